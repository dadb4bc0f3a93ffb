"""Routing, norms and a shared expert registered with a context: its steps and iterations against the oracle, and against
the same calls made one by one."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import layer_ops as lo  # noqa: E402
from oracle import moe_layer as om  # noqa: E402
from oracle.cache_policy import LayerCache  # noqa: E402
from paper_2609_33385_b200 import synth  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_2609_33385_b200 import binding, build
    build.build()
    binding.load()
    return binding


def runner(w, **kw):
    from paper_2609_33385_b200.runner import StackRunner
    return StackRunner(w, **kw)


def dev(bits):
    from paper_2609_33385_b200.runner import bits_to_dev
    return bits_to_dev(bits, "cuda:0")


def bits(t):
    from paper_2609_33385_b200.runner import dev_to_bits
    return dev_to_bits(t)


def np64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def routed_sum(run, layer, h_bits, ids, gate):
    """The gate-weighted sum of the routed experts in 64 bits, one expert at a time."""
    w = run.w
    x = om.bf16_to_f32(h_bits)
    out = np.zeros(x.shape)
    hi = w.hidden * w.intermediate
    for e in np.unique(ids):
        t, j = np.nonzero(ids == e)
        blob = run.layer_blobs(layer)[e]
        if run.fp8:
            ws = om.fp8_expert_weights(blob, w.hidden, w.intermediate)
        else:
            ws = [om.bf16_to_f32(v) for v in (blob[:hi].reshape(-1, w.hidden), blob[hi:2 * hi].reshape(-1, w.hidden),
                                             blob[2 * hi:].reshape(w.hidden, -1))]
        np.add.at(out, t, gate[t, j][:, None] * om.expert_ffn(x[t], *ws))
    return out


@pytest.mark.parametrize("n,fp8", [(1, False), (5, True), (40, False), (300, False), (300, True), (1300, False), (1300, True)])
@pytest.mark.parametrize("score,groups,top_groups,group_top,with_bias", [(1, 4, 2, 2, True), (0, 1, 1, 1, False), (0, 8, 3, 1, True)])
def test_step_with_registered_routing(b, n, fp8, score, groups, top_groups, group_top, with_bias):
    e, k = 32, 4
    w = synth.tiny(n_layers=1, n_experts=e, top_k=k, hidden=512, intermediate=256)
    run = runner(w, capacity=[12], max_tokens=max(n, 8), fp8=fp8)
    try:
        bias = (0.05 * np.random.default_rng(1).normal(size=e)).astype(np.float32) if with_bias else None
        bias_dev = None if bias is None else torch.from_numpy(bias).cuda()
        routing = b.Routing(e, k, score=score, n_groups=groups, top_groups=top_groups, group_top=group_top)
        run.ctx.register_routing(0, routing, None if bias is None else bias_dev.data_ptr())
        cache = LayerCache(e, 12, 1)
        out = torch.empty((n, w.hidden), dtype=torch.bfloat16, device="cuda:0")
        for step in range(3):
            h_bits, conf = synth.flat_tokens(w, n, step)
            x, c = dev(h_bits), torch.from_numpy(conf).cuda()
            run.step(0, x, c, out)
            got = run.ctx.debug_last(0, n)
            order = run.ctx.debug_perm(0, n)
            logits = run.ctx.debug_logits(0, n)
            assert np.array_equal(logits.view(np.uint32), om.gate_logits(om.bf16_to_f32(h_bits), om.bf16_to_f32(run.router_bits[0]), None).view(np.uint32))
            ids, gate, counts, offsets, perm = lo.route_scored(logits, bias, k, softmax=score == 0, n_groups=groups, top_groups=top_groups,
                                                               group_top=group_top)
            assert np.array_equal(got["ids"], ids) and np.array_equal(got["counts"], counts) and np.array_equal(got["perm"], perm)
            assert np.array_equal(order["offsets"], offsets)
            # (a weight is off by 2^-17 of itself at most: exponential, its argument, the softmax's sum, quotients)
            assert np.all(np.abs(got["gate"] - gate) <= 2.0 ** -17 * gate)
            # the cache's decisions follow from the weights as they are
            ref = cache.step(got["ids"], got["gate"], conf)
            assert [int(v) for v in got["scores"]] == list(ref["scores"])
            assert set(np.flatnonzero(got["resident_after"])) == ref["resident_after"]
            want = routed_sum(run, 0, h_bits, got["ids"], got["gate"].astype(np.float64))
            err = np64(out) - want
            assert np.abs(err).max() <= 2e-2 and np.linalg.norm(err) <= 1e-2 * np.linalg.norm(want)
        # taken away again: the plain gate
        run.ctx.register_routing(0, None)
        run.step(0, x, c, out)
        ids, gate = om.topk_route(logits, k)
        got = run.ctx.debug_last(0, n)
        assert np.array_equal(got["ids"], ids) and np.array_equal(got["gate"].view(np.uint32), gate.view(np.uint32))
    finally:
        run.close()


def test_routing_scale_and_score_numerators(b):
    """The scale multiplies the weights and leaves the reuse scores alone."""
    e, k, n = 16, 3, 64
    w = synth.tiny(n_layers=1, n_experts=e, top_k=k, hidden=256)
    run = runner(w, capacity=[e], max_tokens=n)
    try:
        h_bits, conf = synth.flat_tokens(w, n, 3)
        x, c = dev(h_bits), torch.from_numpy(conf).cuda()
        out = torch.empty((n, w.hidden), dtype=torch.bfloat16, device="cuda:0")
        seen = []
        for scale in (1.0, 4.0):
            run.ctx.register_routing(0, b.Routing(e, k, score=b.SCORE_SIGMOID, scale=scale))
            run.step(0, x, c, out)
            seen.append(run.ctx.debug_last(0, n))
        assert np.array_equal(seen[0]["scores"], seen[1]["scores"]) and np.array_equal(4 * seen[0]["gate"], seen[1]["gate"])
    finally:
        run.close()


def shared_expert(b, hidden, inter, seed):
    g = torch.Generator().manual_seed(seed)

    def codes(n, k):
        v = 0.05 * torch.randn(n, k, generator=g)
        s = v.view(n // 128, 128, k // 128, 128).abs().amax(dim=(1, 3)) / 448
        q = (v.view(n // 128, 128, k // 128, 128) / s[:, None, :, None]).view(n, k).to(torch.float8_e4m3fn)
        return q.view(torch.uint8).cuda(), s.cuda()
    (c1, s1), (c2, s2) = codes(2 * inter, hidden), codes(hidden, inter)
    return (c1, s1, c2, s2), b.SharedExpert(inter, c1.data_ptr(), s1.data_ptr(), c2.data_ptr(), s2.data_ptr())


def add_shared(b, keep, x, routed):
    """The shared expert by the public calls; x, routed: [n, hidden] bf16."""
    c1, s1, c2, s2 = keep
    n, h = x.shape
    inter = c2.shape[1]
    st = torch.cuda.current_stream().cuda_stream
    xc, xs = torch.empty((n, h), dtype=torch.uint8, device="cuda"), torch.empty((n, h // 128), device="cuda")
    mid = torch.empty((n, 2 * inter), dtype=torch.bfloat16, device="cuda")
    mc, ms = torch.empty((n, inter), dtype=torch.uint8, device="cuda"), torch.empty((n, inter // 128), device="cuda")
    out = torch.empty_like(x)
    p1 = b.ProductShape(n=2 * inter, k=h, out=0, a_stride=h, a_scale_stride=h // 128, b_stride=h, b_scale_stride=h // 128, add_stride=0, out_stride=2 * inter)
    p2 = b.ProductShape(n=h, k=inter, out=0, a_stride=inter, a_scale_stride=inter // 128, b_stride=inter, b_scale_stride=inter // 128, add_stride=h, out_stride=h)
    assert b.quantize_blocks(x.data_ptr(), h, n, h, 0, st, xc.data_ptr(), h, xs.data_ptr(), h // 128) == 0
    assert b.matmul_blocks(p1, xc.data_ptr(), xs.data_ptr(), c1.data_ptr(), s1.data_ptr(), None, n, st, mid.data_ptr()) == 0
    assert b.quantize_blocks(mid.data_ptr(), 2 * inter, n, inter, 1, st, mc.data_ptr(), inter, ms.data_ptr(), inter // 128) == 0
    assert b.matmul_blocks(p2, mc.data_ptr(), ms.data_ptr(), c2.data_ptr(), s2.data_ptr(), routed.data_ptr(), n, st, out.data_ptr()) == 0
    return out


@pytest.mark.parametrize("n", [1, 33, 700])
def test_step_with_shared_expert(b, n):
    w = synth.tiny(n_layers=1, n_experts=8, top_k=2, hidden=512, intermediate=256)
    run = runner(w, capacity=[4], max_tokens=n)
    try:
        out, plain = (torch.empty((n, 512), dtype=torch.bfloat16, device="cuda:0") for _ in range(2))
        h_bits, conf = synth.flat_tokens(w, n, 5)
        x, c = dev(h_bits), torch.from_numpy(conf).cuda()
        run.step(0, x, c, plain)
        for inter, seed in ((384, 1), (128, 2), (640, 3)):       # (a larger one makes room for itself)
            keep, desc = shared_expert(b, 512, inter, seed)
            run.ctx.register_shared_expert(0, desc)
            run.step(0, x, c, out)
            want = add_shared(b, keep, x, plain)
            torch.cuda.synchronize()
            assert torch.equal(out.view(torch.int16), want.view(torch.int16))
            # and by the definition: the codes of input and activations as the products read them
            c1, s1, c2, s2 = (v.cpu().numpy() for v in keep)
            mid, _ = lo.matmul(*lo.quantize(x.float().cpu().numpy()), c1, s1)
            act = lo.swiglu(mid)
            down = act @ (lo.e4m3_decode(c2) * np.repeat(np.repeat(s2.astype(np.float64), 128, axis=0), 128, axis=1)).T
            # (activations: bf16 2^-8 twice, e4m3 2^-4 of each, which add up as the root of their squares: 2^-4 of the whole at most)
            assert np.linalg.norm(np64(out) - np64(plain) - down) <= 2.0 ** -3 * np.linalg.norm(down) + 2.0 ** -8 * np.linalg.norm(np64(out))
        run.ctx.register_shared_expert(0, None)
        run.step(0, x, c, out)
        assert torch.equal(out.view(torch.int16), plain.view(torch.int16))
    finally:
        run.close()


@pytest.mark.parametrize("n", [1, 20, 600])
def test_iteration_with_everything_around_the_layers(b, n):
    """Three layers, each with other neighbours, in one iteration: bit for bit what the single calls give."""
    h, e, k = 512, 16, 2
    w = synth.tiny(n_layers=3, n_experts=e, top_k=k, hidden=h, intermediate=256)
    run, one = runner(w, capacity=[6, 16, 3], max_tokens=n), runner(w, capacity=[6, 16, 3], max_tokens=n)
    g = torch.Generator().manual_seed(4)
    bf = lambda *s: (1 + 0.2 * torch.randn(*s, generator=g)).to(torch.bfloat16).cuda()  # noqa: E731
    pre, post, gates = [bf(h), None, bf(h)], [bf(h), bf(h), None], [None, bf(1, h), bf(-(-n // 8), h)]
    eps, scale, period = [1e-5, 1e-6, 1e-6], [1.0, 0.5, 0.7], [0, 0, 8]
    try:
        keep, desc = shared_expert(b, h, 256, 7)
        bias = 0.1 * torch.randn(e, generator=g).cuda()
        routing = b.Routing(e, k, score=b.SCORE_SIGMOID, n_groups=4, top_groups=2, group_top=2, scale=1.5)
        for r in (run, one):
            r.ctx.register_shared_expert(1, desc)
            r.ctx.register_routing(0, routing, bias.data_ptr())
            r.ctx.register_routing(2, routing)
        p = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        for layer in range(3):
            run.ctx.register_norms(layer, b.LayerNorms(p(pre[layer]), p(post[layer]), p(gates[layer]), period[layer], eps[layer], scale[layer]))
        st = torch.cuda.current_stream().cuda_stream

        def norm(x, y, layer, w_pre, e_):
            shape = b.NormShape(hidden=h, residual=0, gate_tokens=period[layer] if y is not None else 0, eps=e_, residual_scale=scale[layer] if y is not None else 1.0,
                                x_stride=h, y_stride=h, gate_stride=h, x_out_stride=h, h_stride=h, codes_stride=h, scales_stride=4)
            xo, ho = torch.empty_like(x), torch.empty_like(x)
            assert b.norm_residual(shape, p(x), p(y), p(post[layer]) if y is not None else None, p(gates[layer]) if y is not None else None, p(w_pre), n, st,
                                   p(xo), p(ho) if w_pre is not None else None, None, None) == 0
            return xo, ho if w_pre is not None else xo

        for it in range(2):
            h_bits, conf = synth.flat_tokens(w, n, 20 + it)
            x0, c = dev(h_bits), torch.from_numpy(conf).cuda()
            got, out = torch.empty_like(x0), torch.empty_like(x0)
            run.ctx.denoise_iteration(x0.data_ptr(), c.data_ptr(), n, got.data_ptr())
            x, inp = x0, norm(x0, None, 0, pre[0], eps[0])[1]
            for layer in range(3):
                one.step(layer, inp, c, out)
                # (the call that makes the next layer's input has one eps; layers 1 and 2 share theirs, layer 1 has no norm in front)
                xo, _ = norm(x, out, layer, None, eps[layer])
                nxt = pre[layer + 1] if layer < 2 else None
                if nxt is not None:
                    full = b.NormShape(hidden=h, residual=0, gate_tokens=period[layer], eps=eps[layer], residual_scale=scale[layer], x_stride=h, y_stride=h, gate_stride=h,
                                       x_out_stride=h, h_stride=h, codes_stride=h, scales_stride=4)
                    ho = torch.empty_like(x)
                    assert eps[layer] == eps[layer + 1]
                    assert b.norm_residual(full, p(x), p(out), p(post[layer]), p(gates[layer]), p(nxt), n, st, None, p(ho), None, None) == 0
                    inp = ho
                else:
                    inp = xo
                x = xo
            torch.cuda.synchronize()
            assert torch.equal(got.view(torch.int16), x.view(torch.int16))
            assert (run.ctx.stats().hits, run.ctx.stats().misses) == (one.ctx.stats().hits, one.ctx.stats().misses)
        # norms taken away again: the plain residual
        for layer in range(3):
            run.ctx.register_norms(layer, None)
        run.ctx.denoise_iteration(x0.data_ptr(), c.data_ptr(), n, got.data_ptr())
        x = x0
        for layer in range(3):
            one.step(layer, x, c, out)
            nxt = torch.empty_like(x)
            one.ctx.residual_add(x.data_ptr(), out.data_ptr(), nxt.data_ptr(), x.numel())
            x = nxt
        torch.cuda.synchronize()
        assert torch.equal(got.view(torch.int16), x.view(torch.int16))
    finally:
        run.close()
        one.close()


def test_host_iteration_and_self_check(b):
    """The host-buffer iteration takes the same path, and the self-check finds nothing to report."""
    h, n = 256, 50
    w = synth.tiny(n_layers=2, n_experts=16, top_k=3, hidden=h, intermediate=128)
    run = runner(w, capacity=[5, 5], max_tokens=n)
    try:
        run.ctx.set_option(b.OPT_SELF_CHECK, 1)
        keep, desc = shared_expert(b, h, 128, 9)
        ones = torch.ones(h, dtype=torch.bfloat16, device="cuda:0")
        for layer in range(2):
            run.ctx.register_shared_expert(layer, desc)
            run.ctx.register_routing(layer, b.Routing(16, 3, score=b.SCORE_SIGMOID))
            run.ctx.register_norms(layer, b.LayerNorms(ones.data_ptr(), ones.data_ptr(), None, 0, 1e-6, 1.0))
        h_bits, conf = synth.flat_tokens(w, n, 1)
        x, c = dev(h_bits), torch.from_numpy(conf).cuda()
        got = torch.empty_like(x)
        run.ctx.denoise_iteration(x.data_ptr(), c.data_ptr(), n, got.data_ptr())
        run.ctx.synchronize()
        hx, hc, ho = x.cpu().pin_memory(), c.cpu().pin_memory(), torch.empty((n, h), dtype=torch.bfloat16).pin_memory()
        run.ctx.denoise_iteration_host(hx.data_ptr(), hc.data_ptr(), n, ho.data_ptr())
        assert torch.equal(ho.view(torch.int16), got.cpu().view(torch.int16))
        assert run.ctx.self_check_report()[0] == []
        run.ctx.denoise_iteration(x.data_ptr(), c.data_ptr(), 0, got.data_ptr())
    finally:
        run.close()


def test_registrations_refuse(b):
    w = synth.tiny(n_layers=1, n_experts=8, top_k=2, hidden=256)
    run = runner(w, capacity=[8], max_tokens=8)
    ctx, lib = run.ctx, b.load()
    try:
        good = b.Routing(8, 2)
        ones = torch.ones(256, dtype=torch.bfloat16, device="cuda:0")
        f32 = torch.zeros(64, device="cuda:0")
        q = ones.data_ptr()
        keep, desc = shared_expert(b, 256, 128, 1)
        for rc in (lib.oled_register_routing(None, 0, good, None), lib.oled_register_routing(ctx._h, 1, good, None), lib.oled_register_routing(ctx._h, -1, good, None),
                   lib.oled_register_routing(ctx._h, 0, b.Routing(16, 2), None), lib.oled_register_routing(ctx._h, 0, b.Routing(8, 3), None),
                   lib.oled_register_routing(ctx._h, 0, b.Routing(8, 2, n_groups=3), None), lib.oled_register_routing(ctx._h, 0, None, f32.data_ptr()),
                   lib.oled_register_routing(ctx._h, 0, good, f32.data_ptr() + 2),
                   lib.oled_register_norms(None, 0, b.LayerNorms(q, q, None, 0, 1e-6, 1.0)), lib.oled_register_norms(ctx._h, 1, b.LayerNorms(q, q, None, 0, 1e-6, 1.0)),
                   lib.oled_register_norms(ctx._h, 0, b.LayerNorms(q, q, None, -1, 1e-6, 1.0)), lib.oled_register_norms(ctx._h, 0, b.LayerNorms(q, q, None, 0, 0.0, 1.0)),
                   lib.oled_register_norms(ctx._h, 0, b.LayerNorms(q + 1, q, None, 0, 1e-6, 1.0)),
                   lib.oled_register_norms(ctx._h, 0, b.LayerNorms(q, q, None, 0, 1e-6, float("nan"))),
                   lib.oled_register_shared_expert(None, 0, desc), lib.oled_register_shared_expert(ctx._h, 1, desc),
                   lib.oled_register_shared_expert(ctx._h, 0, b.SharedExpert(100, desc.gate_up, desc.gate_up_scale, desc.down, desc.down_scale)),
                   lib.oled_register_shared_expert(ctx._h, 0, b.SharedExpert(0, desc.gate_up, desc.gate_up_scale, desc.down, desc.down_scale)),
                   lib.oled_register_shared_expert(ctx._h, 0, b.SharedExpert(128, None, desc.gate_up_scale, desc.down, desc.down_scale)),
                   lib.oled_register_shared_expert(ctx._h, 0, b.SharedExpert(128, desc.gate_up + 8, desc.gate_up_scale, desc.down, desc.down_scale))):
            assert rc == b.ERR_INVALID_ARG
        # nothing of that stayed: a step is the plain one
        h_bits, conf = synth.flat_tokens(w, 8, 1)
        out = torch.empty((8, 256), dtype=torch.bfloat16, device="cuda:0")
        run.step(0, dev(h_bits), torch.from_numpy(conf).cuda(), out)
        got = ctx.debug_last(0, 8)
        assert np.array_equal(got["ids"], om.topk_route(ctx.debug_logits(0, 8), 2)[0])
    finally:
        run.close()


@pytest.mark.parametrize("n", [4, 300])
def test_profile_counts_what_stands_around_the_layers(b, n):
    """Every launch of an iteration with routing, norms and shared experts is in the profile, under its own name."""
    h, layers = 256, 2
    w = synth.tiny(n_layers=layers, n_experts=16, top_k=3, hidden=h, intermediate=256)
    run = runner(w, capacity=[16, 16], max_tokens=n)
    try:
        keep, desc = shared_expert(b, h, 128, 9)
        ones = torch.ones(h, dtype=torch.bfloat16, device="cuda:0")
        h_bits, conf = synth.flat_tokens(w, n, 1)
        x, c = dev(h_bits), torch.from_numpy(conf).cuda()
        got = torch.empty_like(x)

        def launched():
            run.ctx.denoise_iteration(x.data_ptr(), c.data_ptr(), n, got.data_ptr())   # (fetches what it misses)
            run.ctx.synchronize()
            run.ctx.profile_read()
            before = run.ctx.launch_count()
            run.ctx.denoise_iteration(x.data_ptr(), c.data_ptr(), n, got.data_ptr())
            count = run.ctx.launch_count() - before
            prof = run.ctx.profile_read()
            assert all(p["ms"] > 0 and p["bytes"] > 0 for p in prof.values() if p["launches"])
            return count, {k: p["launches"] for k, p in prof.items()}

        run.ctx.set_option(b.OPT_PROFILE, 1)
        count, plain = launched()
        assert plain["shared_expert"] == plain["norm"] == 0 and plain["route"] == layers and sum(plain.values()) == count
        for layer in range(layers):
            run.ctx.register_shared_expert(layer, desc)
            run.ctx.register_routing(layer, b.Routing(16, 3, score=b.SCORE_SIGMOID))
        count, prof = launched()
        assert prof["shared_expert"] == 4 * layers and prof["norm"] == 0 and prof["route"] == 2 * layers and prof["combine"] == 2 * layers
        assert sum(prof.values()) == count
        for layer in range(layers):
            run.ctx.register_norms(layer, b.LayerNorms(ones.data_ptr(), ones.data_ptr(), None, 0, 1e-6, 1.0))
        count, prof = launched()
        assert prof["shared_expert"] == 4 * layers and prof["norm"] == layers + 1 and prof["combine"] == layers and sum(prof.values()) == count
    finally:
        run.close()


@pytest.mark.parametrize("n", [1, 4, 20, 200, 600])
def test_combine_left_to_a_gate_kernel_that_chooses_nothing(b, n):
    """A layer's combine is left to the next layer's gate kernel; with a registered routing that kernel makes the logits only."""
    h, e, k, layers = 512, 16, 3, 4
    w = synth.tiny(n_layers=layers, n_experts=e, top_k=k, hidden=h, intermediate=256)
    run, one = runner(w, capacity=[6, 16, 3, 9], max_tokens=n), runner(w, capacity=[6, 16, 3, 9], max_tokens=n)
    try:
        bias = 0.1 * torch.randn(e, generator=torch.Generator().manual_seed(1)).cuda()
        for r in (run, one):
            r.ctx.register_routing(1, b.Routing(e, k, score=b.SCORE_SIGMOID, n_groups=4, top_groups=2, group_top=2, scale=1.5), bias.data_ptr())
            r.ctx.register_routing(2, b.Routing(e, k))
        for it in range(3):
            h_bits, conf = synth.flat_tokens(w, n, 30 + it)
            x, c = dev(h_bits), torch.from_numpy(conf).cuda()
            got, out = torch.empty_like(x), torch.empty_like(x)
            before = run.ctx.launch_count()
            run.ctx.denoise_iteration(x.data_ptr(), c.data_ptr(), n, got.data_ptr())
            fused = run.ctx.launch_count() - before
            before = one.ctx.launch_count()
            for layer in range(layers):
                one.step(layer, x, c, out)
                nxt = torch.empty_like(x)
                one.ctx.residual_add(x.data_ptr(), out.data_ptr(), nxt.data_ptr(), x.numel())
                x = nxt
            single = one.ctx.launch_count() - before
            torch.cuda.synchronize()
            assert single - fused >= layers - 1            # (every combine but the last one is another kernel's)
            assert torch.equal(got.view(torch.int16), x.view(torch.int16))
            assert (run.ctx.stats().hits, run.ctx.stats().misses) == (one.ctx.stats().hits, one.ctx.stats().misses)
    finally:
        run.close()
        one.close()
