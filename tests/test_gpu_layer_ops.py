"""The operators around the routed experts against the oracle in 64 bits (oracle/layer_ops.py).

Roundings are counted as half a step relative to the value: bf16 2^-8, e4m3 2^-4 (and 2^-10 of its scale below the normal
codes), fp32 2^-24.  The bounds of the fp32 arithmetic stand beside the tests that use them.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import layer_ops as lo  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def b():
    from paper_2609_33385_b200 import binding, build
    build.build()
    binding.load()
    return binding


def stream():
    return torch.cuda.current_stream().cuda_stream


def ok(b, rc):
    assert rc == b.OLED_OK, b.strerror(rc)


def ptr(t):
    return None if t is None else t.data_ptr()


def np64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rows(values, dtype, stride, guard):
    """A [rows, cols] view into a buffer with `stride` elements a row, filled with `guard` around the values."""
    r, c = values.shape
    buf = torch.full((r, stride), guard, dtype=torch.float32, device=DEV).to(dtype)
    buf[:, :c] = values.to(device=DEV, dtype=dtype)
    return buf


# ---- routing -------------------------------------------------------------------------------------

def run_route(b, logits, bias, stride=None, order=True, **kw):
    t, e = logits.shape
    r = b.Routing(n_experts=e, **kw)
    k = kw["top_k"]
    stride = stride or e
    x = torch.full((t, stride), 1e30, device=DEV)
    x[:, :e] = torch.from_numpy(logits)
    bi = None if bias is None else torch.from_numpy(bias).to(DEV)
    ids = torch.full((t + 1, k), -7, dtype=torch.int32, device=DEV)
    gate = torch.full((t + 1, k), -7.0, device=DEV)
    counts, offsets = (torch.full((n,), -7, dtype=torch.int32, device=DEV) for n in (e + 1, e + 2))
    perm = torch.full((t * k + 1,), -7, dtype=torch.int32, device=DEV)
    need = b.route_scored_scratch(r, t)
    scratch = torch.full((need // 4 + 1,), -7, dtype=torch.int32, device=DEV)
    ok(b, b.route_scored(r, x.data_ptr(), stride, ptr(bi), t, stream(), ids.data_ptr(), gate.data_ptr(), *([ptr(counts), ptr(offsets), ptr(perm)] if order else [None] * 3),
                         scratch.data_ptr(), need))
    torch.cuda.synchronize()
    assert bool((ids[t] == -7).all()) and bool((gate[t] == -7).all()) and int(perm[t * k]) == -7 and int(counts[e]) == -7
    assert int(offsets[e + 1]) == -7 and int(scratch[-1]) == -7
    return ids[:t].cpu().numpy(), gate[:t].cpu().numpy(), counts[:e].cpu().numpy(), offsets[:e + 1].cpu().numpy(), perm[:t * k].cpu().numpy()


# relative error of a weight: the exponential 2^-22, its argument (|l - max| <= 16 here) 16 * 2^-24, the softmax's sum 2^-18,
# quotient and scale 2^-23
GATE_RTOL = 2.0 ** -22 + 2.0 ** -20 + 2.0 ** -18 + 2.0 ** -23


def check_route(b, logits, bias, stride=None, **kw):
    got = run_route(b, logits, bias, stride, **kw)
    ref_kw = {k: v for k, v in kw.items() if k not in ("score", "renormalise")}
    ids, gate, counts, offsets, perm = lo.route_scored(logits, bias, softmax=kw.get("score", 0) == b.SCORE_SOFTMAX,
                                                       renormalise=bool(kw.get("renormalise", 1)), **ref_kw)
    assert np.array_equal(got[0], ids)
    assert np.all(np.abs(got[1] - gate) <= GATE_RTOL * np.abs(gate) + 1e-30)
    assert np.array_equal(got[2], counts) and np.array_equal(got[3], offsets) and np.array_equal(got[4], perm)


@pytest.mark.parametrize("t", [1, 2, 7, 33, 513, 1500])
@pytest.mark.parametrize("score,with_bias,groups,top_groups,group_top", [
    (0, False, 1, 1, 1), (0, True, 1, 1, 1), (1, False, 1, 1, 1), (1, True, 1, 1, 1), (1, True, 8, 4, 2), (1, True, 8, 3, 1), (0, False, 4, 2, 1),
    (1, False, 8, 4, 2), (0, False, 8, 2, 2), (0, True, 4, 1, 2), (1, True, 4, 4, 2)])
def test_route_matches_oracle(b, t, score, with_bias, groups, top_groups, group_top):
    rng = np.random.default_rng(t * 100 + score * 10 + groups)
    e = 64
    logits = rng.normal(size=(t, e)).astype(np.float32)
    bias = (0.1 * rng.normal(size=e)).astype(np.float32) if with_bias else None
    check_route(b, logits, bias, top_k=8, score=score, n_groups=groups, top_groups=top_groups, group_top=group_top,
                renormalise=t % 2, scale=2.5 if t % 3 else 1.0)


@pytest.mark.parametrize("e,k,groups,top_groups", [(1, 1, 1, 1), (2, 2, 1, 1), (5, 3, 1, 1), (60, 6, 4, 2), (96, 32, 3, 2), (100, 10, 5, 2), (160, 6, 8, 3), (256, 8, 8, 4),
                                                   (510, 9, 17, 5), (512, 32, 1, 1), (512, 8, 32, 8), (384, 8, 8, 4), (510, 7, 3, 1)])
@pytest.mark.parametrize("with_bias", [False, True])
def test_route_shapes(b, e, k, groups, top_groups, with_bias):
    rng = np.random.default_rng(e + k)
    logits = (2 * rng.normal(size=(150, e))).astype(np.float32)
    bias = (0.05 * rng.normal(size=e)).astype(np.float32) if with_bias else None
    for score in (0, 1):
        check_route(b, logits, bias, stride=e + 3, top_k=k, score=score, n_groups=groups, top_groups=top_groups, group_top=min(2, e // groups))


@pytest.mark.parametrize("score", [0, 1])
def test_route_ties_and_near_ties(b, score):
    """Equal logits, equal choices, and choices that differ by less than fp32 can say: the ids are those of 64 bits."""
    rng = np.random.default_rng(5)
    e, t = 64, 200
    coarse = (rng.integers(-3, 4, size=(t, e)) * 0.5).astype(np.float32)     # many equal logits
    check_route(b, coarse, None, top_k=8, score=score)
    check_route(b, coarse, None, top_k=8, score=score, n_groups=8, top_groups=3, group_top=2)
    zero = np.zeros(e, np.float32)
    check_route(b, coarse, zero, top_k=8, score=score)
    check_route(b, np.zeros((3, e), np.float32), None, top_k=8, score=score)
    # a bias that undoes the scores' differences up to their rounding
    one = rng.normal(size=(1, e)).astype(np.float32)
    s = 1 / (1 + np.exp(-one[0].astype(np.float64))) if score else np.exp(one[0].astype(np.float64)) / np.exp(one[0].astype(np.float64)).sum()
    check_route(b, np.repeat(one, 9, axis=0), (0.75 - s).astype(np.float32), top_k=12, score=score)
    check_route(b, np.repeat(one, 9, axis=0), (0.75 - s).astype(np.float32), top_k=12, score=score, n_groups=4, top_groups=2, group_top=2)
    nudged = one + (rng.integers(-2, 3, size=(t, e)) * 2.0 ** -23).astype(np.float32)
    check_route(b, nudged, (0.75 - s).astype(np.float32), top_k=8, score=score, n_groups=8, top_groups=4, group_top=2)


@pytest.mark.parametrize("groups", [(1, 1, 1), (8, 4, 2), (8, 4, 1)])
def test_route_saturated_scores(b, groups):
    """Sigmoids that are the same number in fp32 and are not in 64 bits, in ascending order of the index."""
    e, t = 64, 20
    rng = np.random.default_rng(8)
    logits = (16 + np.sort(rng.uniform(0, 4, size=(t, e)), axis=1)).astype(np.float32)
    for bias in (np.zeros(e, np.float32), np.full(e, 0.25, np.float32)):
        check_route(b, logits, bias, top_k=8, score=1, n_groups=groups[0], top_groups=groups[1], group_top=groups[2])


def test_route_groups_of_equal_fp32_value(b):
    """Two groups far above the others, equal in fp32 and told apart in 64 bits by their index's opposite: one may stay."""
    e, t = 64, 8
    logits = np.full((t, e), -3.0, np.float32)
    for i in range(t):
        lo_g, hi_g = i, (i + 3) % 8
        logits[i, lo_g * 8:lo_g * 8 + 2] = 18.0
        logits[i, hi_g * 8:hi_g * 8 + 2] = np.nextafter(np.float32(18.0), np.float32(19.0))
    for bias in (None, np.zeros(e, np.float32)):
        for top_groups in (1, 2, 3):
            for group_top in (1, 2):
                check_route(b, logits, bias, top_k=6, score=1, n_groups=8, top_groups=top_groups, group_top=group_top)


@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("e,groups,top_groups,k,alike", [(64, 8, 3, 8, 2), (64, 8, 1, 5, 8), (512, 16, 9, 32, 2), (96, 3, 2, 6, 4), (40, 20, 7, 3, 2), (512, 32, 30, 8, 3)])
def test_route_groups_whose_border_fp32_cannot_tell(b, score, e, groups, top_groups, k, alike):
    """Groups whose best experts differ by a few units in the last place; of some tokens all groups, of others those around the border.
    `alike` experts of a group are that near to each other's counterparts (and, in every second token, to each other)."""
    rng = np.random.default_rng(9)
    t, size = 120, e // groups
    logits = rng.uniform(-3, 0, size=(t, groups, size)).astype(np.float32)
    for i in range(t):
        best = np.full(alike, 1.5) if i % 2 else 1.0 + 0.5 * np.arange(alike)
        for g in range(groups):
            at = rng.choice(size, min(alike, size), replace=False)
            logits[i, g, at] = best[:len(at)].astype(np.float32) + (rng.integers(-2, 3, size=len(at)) * 2.0 ** -23).astype(np.float32)
        if i % 3:
            far = rng.choice(groups, groups // 2, replace=False)
            logits[i, far] += rng.choice([-0.5, 0.5], size=(len(far), 1)).astype(np.float32)
    logits = logits.reshape(t, e)
    for bias in (None, np.zeros(e, np.float32), np.full(e, 0.25, np.float32)):
        for group_top in (1, 2):
            check_route(b, logits, bias, top_k=k, score=score, n_groups=groups, top_groups=top_groups, group_top=group_top)


@pytest.mark.parametrize("t,e,k", [(4500, 1, 1), (4111, 2, 1), (2500, 3, 2), (1200, 7, 7), (900, 13, 5), (700, 40, 17), (150, 510, 32), (129, 512, 32), (40001, 9, 1), (1 << 20, 5, 2)])
def test_route_order_of_many_assignments(b, t, e, k):
    """The order of more assignments than one launch takes: few and odd numbers of experts, tokens that do not fill the CTAs."""
    gen = torch.Generator(device=DEV).manual_seed(t)
    logits = torch.randn((t, e), device=DEV, generator=gen)
    r = b.Routing(e, k)
    ids, gate = torch.empty((t, k), dtype=torch.int32, device=DEV), torch.empty((t, k), device=DEV)
    counts, offsets = torch.full((e + 1,), -7, dtype=torch.int32, device=DEV), torch.full((e + 2,), -7, dtype=torch.int32, device=DEV)
    perm = torch.full((t * k + 1,), -7, dtype=torch.int32, device=DEV)
    need = b.route_scored_scratch(r, t)
    for shift in (0, 1):  # scratch on 8-byte boundaries, and on 4-byte ones alone
        scratch = torch.full((need // 4 + 3,), -7, dtype=torch.int32, device=DEV)
        ok(b, b.route_scored(r, logits.data_ptr(), e, None, t, stream(), ids.data_ptr(), gate.data_ptr(), counts.data_ptr(), offsets.data_ptr(), perm.data_ptr(),
                             scratch.data_ptr() + 4 * shift, need))
        torch.cuda.synchronize()
        assert bool((scratch[shift + need // 4:] == -7).all()) and bool((scratch[:shift] == -7).all())
        expected = torch.sort(logits.double(), dim=1, descending=True, stable=True).indices[:, :k]
        assert bool((ids == expected).all())
        flat = ids.flatten().long()
        assert bool((perm[:-1] == torch.sort(flat, stable=True).indices).all()) and int(perm[-1]) == -7
        n = torch.bincount(flat, minlength=e)
        assert bool((counts[:e] == n).all()) and int(counts[e]) == -7
        assert bool((offsets[1:e + 1] == torch.cumsum(n, 0)).all()) and int(offsets[0]) == 0 and int(offsets[e + 1]) == -7


@pytest.mark.parametrize("score", [0, 1])
def test_route_with_fewer_finite_choices_than_wanted(b, score):
    """Groups that stay and have fewer experts than wanted that are not at -inf, by their logits or by their bias."""
    rng = np.random.default_rng(10)
    t, e, groups = 90, 48, 4
    logits = rng.normal(size=(t, e)).astype(np.float32)
    for i in range(t):
        for g in range(groups):
            keep = rng.choice(12, rng.integers(0 if i % 3 == 0 else 1, 5), replace=False)
            gone = np.setdiff1d(np.arange(12), keep)
            logits[i, g * 12 + gone] = -np.inf
    masked = np.where(np.arange(e) % 12 < 2, 0.1, -np.inf).astype(np.float32)
    finite = rng.normal(size=(t, e)).astype(np.float32)
    for group_top in (1, 2):
        for top_groups in (2, 3):
            check_route(b, logits, None, top_k=7, score=score, n_groups=groups, top_groups=top_groups, group_top=group_top)
            check_route(b, finite, masked, top_k=7, score=score, n_groups=groups, top_groups=top_groups, group_top=group_top)
    check_route(b, logits, None, top_k=9, score=score)
    check_route(b, finite, masked, top_k=9, score=score)


@pytest.mark.parametrize("score", [0, 1])
def test_route_non_finite(b, score):
    rng = np.random.default_rng(6)
    e = 32
    l = rng.normal(size=(12, e)).astype(np.float32)
    l[0, 3] = np.nan
    l[1, :] = np.nan
    l[2, :] = -np.inf
    l[3, 5:] = -np.inf
    l[4, 7] = np.inf
    l[5, [2, 9]] = np.inf
    l[6, :] = np.finfo(np.float32).min
    l[7, 4] = np.finfo(np.float32).max
    l[8, ::2] = np.nan
    l[9, 1:] = np.nan
    l[10, :] = 100.0
    l[11, :] = -200.0
    bias = (0.1 * rng.normal(size=e)).astype(np.float32)
    masked = bias.copy()
    masked[::3] = -np.inf
    for bi in (None, bias, masked, np.full(e, -np.inf, np.float32)):
        for groups in ((1, 1, 1), (4, 2, 2)):
            got = run_route(b, l, bi, top_k=6, score=score, n_groups=groups[0], top_groups=groups[1], group_top=groups[2])
            ids, gate, counts, offsets, perm = lo.route_scored(l, bi, 6, softmax=score == 0, n_groups=groups[0], top_groups=groups[1], group_top=groups[2])
            assert np.array_equal(got[0], ids)
            assert all(len(set(r)) == 6 for r in got[0].tolist())
            # (scores next to the smallest fp32 numbers keep no relative precision)
            assert np.all(np.abs(got[1] - gate) <= GATE_RTOL * np.abs(gate) + 1e-15)
            assert np.array_equal(got[4], perm) and np.array_equal(got[2], counts)


def test_route_without_order_and_large(b):
    rng = np.random.default_rng(7)
    l = rng.normal(size=(4099, 128)).astype(np.float32)
    bias = (0.1 * rng.normal(size=128)).astype(np.float32)
    kw = dict(top_k=8, score=1)
    check_route(b, l, bias, **kw)
    got = run_route(b, l, bias, order=False, **kw)
    assert np.array_equal(got[0], lo.route_scored(l, bias, 8)[0]) and set(got[2].tolist()) == {-7}
    skew = l.copy()
    skew[:, 17] += 50                                    # every token has it
    check_route(b, skew, None, top_k=1, score=1)


# ---- norms ---------------------------------------------------------------------------------------

def run_norm(b, x, y, post, gate, pre, gate_tokens, residual, eps, scale, outs, pad):
    t, h = x.shape
    kind = torch.float32 if residual else torch.bfloat16
    s = h + pad
    xd = rows(x, kind, s, 7.0)
    yd = None if y is None else rows(y, torch.bfloat16, s, 7.0)
    gd = None if gate is None else rows(gate, torch.bfloat16, s, 7.0)
    vec = [None if w is None else w.to(device=DEV, dtype=torch.bfloat16) for w in (post, pre)]
    nb = -(-h // 128)
    xo = torch.full((t, s), 5.0, dtype=kind, device=DEV)
    ho = torch.full((t, s), 5.0, dtype=torch.bfloat16, device=DEV) if "h" in outs else None
    co = torch.full((t, s), 0x55, dtype=torch.uint8, device=DEV) if "q" in outs else None
    so = torch.full((t, nb + 1), 5.0, device=DEV) if "q" in outs else None
    shape = b.NormShape(hidden=h, residual=residual, gate_tokens=gate_tokens, eps=eps, residual_scale=scale, x_stride=s, y_stride=s,
                        gate_stride=s, x_out_stride=s, h_stride=s, codes_stride=s, scales_stride=nb + 1)
    ok(b, b.norm_residual(shape, ptr(xd), ptr(yd), ptr(vec[0]), ptr(gd), ptr(vec[1]), t, stream(), ptr(xo) if "x" in outs else None, ptr(ho), ptr(co), ptr(so)))
    torch.cuda.synchronize()
    if pad:
        for o, g in ((xo, 5.0), (ho, 5.0), (co, 0x55)):
            assert o is None or bool((o[:, h:] == g).all())
    assert so is None or bool((so[:, nb:] == 5.0).all())
    return xd, yd, vec, gd, xo[:, :h], None if ho is None else ho[:, :h], None if co is None else co[:, :h], None if so is None else so[:, :nb]


def check_norm(b, t, h, residual=0, post=True, gate_tokens=-1, outs="xhq", pad=0, scale=1.0, with_y=True, eps=1e-6, seed=0):
    g = torch.Generator().manual_seed(seed + h)
    x, y = 3 * torch.randn(t, h, generator=g), torch.randn(t, h, generator=g)
    wpost = 1 + 0.1 * torch.randn(h, generator=g) if post and with_y else None
    wpre = 1 + 0.1 * torch.randn(h, generator=g) if "h" in outs or "q" in outs else None
    n_gate = 1 if gate_tokens == 0 else -(-t // max(1, gate_tokens))
    gate = torch.randn(n_gate, h, generator=g) if gate_tokens >= 0 and with_y else None
    xd, yd, vec, gd, xo, ho, co, so = run_norm(b, x, y if with_y else None, wpost, gate, wpre, max(0, gate_tokens), residual, eps, scale, outs, pad)
    f = lambda v: None if v is None else np64(v)[..., :h]  # noqa: E731
    ref_x, ref_h, step = lo.norm_residual(f(xd), f(yd), f(vec[0]), f(gd), f(vec[1]), max(0, gate_tokens), eps, scale)
    # a norm's factor: its sum of squares in at most 32 rounded steps per thread and 5 + 16 to join them, halved by the root
    # (53 * 2^-25), mean, eps, root 2^-22 + 2^-24; its product with value, weight, gate and scale 4 * 2^-24
    rel = 53 * 2.0 ** -25 + 2.0 ** -22 + 5 * 2.0 ** -24
    ex = rel * np.abs(step) + 2.0 ** -24 * np.abs(ref_x)
    if "x" in outs:
        bound = ex + (0 if residual else 2.0 ** -8 * np.abs(ref_x)) + 1e-37
        assert np.all(np.abs(np64(xo) - ref_x) <= bound)
    if ref_h is None:
        return
    inv = np.abs(f(vec[1])) / np.sqrt((ref_x * ref_x).mean(axis=1, keepdims=True) + eps)
    # (the sum of squares takes each element's error too: at most twice the largest relative one of the row, halved by the root)
    row = np.sqrt((ex * ex).sum(axis=1, keepdims=True) / np.maximum((ref_x * ref_x).sum(axis=1, keepdims=True), 1e-300))
    eh = inv * ex + (rel + row) * np.abs(ref_h)
    if "h" in outs:
        assert np.all(np.abs(np64(ho) - ref_h) <= (1 + 2.0 ** -8) * eh + 2.0 ** -8 * np.abs(ref_h) + 1e-37)
    if "q" in outs:
        sc = so.cpu().numpy().astype(np.float64)
        per = np.repeat(sc, 128, axis=1)[:, :h]
        want = lo.block_amax(ref_h) / 448
        assert np.all(np.abs(sc - want) <= want * 2.0 ** -23 + lo.block_amax(eh) / 448)
        got = lo.dequantize(co.cpu().numpy(), sc)
        assert np.all(np.abs(got - ref_h) <= (1 + 2.0 ** -4) * eh + (2.0 ** -4 + 2.0 ** -22) * np.abs(ref_h) + 2.0 ** -10 * per)


@pytest.mark.parametrize("t,h", [(1, 1), (3, 7), (2, 8), (5, 100), (9, 128), (6, 256), (1, 264), (4, 1000), (7, 1024), (33, 2048), (3, 2056), (17, 3760), (5, 4096),
                                 (3, 4111), (2, 8192), (2, 8200), (1, 16384), (700, 512)])
@pytest.mark.parametrize("residual", [0, 1])
def test_norm_matches_oracle(b, t, h, residual):
    check_norm(b, t, h, residual, gate_tokens=2, pad=0, scale=0.5)
    check_norm(b, t, h, residual, gate_tokens=0, pad=3)
    check_norm(b, t, h, residual, gate_tokens=1, pad=16, post=False)


@pytest.mark.parametrize("outs", ["x", "h", "q", "xh", "xq", "hq"])
@pytest.mark.parametrize("with_y", [True, False])
def test_norm_outputs(b, outs, with_y):
    check_norm(b, 37, 640, outs=outs, with_y=with_y, gate_tokens=5)
    check_norm(b, 37, 333, residual=1, outs=outs, with_y=with_y)


def test_norm_in_place_and_non_finite(b):
    t, h = 8, 512
    g = torch.Generator().manual_seed(2)
    x0 = torch.randn(t, h, generator=g).to(torch.bfloat16).to(DEV)
    y0 = torch.randn(t, h, generator=g).to(torch.bfloat16).to(DEV)
    y0[2, 100] = float("inf")
    y0[3, 5] = float("nan")
    x0[4, 7] = float("nan")
    y0[5] = 0
    x0[5] = 0                                            # the norm of zeros is zeros
    w = torch.ones(h, dtype=torch.bfloat16, device=DEV)
    shape = b.NormShape(hidden=h, residual=0, gate_tokens=0, eps=1e-6, residual_scale=1.0, x_stride=h, y_stride=h, gate_stride=h,
                        x_out_stride=h, h_stride=h, codes_stride=h, scales_stride=4)
    xo, ho = torch.empty_like(x0), torch.empty_like(x0)
    ok(b, b.norm_residual(shape, ptr(x0), ptr(y0), ptr(w), None, ptr(w), t, stream(), ptr(xo), ptr(ho), None, None))
    x1, y1 = x0.clone(), y0.clone()
    ok(b, b.norm_residual(shape, ptr(x1), ptr(y1), ptr(w), None, ptr(w), t, stream(), ptr(x1), ptr(y1), None, None))
    torch.cuda.synchronize()
    assert torch.equal(x1.view(torch.int16), xo.view(torch.int16)) and torch.equal(y1.view(torch.int16), ho.view(torch.int16))
    assert not bool(xo[5].any()) and not bool(ho[5].any())
    fine = [0, 1, 5, 6, 7]
    assert bool(torch.isfinite(ho[fine].float()).all()) and bool(torch.isnan(ho[[2, 3, 4]].float()).any(dim=1).all())


# ---- quantisation --------------------------------------------------------------------------------

@pytest.mark.parametrize("r,k", [(1, 16), (1, 128), (3, 144), (5, 1024), (2, 1040), (33, 2048), (4, 16384), (1000, 384)])
def test_quantize_is_bit_exact(b, r, k):
    g = torch.Generator().manual_seed(k)
    x = torch.randn(r, k, generator=g) * torch.exp(3 * torch.randn(r, 1, generator=g))
    x[0, :min(k, 128)] = 0
    if r > 2:
        x[2] *= 1e-36                                    # blocks below the floor of the scales
        x[1, 3] = 3e38
    xd = rows(x, torch.bfloat16, k + 8, 9.0)
    codes = torch.full((r, k + 16), 0x55, dtype=torch.uint8, device=DEV)
    nb = -(-k // 128)
    scales = torch.full((r, nb + 2), 5.0, device=DEV)
    ok(b, b.quantize_blocks(xd.data_ptr(), k + 8, r, k, 0, stream(), codes.data_ptr(), k + 16, scales.data_ptr(), nb + 2))
    want_c, want_s = lo.quantize(xd[:, :k].float().cpu().numpy())
    assert np.array_equal(scales[:, :nb].cpu().numpy(), want_s)
    got = codes.cpu().numpy()
    assert np.array_equal(lo.e4m3_decode(got[:, :k]), lo.e4m3_decode(want_c))
    assert bool((codes[:, k:] == 0x55).all()) and bool((scales[:, nb:] == 5.0).all())


@pytest.mark.parametrize("r,k", [(1, 16), (4, 1024), (9, 528), (300, 768)])
def test_quantize_swiglu(b, r, k):
    g = torch.Generator().manual_seed(k + 1)
    x = (3 * torch.randn(r, 2 * k, generator=g)).to(torch.bfloat16).to(DEV)
    codes, nb = torch.zeros((r, k), dtype=torch.uint8, device=DEV), -(-k // 128)
    scales = torch.zeros((r, nb), device=DEV)
    ok(b, b.quantize_blocks(x.data_ptr(), 2 * k, r, k, 1, stream(), codes.data_ptr(), k, scales.data_ptr(), nb))
    ref = lo.swiglu(np64(x))
    # silu: the exponential's argument |g| <= 16 (16 * 2^-24) and itself 2^-22, sum, quotient 2^-22, product: 2^-19 together
    s = scales.cpu().numpy().astype(np.float64)
    want = lo.block_amax(ref) / 448
    assert np.all(np.abs(s - want) <= want * 2.0 ** -19)
    got = lo.dequantize(codes.cpu().numpy(), s)
    assert np.all(np.abs(got - ref) <= (2.0 ** -4 + 2.0 ** -18) * np.abs(ref) + 2.0 ** -10 * np.repeat(s, 128, axis=1)[:, :k])


def test_quantize_non_finite(b):
    x = torch.ones((3, 512), dtype=torch.bfloat16, device=DEV)
    x[0, 130], x[1, 5], x[1, 400] = float("inf"), float("nan"), float("-inf")
    codes, scales = torch.zeros((3, 512), dtype=torch.uint8, device=DEV), torch.zeros((3, 4), device=DEV)
    ok(b, b.quantize_blocks(x.data_ptr(), 512, 3, 512, 0, stream(), codes.data_ptr(), 512, scales.data_ptr(), 4))
    v = lo.dequantize(codes.cpu().numpy(), scales.cpu().numpy())
    bad = np.isnan(v).reshape(3, 4, 128)
    assert bad.all(axis=2).tolist() == [[False, True, False, False], [True, False, False, True], [False] * 4]
    # (ones: code 448 times fl(1 / 448), which is off by 2^-24 of itself at most)
    assert np.all(np.abs(v[2] - 1.0) <= 2.0 ** -24) and not bad[~bad.all(axis=2)].any()


# ---- products ------------------------------------------------------------------------------------

def product_inputs(m, n, k, seed=0):
    g = torch.Generator().manual_seed(seed + m * 7 + n * 3 + k)
    kb, nb = -(-k // 128), -(-n // 128)
    a = (40 * torch.randn(m, k, generator=g)).to(torch.float8_e4m3fn).view(torch.uint8)
    w = (40 * torch.randn(n, k, generator=g)).to(torch.float8_e4m3fn).view(torch.uint8)
    sa, sb = (torch.exp(torch.randn(r, kb, generator=g)) * 0.02 for r in (m, nb))
    return a, sa, w, sb


def padded(t, stride, fill):
    buf = torch.full((t.shape[0], stride), fill, dtype=t.dtype, device=DEV)
    buf[:, :t.shape[1]] = t.to(DEV)
    return buf


def run_product(b, a, sa, w, sb, fp32, add=None, pad=0, in_place=False):
    (m, k), n, kb = a.shape, w.shape[0], sa.shape[1]
    ad, wd = padded(a, k + 16 * pad, 0x7F), padded(w, k + 16 * pad, 0x7F)   # (codes between the rows would make everything NaN)
    sad, sbd = padded(sa, kb + pad, float("nan")), padded(sb, kb + pad, float("nan"))
    kind = torch.float32 if fp32 else torch.bfloat16
    out = torch.full((m + 1, n + pad), 5.0, dtype=kind, device=DEV)
    addd = None
    if add is not None:
        addd = padded(add, n + pad, 5.0)
        if in_place:
            out[:m] = addd
            addd = out
    shape = b.ProductShape(n=n, k=k, out=b.FP32 if fp32 else b.BF16, a_stride=k + 16 * pad, a_scale_stride=kb + pad, b_stride=k + 16 * pad,
                           b_scale_stride=kb + pad, add_stride=n + pad, out_stride=n + pad)
    ok(b, b.matmul_blocks(shape, ptr(ad), ptr(sad), ptr(wd), ptr(sbd), ptr(addd), m, stream(), ptr(out)))
    torch.cuda.synchronize()
    assert bool((out[m] == 5.0).all()) and bool((out[:, n:] == 5.0).all())
    return out[:m, :n]


def check_product(b, m, n, k, fp32=False, with_add=False, pad=0, in_place=False):
    a, sa, w, sb = product_inputs(m, n, k)
    add = torch.randn(m, n, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16) if with_add else None
    got = np64(run_product(b, a, sa, w, sb, fp32, add, pad, in_place))
    ref, size = lo.matmul(a.numpy(), sa.numpy(), w.numpy(), sb.numpy(), None if add is None else np64(add))
    kb = sa.shape[1]
    # a block's 128 products are exact; their sum takes 128 steps of at most 2^-23 (whether the tensor core rounds or cuts), the
    # scale 2^-24, every block's addition 2^-24, up to eight joined parts and the addend 9 * 2^-24; all relative to the sum of magnitudes
    bound = size * (128 * 2.0 ** -23 + (kb + 10) * 2.0 ** -24)
    bound = bound + (0 if fp32 else 2.0 ** -8 * (np.abs(ref) + bound))
    assert np.all(np.abs(got - ref) <= bound + 1e-37)


@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 32, 33, 64, 65, 128, 129, 200])
@pytest.mark.parametrize("n,k", [(128, 128), (1, 16), (130, 272), (1000, 1024)])
def test_product_matches_oracle(b, m, n, k):
    check_product(b, m, n, k, fp32=m % 2 == 0)
    check_product(b, m, n, k, fp32=m % 2 == 1, with_add=True, pad=1)


@pytest.mark.parametrize("m,n,k", [(1, 2048, 2048), (1, 77, 16384), (5, 256, 4096), (32, 2048, 1024), (250, 4096, 2048), (128, 300, 16384), (300, 128, 16384), (700, 777, 528),
                                   (1000, 1536, 640), (2049, 513, 384), (4000, 2304, 272)])
def test_product_larger(b, m, n, k):
    check_product(b, m, n, k)
    check_product(b, m, n, k, fp32=True, with_add=True)
    check_product(b, m, n, k, with_add=True, in_place=True, pad=2)


@pytest.mark.parametrize("m,n", [(128, 5000), (64, 9600), (9, 10000)])
def test_product_long_k_without_many_ctas_to_a_tile(b, m, n):
    check_product(b, m, n, 16384)


def test_offsets_past_32_bits(b):
    """Arrays of more than 2^32 elements: the last rows are those of a small call, the ones in front of them stay zeros."""
    r, k = 265000, 16384                                  # 4.3e9 elements
    last = torch.randn(3, k, device=DEV).to(torch.bfloat16)
    x = torch.zeros((r, k), dtype=torch.bfloat16, device=DEV)
    x[-3:] = last
    codes, scales = torch.full((r, k), 1, dtype=torch.uint8, device=DEV), torch.empty((r, k // 128), device=DEV)
    c1, s1 = torch.empty((3, k), dtype=torch.uint8, device=DEV), torch.empty((3, k // 128), device=DEV)
    ok(b, b.quantize_blocks(ptr(x), k, r, k, 0, stream(), ptr(codes), k, ptr(scales), k // 128))
    ok(b, b.quantize_blocks(ptr(last), k, 3, k, 0, stream(), ptr(c1), k, ptr(s1), k // 128))
    assert torch.equal(codes[-3:], c1) and torch.equal(scales[-3:], s1) and not bool(codes[:-3].any())
    w = torch.ones(k, dtype=torch.bfloat16, device=DEV)
    shape = b.NormShape(hidden=k, residual=0, gate_tokens=0, eps=1e-6, residual_scale=1.0, x_stride=k, y_stride=k, gate_stride=k, x_out_stride=k, h_stride=k,
                        codes_stride=k, scales_stride=k // 128)
    h1 = torch.empty_like(last)
    ok(b, b.norm_residual(shape, ptr(last), None, None, None, ptr(w), 3, stream(), None, ptr(h1), None, None))
    ok(b, b.norm_residual(shape, ptr(x), None, None, None, ptr(w), r, stream(), None, ptr(x), None, None))
    assert torch.equal(x[-3:].view(torch.int16), h1.view(torch.int16)) and not bool(x[:-3].any())
    del x, codes, scales
    m, n, kk = 70000, 65536, 16                           # 4.6e9 results
    a, wt = torch.zeros((m, kk), dtype=torch.uint8, device=DEV), torch.full((n, kk), 0x38, dtype=torch.uint8, device=DEV)
    a[-1], a[1] = 0x38, 0x40                              # 1.0, 2.0
    sa, sb = torch.ones((m, 1), device=DEV), torch.ones((n // 128, 1), device=DEV)
    out = torch.empty((m, n), dtype=torch.bfloat16, device=DEV)
    ps = b.ProductShape(n=n, k=kk, out=0, a_stride=kk, a_scale_stride=1, b_stride=kk, b_scale_stride=1, add_stride=0, out_stride=n)
    ok(b, b.matmul_blocks(ps, ptr(a), ptr(sa), ptr(wt), ptr(sb), None, m, stream(), ptr(out)))
    assert bool((out[-1] == 16).all()) and bool((out[1] == 32).all()) and not bool(out[2:-1].any()) and not bool(out[0].any())


@pytest.mark.parametrize("m", [3, 200, 1200])
def test_product_nan_stays_in_its_row_and_column(b, m):
    a, sa, w, sb = product_inputs(m, 512, 512)
    a[2, 130], w[300, 400] = 0x7F, 0xFF
    sa[1, 1] = float("inf")
    got = np64(run_product(b, a, sa, w, sb, True))
    bad = ~np.isfinite(got)
    assert bad[1].all() and bad[2].all() and bad[:, 300].all()
    bad[1:3], bad[:, 300] = False, False
    assert not bad.any()


@pytest.mark.parametrize("m,n,k", [(2100, 1531, 384), (1300, 1536, 2192), (4100, 600, 144), (257, 9600, 2064), (2304, 2048, 1024), (5000, 1024, 128)])
def test_product_on_pairs(b, m, n, k):
    """Shapes that go to pairs of CTAs: ragged rows, columns and k, rows of C on and off 16-byte boundaries."""
    check_product(b, m, n, k)
    check_product(b, m, n, k, fp32=True, with_add=True, pad=1)
    check_product(b, m, n, k, fp32=True)
    check_product(b, m, n, k, with_add=True, in_place=True, pad=8)


def test_product_on_pairs_keeps_nan_in_its_row_and_column(b):
    a, sa, w, sb = product_inputs(2300, 2048, 256)
    a[1000, 130], w[300, 40] = 0x7F, 0xFF
    sa[1400, 1] = float("inf")
    bad = ~torch.isfinite(run_product(b, a, sa, w, sb, True))
    assert bool(bad[1000].all()) and bool(bad[1400].all()) and bool(bad[:, 300].all())
    bad[[1000, 1400]], bad[:, 300] = False, False
    assert not bool(bad.any())


def test_product_scales_of_zero_and_spread(b):
    """Zero scales, and blocks of very different scales: a block counts by its scale alone."""
    a, sa, w, sb = product_inputs(40, 256, 1024)
    sa[:, 1::2] = 0
    sb[1, :] *= 1e-20
    sa[7] *= 1e15
    got = np64(run_product(b, a, sa, w, sb, True))
    ref, size = lo.matmul(a.numpy(), sa.numpy(), w.numpy(), sb.numpy())
    assert np.all(np.abs(got - ref) <= size * (128 * 2.0 ** -23 + 18 * 2.0 ** -24) + 1e-37)


# ---- together, captured, side by side ------------------------------------------------------------

def test_layer_around_the_routed_experts(b):
    """What a layer does next to its routed experts, as it would be run: norm to bf16 and codes, routing from the gate's logits,
    a dense SwiGLU expert from codes whose down projection is added to the routed experts' sum, and the next norm."""
    t, h, inter, e, k = 77, 512, 384, 32, 4
    g = torch.Generator().manual_seed(9)
    bf = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).to(DEV)  # noqa: E731
    x, y, routed = bf(t, h), bf(t, h), bf(t, h)
    ones = torch.ones(h, dtype=torch.bfloat16, device=DEV)
    w1, w2 = 0.05 * torch.randn(2 * inter, h, generator=g), 0.05 * torch.randn(h, inter, generator=g)
    wr = torch.randn(e, h, generator=g).to(DEV) * 0.05

    def codes_of(w):
        n, c = w.shape
        blocks = w.view(n // 128, 128, c // 128, 128)
        s = blocks.abs().amax(dim=(1, 3)) / 448
        return (blocks / s[:, None, :, None]).view(n, c).to(torch.float8_e4m3fn).view(torch.uint8).to(DEV), s.to(DEV)

    (c1, s1), (c2, s2) = codes_of(w1), codes_of(w2)
    xo, hh = torch.empty_like(x), torch.empty_like(x)
    hc, hs = torch.empty((t, h), dtype=torch.uint8, device=DEV), torch.empty((t, h // 128), device=DEV)
    mid = torch.empty((t, 2 * inter), dtype=torch.bfloat16, device=DEV)
    mc, ms = torch.empty((t, inter), dtype=torch.uint8, device=DEV), torch.empty((t, inter // 128), device=DEV)
    out, x2, h2 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    logits = torch.empty((t, e), device=DEV)
    ids, gate = torch.empty((t, k), dtype=torch.int32, device=DEV), torch.empty((t, k), device=DEV)
    counts, offsets, perm = (torch.empty(n, dtype=torch.int32, device=DEV) for n in (e, e + 1, t * k))
    ns = b.NormShape(hidden=h, residual=0, gate_tokens=0, eps=1e-6, residual_scale=1.0, x_stride=h, y_stride=h, gate_stride=h, x_out_stride=h,
                     h_stride=h, codes_stride=h, scales_stride=h // 128)
    p1 = b.ProductShape(n=2 * inter, k=h, out=0, a_stride=h, a_scale_stride=h // 128, b_stride=h, b_scale_stride=h // 128, add_stride=0, out_stride=2 * inter)
    p2 = b.ProductShape(n=h, k=inter, out=0, a_stride=inter, a_scale_stride=inter // 128, b_stride=inter, b_scale_stride=inter // 128, add_stride=h, out_stride=h)
    r = b.Routing(n_experts=e, top_k=k, score=b.SCORE_SIGMOID, n_groups=4, top_groups=2, group_top=2, scale=2.5)
    bias = (0.1 * torch.randn(e, generator=g)).to(DEV)

    def layer():
        st = stream()
        ok(b, b.norm_residual(ns, ptr(x), ptr(y), ptr(ones), None, ptr(ones), t, st, ptr(xo), ptr(hh), ptr(hc), ptr(hs)))
        torch.matmul(hh.float(), wr.t(), out=logits)
        ok(b, b.route_scored(r, ptr(logits), e, ptr(bias), t, st, ptr(ids), ptr(gate), ptr(counts), ptr(offsets), ptr(perm), None, 0))
        ok(b, b.matmul_blocks(p1, ptr(hc), ptr(hs), ptr(c1), ptr(s1), None, t, st, ptr(mid)))
        ok(b, b.quantize_blocks(ptr(mid), 2 * inter, t, inter, 1, st, ptr(mc), inter, ptr(ms), inter // 128))
        ok(b, b.matmul_blocks(p2, ptr(mc), ptr(ms), ptr(c2), ptr(s2), ptr(routed), t, st, ptr(out)))
        ok(b, b.norm_residual(ns, ptr(xo), ptr(out), ptr(ones), None, ptr(ones), t, st, ptr(x2), ptr(h2), None, None))

    layer()
    torch.cuda.synchronize()
    want = [v.clone() for v in (xo, hh, hc, hs, ids, gate, perm, mid, mc, ms, out, x2, h2)]
    # every stage against the oracle on the stage's own inputs
    ref_ids, _, _, _, ref_perm = lo.route_scored(logits.cpu().numpy(), bias.cpu().numpy(), k, n_groups=4, top_groups=2, group_top=2, scale=2.5)
    assert np.array_equal(ids.cpu().numpy(), ref_ids) and np.array_equal(perm.cpu().numpy(), ref_perm)
    ref, size = lo.matmul(hc.cpu().numpy(), hs.cpu().numpy(), c1.cpu().numpy(), s1.cpu().numpy())
    assert np.all(np.abs(np64(mid) - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -15 * size)
    ref, size = lo.matmul(mc.cpu().numpy(), ms.cpu().numpy(), c2.cpu().numpy(), s2.cpu().numpy(), np64(routed))
    assert np.all(np.abs(np64(out) - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -15 * size)
    # the layer as a whole in 64 bits, without the codes: three roundings to e4m3 (input, weights, activations: 2^-4 at most,
    # uniform within it 2^-4 / sqrt(3) each) on the dense expert's part of the sum
    fx, fh, _ = lo.norm_residual(np64(x), np64(y), np64(ones), None, np64(ones), 0, 1e-6, 1.0)
    dense = lo.swiglu(fh @ w1.double().numpy().T) @ w2.double().numpy().T
    assert np.linalg.norm(np64(out) - np64(routed) - dense) <= 4 * 2.0 ** -4 * np.linalg.norm(dense) + 2.0 ** -8 * np.linalg.norm(np64(out))
    # captured and replayed on another stream, next to other work: the same bits
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        layer()
    for v in (xo, hh, hc, hs, ids, gate, perm, mid, mc, ms, out, x2, h2):
        v.zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for a, c in zip((xo, hh, hc, hs, ids, gate, perm, mid, mc, ms, out, x2, h2), want):
        assert torch.equal(a.view(torch.uint8), c.view(torch.uint8))


def test_products_on_two_streams(b):
    """Calls of different shapes that overlap share nothing."""
    shapes = [(1, 2048, 2048), (40, 1024, 2048), (200, 512, 1024), (9, 128, 8192), (1500, 768, 512)]
    sets = []
    for m, n, k in shapes:
        a, sa, w, sb = (t.to(DEV) for t in product_inputs(m, n, k))
        shape = b.ProductShape(n=n, k=k, out=0, a_stride=k, a_scale_stride=sa.shape[1], b_stride=k, b_scale_stride=sa.shape[1], add_stride=0, out_stride=n)
        sets.append((shape, a, sa, w, sb, m, torch.empty((m, n), dtype=torch.bfloat16, device=DEV)))
    streams = [torch.cuda.Stream() for _ in range(3)]
    want = []
    for shape, a, sa, w, sb, m, out in sets:
        ok(b, b.matmul_blocks(shape, ptr(a), ptr(sa), ptr(w), ptr(sb), None, m, stream(), ptr(out)))
        want.append(out.clone())
    torch.cuda.synchronize()
    outs = [[torch.empty_like(s[6]) for s in sets] for _ in streams]
    for _ in range(30):
        for st, o in zip(streams, outs):
            for (shape, a, sa, w, sb, m, _), out in zip(sets, o):
                ok(b, b.matmul_blocks(shape, ptr(a), ptr(sa), ptr(w), ptr(sb), None, m, st.cuda_stream, ptr(out)))
    torch.cuda.synchronize()
    for o in outs:
        for got, ref in zip(o, want):
            assert torch.equal(got.view(torch.int16), ref.view(torch.int16))


def border_ties(e, k, rng, pairs):
    """Logits of a token per pair (a, b): the K-1 largest are distinct, the two next are equal and at a and b, the others are distinct and lower."""
    t = len(pairs)
    logits = -1 - 0.001 * np.argsort(rng.random((t, e)), axis=1).astype(np.float32)
    for i, (x, y) in enumerate(pairs):
        others = rng.permutation(np.setdiff1d(np.arange(e), (x, y)))[:k - 1]
        logits[i, others] = 1 + 0.01 * np.arange(k - 1, dtype=np.float32)
        logits[i, [x, y]] = 0.5
    return logits


@pytest.mark.parametrize("k", [1, 8])
@pytest.mark.parametrize("e,groups,top_groups", [(40, 1, 1), (64, 1, 1), (128, 1, 1), (160, 1, 1), (256, 1, 1), (384, 1, 1), (512, 1, 1), (96, 3, 2), (256, 8, 4), (512, 16, 9), (504, 18, 9), (512, 32, 20)])
def test_route_ties_between_the_last_choice_and_the_next_one(b, e, groups, top_groups, k):
    """Without a bias, equal logits of which one is the K-th choice: the lower index has it, wherever the two lie."""
    rng = np.random.default_rng(11)
    near = [(x, x + 1) for x in range(e - 1)]                                  # (mostly of one lane)
    far = [tuple(sorted(rng.choice(e, 2, replace=False))) for _ in range(100)]
    logits = border_ties(e, k, rng, near + far)
    for group_top in (1, 2):
        for score in (0, 1):
            check_route(b, logits, None, top_k=k, score=score, n_groups=groups, top_groups=top_groups, group_top=group_top)


@pytest.mark.parametrize("e,groups,top_groups", [(64, 1, 1), (256, 1, 1), (512, 1, 1), (256, 8, 4), (504, 18, 9)])
def test_route_logits_that_were_bf16(b, e, groups, top_groups):
    """Logits of a bf16 gate: equal ones are common, and some of them lie at the border of the choice."""
    logits = torch.randn(3000, e, generator=torch.Generator().manual_seed(e)).to(torch.bfloat16).float().numpy()
    for score, group_top in ((0, 1), (1, 2)):
        check_route(b, logits, None, top_k=8, score=score, n_groups=groups, top_groups=top_groups, group_top=group_top)


@pytest.mark.parametrize("score", [0, 1])
def test_route_choices_next_to_the_smallest_numbers(b, score):
    """Scores that only the range of 64-bit numbers tells apart, down to its smallest ones, beside a bias that does not cover them."""
    check_route(b, np.float32([[0, -740, -720, -800]]), np.zeros(4, np.float32), top_k=3, score=score)
    rng = np.random.default_rng(12)
    for e, groups, top_groups in ((24, 1, 1), (64, 1, 1), (256, 1, 1), (64, 4, 2), (256, 8, 3)):
        logits = rng.uniform(-755, -690, size=(60, e)).astype(np.float32)
        logits[::3] = rng.uniform(-755, -80, size=(20, e)).astype(np.float32)
        logits[np.arange(60), rng.integers(0, e, 60)] = 0.0 if score == 0 else -690.0
        for bias in (np.zeros(e, np.float32), np.where(np.arange(e) % 3 == 0, -np.inf, 0).astype(np.float32)):
            for group_top in (1, 2):
                check_route(b, logits, bias, top_k=min(e // 2, 12), score=score, n_groups=groups, top_groups=top_groups, group_top=group_top, renormalise=0)
        for group_top in (1, 2):  # without a bias the two largest scores of a group are added all the same
            check_route(b, logits, None, top_k=min(e // 2, 12), score=score, n_groups=groups, top_groups=top_groups, group_top=group_top, renormalise=0)


@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("size,groups,top_groups", [(4, 8, 3), (8, 8, 4), (2, 32, 9), (16, 3, 1)])
def test_route_groups_whose_two_choices_cancel(b, score, size, groups, top_groups):
    """The two largest choices of a group are far larger than their sum, so that their fp32 forms are off by more than the sums are apart."""
    rng = np.random.default_rng(13)
    t, e = 150, size * groups
    for big in (10.0, 100.0, 3e4):
        bias = np.full((groups, size), -8 * big, np.float32)
        bias[:, 0], bias[:, 1] = big, -big
        bias = np.stack([rng.permutation(r) for r in bias]).reshape(-1)
        logits = rng.normal(size=(t, 1, 1)) + np.zeros((t, groups, size))
        logits = logits + rng.uniform(-1, 1, size=logits.shape) * (2.0 ** -rng.integers(4, 24, size=(t, 1, 1)))  # sums apart by 1e-7 to 0.1
        check_route(b, logits.reshape(t, e).astype(np.float32), bias, top_k=min(top_groups * size, 4), score=score, n_groups=groups, top_groups=top_groups,
                    group_top=2)


def test_products_on_pairs_beside_others(b):
    """Launches on pairs of CTAs in several streams, next to one another and to the smallest calls: they share nothing, tensor memory apart."""
    shapes = [(2304, 2048, 1024), (1, 128, 128), (16, 4096, 128), (1300, 4096, 384), (9, 2048, 512)]
    sets = []
    for m, n, k in shapes:
        a, sa, w, sb = (t.to(DEV) for t in product_inputs(m, n, k))
        shape = b.ProductShape(n=n, k=k, out=0, a_stride=k, a_scale_stride=sa.shape[1], b_stride=k, b_scale_stride=sa.shape[1], add_stride=0, out_stride=n)
        sets.append((shape, a, sa, w, sb, m, torch.empty((m, n), dtype=torch.bfloat16, device=DEV)))
    want = []
    for shape, a, sa, w, sb, m, out in sets:
        ok(b, b.matmul_blocks(shape, ptr(a), ptr(sa), ptr(w), ptr(sb), None, m, stream(), ptr(out)))
        want.append(out.clone())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    outs = [[torch.full_like(s[6], 7.0) for s in sets] for _ in streams]
    for r in range(40):
        for i, (st, o) in enumerate(zip(streams, outs)):
            for j in range(len(sets)):  # (each stream begins with another shape)
                shape, a, sa, w, sb, m, _ = sets[(i + j) % len(sets)]
                ok(b, b.matmul_blocks(shape, ptr(a), ptr(sa), ptr(w), ptr(sb), None, m, st.cuda_stream, ptr(o[(i + j) % len(sets)])))
    torch.cuda.synchronize()
    for o in outs:
        for got, ref in zip(o, want):
            assert torch.equal(got.view(torch.int16), ref.view(torch.int16))


@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("e,k,groups,top_groups,group_top", [(32, 32, 1, 1, 1), (7, 7, 1, 1, 1), (64, 32, 8, 4, 2), (256, 32, 8, 1, 1), (256, 32, 8, 1, 2), (60, 30, 4, 2, 1), (17, 17, 17, 17, 1)])
def test_route_takes_every_expert_that_stays(b, e, k, groups, top_groups, group_top, score):
    """As many experts wanted as the groups that stay have: nothing is left behind the last choice."""
    rng = np.random.default_rng(e + k)
    logits = (2 * rng.normal(size=(300, e))).astype(np.float32)
    masked = np.where(rng.random(e) < 0.3, -np.inf, 0.1).astype(np.float32)
    for bias in (None, (0.05 * rng.normal(size=e)).astype(np.float32), masked):
        check_route(b, logits, bias, top_k=k, score=score, n_groups=groups, top_groups=top_groups, group_top=group_top)


@pytest.mark.parametrize("renormalise", [0, 1])
@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("e,groups", [(64, 1), (256, 8), (512, 1)])
def test_route_weights_by_their_roundings(b, e, groups, score, renormalise):
    """The weights against the formulas' roundings, each in units of 2^-24 of the value (expf 2 units in the last place: 4, the fast quotient
    2: 4, an addition or product 1)."""
    rng = np.random.default_rng(14)
    logits = (3 * rng.normal(size=(400, e))).astype(np.float32)
    kw = dict(top_k=8, n_groups=groups, top_groups=max(1, groups // 2), group_top=min(2, groups), scale=2.5)
    ids, gate, *_ = run_route(b, logits, None, score=score, renormalise=renormalise, **kw)
    want_ids, want, *_ = lo.route_scored(logits, None, softmax=score == 0, renormalise=bool(renormalise), **kw)
    assert np.array_equal(ids, want_ids)
    chosen = np.take_along_axis(logits.astype(np.float64), ids, axis=1)
    below = logits.max(axis=1, keepdims=True) - chosen      # (a logit minus the largest one, rounded: as many units)
    if score == 1:
        units = 9.0                                          # exponential 4, one added 1, quotient 4
        units += 1 + (9 + 5 + 1 + 4 if renormalise else 0)   # scale; the sum's terms, five additions, 1e-20, quotient
    elif renormalise:
        units = (below + 4) + (below.max(axis=1, keepdims=True) + 4 + 5 + 1) + 4 + 1
    else:
        # the sum of all: its terms 15 together (a term x below the largest is 3 x + 4 off, and counts by exp(-x)), an addition per
        # expert of a lane and five
        units = (below + 4) + (15 + e / 32 + 5) + 4 + 1
    assert np.all(np.abs(gate - want) <= 1.01 * units * 2.0 ** -24 * want)


@pytest.mark.parametrize("h", [512, 333])
def test_norm_of_rows_beyond_fp32(b, h):
    """Finite rows whose sum of squares is not an fp32 number: their norms are zeros, their neighbours' what they are."""
    x = torch.randn(5, h, generator=torch.Generator().manual_seed(3))
    x[1] *= 1e25
    x[3, 7] = 3e38
    w = torch.ones(h, dtype=torch.bfloat16, device=DEV)
    for residual, kind in ((0, torch.bfloat16), (1, torch.float32)):
        xd, ho = x.to(kind).to(DEV), torch.full((5, h), 5.0, dtype=torch.bfloat16, device=DEV)
        shape = b.NormShape(hidden=h, residual=residual, gate_tokens=0, eps=1e-6, residual_scale=1.0, x_stride=h, y_stride=h, gate_stride=h, x_out_stride=h, h_stride=h,
                            codes_stride=h, scales_stride=-(-h // 128))
        ok(b, b.norm_residual(shape, ptr(xd), None, None, None, ptr(w), 5, stream(), None, ptr(ho), None, None))
        rms = (ho.double() ** 2).mean(dim=1).sqrt().cpu()
        assert not bool(ho[[1, 3]].any()) and bool(((rms[[0, 2, 4]] - 1).abs() <= 2.0 ** -8).all())
