"""The operators around the routed experts of an MoE layer, as cases for timing and comparison.

``route``     ``binding.route_scored``: from gate logits to expert ids and gate weights (softmax or
              sigmoid scores, a bias that takes part in the choice only, groups of experts, top-k,
              renormalised and scaled weights), with counts, offsets and the stable order by expert
``norm``      ``binding.norm_residual``: the norm behind a block, its gate, the residual scale, the
              residual addition and the norm in front of the next block
``product``   ``binding.matmul_blocks``: a matrix product of e4m3 codes, one fp32 scale per row
              and 128 columns of the left operand and per 128 x 128 block of the right one
``quantize``  ``binding.quantize_blocks``: bf16 rows, or SwiGLU of rows, to codes and scales

``run`` computes them in elementary torch operations, or, where ``own`` is true, with the library.
"""
import math

import torch

own = False

BLOCK = 128
E4M3_MAX = 448.0
TINY = 2.0 ** -100  # blocks whose largest magnitude is below it are scaled as if it were this


# ---- cases -----------------------------------------------------------------------------------------

def _route(name, tokens, experts, top_k, score="softmax", bias=False, groups=1, top_groups=1, group_top=1, renorm=True,
           scale=1.0):
    return _named(name, dict(op="route", tokens=tokens, experts=experts, top_k=top_k, score=score, bias=bias, groups=groups,
                             top_groups=top_groups, group_top=group_top, renorm=renorm, scale=scale))


def _norm(name, tokens, hidden, residual="bf16", post=True, gate_tokens=-1, out="bf16", scale=1.0):
    """gate_tokens: tokens that share a row of gates, 0: one row for all of them, -1: no gates."""
    return _named(name, dict(op="norm", tokens=tokens, hidden=hidden, residual=residual, post=post, gate_tokens=gate_tokens,
                             out=out, scale=scale))


def _product(name, m, n, k, out="bf16", add=False):
    return _named(name, dict(op="product", m=m, n=n, k=k, out=out, add=add))


def _quantize(name, rows, cols, swiglu):
    return _named(name, dict(op="quantize", rows=rows, cols=cols, swiglu=swiglu))


def _named(name, c):
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # Token-by-token decoding on the 64-expert stack: latency.
        _route("route 1 token", 1, 64, 8),
        # A ragged batch of blocks on the 128-expert stack, with a bias that keeps the experts' loads even.
        _route("route 250 tokens sigmoid", 250, 128, 8, score="sigmoid", bias=True),
        # The prompts of a batch, 256 experts in eight groups of which a token may use four.
        _route("route 32768 tokens in groups", 32768, 256, 8, score="sigmoid", bias=True, groups=8, top_groups=4,
               group_top=2, scale=2.5),
        # One token between two layers of the 2048-wide stack: latency.
        _norm("norm 1 token", 1, 2048),
        # A ragged batch of blocks of 32, a row of gates per block, the result for the gate and for fp8 products.
        _norm("norm 250 tokens fp8", 250, 2048, gate_tokens=32, out="both"),
        # A batch of prompts on the 4096-wide layer, the residual stream kept in fp32.
        _norm("norm 16384 tokens", 16384, 4096, residual="fp32", gate_tokens=0, scale=0.5),
        # One token through the gate and up projections of a dense expert (intermediate 1024): the weights' bytes.
        _product("product 1 token", 1, 2048, 2048),
        # A block of 32 through its down projection, added to the routed experts' sum.
        _product("product 32 tokens added", 32, 2048, 1024, add=True),
        # A ragged batch of blocks, fp32 results.
        _product("product 250 tokens fp32", 250, 4096, 2048, out="fp32"),
        # A batch of prompts on the 4096-wide layer: the tensor cores.
        _product("product 8192 tokens", 8192, 4096, 4096),
        # The activations of a block between a dense expert's two products.
        _quantize("quantize 32 tokens swiglu", 32, 1024, True),
        # A batch of prompts in front of a product.
        _quantize("quantize 16384 tokens", 16384, 4096, False),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("route", "norm", "product", "product", "quantize"))
    if op == "route":
        groups = rng.choice((1, 1, 2, 4, 8))
        experts = groups * rng.randint(max(2, 8 // groups), 384 // groups)
        top_groups = rng.randint(1, groups)
        return _route(None, _spread(rng, 1, 21000), experts, rng.randint(1, min(16, top_groups * (experts // groups))),
                      score=rng.choice(("softmax", "sigmoid")), bias=rng.random() < 0.6, groups=groups,
                      top_groups=top_groups, group_top=rng.choice((1, 2)), renorm=rng.random() < 0.7,
                      scale=rng.choice((1.0, 2.5)))
    if op == "norm":
        tokens, hidden = _spread(rng, 1, 16384), rng.choice((BLOCK * rng.randint(1, 32), 8 * rng.randint(16, 512), rng.randint(100, 4096)))
        return _norm(None, tokens, hidden, residual=rng.choice(("bf16", "fp32")), post=rng.random() < 0.7,
                     gate_tokens=rng.choice((-1, 0, 1, 32)), out=rng.choice(("bf16", "bf16", "fp8", "both")),
                     scale=rng.choice((1.0, 0.5)))
    if op == "product":
        m, n = _spread(rng, 1, 8192), rng.choice((BLOCK * rng.randint(1, 32), rng.randint(64, 4096)))
        return _product(None, m, n, 16 * rng.randint(4, 256), out=rng.choice(("bf16", "bf16", "fp32")),
                        add=rng.random() < 0.3)
    swiglu = rng.random() < 0.5
    return _quantize(None, _spread(rng, 1, 16384 // (2 if swiglu else 1)), 16 * rng.randint(4, 256), swiglu)


def work(case):
    c = case
    if c["op"] == "route":
        t, e, k = c["tokens"], c["experts"], c["top_k"]
        return {"bytes": 4.0 * t * e + 4.0 * e * c["bias"] + 12.0 * t * k + 4.0 * (2 * e + 1), "flops": 12.0 * t * e}
    if c["op"] == "norm":
        t, h = c["tokens"], c["hidden"]
        item = 2 if c["residual"] == "bf16" else 4
        gates = 0 if c["gate_tokens"] < 0 else 1 if c["gate_tokens"] == 0 else -(-t // c["gate_tokens"])
        out = (2 if c["out"] in ("bf16", "both") else 0) + (1 + 4.0 / BLOCK if c["out"] in ("fp8", "both") else 0)
        return {"bytes": t * h * (2.0 * item + 2 + out) + 2.0 * h * (1 + c["post"] + gates), "flops": 10.0 * t * h}
    if c["op"] == "product":
        m, n, k = c["m"], c["n"], c["k"]
        blocks = -(-k // BLOCK)
        item = 2 if c["out"] == "bf16" else 4
        return {"bytes": 1.0 * m * k + 1.0 * n * k + 4.0 * m * blocks + 4.0 * -(-n // BLOCK) * blocks +
                m * n * (item + 2.0 * c["add"]), "flops": 2.0 * m * n * k}
    r, k = c["rows"], c["cols"]
    return {"bytes": r * k * (4.0 if c["swiglu"] else 2.0) + r * k + 4.0 * r * -(-k // BLOCK),
            "flops": r * k * (12.0 if c["swiglu"] else 4.0)}


# ---- inputs ----------------------------------------------------------------------------------------

def _randn(gen, *shape):
    return torch.randn(shape, device="cuda", generator=gen)


def _rows(gen, rows, cols):
    """Activations: N(0, 1), a few channels eight times as large, as hidden states have them."""
    x = _randn(gen, rows, cols)
    x[:, ::97] *= 8.0
    return x


def _codes(w):
    """e4m3 codes and scales of a weight matrix by blocks of 128 x 128, as a checkpoint holds them."""
    n, k = w.shape
    nb, kb = -(-n // BLOCK), -(-k // BLOCK)
    full = torch.zeros((nb * BLOCK, kb * BLOCK), device=w.device)
    full[:n, :k] = w
    scale = full.view(nb, BLOCK, kb, BLOCK).abs().amax(dim=(1, 3)).clamp_min(TINY) / E4M3_MAX
    codes = (full.view(nb, BLOCK, kb, BLOCK) / scale[:, None, :, None]).view(nb * BLOCK, kb * BLOCK)[:n, :k]
    return codes.clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).contiguous(), scale.contiguous()


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}

    def out(shape, dtype):
        return torch.zeros(shape, dtype=dtype, device="cuda")

    if c["op"] == "route":
        t, e, k = c["tokens"], c["experts"], c["top_k"]
        s["logits"] = _randn(gen, t, e) + 0.5 * _randn(gen, e)  # some experts are more popular
        s["bias"] = 0.1 * _randn(gen, e) if c["bias"] else None
        s["ids"], s["gate"] = out((t, k), torch.int32), out((t, k), torch.float32)
        s["counts"], s["offsets"], s["perm"] = (out((n,), torch.int32) for n in (e, e + 1, t * k))
    elif c["op"] == "norm":
        t, h = c["tokens"], c["hidden"]
        kind = torch.bfloat16 if c["residual"] == "bf16" else torch.float32
        s["x"] = (3.0 * _rows(gen, t, h)).to(kind)
        s["y"] = _randn(gen, t, h).to(torch.bfloat16)
        s["post"] = (1.0 + 0.1 * _randn(gen, h)).to(torch.bfloat16) if c["post"] else None
        s["pre"] = (1.0 + 0.1 * _randn(gen, h)).to(torch.bfloat16)
        rows = 1 if c["gate_tokens"] == 0 else -(-t // max(1, c["gate_tokens"]))
        s["gates"] = (0.5 * _randn(gen, rows, h)).to(torch.bfloat16) if c["gate_tokens"] >= 0 else None
        s["x_out"] = out((t, h), kind)
        s["h"] = out((t, h), torch.bfloat16) if c["out"] != "fp8" else None
        s["codes"] = out((t, h), torch.float8_e4m3fn) if c["out"] != "bf16" else None
        s["scales"] = out((t, -(-h // BLOCK)), torch.float32) if c["out"] != "bf16" else None
    elif c["op"] == "product":
        m, n, k = c["m"], c["n"], c["k"]
        a = _rows(gen, m, k)
        kb = -(-k // BLOCK)
        full = torch.zeros((m, kb * BLOCK), device="cuda")
        full[:, :k] = a
        s["a_scale"] = full.view(m, kb, BLOCK).abs().amax(dim=2).clamp_min(TINY) / E4M3_MAX
        s["a"] = (full.view(m, kb, BLOCK) / s["a_scale"][:, :, None]).view(m, -1)[:, :k].clamp(-E4M3_MAX, E4M3_MAX).to(
            torch.float8_e4m3fn).contiguous()
        s["b"], s["b_scale"] = _codes(0.02 * _randn(gen, n, k))
        s["add"] = _randn(gen, m, n).to(torch.bfloat16) if c["add"] else None
        s["out"] = out((m, n), torch.bfloat16 if c["out"] == "bf16" else torch.float32)
    else:
        r, k = c["rows"], c["cols"]
        s["x"] = _rows(gen, r, 2 * k if c["swiglu"] else k).to(torch.bfloat16)
        s["codes"] = out((r, k), torch.float8_e4m3fn)
        s["scales"] = out((r, -(-k // BLOCK)), torch.float32)
    return s


# ---- the plain form --------------------------------------------------------------------------------

def _plain_choice(x, c):
    """Order of the last axis's best c, ties to the lowest index."""
    return torch.sort(x, dim=-1, descending=True, stable=True)[1][..., :c]


def _plain_route(s):
    c = s["case"]
    t, e, k, groups = c["tokens"], c["experts"], c["top_k"], c["groups"]
    x = s["logits"].double()  # (what stands next to a border is told apart in 64 bits)
    if c["score"] == "sigmoid":
        score = 1.0 / (1.0 + torch.exp(-x))
    else:
        z = torch.exp(x - x.max(dim=1, keepdim=True)[0])
        score = z / z.sum(dim=1, keepdim=True)
    value = score if s["bias"] is None else score + s["bias"].double()
    order = x if s["bias"] is None else value  # (scores rise with the logits)
    if groups > 1:
        if c["group_top"] == 1:
            best = order.view(t, groups, -1).max(dim=2)[0]
        else:
            best = torch.sort(value.view(t, groups, -1), dim=2, descending=True)[0][:, :, :2].sum(dim=2)
        allowed = torch.zeros((t, groups), dtype=torch.bool, device=x.device)
        allowed.scatter_(1, _plain_choice(best, c["top_groups"]), True)
        order = torch.where(allowed.repeat_interleave(e // groups, dim=1), order, -math.inf)
    ids = _plain_choice(order, k)
    gate = torch.gather(score, 1, ids)
    if c["renorm"]:
        gate = gate / (gate.sum(dim=1, keepdim=True) + 1e-20)
    flat = ids.reshape(-1)
    counts = torch.bincount(flat, minlength=e)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    perm = torch.sort(flat, stable=True)[1]
    return {"ids": ids.int(), "gate": (gate * c["scale"]).float(), "counts": counts.int(), "offsets": offsets.int(),
            "perm": perm.int()}


def _plain_codes(v):
    """fp32 rows to e4m3 codes and one scale per 128 columns."""
    r, k = v.shape
    kb = -(-k // BLOCK)
    full = torch.nn.functional.pad(v, (0, kb * BLOCK - k)).view(r, kb, BLOCK)
    big = full.abs().amax(dim=2).clamp_min(TINY)
    codes = (full * (E4M3_MAX / big)[:, :, None]).clamp(-E4M3_MAX, E4M3_MAX).view(r, -1)[:, :k]
    return codes.to(torch.float8_e4m3fn), big / E4M3_MAX


def _plain_rms(v):
    return v * torch.rsqrt(v.square().mean(dim=1, keepdim=True) + 1e-6)


def _plain_norm(s):
    c = s["case"]
    z = s["y"].float()
    if s["post"] is not None:
        z = _plain_rms(z) * s["post"].float()
    if s["gates"] is not None:
        gates = s["gates"].float()
        z = z * (gates if c["gate_tokens"] == 0 else gates.repeat_interleave(c["gate_tokens"], dim=0)[:c["tokens"]])
    x = s["x"].float() + c["scale"] * z
    h = _plain_rms(x) * s["pre"].float()
    out = {"x": x.to(s["x"].dtype)}
    if s["h"] is not None:
        out["h"] = h.to(torch.bfloat16)
    if s["codes"] is not None:
        out["codes"], out["scales"] = _plain_codes(h)
    return out


def _plain_product(s):
    c = s["case"]
    m, n, k = c["m"], c["n"], c["k"]
    a = s["a"].float() * s["a_scale"].repeat_interleave(BLOCK, dim=1)[:, :k]
    b = s["b"].float() * s["b_scale"].repeat_interleave(BLOCK, dim=0)[:n].repeat_interleave(BLOCK, dim=1)[:, :k]
    out = a @ b.t()
    if s["add"] is not None:
        out = out + s["add"].float()
    return out.to(s["out"].dtype)


def _plain_quantize(s):
    x = s["x"].float()
    if s["case"]["swiglu"]:
        gate, up = x.chunk(2, dim=1)
        x = gate / (1.0 + torch.exp(-gate)) * up
    codes, scales = _plain_codes(x)
    return {"codes": codes, "scales": scales}


# ---- the library -----------------------------------------------------------------------------------

def _ptr(t):
    return None if t is None else t.data_ptr()


def _own(s):
    from paper_2609_33385_b200 import binding

    c = s["case"]
    stream = torch.cuda.current_stream().cuda_stream
    if c["op"] == "route":
        if "routing" not in s:  # what a program keeps: the layer's routing and the scratch it asks for
            s["routing"] = binding.Routing(n_experts=c["experts"], top_k=c["top_k"],
                                           score=binding.SCORE_SIGMOID if c["score"] == "sigmoid" else binding.SCORE_SOFTMAX,
                                           n_groups=c["groups"], top_groups=c["top_groups"], group_top=c["group_top"],
                                           renormalise=1 if c["renorm"] else 0, scale=c["scale"])
            s["scratch"] = torch.empty(max(16, binding.route_scored_scratch(s["routing"], c["tokens"])), dtype=torch.uint8,
                                       device="cuda")
        rc = binding.route_scored(s["routing"], s["logits"].data_ptr(), c["experts"], _ptr(s["bias"]), c["tokens"], stream,
                                  s["ids"].data_ptr(), s["gate"].data_ptr(), s["counts"].data_ptr(), s["offsets"].data_ptr(),
                                  s["perm"].data_ptr(), s["scratch"].data_ptr(), s["scratch"].numel())
        got = {"ids": s["ids"], "gate": s["gate"], "counts": s["counts"], "offsets": s["offsets"], "perm": s["perm"]}
    elif c["op"] == "norm":
        if "shape" not in s:
            h = c["hidden"]
            s["shape"] = binding.NormShape(hidden=h, residual=binding.FP32 if c["residual"] == "fp32" else binding.BF16,
                                           gate_tokens=max(0, c["gate_tokens"]), eps=1e-6, residual_scale=c["scale"], x_stride=h,
                                           y_stride=h, gate_stride=h, x_out_stride=h, h_stride=h, codes_stride=h,
                                           scales_stride=-(-h // BLOCK))
        rc = binding.norm_residual(s["shape"], s["x"].data_ptr(), s["y"].data_ptr(), _ptr(s["post"]), _ptr(s["gates"]),
                                   s["pre"].data_ptr(), c["tokens"], stream, s["x_out"].data_ptr(), _ptr(s["h"]),
                                   _ptr(s["codes"]), _ptr(s["scales"]))
        got = {"x": s["x_out"]}
        got.update((n, s[n]) for n in ("h", "codes", "scales") if s[n] is not None)
    elif c["op"] == "product":
        if "shape" not in s:
            kb = -(-c["k"] // BLOCK)
            s["shape"] = binding.ProductShape(n=c["n"], k=c["k"], out=binding.FP32 if c["out"] == "fp32" else binding.BF16,
                                              a_stride=c["k"], a_scale_stride=kb, b_stride=c["k"], b_scale_stride=kb,
                                              add_stride=c["n"], out_stride=c["n"])
        rc = binding.matmul_blocks(s["shape"], s["a"].data_ptr(), s["a_scale"].data_ptr(), s["b"].data_ptr(),
                                      s["b_scale"].data_ptr(), _ptr(s["add"]), c["m"], stream, s["out"].data_ptr())
        got = s["out"]
    else:
        k = c["cols"]
        rc = binding.quantize_blocks(s["x"].data_ptr(), s["x"].shape[1], c["rows"], k, 1 if c["swiglu"] else 0, stream,
                                        s["codes"].data_ptr(), k, s["scales"].data_ptr(), -(-k // BLOCK))
        got = {"codes": s["codes"], "scales": s["scales"]}
    if rc != 0:
        raise RuntimeError("%s: %s" % (c["op"], binding.strerror(rc)))
    return got


def run(s):
    if own:
        return _own(s)
    return {"route": _plain_route, "norm": _plain_norm, "product": _plain_product, "quantize": _plain_quantize}[s["case"]["op"]](s)


# ---- the definition in 64 bits ---------------------------------------------------------------------

def _exact_route(s):
    c = s["case"]
    t, e, k = c["tokens"], c["experts"], c["top_k"]
    size = e // c["groups"]
    x = s["logits"].double()
    score = torch.sigmoid(x) if c["score"] == "sigmoid" else torch.softmax(x, dim=1)
    key = x.clone() if s["bias"] is None else score + s["bias"].double()
    value = score if s["bias"] is None else key
    if c["groups"] > 1:
        per = (key if c["group_top"] == 1 else value).reshape(t, c["groups"], size).topk(c["group_top"], dim=2)[0].sum(dim=2)
        # a group stays if fewer than top_groups others come before it
        g = torch.arange(c["groups"], device=x.device)
        ahead = (per[:, None, :] > per[:, :, None]) | ((per[:, None, :] == per[:, :, None]) & (g[None, None, :] < g[None, :, None]))
        drop = ahead.sum(dim=2) >= c["top_groups"]
        key[drop[:, :, None].expand(t, c["groups"], size).reshape(t, e)] = -math.inf
    ids = torch.empty((t, k), dtype=torch.int64, device=x.device)
    rows = torch.arange(t, device=x.device)
    left = torch.ones((t, e), dtype=torch.bool, device=x.device)
    index = torch.arange(e, device=x.device)
    for j in range(k):  # the largest that is left, the lowest index where several are
        top = torch.where(left, key, -math.inf).amax(dim=1, keepdim=True)
        ids[:, j] = torch.where(left & (key == top), index, e).amin(dim=1)
        left[rows, ids[:, j]] = False
    gate = score[rows[:, None], ids]
    if c["renorm"]:
        gate = gate / (gate.sum(dim=1, keepdim=True) + 1e-20)
    hot = torch.zeros((e,), dtype=torch.int64, device=x.device)
    hot.index_add_(0, ids.reshape(-1), torch.ones(t * k, dtype=torch.int64, device=x.device))
    place = ids.reshape(-1) * (t * k) + torch.arange(t * k, device=x.device)
    return {"ids": ids.int(), "gate": gate * c["scale"], "counts": hot.int(),
            "offsets": torch.cat([hot.new_zeros(1), torch.cumsum(hot, 0)]).int(), "perm": torch.argsort(place).int()}


def _exact_codes(v):
    """The codes as the numbers that they are, and the scales."""
    parts, scales = [], []
    for at in range(0, v.shape[1], BLOCK):
        b = v[:, at:at + BLOCK]
        big = torch.clamp(b.abs().max(dim=1)[0], min=TINY)
        scaled = b * (E4M3_MAX / big)[:, None]
        # three fraction bits above 2^-6, steps of 2^-9 below
        step = torch.exp2(torch.clamp(torch.floor(torch.log2(torch.clamp(scaled.abs(), min=2.0 ** -20))), min=-6.0) - 3.0)
        parts.append(torch.clamp(torch.round(scaled / step) * step, -E4M3_MAX, E4M3_MAX))
        scales.append(big / E4M3_MAX)
    return torch.cat(parts, dim=1), torch.stack(scales, dim=1)


def _exact_norm(s):
    c = s["case"]
    t = c["tokens"]
    step = s["y"].double()
    if c["post"]:
        step = step / torch.sqrt((step * step).sum(dim=1, keepdim=True) / c["hidden"] + 1e-6) * s["post"].double()
    if c["gate_tokens"] >= 0:
        row = torch.arange(t, device=step.device) // c["gate_tokens"] if c["gate_tokens"] > 0 else torch.zeros(
            t, dtype=torch.int64, device=step.device)
        step = step * s["gates"].double()[row]
    x = s["x"].double() + step * c["scale"]
    h = x / torch.sqrt((x * x).sum(dim=1, keepdim=True) / c["hidden"] + 1e-6) * s["pre"].double()
    out = {"x": x}
    if c["out"] in ("bf16", "both"):
        out["h"] = h
    if c["out"] in ("fp8", "both"):
        out["codes"], out["scales"] = _exact_codes(h)
    return out


def _exact_product(s):
    c = s["case"]
    out = torch.zeros((c["m"], c["n"]), dtype=torch.float64, device="cuda") if not c["add"] else s["add"].double()
    of_row = torch.arange(c["n"], device="cuda") // BLOCK
    for i, at in enumerate(range(0, c["k"], BLOCK)):
        part = s["a"][:, at:at + BLOCK].double() @ s["b"][:, at:at + BLOCK].double().t()
        out += part * s["a_scale"][:, i:i + 1].double() * s["b_scale"][of_row, i].double()[None, :]
    return out


def _exact_quantize(s):
    x, k = s["x"].double(), s["case"]["cols"]
    if s["case"]["swiglu"]:
        x = x[:, :k] * torch.sigmoid(x[:, :k]) * x[:, k:]
    codes, scales = _exact_codes(x)
    return {"codes": codes, "scales": scales}


def exact(case, seed):
    s = prepare(case, seed)
    return {"route": _exact_route, "norm": _exact_norm, "product": _exact_product, "quantize": _exact_quantize}[case["op"]](s)
