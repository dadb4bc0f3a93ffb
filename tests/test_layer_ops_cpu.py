"""The operators around the routed experts, without a GPU: the oracle against hand-worked and brute-force values, and
every refusal of the entry points (nothing is launched for a refused call, so the pointers are only numbers)."""
import itertools
import math

import numpy as np
import pytest

from oracle import layer_ops as lo

P = 0x7f0000000000          # 16-byte aligned addresses, far apart; never read
STEP = 1 << 36


def ptr(i, off=0):
    return P + i * STEP + off


@pytest.fixture(scope="module")
def b():
    from paper_2609_33385_b200 import build
    build.build()
    from paper_2609_33385_b200 import binding
    binding.load()
    return binding


# ---- oracle --------------------------------------------------------------------------------------

def test_route_oracle_by_hand():
    # sigmoid(0) = .5, sigmoid(ln 3) = .75, sigmoid(-ln 3) = .25; the bias lifts expert 2 over expert 1
    l = np.array([[-math.log(3), 0.0, math.log(3), 0.0]], np.float32)
    ids, gate, counts, offsets, perm = lo.route_scored(l, None, 2)
    assert ids.tolist() == [[2, 1]] and np.allclose(gate, [[0.6, 0.4]])
    ids, gate, *_ = lo.route_scored(l, np.float32([0.6, 0, 0, 0]), 2, renormalise=False, scale=2.0)
    assert ids.tolist() == [[0, 2]] and np.allclose(gate, [[0.5, 1.5]])        # .25 + .6 leads, its weight is .25 * 2
    # groups (0, 1), (2, 3): the sum of two scores decides
    l = np.array([[3.0, -9.0, 1.0, 1.0]], np.float32)
    assert lo.route_scored(l, None, 1, n_groups=2, top_groups=1, group_top=1)[0].tolist() == [[0]]
    assert lo.route_scored(l, None, 1, n_groups=2, top_groups=1, group_top=2)[0].tolist() == [[2]]
    ids, _, counts, offsets, perm = lo.route_scored(np.float32([[0, 1, 0], [1, 0, 0]]), None, 2)
    assert ids.tolist() == [[1, 0], [0, 1]]
    assert counts.tolist() == [2, 2, 0] and offsets.tolist() == [0, 2, 4, 4] and perm.tolist() == [1, 2, 0, 3]


def test_route_oracle_against_enumeration():
    rng = np.random.default_rng(3)
    for _ in range(30):
        l, bias = rng.normal(size=(1, 8)).astype(np.float32), rng.normal(size=8).astype(np.float32) * np.float32(0.2)
        ids, *_ = lo.route_scored(l, bias, 3, n_groups=4, top_groups=2, group_top=2)
        c = 1 / (1 + np.exp(-l[0].astype(float))) + bias.astype(float)
        best = max(itertools.combinations(range(4), 2), key=lambda gs: sum(c[2 * g] + c[2 * g + 1] for g in gs))
        pool = [e for g in best for e in (2 * g, 2 * g + 1)]
        chosen = max(itertools.permutations(pool, 3), key=lambda p: tuple(c[list(p)]))
        assert ids[0].tolist() == list(chosen)


def test_e4m3_oracle():
    v = lo.E4M3
    assert v[0x7E] == 448 and v[0x01] == 2.0 ** -9 and v[0x08] == 2.0 ** -6 and np.isnan(v[0x7F])
    for c in range(256):
        if c & 0x7F != 0x7F:
            assert lo.e4m3_encode(np.array([v[c]]))[0] == c
    # halfway goes to the even code, beyond 448 is clamped
    mid = (v[0x10] + v[0x11]) / 2
    assert lo.e4m3_encode(np.array([mid, np.nextafter(mid, 9), 1e9, -460.0])).tolist() == [0x10, 0x11, 0x7E, 0xFE]


def test_norm_and_product_oracles_by_hand():
    x, y = np.array([[1.0, -1.0]]), np.array([[3.0, 4.0]])
    out, h, _ = lo.norm_residual(x, y, np.ones(2), np.array([[2.0, 0.5]]), np.ones(2), 0, 0.0, 0.5)
    r = math.sqrt(12.5)
    assert np.allclose(out, [[1 + 3 / r, -1 + 1 / r]]) and np.allclose((h * h).mean(), 1)
    codes = np.full((1, 130), 0x38, np.uint8)                    # 1.0
    got, size = lo.matmul(codes, [[2.0, 3.0]], codes, [[1.0, 10.0]], add=[[1.0]])
    assert got[0, 0] == 128 * 2 + 2 * 30 + 1 == size[0, 0]


# ---- refusals ------------------------------------------------------------------------------------

def _routing(b, **kw):
    base = dict(n_experts=64, top_k=8)
    base.update(kw)
    return b.Routing(**base)


@pytest.mark.parametrize("kw", [
    dict(n_experts=0), dict(n_experts=513), dict(top_k=0), dict(top_k=33), dict(top_k=9, n_experts=8), dict(score=2), dict(score=-1),
    dict(n_groups=0), dict(n_groups=3), dict(n_groups=64), dict(n_groups=8, top_groups=9), dict(top_groups=0), dict(group_top=0),
    dict(group_top=3), dict(n_groups=32, n_experts=32, top_groups=32, group_top=2), dict(n_groups=16, top_groups=1, top_k=5),
    dict(renormalise=2), dict(scale=math.inf), dict(scale=math.nan)])
def test_route_refuses_routing(b, kw):
    r = _routing(b, **kw)
    assert b.route_scored(r, ptr(0), 512, None, 4, 0, ptr(1), ptr(2), None, None, None, None, 0) == b.ERR_INVALID_ARG
    assert b.route_scored_scratch(r, 1 << 16) == 0


def _route(b, **kw):
    a = dict(r=_routing(b), logits=ptr(0), stride=64, bias=None, n=4, ids=ptr(1), gate=ptr(2), counts=ptr(3), offsets=ptr(4), perm=ptr(5),
             scratch=None, bytes=0)
    a.update(kw)
    return b.route_scored(a["r"], a["logits"], a["stride"], a["bias"], a["n"], 0, a["ids"], a["gate"], a["counts"], a["offsets"], a["perm"],
                          a["scratch"], a["bytes"])


def test_route_refuses_arguments(b):
    big = dict(n=1000, scratch=ptr(6))                     # 8000 assignments: sorted through scratch
    need = b.route_scored_scratch(_routing(b), 1000)
    assert need > 0 and b.route_scored_scratch(_routing(b), 512) == 0
    for kw in (dict(r=None), dict(n=-1), dict(stride=63), dict(stride=(1 << 36) + 1), dict(logits=None), dict(ids=None), dict(gate=None), dict(counts=None),
               dict(offsets=None), dict(perm=None), dict(logits=ptr(0, 2)), dict(ids=ptr(1, 1)), dict(gate=ptr(2, 2)),
               dict(bias=ptr(7, 2)), dict(counts=ptr(3, 2)), dict(offsets=ptr(4, 1)), dict(perm=ptr(5, 3)), dict(ids=ptr(0, 16)),
               dict(gate=ptr(1, 64)), dict(perm=ptr(2)), dict(bias=ptr(3)), dict(big, scratch=None, bytes=need),
               dict(big, bytes=need - 1), dict(big, bytes=need, scratch=ptr(6, 2)), dict(big, bytes=need, scratch=ptr(5, 16))):
        assert _route(b, **kw) == b.ERR_INVALID_ARG, kw
    assert _route(b, n=b.MAX_ROUTE_TOKENS + 1) == b.ERR_TOO_MANY_TOKENS
    assert _route(b, n=0, logits=None, ids=None, gate=None, counts=None, offsets=None, perm=None) == b.OLED_OK


def _norm(b, shape=None, **kw):
    s = dict(hidden=256, residual=b.BF16, gate_tokens=0, eps=1e-6, residual_scale=1.0, x_stride=256, y_stride=256, gate_stride=256,
             x_out_stride=256, h_stride=256, codes_stride=256, scales_stride=2)
    s.update(shape or {})
    a = dict(x=ptr(0), y=ptr(1), post=ptr(2), gate=ptr(3), pre=ptr(4), n=4, x_out=ptr(5), h=ptr(6), codes=ptr(7), scales=ptr(8))
    a.update(kw)
    return b.norm_residual(b.NormShape(**s) if shape != "none" else None, a["x"], a["y"], a["post"], a["gate"], a["pre"], a["n"], 0, a["x_out"],
                           a["h"], a["codes"], a["scales"])


@pytest.mark.parametrize("shape", [
    dict(hidden=0), dict(hidden=16385), dict(residual=2), dict(gate_tokens=-1), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan),
    dict(eps=math.inf), dict(residual_scale=math.nan), dict(x_stride=255), dict(y_stride=255), dict(gate_stride=0), dict(x_out_stride=1),
    dict(h_stride=255), dict(codes_stride=255), dict(scales_stride=1), dict(x_stride=1 << 60), dict(scales_stride=1 << 37)])
def test_norm_refuses_shape(b, shape):
    assert _norm(b, shape) == b.ERR_INVALID_ARG


def test_norm_refuses_arguments(b):
    for kw in (dict(n=-1), dict(x=None), dict(y=None), dict(y=None, post=None), dict(y=None, gate=None), dict(pre=None),
               dict(h=None, codes=None, scales=None), dict(codes=None), dict(scales=None),
               dict(x_out=None, h=None, codes=None, scales=None, pre=None), dict(x=ptr(0, 1)), dict(y=ptr(1, 1)), dict(post=ptr(2, 1)),
               dict(gate=ptr(3, 1)), dict(pre=ptr(4, 1)), dict(x_out=ptr(5, 1)), dict(h=ptr(6, 1)), dict(scales=ptr(8, 2)),
               dict(x_out=ptr(0, 2)), dict(h=ptr(1, 512)), dict(x_out=ptr(2)), dict(h=ptr(3)), dict(codes=ptr(0)), dict(codes=ptr(1)),
               dict(scales=ptr(4)), dict(h=ptr(5)), dict(codes=ptr(6)), dict(scales=ptr(7))):
        assert _norm(b, **kw) == b.ERR_INVALID_ARG, kw
    assert _norm(b, dict(residual=b.FP32), x=ptr(0, 2)) == b.ERR_INVALID_ARG
    assert _norm(b, dict(residual=b.FP32), h=ptr(0)) == b.ERR_INVALID_ARG            # h in place of an fp32 x
    assert _norm(b, dict(x_stride=512), x_out=ptr(0)) == b.ERR_INVALID_ARG           # the same address, another stride
    assert b.norm_residual(None, *[ptr(i) for i in range(5)], 4, 0, ptr(5), ptr(6), None, None) == b.ERR_INVALID_ARG
    assert _norm(b, n=0, x=None, y=None, post=None, gate=None, pre=None, x_out=None, h=None, codes=None, scales=None) == b.OLED_OK


def test_quantize_refuses(b):
    def q(**kw):
        a = dict(x=ptr(0), xs=256, rows=4, cols=256, sw=0, codes=ptr(1), cs=256, scales=ptr(2), ss=2)
        a.update(kw)
        return b.quantize_blocks(a["x"], a["xs"], a["rows"], a["cols"], a["sw"], 0, a["codes"], a["cs"], a["scales"], a["ss"])
    for kw in (dict(rows=-1), dict(cols=0), dict(cols=264), dict(cols=16400, xs=16400, cs=16400, ss=200), dict(sw=2), dict(xs=248),
               dict(xs=257), dict(xs=1 << 40), dict(sw=1), dict(cs=240), dict(cs=264), dict(ss=1), dict(x=None), dict(codes=None), dict(scales=None),
               dict(x=ptr(0, 8)), dict(codes=ptr(1, 8)), dict(scales=ptr(2, 2)), dict(codes=ptr(0)), dict(scales=ptr(0, 64)),
               dict(scales=ptr(1, 64))):
        assert q(**kw) == b.ERR_INVALID_ARG, kw
    assert q(rows=0, x=None, codes=None, scales=None) == b.OLED_OK


def test_matmul_refuses(b):
    def mm(m=4, **kw):
        s = dict(n=256, k=256, out=b.BF16, a_stride=256, a_scale_stride=2, b_stride=256, b_scale_stride=2, add_stride=256, out_stride=256)
        a = dict(a=ptr(0), sa=ptr(1), b=ptr(2), sb=ptr(3), add=None, out=ptr(4))
        s.update({k: v for k, v in kw.items() if k in s and k not in ("out",)})
        if "type" in kw:
            s["out"] = kw["type"]
        a.update({k: v for k, v in kw.items() if k in a})
        return b.matmul_blocks(b.ProductShape(**s), a["a"], a["sa"], a["b"], a["sb"], a["add"], m, 0, a["out"])
    for kw in (dict(m=-1), dict(n=0), dict(n=(1 << 20) + 1, out_stride=1 << 21), dict(k=0), dict(k=24), dict(k=16400, a_stride=16400, b_stride=16400, a_scale_stride=200, b_scale_stride=200),
               dict(type=2), dict(a_stride=240), dict(a_stride=264), dict(b_stride=240), dict(b_stride=264), dict(a_scale_stride=1), dict(b_scale_stride=1),
               dict(out_stride=255), dict(add=ptr(5), add_stride=255), dict(a=None), dict(sa=None), dict(b=None), dict(sb=None), dict(out=None),
               dict(a=ptr(0, 8)), dict(b=ptr(2, 8)), dict(sa=ptr(1, 2)), dict(sb=ptr(3, 2)), dict(add=ptr(5, 1)), dict(out=ptr(4, 1)),
               dict(type=1, out=ptr(4, 2)), dict(out=ptr(0)), dict(out=ptr(1)), dict(out=ptr(2)), dict(out=ptr(3)), dict(add=ptr(4, 64)),
               dict(type=1, add=ptr(4)), dict(a_stride=1 << 40), dict(out_stride=1 << 62)):
        assert mm(**kw) == b.ERR_INVALID_ARG, kw
    assert b.matmul_blocks(None, ptr(0), ptr(1), ptr(2), ptr(3), None, 4, 0, ptr(4)) == b.ERR_INVALID_ARG
    assert mm(m=b.MAX_ROUTE_TOKENS + 1) == b.ERR_TOO_MANY_TOKENS
    assert mm(m=0, a=None, sa=None, b=None, sb=None, out=None) == b.OLED_OK
