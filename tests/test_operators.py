"""The operators around the block, on the CPU: their oracles against brute force
and against differences, the error model of the decode linear emulated in IEEE
float32, and every refusal of the C ABI (validation returns before anything is
enqueued; the pointers below are never dereferenced)."""

import ctypes as C
import math

import numpy as np
import pytest

from oracle import mxmoe_oracle as O
from paper_2505_05799_amd import mxmoe as M
from paper_2505_05799_amd import workloads as W
from tests import tolerance as TL


@pytest.fixture(scope="module")
def lib():
    return M.load_library()


def at(mb, off=0):             # an address; the buffers of the calls below lie MB apart
    return C.c_void_p((mb << 20) + off)


# ------------------------------------------------------------------- oracles
@pytest.mark.parametrize("act", ["bf16", "fp16"])
def test_norm_oracle_brute_force(act):
    rng = np.random.default_rng(3)
    x = O.act_values(W.f64_to_act(rng.standard_normal((5, 19)) * 3, act), act)
    r = O.act_values(W.f64_to_act(rng.standard_normal((5, 19)), act), act)
    w = O.act_values(W.f64_to_act(1 + 0.1 * rng.standard_normal(19), act), act)
    x[3], r[3] = 0.0, 0.0
    y, z, y64 = O.add_rms_norm(x, r, w, act, 1e-6)
    for i in range(5):
        ss = 0.0
        for j in range(19):
            zz = float(O.round_to_act(np.float64(np.float32(x[i, j] + r[i, j])), act))
            assert zz == z[i, j]
            ss += zz * zz
        root = 1.0 / math.sqrt(ss / 19 + 1e-6)
        for j in range(19):
            want = z[i, j] * root * w[j]
            assert abs(y64[i, j] - want) <= 1e-14 * abs(want)
            # three roundings to fp32 (the factor, two products) and one to the dtype
            assert abs(y[i, j] - want) <= TL.slot_bound(np.float64(want), 3.5 * TL.U32 * abs(want), act) + 1e-300
    assert not y[3].any()
    # a row of equal values v has y = v / |v| (eps aside)
    y, _, _ = O.add_rms_norm(np.full((1, 64), -2.0), None, np.ones(64), act, 1e-30)
    assert np.all(y == -1.0)


def test_balance_oracle_gradient_is_the_difference():
    rng = np.random.default_rng(11)
    T, E, k = 13, 7, 3
    l = rng.standard_normal((T, E)) * 2
    ids = np.argsort(-l, axis=1)[:, :k]
    ids[2, 1] = ids[2, 0]                       # the same expert twice counts twice
    ids[4, 0] = -1                              # not counted
    mask = np.ones(T, bool)
    mask[[5, 9]] = False
    L, c, p, g = O.balance_loss(l, ids, mask, alpha=0.3)
    assert c.sum() == 11 * k - 1 and abs(p.sum() - 1) < 1e-12
    assert not g[~mask].any()
    assert np.abs(g.sum(axis=1)).max() < 1e-15    # a shift of a token's logits changes nothing
    h = 1e-5
    for t in range(T):
        for e in range(E):
            d = np.zeros_like(l)
            d[t, e] = h
            lp = O.balance_loss(l + d, ids, mask, 0.3, counts=c)[0]
            lm = O.balance_loss(l - d, ids, mask, 0.3, counts=c)[0]
            assert abs((lp - lm) / (2 * h) - g[t, e]) <= 1e-9


def test_balance_oracle_closed_forms():
    # even counts and even probabilities: alpha; everything on one expert: alpha E
    l = np.zeros((8, 4))
    ids = np.arange(8)[:, None] % 4
    assert abs(O.balance_loss(l, ids, None, 2.0)[0] - 2.0) < 1e-12
    l[:, 1] = 200.0
    assert abs(O.balance_loss(l, np.ones((8, 1), int), None, 1.0)[0] - 4.0) < 1e-12
    assert O.balance_loss(l, ids, np.zeros(8, bool))[0] == 0.0


# ------------------------------------------- error model of the decode linear
@pytest.mark.parametrize("act", ["bf16", "fp16"])
@pytest.mark.parametrize("k", [128, 2048, 14336])
def test_decode_w4_error_model(act, k):
    """The kernel's arithmetic for w4g128 in IEEE float32, one term after another
    (the longest chain of roundings an MFMA may form), stays at least four times
    inside ACC16_EPS sum |a||w|: bf16 sums a (128 + q) and a over a group, takes
    (128 + z) times the latter off, multiplies by the scale and adds the groups,
    here up to 16 partial sums of every 16th group; fp16 sums a (q - z)."""
    rng = np.random.default_rng(k)
    m, n = 2, 8
    a = O.act_values(W.f64_to_act(rng.standard_normal((m, k)), act), act)
    a[1] = np.abs(a[1])                          # one sign: nothing cancels in the bias
    q = W.quantize_linear(W.draw_weight(7, 0, 0, 16, k), W.W4G128)
    f = np.float32
    s = q.scales[:n].astype(f)
    z = q.zeros[:n].astype(f)
    code = q.codes[:n].astype(f)
    part = np.zeros((16, m, n), f)
    for g in range(k // 128):
        acc, rs = np.zeros((m, n), f), np.zeros((m, 1), f)
        for c in range(128 * g, 128 * g + 128):
            b = code[:, c] + f(128) if act == "bf16" else code[:, c] - z[:, g]
            acc = acc + a[:, c:c + 1].astype(f) * b[None]
            rs = rs + a[:, c:c + 1].astype(f)
        if act == "bf16":
            acc = (acc.astype(np.float64) - (f(128) + z[:, g])[None].astype(np.float64) * rs).astype(f)   # one fma
        i = g % 16
        part[i] = (part[i].astype(np.float64) + s[:, g][None].astype(np.float64) * acc).astype(f)
    tot = part[0]
    for i in range(1, 16):
        tot = tot + part[i]
    wd = O.dequant(q, act)[:n]
    err = np.abs(tot - a @ wd.T)
    assert np.all(4 * err <= TL.acc_bound(np.abs(a), np.abs(wd))), float((err / TL.acc_bound(np.abs(a), np.abs(wd))).max())


def w4_bf16_emulated(a, q, offset):
    """The decode linear of w4g128 on bf16 rows in IEEE float32, one term after another: a group's
    sums of a (offset + q) and of a, (offset + z) times the latter taken off, times the scale, over
    up to 16 partial sums of every 16th group."""
    f = np.float32
    (m, k), n = a.shape, q.n
    s, z, code = q.scales.astype(f), q.zeros.astype(f), q.codes.astype(f)
    part = np.zeros((16, m, n), f)
    for g in range(k // 128):
        acc, rs = np.zeros((m, n), f), np.zeros((m, 1), f)
        for c in range(128 * g, 128 * g + 128):
            acc = acc + a[:, c:c + 1].astype(f) * (code[:, c] + f(offset))[None]
            rs = rs + a[:, c:c + 1].astype(f)
        acc = (acc.astype(np.float64) - (f(offset) + z[:, g])[None].astype(np.float64) * rs).astype(f)   # one fma
        part[g % 16] = (part[g % 16].astype(np.float64) + s[:, g][None].astype(np.float64) * acc).astype(f)
    tot = part[0]
    for i in range(1, 16):
        tot = tot + part[i]
    return tot


@pytest.mark.parametrize("k", [128, 2048, 14336])
def test_decode_w4_bf16_offset(k):
    """Codes as 16 + q, as the kernel has them: at least four times inside ACC16_EPS sum |a||w|
    for weights that use their codes; and, where one weight stretches each group's range and the
    others sit on the zero point, the error is of sum |a| (16 + q), a third at the most of what
    an offset of 128 leaves (143 / 31 = 4.6 times as much)."""
    rng = np.random.default_rng(k)
    a = O.act_values(W.f64_to_act(np.abs(rng.standard_normal((4, k))), "bf16"), "bf16")   # one sign
    a[0] *= rng.choice([-1.0, 1.0], k)
    q = W.quantize_linear(W.draw_weight(7, 0, 0, 16, k), W.W4G128)
    wd = O.dequant(q, "bf16")
    err = np.abs(w4_bf16_emulated(a, q, 16) - a @ wd.T)
    assert np.all(4 * err <= TL.acc_bound(np.abs(a), np.abs(wd)))
    w = np.zeros((16, k), np.float32)
    w[:, 5::128] = 1.0
    q = W.quantize_linear(w, W.W4G128)
    want = a @ O.dequant(q, "bf16").T
    rms = [np.sqrt(np.mean((w4_bf16_emulated(a, q, off) - want) ** 2)) for off in (16, 128)]
    assert rms[0] <= rms[1] / 3, rms


# ------------------------------------------------------------------ refusals
def norm_call(lib, x=at(1), ldx=64, res=at(2), ldr=64, w=at(3), act=M.BF16, rows=4, cols=64, eps=1e-6, sum_=at(4), lds=64,
              y=at(5), ldy=64, qmax=127, codes=at(6), scales=at(7)):
    return lib.mxmoe_add_rms_norm(x, ldx, res, ldr, w, act, rows, cols, eps, sum_, lds, y, ldy, qmax, codes, scales, None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(w=None), dict(act=2), dict(rows=-1), dict(cols=0), dict(eps=0.0), dict(eps=-1.0),
    dict(eps=float("nan")), dict(eps=1e-31), dict(eps=float("inf")), dict(ldx=63), dict(ldr=63), dict(lds=63), dict(ldy=63),
    dict(ldx=1 << 40), dict(ldy=1 << 62), dict(res=None), dict(qmax=127, codes=None), dict(qmax=127, scales=None),
    dict(qmax=0), dict(qmax=0, codes=None), dict(qmax=0, codes=None, scales=None, y=None), dict(x=at(1, 1)),
    dict(w=at(3, 1)), dict(scales=at(7, 2)),
    dict(y=at(4)), dict(y=at(4, 4 * 128 - 2)),         # y and the sum share bytes
    dict(sum_=at(1, 2)), dict(y=at(1, 128)),            # shifted over an input
    dict(sum_=at(2), lds=72),                           # in place with another stride
    dict(codes=at(1)), dict(codes=at(5, 8)), dict(scales=at(6, 252)), dict(y=at(3)), dict(scales=at(3, 124)),
    dict(ldx=80, ldy=80, y=at(1, 2 * 60)),              # slices of one wider tensor that overlap
])
def test_norm_refuses(lib, bad):
    assert norm_call(lib, **bad) == M.ERR_INVALID_ARG


def test_norm_refuses_unsupported_and_takes_nothing(lib):
    for q in (7, 8, 128, -1):
        assert norm_call(lib, qmax=q) == M.ERR_UNSUPPORTED
    assert norm_call(lib, cols=(1 << 24) + 8, ldx=1 << 25, ldr=1 << 25, lds=1 << 25, ldy=1 << 25) == M.ERR_UNSUPPORTED
    assert norm_call(lib, rows=0, x=None, res=None, w=None, sum_=None, y=None, codes=None, scales=None) == M.OK


def test_norm_refuses_spans_past_any_memory(lib):
    """Strides whose product with the rows passes 2^40 bytes (2^63 among them)."""
    far = 1 << 37
    for bad in (dict(ldx=far), dict(ldr=far), dict(lds=far), dict(ldy=far)):
        assert norm_call(lib, rows=1 << 30, **bad) == M.ERR_INVALID_ARG
        assert norm_call(lib, rows=8, **bad) == M.ERR_INVALID_ARG


def decode_call(lib, scheme=W.W4G128, n=64, k=256, act=M.BF16, packed=at(1), m=4, a=at(2), lda=256, scales=None,
                bias=at(4), out=at(5), ldo=64):
    L = M.Linear_t(n, k, M.scheme_t(scheme))
    return lib.mxmoe_linear_decode(C.byref(L), act, packed, m, a, lda, scales, bias, out, ldo, None)


@pytest.mark.parametrize("bad", [
    dict(packed=None), dict(a=None), dict(out=None), dict(act=5), dict(m=-1), dict(lda=255), dict(ldo=63),
    dict(lda=1 << 50), dict(ldo=1 << 50), dict(packed=at(1, 128)), dict(a=at(2, 8)), dict(lda=257), dict(bias=at(4, 1)),
    dict(out=at(5, 1)), dict(scales=at(3)),             # scales with 16-bit rows
    dict(scheme=W.W8A8), dict(scheme=W.FP8),            # codes without scales
    dict(scheme=W.W8A8, scales=at(3, 2)), dict(scheme=W.W8A8, scales=at(3), lda=264),
    dict(n=0), dict(k=0),
    dict(out=at(2)), dict(out=at(4)), dict(out=at(1, 512)), dict(scheme=W.FP8, scales=at(3), out=at(3, 8)),
    dict(lda=512, ldo=512, out=at(2, 2 * 200)),         # a slice that overlaps the rows'
])
def test_decode_refuses(lib, bad):
    assert decode_call(lib, **bad) == M.ERR_INVALID_ARG


def test_decode_refuses_unsupported_and_takes_nothing(lib):
    for s in W.ALL_SCHEMES:
        if s not in (W.W4G128, W.W8A8, W.FP8):
            assert decode_call(lib, scheme=s, scales=at(3) if s.a_bits < 16 else None) == M.ERR_UNSUPPORTED
    assert decode_call(lib, m=M.DECODE_ROWS + 1) == M.ERR_UNSUPPORTED
    assert decode_call(lib, n=72) == M.ERR_UNSUPPORTED
    assert decode_call(lib, k=200) == M.ERR_UNSUPPORTED
    # codes of -128 on both sides: 2^17 products of 2^14 pass the int32 sums
    assert decode_call(lib, scheme=W.W8A8, scales=at(3), k=1 << 17, lda=1 << 17) == M.ERR_UNSUPPORTED
    assert decode_call(lib, m=0, packed=None, a=None, out=None) == M.OK


def balance_call(lib, logits=at(1), ids=at(2), mask=at(3), T=5000, E=16, k=2, alpha=1.0, counts=at(4), probs=at(5),
                 loss=at(6), grad=at(7), ws=at(8), wsb=None):
    wsb = lib.mxmoe_balance_workspace_bytes(max(T, 0), 16) if wsb is None else wsb
    return lib.mxmoe_balance_loss(logits, ids, mask, T, E, k, alpha, counts, probs, loss, grad, ws, wsb, None)


@pytest.mark.parametrize("bad", [
    dict(logits=None), dict(ids=None), dict(counts=None), dict(probs=None), dict(loss=None), dict(ws=None), dict(T=-1),
    dict(E=0), dict(E=1025), dict(k=0), dict(k=17), dict(alpha=float("nan")), dict(alpha=float("inf")),
    dict(T=1 << 30, k=2, wsb=1 << 40), dict(logits=at(1, 2)), dict(grad=at(7, 1)), dict(ws=at(8, 64)),
    dict(grad=at(1, 64)), dict(counts=at(2)), dict(probs=at(4, 60)), dict(loss=at(5, 60)), dict(grad=at(2)),
    dict(ws=at(7)), dict(loss=at(3)), dict(ws=at(1)),
])
def test_balance_refuses(lib, bad):
    assert balance_call(lib, **bad) == M.ERR_INVALID_ARG


def test_balance_workspace(lib):
    assert balance_call(lib, wsb=lib.mxmoe_balance_workspace_bytes(5000, 16) - 1) == M.ERR_WORKSPACE
    for T, E in ((-1, 8), (8, 0), (8, 1025)):
        assert lib.mxmoe_balance_workspace_bytes(T, E) == 0
    last = 0
    for T in (0, 1, 17, 512, 4096, 65536, 1 << 20):   # a workspace serves every smaller batch
        b = lib.mxmoe_balance_workspace_bytes(T, 64)
        assert b >= last
        last = b
    assert last < 1 << 20


def test_binding_refuses_host_tensors():
    import torch
    x = torch.zeros(2, 16, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        M.add_rms_norm(x, x[0])
    with pytest.raises(ValueError):
        M.balance_loss(torch.zeros(2, 4), torch.zeros(2, 1, dtype=torch.int32))
