"""GPU parity of the operators around the block against their oracles: the
residual and RMS norm with 8-bit rows (every output bit for bit), the decode
linear (int8 within the epilogue's roundings, the others within the error models
of tests/tolerance.py plus the output's rounding) and the balance loss."""

import ctypes as C

import numpy as np
import pytest

from oracle import mxmoe_oracle as O
from paper_2505_05799_amd import mxmoe as M
from paper_2505_05799_amd import workloads as W
from tests import tolerance as TL
from tests.gpuhelp import say, torch_mod

pytestmark = pytest.mark.gpu


def bits(t):
    return t.contiguous().view(__import__("torch").int16).cpu().numpy().view(np.uint16)


def act_bits(v, act):
    """fp64 values that the dtype holds -> their bit patterns (-0 kept)."""
    if act == "fp16":
        return v.astype(np.float16).view(np.uint16)
    return W.f32_to_bf16_bits(v.astype(np.float32))


# ---------------------------------------------------------------------- norm
def norm_rows(rng, rows, cols, act, scale=1.0):
    x = rng.standard_normal((rows, cols)) * scale
    x[:, rng.random(cols) < 0.01] *= 8
    return W.f64_to_act(x, act)


def strided(torch, a, act, pad, off=0):
    """The rows on the GPU as a slice of wider ones (pad extra elements, off of
    them in front), the rest a value that must not be read or written."""
    rows, cols = a.shape
    t = torch.full((rows, cols + pad), 77.0, dtype=torch.bfloat16 if act == "bf16" else torch.float16, device="cuda")
    v = t[:, off:off + cols]
    v.copy_(M.act_tensor(a, act))
    return v, t


def check_norm(x, res, w, act, qmax, got, eps=1e-6):
    xa, ra, wa = O.act_values(x, act), None if res is None else O.act_values(res, act), O.act_values(w, act)
    y, z, _ = O.add_rms_norm(xa, ra, wa, act, eps)
    gy, gz, codes, scales = got
    if gy is not None:
        assert np.array_equal(bits(gy), act_bits(y, act))
    if res is None:
        assert gz is None
    else:
        assert np.array_equal(bits(gz), act_bits(z, act))
    if not qmax:
        assert codes is None and scales is None
        return
    q, s = O.act_quant(y, qmax) if qmax == 127 else O.fp8_quant(y)
    assert np.array_equal(scales.cpu().numpy().view(np.uint32), s.view(np.uint32))
    assert np.array_equal(codes.cpu().numpy().view(np.uint8), q.view(np.uint8))


NORM_SHAPES = [(1, 1), (3, 2), (2, 7), (1, 8), (5, 64), (4, 127), (7, 128), (1, 513), (9, 1024), (1, 2048), (33, 2056),
               (2, 3584), (130, 4096), (3, 4104), (5, 7168), (2, 16384), (1, 16392), (1, 32768), (2, 33000), (1, 70001),
               (700, 72), (1500, 256), (4100, 128), (4097, 1000), (4096, 1600), (4099, 2056), (513, 5000), (512, 16000)]


@pytest.mark.parametrize("act", ["bf16", "fp16"])
@pytest.mark.parametrize("qmax", [0, 127, 448])
@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
def test_norm(rows, cols, qmax, act):
    torch = torch_mod()
    rng = np.random.default_rng(rows * 1000 + cols)
    x, res, w = (norm_rows(rng, r, cols, act, s) for r, s in ((rows, 1.0), (rows, 0.5), (1, 1.0)))
    xt, rt, wt = M.act_tensor(x, act), M.act_tensor(res, act), M.act_tensor(w, act)[0]
    check_norm(x, res, w[0][None], act, qmax, M.add_rms_norm(xt, wt, residual=rt, qmax=qmax))
    check_norm(x, None, w[0][None], act, qmax, M.add_rms_norm(xt, wt, qmax=qmax, want_y=qmax == 0))


@pytest.mark.parametrize("act", ["bf16", "fp16"])
@pytest.mark.parametrize("cols,pad,off", [(256, 8, 8), (256, 13, 0), (256, 8, 1), (255, 9, 3), (4096, 24, 16), (5000, 1, 1)])
def test_norm_strides_and_in_place(cols, pad, off, act):
    torch = torch_mod()
    rng = np.random.default_rng(cols + pad)
    rows = 19
    x, res, w = norm_rows(rng, rows, cols, act), norm_rows(rng, rows, cols, act), norm_rows(rng, 1, cols, act)
    wt = M.act_tensor(w, act)[0]
    for qmax in (127, 448):
        xt, xw = strided(torch, x, act, pad, off)
        rt, rw = strided(torch, res, act, pad, off)
        out = M.add_rms_norm(xt, wt, residual=rt, qmax=qmax, sum_out=rt)      # the sum takes the residual's place
        assert out[1].data_ptr() == rt.data_ptr()
        check_norm(x, res, w, act, qmax, out)
        for t in (xw, rw):                                                     # nothing beside the rows is touched
            t[:, off:off + cols] = 77.0
            assert bool((t == 77.0).all())
    # y in the place of x, the sum in the place of the residual, through the C ABI
    xt, xw = strided(torch, x, act, pad, off)
    rt, rw = strided(torch, res, act, pad, off)
    ld = cols + pad
    st = M.load_library().mxmoe_add_rms_norm(xt.data_ptr(), ld, rt.data_ptr(), ld, wt.data_ptr(), M.act_code(act), rows, cols,
                                             1e-6, rt.data_ptr(), ld, xt.data_ptr(), ld, 0, None, None, M._stream_ptr())
    assert st == M.OK
    check_norm(x, res, w, act, 0, (xt, rt, None, None))
    # slices of one tensor beside each other: read one, write the other
    both = torch.full((rows, 2 * cols + 32), 5.0, dtype=xt.dtype, device="cuda")
    a, b = both[:, 16:16 + cols], both[:, 32 + cols:]
    a.copy_(M.act_tensor(x, act))
    ldb = both.stride(0)
    st = M.load_library().mxmoe_add_rms_norm(a.data_ptr(), ldb, None, 0, wt.data_ptr(), M.act_code(act), rows, cols, 1e-6,
                                             None, 0, b.data_ptr(), ldb, 0, None, None, M._stream_ptr())
    assert st == M.OK
    check_norm(x, None, w, act, 0, (b, None, None, None))
    assert np.array_equal(bits(a), bits(M.act_tensor(x, act)))
    assert bool((both[:, :16] == 5.0).all()) and bool((both[:, 16 + cols:32 + cols] == 5.0).all())


@pytest.mark.parametrize("act", ["bf16", "fp16"])
@pytest.mark.parametrize("cols", [264, 4096, 20000, 131])
def test_norm_special_rows(cols, act):
    """Zero rows, huge and tiny rows (the squares pass the range of 32 bits), and
    rows that are not finite: those have scale NaN and leave the others alone."""
    torch = torch_mod()
    rng = np.random.default_rng(cols)
    big, small = (3e38, 1e-38) if act == "bf16" else (6e4, 6e-8)
    v = rng.uniform(0.2, 1.0, (8, cols)) * rng.choice([-1, 1], (8, cols))
    v[0] = 0.0
    v[1] *= big
    v[2] *= small
    v[3, :] = 0.0
    v[3, cols - 1] = 1.0                               # one element
    x = W.f64_to_act(v, act)
    w = W.f64_to_act(np.ones((1, cols)), act)
    for qmax in (127, 448):
        xt = M.act_tensor(x, act)
        out = M.add_rms_norm(xt, M.act_tensor(w, act)[0], qmax=qmax, eps=1e-12)
        check_norm(x, None, w, act, qmax, out, eps=1e-12)
        assert float(out[3][0]) == 0.0 and not bool(out[2][0].any())
        xt[4, cols // 2] = float("nan")
        xt[6, 0] = float("inf")
        y, _, codes, scales = M.add_rms_norm(xt, M.act_tensor(w, act)[0], qmax=qmax, eps=1e-12)
        assert bool(torch.isnan(scales[[4, 6]]).all()) and not bool(codes[[4, 6]].any())
        assert bool(torch.isnan(y[4]).all()) and bool(torch.isnan(y[6, 0]))
        keep = [0, 1, 2, 3, 5, 7]
        check_norm(x[keep], None, w, act, qmax, (y[keep], None, codes[keep], scales[keep]), eps=1e-12)
        # a row so small that q / amax would overflow counts as zero
        if act == "bf16":
            tiny = torch.full((1, cols), 2.0 ** -70, dtype=torch.bfloat16, device="cuda")
            _, _, codes, scales = M.add_rms_norm(tiny, tiny[0], qmax=qmax, eps=1.0)
            assert float(scales) == 0.0 and not bool(codes.any())


def test_norm_refusals():
    torch = torch_mod()
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    w = x[0].clone()
    for bad in (lambda: M.add_rms_norm(x.float(), w.float()), lambda: M.add_rms_norm(x, w.half()),
                lambda: M.add_rms_norm(x, w[:32]), lambda: M.add_rms_norm(x, w, residual=x[:2]),
                lambda: M.add_rms_norm(x.t(), w), lambda: M.add_rms_norm(x, w, sum_out=x),
                lambda: M.add_rms_norm(x[0], w), lambda: M.add_rms_norm(x[:1].expand(4, 64), w),
                lambda: M.add_rms_norm(x, w.cpu())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: M.add_rms_norm(x, w, qmax=7), lambda: M.add_rms_norm(x, w, want_y=False),
                lambda: M.add_rms_norm(x, w, eps=0.0)):
        with pytest.raises(M.MxmoeError):
            bad()
    y, z, c, s = M.add_rms_norm(x[:0], w, residual=x[:0], qmax=127)
    assert y.shape == z.shape == c.shape == (0, 64) and s.shape == (0,)


# -------------------------------------------------------------------- linear
def decode_case(scheme, act, m, n, k, seed, bias, pad=0):
    torch = torch_mod()
    rng = np.random.default_rng(seed)
    q = W.quantize_linear(W.draw_weight(seed, 1, 0, n, k), scheme)
    x = W.f64_to_act(rng.standard_normal((m, k)), act)
    b = W.f64_to_act(rng.standard_normal((1, n)), act) if bias else None
    pl = M.PackedLinear(q, act)
    xv = O.act_values(x, act)
    if scheme == W.W4G128:
        a, scales = M.act_tensor(x, act), None
        ad = xv
    else:
        codes, s = O.act_quant(xv, 127) if scheme == W.W8A8 else O.fp8_quant(xv)
        a, scales = torch.from_numpy(codes.view(np.int8).copy()).cuda(), torch.from_numpy(s.copy()).cuda()
        ad = (codes.astype(np.float64) if scheme == W.W8A8 else O.e4m3_values(codes)) * s.astype(np.float64)[:, None]
    if pad:
        wide = torch.full((m, k + pad), 1, dtype=a.dtype, device="cuda")
        wide[:, :k] = a
        a = wide[:, :k]
    return q, pl, a, scales, None if b is None else M.act_tensor(b, act)[0], ad, b


def check_decode(q, ad, b, act, got):
    want = ad @ O.dequant(q, act).T
    wd = O.dequant(q, act)
    if q.scheme == W.W8A8:      # the exact sum, rounded to fp32, times two scales (and added to the bias)
        bound = 4 * TL.U32 * np.abs(want)
    elif q.scheme == W.FP8:
        bound = TL.fp8_block_bound(ad, wd) + 4 * TL.U32 * np.abs(want)
    else:
        bound = TL.acc_bound(np.abs(ad), np.abs(wd))
    if b is not None:
        want = want + O.act_values(b, act)
    bound = TL.slot_bound(want, bound + 2 * TL.U32 * np.abs(want) + 1e-30, act)
    err = np.abs(O.act_values(M.act_numpy(got, act), act) - want)
    assert np.all(err <= bound), float((err / bound).max())
    return float((err / bound).max())


DECODE_SCHEMES = [W.W4G128, W.W8A8, W.FP8]


@pytest.mark.parametrize("act", ["bf16", "fp16"])
@pytest.mark.parametrize("m", [1, 2, 7, 15, 16, 17, 31, 32, 33, 48, 49, 63, 64])
@pytest.mark.parametrize("scheme", DECODE_SCHEMES, ids=lambda s: s.name)
def test_decode_rows(scheme, m, act):
    for n, k, bias in ((16, 128, False), (48, 384, True), (272, 1408, m % 2 == 0)):
        q, pl, a, sc, bt, ad, b = decode_case(scheme, act, m, n, k, m + n, bias)
        worst = check_decode(q, ad, b, act, M.linear_decode(pl, a, scales=sc, bias=bt))
        say(f"decode {scheme.name} {act} {m}x{n}x{k}: {worst:.3f} of the bound")


@pytest.mark.parametrize("scheme", DECODE_SCHEMES, ids=lambda s: s.name)
@pytest.mark.parametrize("m,n,k", [(1, 4096, 2048), (3, 2048, 14336), (16, 5632, 2048), (64, 1024, 4096), (33, 20480, 256),
                                   (1, 16, 16384)])
def test_decode_shapes(scheme, m, n, k):
    for act in ("bf16", "fp16"):
        q, pl, a, sc, bt, ad, b = decode_case(scheme, act, m, n, k, 5, True)
        worst = check_decode(q, ad, b, act, M.linear_decode(pl, a, scales=sc, bias=bt))
        say(f"decode {scheme.name} {act} {m}x{n}x{k}: {worst:.3f} of the bound")


@pytest.mark.parametrize("scheme", DECODE_SCHEMES, ids=lambda s: s.name)
@pytest.mark.parametrize("n", [4112, 6000, 8208, 10000, 12304, 16400, 19232, 24592])
def test_decode_wide(scheme, n):
    """Every number of channel blocks to a workgroup, the last one not full, for each
    number of row fragments."""
    k = 384
    for m, act in ((1, "fp16"), (9, "bf16"), (24, "fp16"), (40, "bf16")):
        q, pl, a, sc, bt, ad, b = decode_case(scheme, act, m, n, k, n, True)
        worst = check_decode(q, ad, b, act, M.linear_decode(pl, a, scales=sc, bias=bt))
        say(f"decode {scheme.name} {act} {m}x{n}x{k}: {worst:.3f} of the bound")


@pytest.mark.parametrize("scheme", DECODE_SCHEMES, ids=lambda s: s.name)
def test_decode_strides(scheme):
    """Rows and outputs of wider tensors, rows that are not 16-byte aligned (the
    binding copies them), and what lies beside the output stays as it was."""
    torch = torch_mod()
    for m in (1, 5, 20):
        for pad in (16, 5):
            q, pl, a, sc, bt, ad, b = decode_case(scheme, "bf16", m, 96, 512, 3, True, pad)
            wide = torch.full((m + 2, 96 + 11), 9.0, dtype=torch.bfloat16, device="cuda")
            out = wide[1:m + 1, 3:99]
            assert M.linear_decode(pl, a, scales=sc, bias=bt, out=out) is out
            check_decode(q, ad, b, "bf16", out)
            ref = M.linear_decode(pl, a.contiguous(), scales=sc, bias=bt)
            assert np.array_equal(bits(ref), bits(out))
            out[:] = 9.0
            assert bool((wide == 9.0).all())


@pytest.mark.parametrize("scheme", DECODE_SCHEMES, ids=lambda s: s.name)
def test_decode_rows_are_independent(scheme):
    """A row's result does not depend on the other rows' values: NaN or inf in one
    row stays there; the same row in another batch of the same size has the same
    bits."""
    torch = torch_mod()
    for m in (3, 16, 40):
        q, pl, a, sc, bt, ad, b = decode_case(scheme, "bf16", m, 64, 640, 8, False)
        ref = M.linear_decode(pl, a, scales=sc)
        a2, sc2 = a.clone(), None if sc is None else sc.clone()
        if sc is None:
            a2[1, 77] = float("nan")
        else:
            sc2[1] = float("nan")
        got = M.linear_decode(pl, a2, scales=sc2)
        assert bool(torch.isnan(got[1]).all())
        keep = [i for i in range(m) if i != 1]
        assert torch.equal(got[keep].view(torch.int16), ref[keep].view(torch.int16))


def test_decode_refusals():
    torch = torch_mod()
    q, pl, a, sc, bt, ad, b = decode_case(W.W4G128, "bf16", 4, 64, 256, 1, True)
    q8, pl8, a8, s8, *_ = decode_case(W.W8A8, "bf16", 4, 64, 256, 1, True)
    for bad in (lambda: M.linear_decode(pl, a.half()), lambda: M.linear_decode(pl, a[:, :128].contiguous()),
                lambda: M.linear_decode(pl, a, scales=s8), lambda: M.linear_decode(pl8, a8),
                lambda: M.linear_decode(pl8, a, scales=s8), lambda: M.linear_decode(pl8, a8, scales=s8[:2]),
                lambda: M.linear_decode(pl, a, bias=bt.float()), lambda: M.linear_decode(pl, a, out=a),
                lambda: M.linear_decode(pl, a.cpu())):
        with pytest.raises(ValueError):
            bad()
    w16 = M.PackedLinear(W.quantize_linear(W.draw_weight(1, 1, 0, 64, 256), W.W16), "bf16")
    with pytest.raises(M.MxmoeError):
        M.linear_decode(w16, a)
    with pytest.raises(M.MxmoeError):
        M.linear_decode(pl, torch.zeros(65, 256, dtype=torch.bfloat16, device="cuda"))
    assert M.linear_decode(pl, a[:0]).shape == (0, 64)


# ------------------------------------------------------------------- balance
def balance_case(T, E, k, seed, masked=0.0):
    rng = np.random.default_rng(seed)
    l = (rng.standard_normal((T, E)) * 1.5 - np.log1p(rng.permutation(E))).astype(np.float32)
    ids = np.argsort(-l, axis=1, kind="stable")[:, :k].astype(np.int32)
    mask = rng.random(T) >= masked if masked else None
    return l, ids, mask


def check_balance(l, ids, mask, alpha, got):
    """fp32 softmax of E terms: exp within 2 ulp of an argument that is rounded once
    (|l - max| U32, below 40 U32 here where p counts), E - 1 additions of positive terms
    and a quotient: p within (E + 50) U32.  A column's sum of positive terms takes at
    most T more additions; f - sum f p errs by the same share of f + sum f p."""
    loss, counts, probs, grad = got
    T, E = l.shape
    L, c, P, g = O.balance_loss(l, ids, mask, alpha)
    u = (E + 50) * TL.U32
    assert np.array_equal(counts.cpu().numpy(), c)
    assert np.all(np.abs(probs.cpu().numpy() - P) <= (u + T * TL.U32) * P + 1e-38)
    assert abs(float(loss) - L) <= (u + T * TL.U32) * abs(L) + 1e-38
    if grad is None:
        return
    n = T if mask is None else int(np.sum(mask))
    f = c / max(1, n * ids.shape[1])
    with np.errstate(invalid="ignore", divide="ignore"):
        p = np.exp(l.astype(np.float64) - l.max(axis=1, keepdims=True).astype(np.float64))
        p = np.nan_to_num(p / p.sum(axis=1, keepdims=True))
    if mask is not None:
        p[~np.asarray(mask, bool)] = 0
    size = abs(alpha) * E / max(1, n) * p * (f[None] + (f * p).sum(axis=1, keepdims=True))
    err = np.abs(grad.cpu().numpy() - g)
    assert np.all(err <= 3 * u * size + 1e-38), float((err / (3 * u * size + 1e-38)).max())


BALANCE = [(1, 1, 1), (1, 8, 2), (2, 2, 2), (3, 5, 5), (17, 8, 2), (64, 60, 4), (100, 64, 6), (257, 33, 1), (300, 128, 8),
           (511, 160, 6), (1000, 3, 2), (1025, 256, 8), (2048, 60, 4), (33, 1024, 8), (700, 1000, 3), (4099, 64, 8),
           (20000, 8, 2), (4200, 128, 3), (9000, 120, 2), (1100, 200, 2)]


@pytest.mark.parametrize("masked", [0.0, 0.3])
@pytest.mark.parametrize("T,E,k", BALANCE)
def test_balance(T, E, k, masked):
    torch = torch_mod()
    l, ids, mask = balance_case(T, E, k, T + E, masked)
    lt, it = torch.from_numpy(l).cuda(), torch.from_numpy(ids).cuda()
    mt = None if mask is None else torch.from_numpy(mask).cuda()
    got = M.balance_loss(lt, it, alpha=0.7, token_mask=mt)
    check_balance(l, ids, mask, 0.7, got)
    if mask is not None:
        assert not bool(got[3][~mt].any())
    none = M.balance_loss(lt, it, alpha=0.7, token_mask=mt, want_grad=False)
    assert none[3] is None
    for a, b in zip(none[:3], got[:3]):
        assert torch.equal(a, b)


def test_balance_odd_inputs():
    """Ids that are repeated or out of range, experts and whole tokens at -inf,
    padding that holds NaN, a batch of padding alone and an empty one."""
    torch = torch_mod()
    for T, E in ((200, 60), (40, 8), (3000, 200)):
        l, ids, _ = balance_case(T, E, 4, 5)
        rng = np.random.default_rng(1)
        ids[rng.random(ids.shape) < 0.1] = -1
        ids[rng.random(ids.shape) < 0.1] = E
        ids[rng.random(ids.shape) < 0.1] = 2 ** 31 - 1
        ids[7] = 3                                          # one expert four times
        l[:, 5] = -np.inf
        l[11] = -np.inf
        l[12, 1:] = -np.inf
        mask = np.ones(T, np.uint8)
        mask[20:30] = 0
        mask[::3] *= 7                                      # any value but 0 keeps
        lt = torch.from_numpy(l).cuda()
        lt[20:25] = float("nan")
        lt[25:30] = float("inf")
        check_balance(l, ids, mask, 1.0, M.balance_loss(lt, torch.from_numpy(ids).cuda(), token_mask=torch.from_numpy(mask).cuda()))
        none = torch.zeros(T, dtype=torch.bool, device="cuda")
        for t in M.balance_loss(lt, torch.from_numpy(ids).cuda(), token_mask=none):
            assert not bool(t.any())
        lt[0, 1] = float("nan")
        loss, counts, probs, grad = M.balance_loss(lt, torch.from_numpy(ids).cuda(), token_mask=torch.from_numpy(mask).cuda())
        assert bool(torch.isnan(loss)) and bool(torch.isnan(probs).any()) and bool(torch.isnan(grad[0]).any())
        assert not bool(torch.isnan(grad[1:]).any())
    loss, counts, probs, grad = M.balance_loss(torch.zeros(0, 8, device="cuda"), torch.zeros(0, 2, dtype=torch.int32, device="cuda"))
    assert float(loss) == 0 and not bool(counts.any()) and not bool(probs.any()) and grad.shape == (0, 8)


@pytest.mark.parametrize("T,E,k", [(65, 8, 2), (2000, 60, 4)])
def test_balance_gradient_against_differences(T, E, k):
    """(L(l + h d) - L(l - h d)) / 2h of the GPU's losses against the GPU's gradient
    along d.  The quotient differs from the derivative by what it does in 64 bits
    (measured on the oracle) and by the losses' own error over 2h; the gradient's
    elements are within the bound of check_balance."""
    torch = torch_mod()
    l, ids, _ = balance_case(T, E, k, 3)
    it = torch.from_numpy(ids).cuda()
    d = np.random.default_rng(4).choice([-1.0, 1.0], (T, E))
    h = 2.0 ** -6
    lp, lm = (l + h * d).astype(np.float32), (l - h * d).astype(np.float32)
    at = [float(M.balance_loss(torch.from_numpy(v).cuda(), it)[0]) for v in (lp, lm)]
    g = M.balance_loss(torch.from_numpy(l).cuda(), it)[3].cpu().numpy().astype(np.float64)
    ref = [O.balance_loss(v, ids)[0] for v in (lp, lm)]
    gr = O.balance_loss(l, ids)[3]
    u = (E + 50 + T) * TL.U32
    tol = abs((ref[0] - ref[1]) / (2 * h) - (gr * d).sum()) + 2 * u * max(ref) / (2 * h) + 3 * u * np.abs(gr).sum() * 4
    assert abs((at[0] - at[1]) / (2 * h) - (g * d).sum()) <= tol


def test_balance_in_place_and_refusals():
    torch = torch_mod()
    for T, E, k in ((64, 60, 4), (3000, 64, 2), (5, 1000, 2)):
        l, ids, _ = balance_case(T, E, k, 6)
        lt, it = torch.from_numpy(l).cuda(), torch.from_numpy(ids).cuda()
        want = M.balance_loss(lt, it)
        lib = M.load_library()
        wsb = lib.mxmoe_balance_workspace_bytes(T, E)
        ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
        c, p, s = torch.empty(E, dtype=torch.int32, device="cuda"), torch.empty(E, device="cuda"), torch.empty(1, device="cuda")
        st = lib.mxmoe_balance_loss(lt.data_ptr(), it.data_ptr(), None, T, E, k, 1.0, c.data_ptr(), p.data_ptr(), s.data_ptr(),
                                    lt.data_ptr(), ws.data_ptr(), wsb, M._stream_ptr())
        assert st == M.OK
        for a, b in zip((s[0], c, p, lt), want):
            assert torch.equal(a, b)
    for bad in (lambda: M.balance_loss(lt.half(), it), lambda: M.balance_loss(lt, it.long()),
                lambda: M.balance_loss(lt, it[:2]), lambda: M.balance_loss(lt.t(), it),
                lambda: M.balance_loss(lt, it, token_mask=torch.ones(T, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(M.MxmoeError):
        M.balance_loss(torch.zeros(4, 2, device="cuda"), torch.zeros(4, 3, dtype=torch.int32, device="cuda"))
    with pytest.raises(M.MxmoeError):
        M.balance_loss(lt, it, alpha=float("nan"))


# ------------------------------------------------------------------ together
def _layer(torch, act="bf16", T=24):
    """What surrounds a block in one layer, and the block."""
    H = 256
    blk = W.random_small_block(5, T=T, H=H, F=384, E=6, k=2, n_shared=1, F_shared=256, act=act,
                               schemes=[(W.W4G128,) * 3, (W.W8A8, W.W8A8, W.W2G128), (W.W4A4,) * 3, (W.FP8,) * 3,
                                        (W.W16,) * 3, (W.W8A8,) * 3, (W.FP8, W.FP8, W.W8A8)])
    mb = M.MoEBlock(blk)
    proj = {s.name: M.PackedLinear(W.quantize_linear(W.draw_weight(9, i, 0, H, H), s), act) for i, s in enumerate(DECODE_SCHEMES)}
    rng = np.random.default_rng(2)
    x, res = (M.act_tensor(norm_rows(rng, T, H, act), act) for _ in range(2))
    w = M.act_tensor(norm_rows(rng, 1, H, act), act)[0]
    router = torch.from_numpy(rng.standard_normal((H, 6)).astype(np.float32) * 0.1).cuda()
    return blk, mb, proj, x, res, w, router


def _pass(torch, L, stream=None):
    """norm -> int8 linear on its codes -> norm -> fp8 linear -> norm -> w4 linear ->
    norm -> router, block and balance loss."""
    blk, mb, proj, x, res, w, router = L
    y, z, c, s = M.add_rms_norm(x, w, residual=res, qmax=127, want_y=False, stream=stream)
    o = M.linear_decode(proj["w8a8"], c, scales=s, stream=stream)
    y, z, c, s = M.add_rms_norm(o, w, residual=z, qmax=448, want_y=False, stream=stream)
    o = M.linear_decode(proj["fp8"], c, scales=s, stream=stream)
    y, z, _, _ = M.add_rms_norm(o, w, residual=z, stream=stream)
    o = M.linear_decode(proj["w4g128"], y, bias=w, stream=stream)
    y, z, c, s = M.add_rms_norm(o, w, residual=z, qmax=127, stream=stream)
    if stream is None:
        logits = (y.float()[:, :, None] * router[None]).sum(1)
    else:
        with torch.cuda.stream(stream):
            logits = (y.float()[:, :, None] * router[None]).sum(1)
    ids, gw, _ = M.router_topk(logits, 2, stream=stream)
    out = mb.forward(y, ids, gw, stream=stream)
    loss, counts, probs, grad = M.balance_loss(logits, ids, alpha=0.01, stream=stream)
    return [z, y, c, s, logits, ids, gw, out, loss, counts, probs, grad]


def _same(torch, a, b):
    for i, (u, v) in enumerate(zip(a, b)):
        assert torch.equal(u.reshape(-1).view(torch.uint8), v.reshape(-1).view(torch.uint8)), i


def test_layer_together():
    """The operators as one layer uses them: the codes of a norm are those that
    act_quant gives for its rows, so the int8 linear equals one on act_quant's codes;
    the counts are the routing's; eager, on another stream, and captured and
    replayed, the pass gives the same bits."""
    torch = torch_mod()
    L = _layer(torch)
    blk, mb, proj, x, res, w, router = L
    ref = _pass(torch, L)
    y, z, c, s = M.add_rms_norm(x, w, residual=res, qmax=127)
    qc, qs = M.act_quant(y, "bf16", 127)
    assert torch.equal(c, qc) and torch.equal(s, qs)
    c8, s8 = M.add_rms_norm(x, w, residual=res, qmax=448, want_y=False)[2:]
    qc, qs = M.act_quant(y, "bf16", 448)
    assert torch.equal(c8, qc) and torch.equal(s8, qs)
    # the int8 product is the raw linear's integers times the scales
    raw = M.linear_forward(proj["w8a8"], y)
    sw = torch.from_numpy(proj["w8a8"].q.scales).cuda()
    want = (raw.float() * s[:, None] * sw).to(torch.bfloat16)
    assert torch.equal(M.linear_decode(proj["w8a8"], c, scales=s).view(torch.int16), want.view(torch.int16))
    routed = M.route_permute(ref[5], 6)
    assert torch.equal(routed["counts"], ref[9])
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    other = _pass(torch, L, stream=st)
    torch.cuda.current_stream().wait_stream(st)
    torch.cuda.synchronize()
    _same(torch, ref, other)
    with torch.cuda.stream(st):
        _pass(torch, L)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cap = _pass(torch, L)
    for rep in range(3):
        for t in cap:
            t.reshape(-1).view(torch.uint8).zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        _same(torch, ref, cap)
        _same(torch, ref, _pass(torch, L))           # eager work between replays
        torch.cuda.synchronize()


def test_two_streams_at_once():
    """Two passes in flight on two streams, each with its own buffers."""
    torch = torch_mod()
    L = [_layer(torch, T=t) for t in (24, 40)]
    ref = [_pass(torch, l) for l in L]
    torch.cuda.synchronize()
    st = [torch.cuda.Stream() for _ in L]
    for _ in range(4):
        got = [_pass(torch, l, stream=s) for l, s in zip(L, st)]
        torch.cuda.synchronize()
        for a, b in zip(ref, got):
            _same(torch, a, b)


def test_norm_more_rows_than_workgroups():
    """Row counts past the largest grid (workgroups then take several rows): eight rows
    repeated give their outputs repeated."""
    torch = torch_mod()
    for rows, cols in ((33_600_000, 3), (4_400_000, 300)):
        rng = np.random.default_rng(cols)
        x, w = norm_rows(rng, 8, cols, "bf16"), norm_rows(rng, 1, cols, "bf16")
        few, wt = M.act_tensor(x, "bf16"), M.act_tensor(w, "bf16")[0]
        y8, _, c8, s8 = M.add_rms_norm(few, wt, qmax=127)
        check_norm(x, None, w, "bf16", 127, (y8, None, c8, s8))
        y, _, c, s = M.add_rms_norm(few.repeat(rows // 8, 1), wt, qmax=127)
        assert bool((y.view(rows // 8, 8, cols) == y8).all()) and bool((c.view(rows // 8, 8, cols) == c8).all())
        assert bool((s.view(rows // 8, 8) == s8).all())
        del y, c, s
        torch.cuda.empty_cache()


def test_decode_largest_weight():
    """Weights whose byte offsets pass 31 bits: the last channels of 131056 x 16384."""
    torch = torch_mod()
    n, k, m = 131056, 16384, 3
    g = torch.Generator(device="cuda").manual_seed(1)
    codes = torch.randint(-127, 128, (n, k), generator=g, device="cuda", dtype=torch.int8)
    scales = torch.rand(n, generator=g, device="cuda") * 1e-3
    pl = M.PackedLinear(W.QLinear(W.W8A8, n, k, codes, scales), "bf16")
    a = torch.randint(-127, 128, (m, k), generator=g, device="cuda", dtype=torch.int8)
    sa = torch.rand(m, generator=g, device="cuda") * 1e-2
    out = M.linear_decode(pl, a, scales=sa)
    for lo in (0, n - 64):
        want = (a.double() @ codes[lo:lo + 64].double().t().contiguous()) * sa.double()[:, None] * scales[lo:lo + 64].double()
        want = want.cpu().numpy()
        got = O.act_values(M.act_numpy(out[:, lo:lo + 64], "bf16"), "bf16")
        assert np.all(np.abs(got - want) <= TL.slot_bound(want, 4 * TL.U32 * np.abs(want), "bf16"))
    del codes, pl, out
    torch.cuda.empty_cache()


def test_decode_poisoned_channel():
    """A channel whose packed scale is NaN (a zero point outside its range) is NaN, its
    neighbours are not."""
    torch = torch_mod()
    q = W.quantize_linear(W.draw_weight(3, 1, 0, 48, 512), W.W4G128)
    ref = M.PackedLinear(q, "bf16")
    zeros = q.zeros.copy()
    zeros[19, 2] = 16.0
    bad = M.PackedLinear(W.QLinear(q.scheme, q.n, q.k, q.codes, q.scales, zeros), "bf16")
    for m in (1, 7, 40):
        a = torch.randn(m, 512, device="cuda").bfloat16()
        x, y = M.linear_decode(ref, a), M.linear_decode(bad, a)
        assert bool(torch.isnan(y[:, 19]).all())
        keep = [c for c in range(48) if c != 19]
        assert torch.equal(x[:, keep], y[:, keep])


def _larger(torch):
    """One call of each operator at a size that takes several workgroups and launches."""
    rng = np.random.default_rng(6)
    x, res = (M.act_tensor(norm_rows(rng, 600, 5000, "fp16"), "fp16") for _ in range(2))
    w = M.act_tensor(norm_rows(rng, 1, 5000, "fp16"), "fp16")[0]
    q, pl, a, sc, bt, ad, b = decode_case(W.FP8, "bf16", 40, 2064, 1408, 1, True)
    q4, pl4, a4, *_ = decode_case(W.W4G128, "fp16", 60, 12800, 384, 1, False)
    cases = []
    for T, E, k in ((3000, 200, 4), (5000, 60, 4)):
        l, ids, mask = balance_case(T, E, k, 5, 0.2)
        cases.append([torch.from_numpy(v).cuda() for v in (l, ids, mask)])

    def run():
        out = list(M.add_rms_norm(x, w, residual=res, qmax=448))
        out += [M.linear_decode(pl, a, scales=sc, bias=bt), M.linear_decode(pl4, a4)]
        for l, ids, mask in cases:
            out += M.balance_loss(l, ids, token_mask=mask)
        return out
    return run


def test_larger_calls_in_a_graph():
    """Captured and replayed, with eager calls and synchronizations in between, and twice
    in a row: the same bits."""
    torch = torch_mod()
    run = _larger(torch)
    ref = run()
    _same(torch, ref, run())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cap = run()
    for rep in range(3):
        for t in cap:
            t.reshape(-1).view(torch.uint8).zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        _same(torch, ref, cap)
        _same(torch, ref, run())
        torch.cuda.synchronize()


def test_side_stream_memory_is_kept():
    """Inputs dropped right after a call on another stream stay whole until it has run:
    the calls hold them back from the allocator."""
    torch = torch_mod()
    s = torch.cuda.Stream()
    x = torch.randn(2048, 4096, device="cuda").bfloat16()
    w = torch.ones(4096, dtype=torch.bfloat16, device="cuda")
    want = M.add_rms_norm(x, w)[0]
    torch.cuda.synchronize()
    for _ in range(5):
        tmp = x.clone()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            torch.cuda._sleep(2_000_000)                 # the call waits behind this
        y = M.add_rms_norm(tmp, w, stream=s)[0]
        del tmp
        for _ in range(4):
            torch.full((2048, 4096), 7.0, dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        assert torch.equal(y.view(torch.int16), want.view(torch.int16))


def test_far_offsets():
    """Rows whose byte offsets pass 32 bits: the rows at the end of a 5 GB buffer."""
    torch = torch_mod()
    act, cols = "bf16", 256
    rows, ld = 5, 1 << 29                               # rows 1 GiB apart
    big = torch.empty(4 * ld + 2048, dtype=torch.bfloat16, device="cuda")
    xt = big.as_strided((rows, cols), (ld, 1))
    rng = np.random.default_rng(8)
    x, w = norm_rows(rng, rows, cols, act), norm_rows(rng, 1, cols, act)
    xt.copy_(M.act_tensor(x, act))
    wt = M.act_tensor(w, act)[0]
    check_norm(x, None, w, act, 127, M.add_rms_norm(xt, wt, qmax=127))
    q, pl, a, sc, bt, ad, b = decode_case(W.W4G128, act, rows, 64, cols, 2, False)
    dense = M.linear_decode(pl, M.act_tensor(x, act))
    out = big.as_strided((rows, 64), (ld, 1), 1024)     # outputs as far apart
    M.linear_decode(pl, xt, out=out)
    assert torch.equal(out.contiguous().view(torch.int16), dense.view(torch.int16))
    check_norm(x, None, w, act, 0, (M.add_rms_norm(xt, wt)[0], None, None, None))


# ------------------------------------------- every launch form against its oracle
def decode_want(q, ad, b, act):
    """What a decode linear gives for decoded rows ad, and how far the stored values
    may be from it (the models of check_decode)."""
    wd = O.dequant(q, act)
    want = ad @ wd.T
    if q.scheme == W.W8A8:
        bound = 4 * TL.U32 * np.abs(want)
    elif q.scheme == W.FP8:
        bound = TL.fp8_block_bound(ad, wd) + 4 * TL.U32 * np.abs(want)
    else:
        bound = TL.acc_bound(np.abs(ad), np.abs(wd))
    want = want + O.act_values(b, act)
    return want, TL.slot_bound(want, bound + 2 * TL.U32 * np.abs(want) + 1e-30, act)


@pytest.mark.parametrize("scheme", DECODE_SCHEMES, ids=lambda s: s.name)
@pytest.mark.parametrize("n,k", [(4096, 1408), (4112, 1152), (8208, 1408), (12304, 1152), (16400, 1408), (20480, 1152),
                                 (24592, 1152)])
def test_decode_four_fragments(scheme, n, k):
    """49 to 64 rows: one, two and three blocks of channels to a workgroup, by 4 and by 8
    wavefronts, the last workgroup not full; past 12288 channels the 16-bit rows lie in
    LDS that the workgroup shares, a chunk of 4 k blocks at a time (9 and 11 k blocks: the
    last chunk is not full, and the workgroups start at different ones)."""
    torch = torch_mod()
    q = W.quantize_linear(W.draw_weight(n, 1, 0, n, k), scheme)
    rng = np.random.default_rng(n + k)
    for act in ("bf16", "fp16"):
        pl = M.PackedLinear(q, act)
        b, x = W.f64_to_act(rng.standard_normal((1, n)), act), W.f64_to_act(rng.standard_normal((64, k)), act)
        xv = O.act_values(x, act)
        if scheme == W.W4G128:
            a, sc, ad = M.act_tensor(x, act), None, xv
        else:
            codes, s = O.act_quant(xv, 127) if scheme == W.W8A8 else O.fp8_quant(xv)
            a, sc = torch.from_numpy(codes.view(np.int8).copy()).cuda(), torch.from_numpy(s.copy()).cuda()
            ad = (codes.astype(np.float64) if scheme == W.W8A8 else O.e4m3_values(codes)) * s.astype(np.float64)[:, None]
        want, bound = decode_want(q, ad, b, act)
        for m in (49, 63, 64):
            got = M.linear_decode(pl, a[:m], scales=None if sc is None else sc[:m], bias=M.act_tensor(b, act)[0])
            off = np.abs(O.act_values(M.act_numpy(got, act), act) - want[:m]) / bound[:m]
            assert off.max() <= 1.0, (act, m, float(off.max()))
            say(f"decode {scheme.name} {act} {m}x{n}x{k}: {off.max():.3f} of the bound")


def balance_want(l, ids, mask, alpha):
    """The definition in 64 bits, whole arrays at a time: (loss, counts, probabilities,
    gradient) and how far the kernel's may be from them.

    With d = l - max l of a token, exp errs by the rounding of d (|d| U32 of its value)
    and 4 U32 (2 units in the last place); the sum s by its terms' errors and at most 22
    additions; 1 / s and the product by 2 U32 more: p within e = (|d| + sum p |d| + 32)
    U32 of its value.  The probabilities' sums are held in 64 bits up to four roundings (a
    wavefront's, a workgroup's, a fold's and the result's): 5 U32, however many the tokens.
    f - sum f p errs as f (1 rounding), the products and at most 22 additions do."""
    T, E = l.shape
    k = ids.shape[1]
    kept = np.ones(T, bool) if mask is None else np.asarray(mask, bool)
    n = max(1, int(kept.sum()))
    x = np.where(kept[:, None], l, -np.inf).astype(np.float64)
    top = x.max(axis=1, keepdims=True)
    d = np.where(np.isfinite(x), x - np.where(np.isfinite(top), top, 0.0), -np.inf)
    p = np.exp(d)
    p /= np.where(p.sum(axis=1, keepdims=True) > 0, p.sum(axis=1, keepdims=True), 1.0)
    d = np.where(p > 0, np.abs(d), 0.0)
    e = d + (p * d).sum(axis=1, keepdims=True) + 32
    of = ids[kept]
    c = np.bincount(of[(of >= 0) & (of < E)], minlength=E)
    f = c / (k * n)
    P = p.sum(axis=0) / n
    fp = (p * f).sum(axis=1, keepdims=True)
    g = alpha * E / n * p * (f - fp)
    off_P = TL.U32 * ((p * e).sum(axis=0) / n + 5 * P) + 1e-37
    L = alpha * E * float((f * P).sum())
    off_L = abs(alpha) * E * float((f * off_P).sum()) + 2 * TL.U32 * abs(L) + 1e-37
    off_g = TL.U32 * abs(alpha) * E / n * p * ((e + 6) * (f + fp) + (p * f * (e + 24)).sum(axis=1, keepdims=True)) + 1e-37
    return (L, c, P, g), (off_L, off_P, off_g)


def check_balance64(l, ids, mask, alpha, got):
    loss, counts, probs, grad = [None if t is None else t.cpu().numpy() for t in got]
    (L, c, P, g), (off_L, off_P, off_g) = balance_want(l, ids, mask, alpha)
    assert np.array_equal(counts, c)
    assert np.all(np.abs(probs - P) <= off_P), float((np.abs(probs - P) / off_P).max())
    assert abs(float(loss) - L) <= off_L
    if grad is not None:
        assert np.all(np.abs(grad - g) <= off_g), float((np.abs(grad - g) / off_g).max())


# one workgroup, and two or three launches, for every number of lanes and logits to a lane; batches that take
# a workgroup's loops round again (2000 x 3, 140001 x 64, 300007 x 8), and shares that are folded (30011 x 160)
BALANCE_FORMS = [(300, 12, 2), (5000, 16, 2), (300, 32, 4), (9000, 24, 3), (60, 300, 2), (40, 512, 8), (900, 512, 8),
                 (2600, 384, 2), (5000, 1, 1), (2500, 3, 2), (3000, 2, 1), (1500, 5, 5), (60, 128, 4), (50, 200, 4),
                 (33, 100, 3), (2000, 3, 3), (30011, 160, 6), (140001, 64, 8), (300007, 8, 2)]


@pytest.mark.parametrize("masked", [0.0, 0.3])
@pytest.mark.parametrize("T,E,k", BALANCE_FORMS)
def test_balance_forms(T, E, k, masked):
    torch = torch_mod()
    l, ids, mask = balance_case(T, E, k, T + E, masked)
    lt, it = torch.from_numpy(l).cuda(), torch.from_numpy(ids).cuda()
    mt = None if mask is None else torch.from_numpy(mask).cuda()
    got = M.balance_loss(lt, it, alpha=0.7, token_mask=mt)
    check_balance64(l, ids, mask, 0.7, got)
    none = M.balance_loss(lt, it, alpha=0.7, token_mask=mt, want_grad=False)
    for a, b in zip(none[:3], got[:3]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("masked", [0.0, 0.3])
@pytest.mark.parametrize("T,E,k", BALANCE_FORMS)
def test_balance_counts_every_token_once(T, E, k, masked):
    """Logits that are 0 for one expert and -inf for the others: probabilities of exactly 0 and
    1, whose sums are whole numbers, so that a token left out or taken twice shows in any
    batch; the gradient is 0."""
    torch = torch_mod()
    rng = np.random.default_rng(T + E)
    hot = (rng.random(T) ** 2 * E).astype(np.int64)
    l = np.full((T, E), -np.inf, np.float32)
    l[np.arange(T), hot] = 0.0
    mask = rng.random(T) >= masked if masked else np.ones(T, bool)
    loss, counts, probs, grad = M.balance_loss(torch.from_numpy(l).cuda(), torch.from_numpy(hot[:, None].astype(np.int32)).cuda(),
                                               token_mask=torch.from_numpy(mask).cuda() if masked else None)
    c, n = np.bincount(hot[mask], minlength=E), int(mask.sum())
    assert np.array_equal(counts.cpu().numpy(), c)
    probs = probs.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(probs - c / n) <= 1.001 * TL.U32 * c / n)      # one rounding, that of the result
    want = E * float(((c / n) ** 2).sum())
    assert abs(float(loss) - want) <= 1.001 * TL.U32 * want
    assert not bool(grad.any())


@pytest.mark.parametrize("T,E,k", [(48, 8, 2), (700, 60, 4)])
def test_balance_gradient_in_a_backward_pass(T, E, k):
    """The gradient enters a backward pass beside another loss of the same logits, as the binding
    says; the reference differentiates the sum of both in 64 bits on the CPU.  The returned
    tensors have no graph of their own."""
    torch = torch_mod()
    alpha, H = 0.25, 32
    g = torch.Generator().manual_seed(T)
    x, r = torch.randn(T, H, generator=g), torch.randn(H, E, generator=g) * 0.3
    v = torch.randn(T, E, generator=g) * 0.01
    xg, rg = x.cuda(), r.cuda().requires_grad_()
    logits = (xg[:, :, None] * rg[None]).sum(1)
    ids = torch.topk(logits.detach(), k, dim=1).indices.to(torch.int32)
    loss, counts, probs, grad = M.balance_loss(logits, ids, alpha=alpha)
    assert not any(t.requires_grad for t in (loss, counts, probs, grad))
    main = (torch.softmax(logits, 1) * v.cuda()).sum()
    torch.autograd.backward([main, logits], [None, grad])
    # in 64 bits, from the same 32-bit logits (their own rounding is not the loss's)
    l = logits.detach().cpu().double().requires_grad_()
    p = torch.softmax(l, 1)
    f = torch.bincount(ids.cpu().reshape(-1).long(), minlength=E).double() / (k * T)
    ((p * v.double()).sum() + alpha * E * (f * p.mean(0)).sum()).backward()
    want = (x.double().t() @ l.grad).numpy()
    # both gradients of the logits are p (u - sum u p) for some u: (|d| + sum p |d| + 32 + 50) U32 of p (|u| + sum |u| p)
    # covers theirs (at most 50 more roundings where sums go one by one); then T products are added up
    with torch.no_grad():
        d = l.amax(1, keepdim=True) - l
        e = d + (p * d).sum(1, keepdim=True) + 32 + 50 + E
        u = v.double().abs() + alpha * E / T * f
        off = TL.U32 * 2 * e * p * (u + (u * p).sum(1, keepdim=True))
        bound = (x.double().abs().t() @ (off + (T + 2) * TL.U32 * l.grad.abs())).numpy()
    assert np.all(np.abs(rg.grad.cpu().numpy() - want) <= bound)


@pytest.mark.parametrize("act", ["bf16", "fp16"])
@pytest.mark.parametrize("cols", [200, 5000, 33000, 40003])
def test_norm_every_place(cols, act):
    """Every output in the place of every input that may give it up, rows held in registers
    and rows that are read again (past 32768 elements), with and without codes; what lies
    beside the rows stays as it was."""
    torch = torch_mod()
    lib = M.load_library()
    rng = np.random.default_rng(cols)
    rows, pad, off = 3, 21, 5
    ld = cols + pad
    x, res, w = norm_rows(rng, rows, cols, act), norm_rows(rng, rows, cols, act), norm_rows(rng, 1, cols, act)
    wt = M.act_tensor(w, act)[0]
    # (residual given, where z goes, where y goes): "x", "r" the inputs' places, "n" new rows, "" nowhere
    for has_res, zp, yp in ((True, "r", "x"), (True, "x", "r"), (True, "x", "n"), (True, "r", ""), (True, "x", ""),
                            (True, "", "x"), (True, "", "r"), (True, "n", "x"), (True, "n", "r"), (False, "", "x")):
        for qmax in (0, 127, 448):
            if not yp and not qmax:
                continue
            at = {"": (None, None), "n": strided(torch, x, act, pad, off), "x": strided(torch, x, act, pad, off),
                  "r": strided(torch, res, act, pad, off)}
            codes = torch.full((rows, cols), 99, dtype=torch.int8, device="cuda") if qmax else None
            scales = torch.full((rows,), 99.0, device="cuda") if qmax else None
            p = {k: None if v[0] is None else v[0].data_ptr() for k, v in at.items()}
            st = lib.mxmoe_add_rms_norm(p["x"], ld, p["r"] if has_res else None, ld, wt.data_ptr(), M.act_code(act), rows, cols,
                                        1e-6, p[zp], ld, p[yp], ld, qmax, M._ptr(codes), M._ptr(scales), M._stream_ptr())
            assert st == M.OK
            y, z, _ = O.add_rms_norm(O.act_values(x, act), O.act_values(res, act) if has_res else None, O.act_values(w, act)[0],
                                     act, 1e-6)
            if zp:
                assert np.array_equal(bits(at[zp][0]), act_bits(z, act)), (has_res, zp, yp, qmax)
            if yp:
                assert np.array_equal(bits(at[yp][0]), act_bits(y, act)), (has_res, zp, yp, qmax)
            if qmax:
                qc, qs = O.act_quant(y, qmax) if qmax == 127 else O.fp8_quant(y)
                assert np.array_equal(scales.cpu().numpy().view(np.uint32), qs.view(np.uint32))
                assert np.array_equal(codes.cpu().numpy().view(np.uint8), qc.view(np.uint8))
            for k in ("x", "r"):                        # an input whose place is not given up is as it was
                v, wide = at[k]
                if k not in (zp, yp):
                    assert np.array_equal(bits(v), bits(M.act_tensor(x if k == "x" else res, act)))
                v[:] = 77.0
                assert bool((wide == 77.0).all())


@pytest.mark.parametrize("m,n,k", [(1, 64, 1408), (1, 4096, 4096), (5, 64, 1408), (20, 4112, 384), (40, 64, 640), (64, 8208, 384),
                                   (64, 12304, 1152)])
def test_decode_w4_large_rows(m, n, k):
    """bf16 rows near the end of the range, of one sign and of both: the sums that a group
    goes through stay below 31 sum |a|, so the outputs are finite and as near as any
    others'.  (sum |a| of a group is below 2^123 here, 31 times it below 2^128.)"""
    torch_mod()
    rng = np.random.default_rng(m + n + k)
    q = W.quantize_linear(W.draw_weight(n, 1, 0, n, k), W.W4G128)
    pl = M.PackedLinear(q, "bf16")
    v = rng.uniform(1.0, 2.0, (m, k)) * 2.0 ** 115
    v[m // 2:] *= rng.choice([-1.0, 1.0], (m - m // 2, k))
    if m == 1:
        v = np.abs(v)
    a, b = W.f64_to_act(v, "bf16"), W.f64_to_act(rng.standard_normal((1, n)), "bf16")
    want, bound = decode_want(q, O.act_values(a, "bf16"), b, "bf16")
    got = O.act_values(M.act_numpy(M.linear_decode(pl, M.act_tensor(a, "bf16"), bias=M.act_tensor(b, "bf16")[0]), "bf16"), "bf16")
    assert np.isfinite(got).all()
    assert np.all(np.abs(got - want) <= bound)


@pytest.mark.parametrize("T,E", [(1 << 22, 8), (1 << 20, 64), (1 << 17, 512)])
def test_balance_like_tokens(T, E):
    """A batch of one token over and over: the mean probabilities are the token's own, at most
    four roundings apart (a wavefront's sum, a workgroup's, a fold's, the result's; the mean
    of 2^j tokens is exact), however many tokens a lane adds up."""
    torch = torch_mod()
    row = torch.from_numpy(np.random.default_rng(E).standard_normal((1, E)).astype(np.float32)).cuda()
    one = M.balance_loss(row, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), want_grad=False)[2].double()
    ids = torch.zeros(T, 1, dtype=torch.int32, device="cuda")
    probs = M.balance_loss(row.expand(T, E).contiguous(), ids, want_grad=False)[2].double()
    assert bool(((probs - one).abs() <= 5 * TL.U32 * one).all()), float(((probs - one).abs() / one).max() / TL.U32)


@pytest.mark.parametrize("act", ["bf16", "fp16"])
@pytest.mark.parametrize("n,k", [(8176, 4096), (8192, 3968), (8192, 4096), (12304, 4224), (16400, 4096), (20480, 3584)])
def test_decode_one_wide_row(n, k, act):
    """One row of w4g128 on both sides of 8192 channels and 4096 k, where the launch form changes,
    contiguous, at an odd place (the binding copies it) and with what follows it in its buffer
    left alone and unread (NaN)."""
    torch = torch_mod()
    q, pl, a, _, bt, ad, b = decode_case(W.W4G128, act, 1, n, k, n + k, True)
    ref = M.linear_decode(pl, a, bias=bt)
    check_decode(q, ad, b, act, ref)
    for off in (8, 3):
        wide = torch.full((2 * k + 64,), float("nan"), dtype=a.dtype, device="cuda")
        wide[off:off + k] = a[0]
        out = torch.full((n + 40,), 9.0, dtype=a.dtype, device="cuda")
        M.linear_decode(pl, wide[off:off + k][None], bias=bt, out=out[20:20 + n][None])
        assert torch.equal(out[20:20 + n].view(torch.int16), ref[0].view(torch.int16))
        assert bool((out[:20] == 9.0).all()) and bool((out[20 + n:] == 9.0).all())
