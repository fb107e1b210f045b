"""GPU parity of the operators of a decode step's attention against the fp64 oracle: heads into
the cache (queries within the fp32 roundings of norm and rotation, cached rows within half a
step of their codes, rows that nothing changes bit for bit), rows back, and the attention
over the cache within the error model below.

Error model of the attention.  With the cached values as given, a weight w_t is off by
  d = ACC16_EPS * scale * sum |q||k|  (fp32 sums of exact products, tests/tolerance.py)
      + 8 * 2^-24 * (1 + |x|_max)     (products by scales, the reference's difference, exp2)
      + min(cap * 2^-20, |x|_max * 2^-19) with a cap (tanh y = 1 - 2 / (1 + e^2y) for y > 0: the quotient
                                       and e^2y to 2^-22 each, twice the cap.  From y = 1/4 on, where
                                       2 / (1 + e^2y) <= 0.76 and tanh y >= 0.24, that is 2^-19 of tanh y;
                                       below, four terms more of its series leave out 2^-26 of it)
relative to itself, in the numerator and in the normalizer; the numerator's weights are rounded
once more, by at most u = eps / 2 of the dtype of the product (2^-8 bf16, 2^-11 fp16), and both
sums are fp32 (ACC16_EPS each).  So |out - ref| <= (2 d + u + 2 ACC16_EPS) * sum p|v|, and half a
step of the output's dtype."""

import ctypes as C

import numpy as np
import pytest

from oracle import mxmoe_oracle as O
from paper_2505_05799_amd import mxmoe as M
from paper_2505_05799_amd import workloads as W
from tests import tolerance as TL
from tests.gpuhelp import say, torch_mod

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


def rows(rng, shape, act, scale=1.0):
    return O.act_values(W.f64_to_act(rng.standard_normal(shape) * scale, act), act)


def up(a, act):
    """fp64 values that the dtype holds -> GPU tensor"""
    torch = torch_mod()
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda").to(torch.bfloat16 if act == "bf16" else torch.float16)


def down(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def i32(a):
    torch = torch_mod()
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to("cuda")


def all_bytes(cache):
    torch = torch_mod()
    return [t.clone().view(torch.uint8) for t in cache.buffers() if t is not None]


# ------------------------------------------------------------------ append, read
def head_error(x, w, positions, freqs, interleaved):
    """(y, e): the oracle's rows and what fp32 may be off by.  Three roundings of the norm (the
    factor, two products), a cosine and a sine to 2^-22.1 (the angle in turns to 2^-26, sincospi
    to 2^-23), two products and a sum: under 9 * 2^-24 of |a| + |b|."""
    y = O.head_rows(x, w, 1e-6, positions, freqs, interleaved)
    y0 = np.abs(O.head_rows(x, w, 1e-6, None, None))
    e = 3 * TL.U32 * y0 if w is not None else 0 * y0
    if freqs is not None and len(freqs):
        half = len(freqs)
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        s = 9 * TL.U32 * (y0[..., a] + y0[..., b])
        e[..., a], e[..., b] = s, s
    return y, e


def check_cached(got, y, e, qmax, act, where=""):
    """Rows read back from the cache against the rows that went in (within e of y)."""
    bound = e.copy()
    if qmax:
        amax = np.abs(y).max(axis=-1, keepdims=True)
        if qmax == 127:
            half = 0.5 * amax / 127
        else:
            half = np.maximum(2.0 ** -4 * (np.abs(y) + e), 2.0 ** -10 * amax / 448)
        # half a step, e of the row's largest in the scale, four roundings of fp32
        bound = bound + half * (1 + 2.0 ** -18) + e.max(axis=-1, keepdims=True) + 4 * TL.U32 * np.abs(y)
    bound = TL.slot_bound(y, bound, act)
    err = np.abs(got - y)
    assert np.all(err <= bound), (where, float((err / bound).max()))


def exact_read(x, qmax, act):
    """What comes back of rows that are cached as they are, bit for bit."""
    codes, scales = O.cache_rows(x, qmax)
    if qmax == 0:
        return x
    v = O.e4m3_values(codes.view(np.uint8)) if qmax == 448 else codes.astype(np.float64)
    return O.round_to_act((v.astype(np.float32) * scales[..., None]).astype(np.float64), act)


APPEND = [  # tokens, q heads, kv heads, dim, rot, interleaved, norm, page, pad
    (1, 32, 8, 128, 128, False, True, 64, 0), (1, 1, 1, 64, 64, True, False, 32, 0), (3, 4, 2, 128, 64, False, True, 32, 8),
    (5, 7, 1, 256, 256, False, True, 128, 13), (33, 5, 5, 64, 32, True, True, 32, 1), (64, 2, 1, 128, 0, False, True, 64, 0),
    (97, 0, 3, 128, 128, False, False, 64, 0), (130, 6, 2, 256, 16, True, True, 1024, 3), (257, 14, 2, 64, 48, False, True, 64, 0),
    (700, 3, 3, 128, 0, False, False, 256, 5), (1100, 2, 2, 128, 128, True, True, 128, 2)]


@pytest.mark.parametrize("act", ["bf16", "fp16"])
@pytest.mark.parametrize("qmax", [0, 127, 448])
@pytest.mark.parametrize("T,hq,kv,dim,rot,inter,norm,page,pad", APPEND)
def test_append(T, hq, kv, dim, rot, inter, norm, page, pad, qmax, act):
    torch = torch_mod()
    rng = np.random.default_rng(T * 100 + dim + rot)
    wide = up(rows(rng, (T, (hq + 2 * kv) * dim + pad), act, 2.0), act)
    host = down(wide)
    part = lambda a, lo, n: a[:, lo * dim:(lo + n) * dim].reshape(T, n, dim)  # noqa: E731
    view = lambda lo, n: wide[:, lo * dim:(lo + n) * dim].unflatten(1, (n, dim)) if n else None  # noqa: E731
    q, k, v = part(host, 0, hq), part(host, hq, kv), part(host, hq + kv, kv)
    qw, kw = (rows(rng, dim, act, 0.2) + 1 if norm else None for _ in range(2))
    qw, kw = (None if w is None else O.round_to_act(w, act) for w in (qw, kw))
    pos = rng.integers(0, 200000, T)
    freqs = 1e6 ** (-np.arange(rot // 2) / max(rot // 2, 1))
    n_pages = -(-T // page) + 2
    slots = rng.permutation(n_pages * page)[:T] if T % 2 else (np.arange(T) + 32)   # anywhere, or a run
    slots = slots.astype(np.int32)
    if T > 4:
        slots[[2, 4]] = (-1, n_pages * page)                                        # not kept
    kept = (slots >= 0) & (slots < n_pages * page)
    cache = M.KVCache(n_pages, kv, dim, page_size=page, act=act, qmax=qmax)
    for t in cache.buffers():
        if t is not None:
            t.view(torch.uint8).fill_(0x55)
    got = M.kv_append(cache, view(hq, kv), view(hq + kv, kv), i32(slots), q=view(0, hq),
                      q_weight=None if qw is None or not hq else up(qw, act), k_weight=None if kw is None else up(kw, act),
                      positions=i32(pos) if rot else None, freqs=torch.from_numpy(freqs).to("cuda") if rot else None,
                      interleaved=inter)
    f = freqs if rot else None
    if hq:
        y, e = head_error(q, qw, pos, f, inter)
        err, bound = np.abs(down(got) - y), TL.slot_bound(y, e, act)
        assert got.shape == (T, hq, dim) and np.all(err <= bound), float((err / bound).max())
    else:
        assert got is None
    kb, vb = M.kv_read(cache, i32(slots))
    gk, gv = down(kb), down(vb)
    assert not gk[~kept].any() and not gv[~kept].any()
    y, e = head_error(k, kw, pos, f, inter)
    check_cached(gk[kept], y[kept], e[kept], qmax, act)
    assert np.array_equal(gv[kept], exact_read(v, qmax, act)[kept])
    if kw is None and not rot:
        assert np.array_equal(gk[kept], exact_read(k, qmax, act)[kept])
    # nothing but the kept slots has been written: every other slot reads as before
    others = np.setdiff1d(np.arange(n_pages * page), slots)
    fresh = M.KVCache(n_pages, kv, dim, page_size=page, act=act, qmax=qmax)
    for t in fresh.buffers():
        if t is not None:
            t.view(torch.uint8).fill_(0x55)
    for a, b in zip(M.kv_read(cache, i32(others)), M.kv_read(fresh, i32(others))):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    assert torch.equal(wide, up(host, act))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("qmax", [0, 127, 448])
def test_append_writes_each_byte_of_a_page(dim, qmax):
    """All slots of a page written, in another order: no byte of the page left, none of its neighbours touched."""
    torch = torch_mod()
    rng = np.random.default_rng(dim)
    kv, page = 2, 64
    cache = M.KVCache(3, kv, dim, page_size=page, act="bf16", qmax=qmax)
    for t in cache.buffers():
        if t is not None:
            t.view(torch.uint8).fill_(0x80)       # (no code of a row below, nor a byte of its scale)
    x = np.abs(rows(rng, (page, kv, dim), "bf16")) + 1.0
    x = O.round_to_act(x, "bf16")
    order = rng.permutation(page)
    M.kv_append(cache, up(x[order], "bf16"), up(x[order], "bf16"), i32(page + order))
    gk, gv = M.kv_read(cache, i32(np.arange(page, 2 * page)))
    want = exact_read(x, qmax, "bf16")
    assert np.array_equal(down(gk), want) and np.array_equal(down(gv), want)
    for t in cache.buffers():
        if t is None:
            continue
        b = t.view(torch.uint8)
        assert bool((b[0] == 0x80).all()) and bool((b[2] == 0x80).all())
        if t.dtype is torch.int8:
            assert not bool((b[1] == 0x80).any())


@pytest.mark.parametrize("act", ["bf16", "fp16"])
def test_append_special_rows(act):
    torch = torch_mod()
    rng = np.random.default_rng(3)
    dim, kv = 128, 2
    x = rows(rng, (8, kv, dim), act)
    x[1, 0] = 0
    x[2, 1, 5] = np.inf
    x[3, 0, 127] = np.nan
    x[4] *= 2.0 ** -12
    x[5, 0, 0] = 60000.0
    x = np.where(np.isfinite(x), O.round_to_act(np.where(np.isfinite(x), x, 0.0), act), x)   # what the dtype holds of them
    for qmax in (127, 448):
        cache = M.KVCache(2, kv, dim, page_size=32, act=act, qmax=qmax)
        M.kv_append(cache, up(x, act), up(x, act), i32(np.arange(8)))
        for g in M.kv_read(cache, i32(np.arange(8))):
            g = down(g)
            assert not g[1, 0].any()
            assert np.isnan(g[2, 1]).all() and np.isnan(g[3, 0]).all()
            with np.errstate(invalid="ignore"):
                ok = np.isfinite(x).all(axis=-1)
            clean = np.where(np.isfinite(x), x, 0)
            assert np.array_equal(g[ok], exact_read(clean, qmax, act)[ok])
    # 16-bit rows pass as they are, the queries' norm of zeros is zero and of infinity NaN
    cache = M.KVCache(2, kv, dim, page_size=32, act=act)
    w = up(np.ones(dim), act)
    q = M.kv_append(cache, up(x, act), up(x, act), i32(np.arange(8)), q=up(x, act), q_weight=w)
    for g in M.kv_read(cache, i32(np.arange(8))):
        assert np.array_equal(down(g), x, equal_nan=True)
    q = down(q)
    assert not q[1, 0].any() and np.isnan(q[3, 0]).all() and not np.isfinite(q[2, 1, 5])
    if act == "bf16":   # squares past the fp32 range, rows below the normal one
        y = np.full((2, kv, dim), 2.0 ** 100)
        y[1] = 2.0 ** -130
        q = M.kv_append(cache, up(y, act), up(y, act), i32([0, 1]), q=up(y, act), q_weight=w, eps=1e-30)
        assert np.array_equal(down(q)[0], np.ones((kv, dim)))
        assert np.all(np.abs(down(q)[1] - 2.0 ** -130 * 1e15) <= 2.0 ** -7 * 2.0 ** -80)
        c8 = M.KVCache(2, kv, dim, page_size=32, act=act, qmax=127)
        M.kv_append(c8, up(y, act), up(y, act), i32([0, 1]))
        got = down(M.kv_read(c8, i32([0, 1]))[0])
        assert np.array_equal(got[0], exact_read(y[:1], 127, act)[0]) and not got[1].any()


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("qmax", [0, 127, 448])
def test_append_large_rows_and_weights(qmax, inter):
    """Rows whose products with the norm's weight pass the largest value, though the normalized rows are ordinary;
    and small ones."""
    torch = torch_mod()
    rng = np.random.default_rng(17)
    T, hq, kv, dim = 40, 2, 2, 128
    x = rows(rng, (T, hq + kv, dim), "bf16") * np.where(np.arange(T) % 2, 2.0 ** 122, 2.0 ** -60)[:, None, None]
    qw, kw = (O.round_to_act(rows(rng, dim, "bf16", 8.0) + 64, "bf16") for _ in range(2))
    pos, freqs = rng.integers(0, 5000, T), 1e4 ** (-np.arange(32) / 32)
    cache = M.KVCache(2, kv, dim, page_size=32, act="bf16", qmax=qmax)
    v = up(rows(rng, (T, kv, dim), "bf16"), "bf16")
    got = M.kv_append(cache, up(x[:, hq:], "bf16"), v, i32(np.arange(T)), q=up(x[:, :hq], "bf16"), q_weight=up(qw, "bf16"),
                      k_weight=up(kw, "bf16"), positions=i32(pos), freqs=torch.from_numpy(freqs).cuda(), interleaved=inter)
    y, e = head_error(x[:, :hq], qw, pos, freqs, inter)
    assert np.all(np.abs(down(got) - y) <= TL.slot_bound(y, e, "bf16"))
    y, e = head_error(x[:, hq:], kw, pos, freqs, inter)
    check_cached(down(M.kv_read(cache, i32(np.arange(T)))[0]), y, e, qmax, "bf16")


@pytest.mark.parametrize("inter", [False, True])
def test_append_in_place_and_far_positions(inter):
    torch = torch_mod()
    rng = np.random.default_rng(4)
    T, hq, dim = 9, 4, 128
    x = rows(rng, (T, hq + 2, dim), "fp16")
    pos = np.array([0, 1, 2 ** 20, 2 ** 24 + 1, 10 ** 9 + 7, 2 ** 31 - 1, -5, -2 ** 31, 131071])
    freqs = 1e4 ** (-np.arange(64) / 64)
    wide = up(x, "fp16")
    cache = M.KVCache(1, 1, dim, page_size=32, act="fp16")
    q, k, v = wide[:, :hq], wide[:, hq:hq + 1], wide[:, hq + 1:]
    got = M.kv_append(cache, k, v, i32(np.arange(T)), q=q, q_out=q, positions=i32(pos), freqs=torch.from_numpy(freqs).cuda(),
                      interleaved=inter)
    assert got.data_ptr() == wide.data_ptr()
    # 2^31 * frequency to 2^-53 twice: 2^-20 radians at the most
    y, e = head_error(x, None, pos, freqs, inter)
    far = 2.0 ** -52 * np.abs(pos.astype(np.float64))[:, None, None] * np.abs(x).max()
    err = np.abs(down(q) - y[:, :hq])
    assert np.all(err <= TL.slot_bound(y, e + far, "fp16")[:, :hq])
    assert np.array_equal(down(wide)[:, hq:], x[:, hq:])
    gk = down(M.kv_read(cache, i32(np.arange(T)))[0])
    assert np.all(np.abs(gk - y[:, hq:hq + 1]) <= TL.slot_bound(y, e + far, "fp16")[:, hq:hq + 1])


# ------------------------------------------------------------------ attention
class Case:
    """A cache of random rows and sequences that lie on its pages in any order."""

    def __init__(self, seed, lengths, n_q=1, hq=4, kv=2, dim=128, act="bf16", qmax=127, page=32, prefix=0, kscale=1.0,
                 vscale=1.0, spread=0.3, extra=1):
        rng = np.random.default_rng(seed)
        self.lengths, self.n_q, self.hq, self.kv, self.dim, self.act, self.qmax = np.array(lengths), n_q, hq, kv, dim, act, qmax
        self.page, self.prefix_len = page, prefix
        B = len(lengths)
        first = -(-prefix // page)
        width = max(-(-max(0, int(n) - prefix) // page) for n in lengths) + extra
        own = [max(0, -(-(int(n) - prefix) // page)) for n in lengths]
        n_pages = first + sum(own) + 2
        ids = rng.permutation(n_pages)
        self.prefix = ids[:first]
        self.table = np.full((B, max(width, 0)), -7)
        at = first
        for b in range(B):
            self.table[b, :own[b]] = ids[at:at + own[b]]
            at += own[b]
        n = n_pages * page
        size = lambda: np.exp(spread * rng.standard_normal((n, kv, 1)))  # noqa: E731
        k = O.round_to_act(rows(rng, (n, kv, dim), act) * size() * kscale, act)
        v = O.round_to_act(rows(rng, (n, kv, dim), act) * size() * vscale, act)
        self.cache = M.KVCache(n_pages, kv, dim, page_size=page, act=act, qmax=qmax)
        M.kv_append(self.cache, up(k, act), up(v, act), i32(np.arange(n)))
        self.k, self.v = (O.cache_values(*O.cache_rows(x, qmax), qmax) for x in (k, v))
        self.q = rows(rng, (B * n_q, hq, dim), act)
        self.scale, self.softcap = dim ** -0.5, 0.0

    def run(self, **kw):
        pre = i32(self.prefix) if self.prefix_len else None
        return M.attention_decode(self.cache, up(self.q, self.act), i32(self.table), i32(self.lengths), prefix=pre,
                                  prefix_len=self.prefix_len, scale=self.scale, softcap=self.softcap, **kw)

    def slots(self, b):
        n, p = int(self.lengths[b]), self.page
        pre = [int(self.prefix[t // p]) * p + t % p for t in range(min(n, self.prefix_len))]
        return np.array(pre + [int(self.table[b, t // p]) * p + t % p for t in range(max(0, n - self.prefix_len))], dtype=int)

    def check(self, got, only=None, where=""):
        got, worst = down(got), 0.0
        u = U["bf16" if self.act == "bf16" and self.qmax == 0 else "fp16"]
        for b in range(len(self.lengths)) if only is None else only:
            at = self.slots(b)
            k, v, q = self.k[at], self.v[at], self.q[b * self.n_q:(b + 1) * self.n_q]
            seen = [len(at) - self.n_q + 1 + j for j in range(self.n_q)]
            ref, mass = O.attention(q, k, v, seen, self.scale, self.softcap)
            g = got[b * self.n_q:(b + 1) * self.n_q]
            if len(at):
                qk = np.einsum("jhd,thd->jht", np.abs(q), np.repeat(np.abs(k), self.hq // self.kv, axis=1)).max(axis=2)
            else:
                qk = np.zeros((self.n_q, self.hq))
            x = abs(self.scale) * qk
            d = TL.ACC16_EPS * x + 8 * TL.U32 * (1 + x) + (np.minimum(self.softcap * 2.0 ** -20, x * 2.0 ** -19) if self.softcap else 0)
            bound = TL.slot_bound(ref, (2 * d[..., None] + u + 2 * TL.ACC16_EPS) * mass, self.act)
            for j in range(self.n_q):
                if seen[j] <= 0:
                    assert not g[j].any(), (where, b, j)
                    continue
                err = np.abs(g[j] - ref[j])
                assert np.all(err <= bound[j]), (where, b, j, float((err / bound[j]).max()))
                worst = max(worst, float((err / bound[j]).max()))
        return worst


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 300, 513]


@pytest.mark.parametrize("act", ["bf16", "fp16"])
@pytest.mark.parametrize("qmax", [0, 127, 448])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attention_lengths(dim, qmax, act):
    c = Case(dim + qmax, LENGTHS, dim=dim, qmax=qmax, act=act)
    say(f"attention {dim} {qmax} {act}: worst err / bound {c.check(c.run()):.3f}")


@pytest.mark.parametrize("n_q,hq,kv,page", [(1, 1, 1, 32), (1, 8, 8, 64), (1, 16, 1, 128), (1, 17, 1, 32), (2, 12, 2, 32),
                                            (4, 14, 2, 64), (5, 21, 3, 32), (16, 2, 1, 32), (3, 40, 1, 256), (16, 16, 2, 64),
                                            (1, 130, 1, 32), (7, 33, 3, 1024)])
@pytest.mark.parametrize("qmax", [0, 127, 448])
def test_attention_heads_and_queries(n_q, hq, kv, page, qmax):
    c = Case(n_q * 100 + hq, [0, 1, n_q - 1, n_q, n_q + 1, 40, 95, 96, 230], n_q=n_q, hq=hq, kv=kv, dim=64, page=page, qmax=qmax)
    c.check(c.run())


@pytest.mark.parametrize("qmax,dim,act", [(127, 128, "bf16"), (448, 64, "fp16"), (0, 256, "bf16"), (0, 128, "fp16")])
def test_attention_long(qmax, dim, act):
    c = Case(qmax + dim, [5000, 1, 20011], hq=4, kv=2, dim=dim, qmax=qmax, act=act, page=128)
    c.check(c.run())
    c = Case(qmax + dim, [33000], n_q=2, hq=4, kv=1, dim=dim, qmax=qmax, act=act, page=256)
    c.check(c.run())


@pytest.mark.parametrize("cap", [0.5, 30.0])
@pytest.mark.parametrize("qmax", [0, 127, 448])
def test_attention_softcap(qmax, cap):
    c = Case(11, [1, 50, 333], n_q=2, qmax=qmax, kscale=4.0)
    c.softcap = cap
    c.check(c.run())
    c.scale = -0.05
    c.check(c.run())


@pytest.mark.parametrize("cap", [1e-30, 1e-3, 300.0, 1e5, 1e9, 1e30])
@pytest.mark.parametrize("qmax", [0, 127, 448])
def test_attention_caps_of_any_size(qmax, cap):
    """Caps far above the scores, which hardly change them, and far below, which leave all tokens alike."""
    c = Case(12, [1, 50, 333, 2100], n_q=2, qmax=qmax)
    c.softcap = cap
    c.check(c.run())


@pytest.mark.parametrize("qmax", [0, 127, 448])
def test_attention_sizes_that_meet(qmax, act="bf16"):
    """Small queries and large keys, and the other way round: the scores are ordinary."""
    for size in (2.0 ** 110, 2.0 ** -105):
        for cap in (0.0, 20.0):
            c = Case(13, [1, 70, 500], qmax=qmax, act=act, kscale=size)
            c.q = O.round_to_act(c.q / size * 2, act)
            c.softcap = cap
            c.check(c.run(), where=f"{size} {cap}")


@pytest.mark.parametrize("prefix", [1, 31, 32, 40, 64, 100, 777])
@pytest.mark.parametrize("qmax,dim", [(0, 128), (127, 128), (448, 64), (127, 256)])
def test_attention_prefix(prefix, qmax, dim):
    """Sequences behind a prefix, some that end inside it; and the same as a table in which its pages come first."""
    torch = torch_mod()
    lengths = [0, 1, max(0, prefix - 1), prefix, prefix + 1, prefix + 33, prefix + 200, prefix // 2, prefix + 64, prefix + 3]
    for n_q, hq, kv in ((1, 4, 2), (3, 6, 1)):
        c = Case(prefix + n_q, lengths, n_q=n_q, hq=hq, kv=kv, dim=dim, qmax=qmax, prefix=prefix, page=32)
        got = c.run()
        c.check(got, where=f"prefix {n_q}")
        if prefix % c.page == 0:
            first = prefix // c.page
            table = np.concatenate([np.repeat(c.prefix[None, :first], len(lengths), axis=0), c.table], axis=1)
            same = M.attention_decode(c.cache, up(c.q, c.act), i32(table), i32(c.lengths))
            c.check(same, where="one table")


def test_attention_prefix_many_rows():
    c = Case(5, [700 + 3 * i for i in range(40)] + [0, 20, 699], n_q=1, hq=8, kv=2, dim=128, qmax=448, prefix=690, page=64)
    c.check(c.run())
    c = Case(6, [300] * 9, n_q=16, hq=8, kv=1, dim=64, qmax=0, prefix=250, page=64)
    c.check(c.run())


@pytest.mark.parametrize("qmax", [0, 127, 448])
def test_attention_large_scores_and_scales(qmax):
    """Scores that leave one token all the weight, growing along the sequence and falling; values of
    very different sizes, behind weights of either order."""
    for seed, kscale in ((1, 40.0), (2, 0.0)):
        c = Case(seed, [1, 64, 500], qmax=qmax, kscale=kscale, act="bf16", spread=1.5)
        c.check(c.run())
    rng = np.random.default_rng(9)
    for sign in (1, -1):
        c = Case(20 + sign, [400], hq=2, kv=1, qmax=qmax, dim=64, act="bf16")
        at = c.slots(0)
        ramp = np.linspace(-30, 30, 400)[::sign, None, None]
        base = rows(rng, (1, 1, 64), "bf16")
        k = O.round_to_act(base * ramp / 8, "bf16")
        v = O.round_to_act(rows(rng, (400, 1, 64), "bf16") * np.exp2(rng.integers(-20, 20, (400, 1, 1))), "bf16")
        M.kv_append(c.cache, up(k, "bf16"), up(v, "bf16"), i32(at))
        c.k[at], c.v[at] = (O.cache_values(*O.cache_rows(x, qmax), qmax) for x in (k, v))
        c.q = O.round_to_act(np.repeat(base, 2, axis=1) * 1.0, "bf16")
        c.check(c.run(), where=f"ramp {sign}")


def test_attention_tiny_and_zero_rows():
    for qmax in (127, 448):
        c = Case(3, [1, 40, 100], qmax=qmax, vscale=2.0 ** -60)
        c.check(c.run())
        c = Case(3, [40], qmax=qmax, vscale=0.0)
        assert not down(c.run()).any()
        c = Case(4, [70], qmax=qmax)
        c.q *= 2.0 ** -100
        c.check(c.run())
        c.q[:] = 0
        c.check(c.run())


def poison(c, slots, what):
    """Bytes of slots' rows replaced by NaN (16-bit rows and scales) or e4m3 NaN codes."""
    torch = torch_mod()
    n = len(slots)
    bad = torch.full((n, c.kv, c.dim), what, dtype=c.cache.dtype, device="cuda")
    M.kv_append(c.cache, bad, bad, i32(slots))


@pytest.mark.parametrize("qmax", [0, 127, 448])
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
def test_what_is_masked_does_not_matter(qmax, what):
    """NaN and inf past the last token (the rest of its page, other pages), e4m3 NaN codes there,
    and table entries past the end."""
    torch = torch_mod()
    lengths = [1, 5, 32, 33, 47, 64, 77]
    c = Case(31, lengths, qmax=qmax, dim=64)
    clean = c.run()
    c.check(clean)
    used = np.concatenate([c.slots(b) for b in range(len(lengths))])
    others = np.setdiff1d(np.arange(c.cache.n_pages * c.page), used)
    poison(c, others, what)
    c.table[c.table < 0] = 10 ** 6
    assert torch.equal(c.run().view(torch.int16), clean.view(torch.int16))
    if qmax == 448:   # codes that kv_append never writes
        whole = M.KVCache(c.cache.n_pages, c.kv, c.dim, page_size=c.page, act=c.act, qmax=qmax)
        k, v = M.kv_read(c.cache, i32(used))
        for t in whole.buffers():
            t.view(torch.uint8).fill_(0x7f)
        M.kv_append(whole, k, v, i32(used))
        c.cache = whole
        k2, v2 = M.kv_read(whole, i32(used))
        assert torch.isfinite(k2).all() and torch.isfinite(v2).all()
        assert torch.isfinite(c.run()).all()


@pytest.mark.parametrize("qmax", [0, 127, 448])
@pytest.mark.parametrize("n_q", [2, 5])
def test_later_tokens_do_not_reach_earlier_queries(qmax, n_q):
    """A value or key that is not finite at one of a sequence's last tokens: the queries before it
    are as without it, those that see it are not finite where it lies."""
    torch = torch_mod()
    for n in (33, 64, 37):
        c = Case(17, [n, 50], n_q=n_q, qmax=qmax, dim=64, hq=4, kv=2)
        clean = c.run()
        at = c.slots(0)
        for back in range(n_q - 1):            # token n - 1 - back is seen by queries n_q - 1 - back ..
            for what in (float("inf"), float("nan")):
                c = Case(17, [n, 50], n_q=n_q, qmax=qmax, dim=64, hq=4, kv=2)
                poison(c, at[n - 1 - back:n - back], what)
                got = c.run()
                first = n_q - 1 - back
                assert torch.equal(got[:first].view(torch.int16), clean[:first].view(torch.int16)), (n, back, what)
                assert not torch.isfinite(got[first:n_q]).any(), (n, back, what)
                assert torch.equal(got[n_q:].view(torch.int16), clean[n_q:].view(torch.int16))
    # inside a prefix: a sequence that ends before the token
    c = Case(18, [20, 60, 9, 39], qmax=qmax, dim=64, prefix=40)
    clean = c.run()
    poison(c, c.slots(1)[30:31], float("inf"))
    got = c.run()
    for b, hit in ((0, False), (1, True), (2, False), (3, True)):
        if hit:
            assert not torch.isfinite(got[b]).any()
        else:
            assert torch.equal(got[b].view(torch.int16), clean[b].view(torch.int16))


@pytest.mark.parametrize("qmax", [0, 127, 448])
def test_bad_pages_and_lengths(qmax):
    """Page ids outside the cache: NaN for the queries that see one of their tokens, nothing else."""
    torch = torch_mod()
    lengths = [70, 70, 31, 200, 64, 33]
    c = Case(41, lengths, n_q=3, qmax=qmax, dim=64)
    clean = c.run()
    c.check(clean)
    for id_ in (-1, c.cache.n_pages, 2 ** 31 - 1, -2 ** 31):
        table = c.table.copy()
        table[0, 2], table[3, 0], table[5, 1], table[2, 1:] = id_, id_, id_, id_    # [2]: past its end
        got = M.attention_decode(c.cache, up(c.q, c.act), i32(table), i32(c.lengths))
        nan = torch.isnan(got).all(dim=2).all(dim=1).cpu().numpy()
        # sequence 0: tokens 64 .. 69 are bad, all its queries see 64; 5: token 32, the last query alone
        want = np.zeros(18, bool)
        want[0:3], want[9:12], want[17] = True, True, True
        assert np.array_equal(nan, want)
        ok = torch.from_numpy(~want).cuda()
        assert torch.equal(got[ok].view(torch.int16), clean[ok].view(torch.int16))
    lengths = c.lengths.copy()
    lengths[[1, 4]] = (c.table.shape[1] * c.page + 1, -3)
    got = M.attention_decode(c.cache, up(c.q, c.act), i32(c.table), i32(lengths))
    assert torch.isnan(got[3:6]).all() and not got[12:15].any()
    keep = torch.tensor([0, 1, 2, 6, 7, 8, 9, 10, 11, 15, 16, 17]).cuda()
    assert torch.equal(got[keep].view(torch.int16), clean[keep].view(torch.int16))
    # a bad page of the prefix
    c = Case(42, [50, 10, 40, 33], qmax=qmax, dim=64, prefix=40)
    clean = c.run()
    c.prefix[1] = -1
    got = c.run()
    assert torch.isnan(got[[0, 2, 3]]).all() and torch.equal(got[1].view(torch.int16), clean[1].view(torch.int16))


def test_queries_that_are_not_finite():
    torch = torch_mod()
    for qmax in (0, 127, 448):
        c = Case(51, [40, 90, 33], n_q=2, qmax=qmax, dim=64, hq=4, kv=2)
        clean = c.run()
        c.q[1, 2, 7], c.q[4, 0, 0] = np.nan, np.inf
        got = c.run()
        assert not torch.isfinite(got[1, 2]).any() and not torch.isfinite(got[4, 0]).any()
        same = torch.ones(6, 4, dtype=torch.bool, device="cuda")
        same[1, 2] = same[4, 0] = False
        assert torch.equal(got[same].view(torch.int16), clean[same].view(torch.int16))


@pytest.mark.parametrize("pad", [8, 13])
def test_attention_strides(pad):
    torch = torch_mod()
    c = Case(61, [1, 77, 200], n_q=2, qmax=127)
    want = c.run()
    wide = torch.full((6, 4 * 128 + pad), 7.0, dtype=torch.bfloat16, device="cuda")
    q = wide[:, 3:3 + 512].unflatten(1, (4, 128))
    q.copy_(up(c.q, c.act))
    dst = torch.full((6, 4 * 128 + pad), 9.0, dtype=torch.bfloat16, device="cuda")
    o = dst[:, 5:5 + 512].unflatten(1, (4, 128))
    got = M.attention_decode(c.cache, q, i32(c.table), i32(c.lengths), out=o)
    assert got is o and torch.equal(o, want)
    assert bool((dst[:, :5] == 9).all()) and bool((dst[:, 517:] == 9).all())


def test_no_sequence_and_no_page():
    torch = torch_mod()
    c = Case(62, [5], qmax=127)
    e = torch.zeros(0, 4, 128, dtype=torch.bfloat16, device="cuda")
    assert M.attention_decode(c.cache, e, i32(np.zeros((0, 3))), i32(np.zeros(0))).shape == (0, 4, 128)
    q = up(c.q, c.act)
    got = M.attention_decode(c.cache, q, i32(np.zeros((1, 0))), i32([0]))
    assert not got.any()
    assert torch.isnan(M.attention_decode(c.cache, q, i32(np.zeros((1, 0))), i32([1]))).all()
    full = Case(63, [40, 20], qmax=127, prefix=40, extra=0)     # nothing but the prefix
    assert full.table.shape[1] == 0
    full.check(full.run())
    empty = torch.zeros(0, 2, 128, dtype=torch.bfloat16, device="cuda")
    assert M.kv_append(c.cache, empty, empty, i32(np.zeros(0))) is None
    assert M.kv_read(c.cache, i32(np.zeros(0)))[0].shape == (0, 2, 128)


def test_repeated_calls_are_equal():
    torch = torch_mod()
    for kw in (dict(lengths=[3000, 17, 900, 1]), dict(lengths=[2500, 2600, 2000], prefix=1990, n_q=2)):
        c = Case(71, qmax=448, **kw)
        a = c.run()
        for _ in range(5):
            assert torch.equal(c.run(), a)


def test_binding_refusals():
    torch = torch_mod()
    c = Case(72, [5, 9], qmax=127)
    q, t, n = up(c.q, c.act), i32(c.table), i32(c.lengths)
    for bad in (dict(q=q[:1]), dict(q=q.half()), dict(q=q[..., :64]), dict(q=q.cpu()), dict(q=q[0]), dict(t=t.long()),
                dict(t=t[:1]), dict(t=t.t()), dict(n=n[:1]), dict(n=n.long()), dict(n=n.cpu()), dict(prefix_len=3),
                dict(prefix=n, prefix_len=5), dict(out=torch.empty_like(q)[:1]), dict(out=q.float()), dict(q=q.transpose(0, 1))):
        kw = dict(q=q, t=t, n=n)
        kw.update(bad)
        with pytest.raises(ValueError):
            M.attention_decode(c.cache, kw.pop("q"), kw.pop("t"), kw.pop("n"), **kw)
    with pytest.raises(M.MxmoeError):
        M.attention_decode(c.cache, q, t, n, out=q)
    k = torch.zeros(3, 2, 128, dtype=torch.bfloat16, device="cuda")
    s, f, p = i32([0, 1, 2]), torch.ones(64, dtype=torch.float64, device="cuda"), i32([0, 1, 2])
    for bad in (dict(k=k[:2]), dict(v=k[:2]), dict(k=k.half()), dict(k=k[:, :1]), dict(k=k[..., :64]), dict(k=k.cpu()),
                dict(slots=s[:2]), dict(slots=s.long()), dict(slots=s.cpu()), dict(q=k[:2]), dict(q=k.float()), dict(q=k[:, :0]),
                dict(q_weight=k[0, 0]), dict(q_out=k), dict(q=k, q_weight=k[0, 0, :64]), dict(k_weight=k[0, 0].float()),
                dict(positions=p), dict(freqs=f), dict(positions=p[:2], freqs=f), dict(positions=p, freqs=f.float()),
                dict(k=k.transpose(0, 1).contiguous().transpose(0, 1)), dict(q=k, q_out=k[:2])):
        kw = dict(k=k, v=k, slots=s)
        kw.update(bad)
        with pytest.raises(ValueError):
            M.kv_append(c.cache, kw.pop("k"), kw.pop("v"), kw.pop("slots"), **kw)
    with pytest.raises(M.MxmoeError):
        M.kv_append(c.cache, k, k, s, positions=p, freqs=f[:4])     # 8 rotated elements
    for bad in (s.long(), s.cpu(), s[None], k):
        with pytest.raises(ValueError):
            M.kv_read(c.cache, bad)


# Every form of the attention: items to a workgroup (4 or 8 wavefronts), the shared list, the prefix taken along or through
# LDS; one and two fragments of rows.
@pytest.mark.parametrize("act", ["bf16", "fp16"])
@pytest.mark.parametrize("qmax", [0, 127, 448])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("hq", [4, 40])
def test_attention_forms(hq, dim, qmax, act):
    for lengths, n_q in (([70, 3, 200], 1), ([2200, 0, 31, 640], 1), ([33] * 130, 2)):
        c = Case(hq + dim, lengths, n_q=n_q, hq=hq, kv=2, dim=dim, qmax=qmax, act=act, page=64)
        c.check(c.run(), only=range(min(4, len(lengths))), where=f"{lengths[:4]}")
    # behind a long prefix, which ends inside a block; sequences that end inside it
    lengths = [2150, 0, 1, 2101, 2100, 1500, 2133, 2099, 2300]
    c = Case(hq + dim + 1, lengths, hq=hq, kv=2, dim=dim, qmax=qmax, act=act, page=64, prefix=2100)
    c.check(c.run(), where="prefix")
    c.softcap = 20.0
    c.check(c.run(), where="prefix, cap")


@pytest.mark.parametrize("qmax,dim", [(0, 64), (0, 128), (0, 256), (127, 128), (448, 64), (448, 128), (448, 256)])
def test_long_prefix_odd_rows(qmax, dim):
    """A long prefix whose rows past its end, and inside it past a sequence's end, are not finite; and
    a value that is not finite where some rows see it; pages that are not the cache's."""
    torch = torch_mod()
    lengths = [2150, 700, 2100, 2101, 0, 64, 1999, 2080]
    make = lambda: Case(19, lengths, n_q=2, hq=12, kv=2, dim=dim, qmax=qmax, page=64, prefix=2090)  # noqa: E731
    c = make()
    clean = c.run()
    c.check(clean)
    ends = np.arange(2090 % 64, 64) + 64 * int(c.prefix[-1])          # behind the prefix in its last page
    for what in (float("nan"), float("inf")):
        c = make()
        poison(c, ends, what)
        assert torch.equal(c.run().view(torch.int16), clean.view(torch.int16))
        for at in (1000, 2085, 63):
            c = make()
            poison(c, c.slots(0)[at:at + 1], what)
            got = c.run()
            for b, n in enumerate(lengths):
                for j in range(2):
                    r = 2 * b + j
                    if n - 1 + j > at:
                        assert not torch.isfinite(got[r]).any(), (what, at, b, j)
                    else:
                        assert torch.equal(got[r].view(torch.int16), clean[r].view(torch.int16)), (what, at, b, j)
    if qmax == 0:   # one element: that element alone
        c = make()
        slot = c.slots(0)[1000:1001]
        k, v = M.kv_read(c.cache, i32(slot))
        v[0, 1, 5] = float("inf")
        M.kv_append(c.cache, k, v, i32(slot))
        got = c.run()
        odd = torch.zeros_like(clean, dtype=torch.bool)
        for b, n in enumerate(lengths):
            for j in range(2):
                if n - 1 + j > 1000:
                    odd[2 * b + j, 6:, 5] = True
        assert not torch.isfinite(got[odd]).any()
        assert torch.equal(got[~odd].view(torch.int16), clean[~odd].view(torch.int16))
    c = make()
    c.prefix[20] = c.cache.n_pages
    got = c.run()
    for b, n in enumerate(lengths):
        for j in range(2):
            r = 2 * b + j
            if n - 1 + j > 20 * 64:
                assert torch.isnan(got[r]).all()
            else:
                assert torch.equal(got[r].view(torch.int16), clean[r].view(torch.int16))


@pytest.mark.parametrize("B,hq,kv,prefix,longest", [
    (40, 16, 8, 2100, 300), (10, 16, 8, 2500, 90), (130, 8, 8, 300, 200),    # taken along by 320, 80 and 1040 items
    (40, 16, 8, 2600, 40), (3, 8, 2, 2100, 40),                              # too long for that
    (40, 16, 1, 8200, 40), (128, 32, 2, 2700, 20), (9, 2, 1, 8200, 30)])     # many rows of many pieces, of some; few of many
@pytest.mark.parametrize("qmax", [0, 127])
def test_prefix_forms(B, hq, kv, prefix, longest, qmax):
    rng = np.random.default_rng(B + prefix)
    lengths = prefix + rng.integers(-40, longest, B)
    lengths[:3] = (0, prefix // 2, prefix + longest)
    c = Case(B, lengths, hq=hq, kv=kv, dim=64, qmax=qmax, prefix=prefix, page=64)
    c.check(c.run(), only=range(min(B, 12)))
    if B > 12:
        c.check(c.run(), only=range(B - 4, B))


@pytest.mark.parametrize("T", [31, 32, 8192])
def test_append_tokens_of_a_workgroup(T):
    """The same rows, each by itself and in a call of many."""
    torch = torch_mod()
    rng = np.random.default_rng(T)
    kv, dim = 1, 64
    x = up(rows(rng, (T, 3 * kv, dim), "bf16"), "bf16")
    w = up(O.round_to_act(rows(rng, dim, "bf16", 0.2) + 1, "bf16"), "bf16")
    pos, freqs = i32(rng.integers(0, 9000, T)), torch.from_numpy(1e4 ** (-np.arange(32) / 32)).cuda()
    a, b = (M.KVCache(-(-T // 64), kv, dim, page_size=64, act="bf16", qmax=127) for _ in range(2))
    slots = i32(np.arange(T))
    args = lambda s: dict(q=x[s, :1], q_weight=w, k_weight=w, positions=pos[s], freqs=freqs)  # noqa: E731
    got = M.kv_append(a, x[:, 1:2], x[:, 2:], slots, **args(slice(0, T)))
    for t in range(0, T, 1 if T < 100 else 1111):
        s = slice(t, t + 1)
        one = M.kv_append(b, x[s, 1:2], x[s, 2:], slots[s], **args(s))
        assert torch.equal(one, got[s])
        for g, h in zip(M.kv_read(a, slots[s]), M.kv_read(b, slots[s])):
            assert torch.equal(g, h)


def test_least_and_largest_lengths():
    torch = torch_mod()
    for prefix in (0, 40, 3000):
        c = Case(44, [prefix + 50] * 4, qmax=127, prefix=prefix)
        clean = c.run()
        n = c.lengths.astype(np.int64)
        n[[0, 2]] = (-2 ** 31, 2 ** 31 - 1)
        got = M.attention_decode(c.cache, up(c.q, c.act), i32(c.table), i32(n), prefix=i32(c.prefix) if prefix else None,
                                 prefix_len=prefix)
        assert not got[0].any() and torch.isnan(got[2]).all()
        assert torch.equal(got[[1, 3]].view(torch.int16), clean[[1, 3]].view(torch.int16))


@pytest.mark.parametrize("qmax,dim,act", [(0, 64, "bf16"), (0, 128, "fp16"), (0, 256, "bf16"), (127, 64, "bf16"), (127, 128, "fp16"),
                                          (448, 128, "bf16"), (448, 256, "fp16")])
def test_runs_of_slots(qmax, dim, act):
    """Calls whose tokens fill blocks of the cache in part: runs that begin and end anywhere, two runs
    that meet inside a block of the call, a run broken by one token."""
    torch = torch_mod()
    rng = np.random.default_rng(dim)
    kv, page, n_pages = 2, 64, 8
    for slots in (np.arange(5, 100), np.arange(64, 64 + 33), np.arange(37, 37 + 40), np.arange(95, 127),
                  np.concatenate([np.arange(70, 110), np.arange(200, 260)]), np.concatenate([np.arange(0, 17), np.arange(400, 440)]),
                  np.concatenate([np.arange(32, 50), [300], np.arange(51, 96)]), np.arange(150, 100, -1),
                  np.concatenate([[-1] * 3, np.arange(131, 190), [10 ** 9]]), np.arange(480, 512), np.arange(0, 512)):
        n = len(slots)
        cache, other = (M.KVCache(n_pages, kv, dim, page_size=page, act=act, qmax=qmax) for _ in range(2))
        for t in (*cache.buffers(), *other.buffers()):
            if t is not None:
                t.view(torch.uint8).fill_(0x33)
        x, y = rows(rng, (n, kv, dim), act), rows(rng, (n, kv, dim), act)
        M.kv_append(cache, up(x, act), up(y, act), i32(slots))
        for i in range(n):                                      # token by token
            M.kv_append(other, up(x[i:i + 1], act), up(y[i:i + 1], act), i32(slots[i:i + 1]))
        for a, b in zip(all_bytes(cache), all_bytes(other)):
            assert torch.equal(a, b), slots
        kept = (slots >= 0) & (slots < n_pages * page)
        gk, gv = M.kv_read(cache, i32(slots))
        assert np.array_equal(down(gk)[kept], exact_read(x, qmax, act)[kept]) and not down(gk)[~kept].any()
        assert np.array_equal(down(gv)[kept], exact_read(y, qmax, act)[kept]) and not down(gv)[~kept].any()


# ------------------------------------------------------------------ together
def test_streams_and_graph():
    """A decode loop captured once: append and attention replayed with new tokens, slots and lengths, against the
    same calls made one by one; with other work of the program between the replays."""
    torch = torch_mod()
    for qmax, prefix in ((127, 0), (448, 96), (0, 0)):
        B, hq, kv, dim, page = 5, 8, 2, 128, 64
        rng = np.random.default_rng(qmax + 1)
        c = Case(81, [prefix + n for n in (1, 60, 63, 700, 129)], hq=hq, kv=kv, dim=dim, qmax=qmax, page=page, prefix=prefix, extra=2)
        used = set(c.table[c.table >= 0].tolist()) | set(c.prefix.tolist())
        free = [i for i in range(c.cache.n_pages) if i not in used]
        c.table[2, 1], c.table[1, 1] = free[0], free[1]                      # the pages that they grow into
        freqs = torch.from_numpy(1e4 ** (-np.arange(64) / 64)).cuda()
        w = up(np.ones(dim), c.act)
        table, pre = i32(c.table), i32(c.prefix) if prefix else None
        x = torch.zeros(B, (hq + 2 * kv) * dim, dtype=torch.bfloat16, device="cuda")
        slots, pos, lengths = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(3))

        def step(cache):
            q, k, v = (t.unflatten(1, (-1, dim)) for t in x.split([hq * dim, kv * dim, kv * dim], 1))
            q = M.kv_append(cache, k, v, slots, q=q, q_weight=w, k_weight=w, positions=pos, freqs=freqs)
            return M.attention_decode(cache, q, table, lengths, prefix=pre, prefix_len=prefix)

        other = M.KVCache(c.cache.n_pages, kv, dim, page_size=page, act=c.act, qmax=qmax)
        for a, b in zip(c.cache.buffers(), other.buffers()):
            if a is not None:
                b.copy_(a)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step(other)
        torch.cuda.current_stream().wait_stream(s)
        for a, b in zip(c.cache.buffers(), other.buffers()):
            if a is not None:
                b.copy_(a)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step(other)
        for it in range(4):
            n = c.lengths + it
            own = n - prefix
            x.copy_(up(rows(rng, tuple(x.shape), "bf16"), "bf16"))
            slots.copy_(i32([int(c.table[b, own[b] // page]) * page + int(own[b]) % page for b in range(B)]))
            pos.copy_(i32(n))
            lengths.copy_(i32(n + 1))
            g.replay()
            torch.cuda.synchronize()
            want = step(c.cache)
            junk = torch.full((1 << 20,), float("nan"), device="cuda")       # freed memory that another call may get
            del junk
            assert torch.equal(out, want), (qmax, it)
            for a, b in zip(all_bytes(c.cache), all_bytes(other)):
                assert torch.equal(a, b)


def test_two_graphs_in_turn():
    """Two captured attentions replayed one after the other, on two streams: neither uses the other's workspace."""
    torch = torch_mod()
    cs = [Case(91 + i, [4000 + 7 * i, 100, 2000], qmax=127, hq=8, kv=2) for i in range(2)]
    want = [c.run() for c in cs]
    gs, outs, args = [], [], []
    for c in cs:
        a = (up(c.q, c.act), i32(c.table), i32(c.lengths))
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            M.attention_decode(c.cache, *a)
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(M.attention_decode(c.cache, *a))
        gs.append(g)
        args.append(a)
    st = [torch.cuda.Stream() for _ in gs]
    for _ in range(4):
        for o in outs:
            o.fill_(5.0)
        torch.cuda.synchronize()
        for g, s in zip(gs, st):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)


def test_side_stream_memory_is_kept():
    """Inputs dropped right after a call on another stream are not reused before it is done."""
    torch = torch_mod()
    c = Case(101, [9000, 8000], qmax=127, hq=8, kv=2, page=128)
    want = c.run()
    s = torch.cuda.Stream()
    for _ in range(4):
        q, t, n = up(c.q, c.act), i32(c.table), i32(c.lengths)
        s.wait_stream(torch.cuda.current_stream())
        got = M.attention_decode(c.cache, q, t, n, stream=s)
        del q, t, n
        trash = [torch.full((c.q.size,), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(8)]
        trash += [torch.full((64,), 7, dtype=torch.int32, device="cuda") for _ in range(8)]
        s.synchronize()
        assert torch.equal(got, want)
        del trash


def test_far_offsets():
    """A cache past 4 GB: its last pages."""
    torch = torch_mod()
    kv, dim, page = 16, 256, 1024
    n_pages = 640                                    # 640 * 16 * 1024 * 256 * 2 = 5.4 GB for keys, the same for values
    cache = M.KVCache(n_pages, kv, dim, page_size=page, act="fp16")
    rng = np.random.default_rng(1)
    n = 70
    k, v = rows(rng, (n, kv, dim), "fp16"), rows(rng, (n, kv, dim), "fp16")
    slots = (n_pages - 1) * page + 100 + np.arange(n)
    M.kv_append(cache, up(k, "fp16"), up(v, "fp16"), i32(slots))
    gk, gv = M.kv_read(cache, i32(slots))
    assert np.array_equal(down(gk), k) and np.array_equal(down(gv), v)
    # tokens 100 .. 169 of the page, behind 100 zero rows
    q = rows(rng, (1, kv, dim), "fp16")
    out = down(M.attention_decode(cache, up(q, "fp16"), i32([[n_pages - 1]]), i32([170])))
    z = np.zeros((100, kv, dim))
    ref, mass = O.attention(q, np.concatenate([z, k]), np.concatenate([z, v]), [170], dim ** -0.5)
    assert np.all(np.abs(out - ref) <= TL.slot_bound(ref, 2.0 ** -9 * mass, "fp16"))
    del cache
    torch.cuda.empty_cache()


def test_layer_together():
    """A decoder layer's step as it would run: norm and codes, the joint projection, heads into the
    cache, attention, the output projection, norm, the block; every operator against its oracle
    on what it was given."""
    torch = torch_mod()
    blk = W.random_small_block(7, T=8, H=512, F=256, E=4, k=2, act="bf16", schemes=[(W.W4G128, W.W4G128, W.W8A8)] * 4)
    mb = M.MoEBlock(blk)
    T, H, hq, kv, dim, act = 8, 512, 8, 2, 64, "bf16"
    rng = np.random.default_rng(2)
    qkv = M.PackedLinear(W.quantize_linear(W.draw_weight(1, 0, 0, (hq + 2 * kv) * dim, H), W.W8A8), act)
    wo = M.PackedLinear(W.quantize_linear(W.draw_weight(1, 0, 1, H, hq * dim), W.W4G128), act)
    x = up(rows(rng, (T, H), act), act)
    g1, g2, gq = (up(1 + rows(rng, n, act, 0.05), act) for n in (H, H, dim))
    c = Case(3, [100 + 13 * b for b in range(T)], hq=hq, kv=kv, dim=dim, qmax=448, page=64, extra=1)
    pos = c.lengths - 1
    slots = i32([int(c.table[b, pos[b] // 64]) * 64 + int(pos[b]) % 64 for b in range(T)])
    freqs = torch.from_numpy(1e4 ** (-np.arange(dim // 2) / (dim // 2))).cuda()
    _, _, codes, scales = M.add_rms_norm(x, g1, qmax=127, want_y=False)
    y = M.linear_decode(qkv, codes, scales=scales)
    q, k, v = (t.unflatten(1, (-1, dim)) for t in y.split([hq * dim, kv * dim, kv * dim], 1))
    q2 = M.kv_append(c.cache, k, v, slots, q=q, q_weight=gq, k_weight=gq, positions=i32(pos), freqs=freqs)
    o = M.attention_decode(c.cache, q2, i32(c.table), i32(c.lengths))
    z = M.linear_decode(wo, o.flatten(1))
    h, s, _, _ = M.add_rms_norm(z, g2, residual=x)
    ids, w = torch.from_numpy(blk.topk_ids.copy()).cuda(), torch.from_numpy(blk.topk_w.copy()).cuda()
    out = mb.forward(h, ids, w)
    torch.cuda.synchronize()
    want, e = head_error(down(q), down(gq), pos, freqs.cpu().numpy(), False)
    assert np.all(np.abs(down(q2) - want) <= TL.slot_bound(want, e, act))
    kb, vb = M.kv_read(c.cache, slots)
    want, e = head_error(down(k), down(gq), pos, freqs.cpu().numpy(), False)
    check_cached(down(kb), want, e, 448, act)
    assert np.array_equal(down(vb), exact_read(down(v), 448, act))
    # the attention on what the cache holds: codes times scales of the rows that were written
    at = slots.cpu().numpy()
    c.v[at] = O.cache_values(*O.cache_rows(down(v), 448), 448)
    ks = c.cache.k_scales.permute(0, 2, 1).reshape(-1, kv)[slots.long()].cpu().numpy().astype(np.float64)
    codes_k = down(kb) / ks[..., None]                # (the read rounds code * scale to bf16)
    byte = np.frombuffer(torch.from_numpy(codes_k).to(torch.float8_e4m3fn).view(torch.uint8).numpy().tobytes(), np.uint8)
    c.k[at] = O.e4m3_values(byte.reshape(codes_k.shape)) * ks[..., None]
    c.q = down(q2)
    c.check(o)
    ref = O.moe_forward(M.act_numpy(h, act), blk.topk_ids, blk.topk_w, blk.linears, blk.cfg.E, act)["y"]
    assert np.all(np.abs(down(out) - ref) <= 1e-2 * np.abs(ref).max(axis=1, keepdims=True))
