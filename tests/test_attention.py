"""The operators of a decode step's attention, on the CPU: their oracle against brute force
and identities, and every refusal of the C ABI and of the binding (validation returns before
anything is enqueued; the pointers below are never dereferenced)."""

import ctypes as C
import math

import numpy as np
import pytest

from oracle import mxmoe_oracle as O
from paper_2505_05799_amd import mxmoe as M


@pytest.fixture(scope="module")
def lib():
    return M.load_library()


def at(mb, off=0):             # an address; the buffers of the calls below lie MB apart
    return (mb << 20) + off


# ------------------------------------------------------------------- oracles
@pytest.mark.parametrize("interleaved", [False, True])
def test_head_rows_brute_force(interleaved):
    rng = np.random.default_rng(5)
    T, H, D, rot = 4, 3, 16, 8
    x, w = rng.standard_normal((T, H, D)), 1 + 0.1 * rng.standard_normal(D)
    pos, freqs = np.array([0, 1, 77, 123456]), 10000.0 ** (-np.arange(rot // 2) / (rot // 2))
    y = O.head_rows(x, w, 1e-6, pos, freqs, interleaved)
    for t in range(T):
        for h in range(H):
            r = 1 / math.sqrt(sum(float(a) ** 2 for a in x[t, h]) / D + 1e-6)
            row = [float(x[t, h, d]) * r * w[d] for d in range(D)]
            want = list(row)
            for i in range(rot // 2):
                a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
                c, s = math.cos(int(pos[t]) * freqs[i]), math.sin(int(pos[t]) * freqs[i])
                want[a], want[b] = row[a] * c - row[b] * s, row[b] * c + row[a] * s
            assert np.abs(y[t, h] - want).max() < 1e-12


def test_rotated_products_depend_on_the_distance_alone():
    rng = np.random.default_rng(6)
    q, k = rng.standard_normal((1, 1, 32)), rng.standard_normal((1, 1, 32))
    freqs = 100.0 ** (-np.arange(16) / 16)
    dots = [float((O.head_rows(q, None, 0, np.array([p + 7]), freqs) * O.head_rows(k, None, 0, np.array([p]), freqs)).sum())
            for p in (0, 3, 1000)]
    assert max(dots) - min(dots) < 1e-10
    n = np.linalg.norm(O.head_rows(q, None, 0, np.array([991]), freqs))
    assert abs(n - np.linalg.norm(q)) < 1e-12


def test_attention_oracle():
    rng = np.random.default_rng(7)
    q, k, v = rng.standard_normal((2, 4, 8)), rng.standard_normal((9, 2, 8)), rng.standard_normal((9, 2, 8))
    out, mass = O.attention(q, k, v, [0, 9], 0.3)
    assert not out[0].any() and not mass[0].any()
    for h in range(4):
        w = [math.exp(0.3 * sum(a * b for a, b in zip(q[1, h], k[t, h // 2]))) for t in range(9)]
        want = sum(w[t] * v[t, h // 2] for t in range(9)) / sum(w)
        assert np.abs(out[1, h] - want).max() < 1e-13
    # one token: its value; equal keys: the mean; a large cap changes nothing, a tiny one gives the mean
    assert np.allclose(O.attention(q, k, v, [1, 1], 5.0)[0], np.repeat(v[0], 2, axis=0)[None])
    mean = np.repeat(v.mean(axis=0), 2, axis=0)
    assert np.allclose(O.attention(q, 0 * k, v, [9, 9], 5.0)[0], mean[None])
    assert np.allclose(O.attention(q, k, v, [9, 9], 0.3, 1e6)[0], O.attention(q, k, v, [9, 9], 0.3)[0])
    assert np.allclose(O.attention(q, k, v, [9, 9], 0.3, 1e-9)[0], mean[None])


@pytest.mark.parametrize("qmax", [127, 448])
def test_cache_rows_are_within_half_a_step(qmax):
    rng = np.random.default_rng(8)
    y = rng.standard_normal((5, 2, 64)).astype(np.float32).astype(np.float64)
    y[3] = 0
    codes, scales = O.cache_rows(y, qmax)
    got = O.cache_values(codes, scales, qmax)
    s = scales.astype(np.float64)[..., None]
    # half a step of the codes (e4m3: 2^-4 of the value, 2^-10 at the least), and the roundings
    # of inv, of the product and of the scale, 2^-24 of it each
    half = 0.5 * s if qmax == 127 else np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * s)
    assert np.all(np.abs(got - y) <= half + 4 * 2.0 ** -24 * np.abs(y) + 1e-300)
    assert not got[3].any()


# ------------------------------------------------------------------ refusals
def cache(n_pages=8, heads=2, dim=64, page=32, act=M.BF16, qmax=127, k=at(1), v=at(2), ks=at(3), vs=at(4)):
    if qmax == 0 and ks == at(3):
        ks = vs = None
    return M.KVCache_t(n_pages, heads, dim, page, act, qmax, k, v, ks, vs)


BAD_CACHES = [dict(n_pages=0), dict(n_pages=-1), dict(heads=0), dict(act=2), dict(k=None), dict(v=None), dict(ks=None),
              dict(vs=None), dict(k=at(1, 8)), dict(v=at(2, 2)), dict(ks=at(3, 4)), dict(vs=at(4, 8)), dict(qmax=0, ks=at(5))]
UNSUPPORTED_CACHES = [dict(qmax=7), dict(qmax=128), dict(qmax=-1), dict(dim=96), dict(dim=512), dict(dim=0), dict(page=16),
                      dict(page=48), dict(page=2048), dict(page=0), dict(heads=1025), dict(n_pages=1 << 26)]


def test_cache_bytes(lib):
    for q, es in ((0, 2), (127, 1), (448, 1)):
        c = cache(n_pages=5, heads=3, dim=128, page=64, qmax=q, k=None, v=None, ks=None, vs=None)
        assert lib.mxmoe_kv_cache_bytes(C.byref(c)) == 5 * 3 * 128 * 64 * es
        assert lib.mxmoe_kv_scale_bytes(C.byref(c)) == (5 * 3 * 64 * 4 if q else 0)
    for bad in BAD_CACHES[:4] + UNSUPPORTED_CACHES:
        c = cache(**bad)
        assert lib.mxmoe_kv_cache_bytes(C.byref(c)) == 0 and lib.mxmoe_kv_scale_bytes(C.byref(c)) == 0
        assert lib.mxmoe_attention_workspace_bytes(C.byref(c), 1, 1, 2, 4, 0) == 0
    assert lib.mxmoe_kv_cache_bytes(None) == 0


def append(lib, c=None, n=4, q=at(10), ldq=256, hq=4, k=at(11), ldk=128, v=at(12), ldv=128, qw=at(13), kw=at(14), eps=1e-6,
           pos=at(15), freqs=at(16), rot=64, inter=0, slots=at(17), out=at(18), ldo=256):
    c = cache() if c is None else c
    return lib.mxmoe_kv_append(C.byref(c), n, q, ldq, hq, k, ldk, v, ldv, qw, kw, eps, pos, freqs, rot, inter, slots, out, ldo, None)


@pytest.mark.parametrize("bad", [
    dict(n=-1), dict(hq=-1), dict(hq=65537), dict(inter=2), dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf")),
    dict(k=None), dict(v=None), dict(slots=None), dict(q=None), dict(out=None), dict(hq=0), dict(pos=None), dict(freqs=None),
    dict(rot=0), dict(ldq=255), dict(ldk=127), dict(ldv=127), dict(ldo=255), dict(ldq=1 << 50), dict(ldk=1 << 62),
    dict(q=at(10, 1)), dict(k=at(11, 1)), dict(v=at(12, 1)), dict(qw=at(13, 1)), dict(kw=at(14, 1)), dict(out=at(18, 1)),
    dict(pos=at(15, 2)), dict(slots=at(17, 2)), dict(freqs=at(16, 4)),
    dict(q=None, out=None, hq=0),                                 # a weight without queries
    dict(out=at(10), ldo=264), dict(out=at(10, 2)),               # in the queries' place, but not row for row
    dict(out=at(11)), dict(out=at(12, 64)), dict(out=at(13)), dict(out=at(14, 64)), dict(out=at(15)), dict(out=at(16, 8)),
    dict(out=at(17)), dict(out=at(1)), dict(out=at(2, 512)), dict(out=at(3)), dict(out=at(4)),
    dict(k=at(1)), dict(v=at(2)), dict(q=at(1)), dict(slots=at(3)), dict(pos=at(4)), dict(freqs=at(1)),
])
def test_append_refuses(lib, bad):
    assert append(lib, **bad) == M.ERR_INVALID_ARG


def test_append_refuses_caches_and_unsupported(lib):
    for bad in BAD_CACHES:
        assert append(lib, cache(**bad)) == M.ERR_INVALID_ARG
    for bad in UNSUPPORTED_CACHES:
        assert append(lib, cache(**bad)) == M.ERR_UNSUPPORTED
    assert append(lib, cache(v=at(1))) == M.ERR_INVALID_ARG       # keys and values share bytes
    assert append(lib, cache(vs=at(3))) == M.ERR_INVALID_ARG
    for rot in (8, 24, 80, -16):
        assert append(lib, rot=rot) == M.ERR_UNSUPPORTED
    assert append(lib, n=(1 << 24) + 1) == M.ERR_UNSUPPORTED and read(lib, n=(1 << 24) + 1) == M.ERR_UNSUPPORTED
    assert append(lib, n=0, q=None, out=None, k=None, v=None, slots=None) == M.OK
    assert lib.mxmoe_kv_append(None, 0, None, 0, 0, None, 0, None, 0, None, None, 1e-6, None, None, 0, 0, None, None, 0, None) \
        == M.ERR_INVALID_ARG


def read(lib, c=None, n=4, slots=at(10), k=at(11), v=at(12)):
    c = cache() if c is None else c
    return lib.mxmoe_kv_read(C.byref(c), n, slots, k, v, None)


@pytest.mark.parametrize("bad", [
    dict(n=-1), dict(slots=None), dict(k=None), dict(v=None), dict(slots=at(10, 2)), dict(k=at(11, 1)), dict(v=at(12, 1)),
    dict(k=at(12, 64)), dict(k=at(1)), dict(v=at(2)), dict(v=at(3)), dict(k=at(4)), dict(k=at(10)), dict(v=at(10)),
])
def test_read_refuses(lib, bad):
    assert read(lib, **bad) == M.ERR_INVALID_ARG


def test_read_refuses_caches(lib):
    for bad in BAD_CACHES:
        assert read(lib, cache(**bad)) == M.ERR_INVALID_ARG
    for bad in UNSUPPORTED_CACHES:
        assert read(lib, cache(**bad)) == M.ERR_UNSUPPORTED
    assert read(lib, n=0, slots=None, k=None, v=None) == M.OK


def attend(lib, c=None, q=at(10), ldq=256, batch=3, n_q=2, hq=4, table=at(11), width=5, lengths=at(12), prefix=at(13), plen=40,
           scale=0.125, cap=0.0, out=at(14), ldo=256, ws=at(64), wsb=None):
    c = cache() if c is None else c
    if wsb is None:
        wsb = lib.mxmoe_attention_workspace_bytes(C.byref(c), batch, n_q, hq, width, plen)
    return lib.mxmoe_attention_decode(C.byref(c), q, ldq, batch, n_q, hq, table, width, lengths, prefix, plen, scale, cap, out,
                                      ldo, ws, wsb, None)


@pytest.mark.parametrize("bad", [
    dict(batch=-1), dict(n_q=0), dict(n_q=-1), dict(hq=0), dict(hq=3), dict(width=-1), dict(plen=-1), dict(q=None),
    dict(out=None), dict(lengths=None), dict(table=None), dict(width=0), dict(prefix=None), dict(plen=0),
    dict(scale=float("nan")), dict(scale=float("inf")), dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")),
    dict(ldq=255), dict(ldo=255), dict(ldq=1 << 50), dict(ldo=1 << 62), dict(q=at(10, 1)), dict(out=at(14, 1)),
    dict(table=at(11, 2)), dict(lengths=at(12, 1)), dict(prefix=at(13, 2)), dict(ws=at(64, 64)),
    dict(out=at(10)), dict(out=at(11)), dict(out=at(12)), dict(out=at(13)), dict(out=at(1)), dict(out=at(2)), dict(out=at(3)),
    dict(out=at(4, 64)),
])
def test_attention_refuses(lib, bad):
    assert attend(lib, **bad) == M.ERR_INVALID_ARG


def test_attention_refuses_caches_and_unsupported(lib):
    for bad in BAD_CACHES:
        assert attend(lib, cache(**bad)) == M.ERR_INVALID_ARG
    for bad in UNSUPPORTED_CACHES:
        assert attend(lib, cache(**bad)) == M.ERR_UNSUPPORTED
    assert attend(lib, n_q=M.ATTENTION_QUERIES + 1) == M.ERR_UNSUPPORTED
    assert attend(lib, batch=65536) == M.ERR_UNSUPPORTED
    assert attend(lib, hq=65538, ldq=1 << 23, ldo=1 << 23) == M.ERR_UNSUPPORTED
    assert attend(lib, batch=65535, n_q=16, hq=128) == M.ERR_UNSUPPORTED
    assert attend(lib, width=1 << 25) == M.ERR_UNSUPPORTED
    assert attend(lib, plen=1 << 30) == M.ERR_UNSUPPORTED
    assert attend(lib, batch=0, q=None, table=None, lengths=None, prefix=None, out=None, ws=None) == M.OK


def test_calls_past_a_launch_are_refused(lib):
    """A launch has fewer than 2^32 threads; these would need more."""
    big = lambda heads, dim=64: cache(n_pages=1, heads=heads, dim=dim, k=at(1 << 19), v=at(1 << 19 | 1 << 18), ks=at(3), vs=at(4))  # noqa: E731
    n = 1 << 24
    assert read(lib, big(16), n=n) == M.ERR_UNSUPPORTED and append(lib, big(16), n=n, ldk=1024, ldv=1024) == M.ERR_UNSUPPORTED
    assert read(lib, big(1024), n=(1 << 17) + 1) == M.ERR_UNSUPPORTED
    c = big(1024)
    assert attend(lib, c, batch=32768, n_q=1, hq=1024, ldq=1 << 16, ldo=1 << 16, width=1, plen=0, prefix=None) == M.ERR_UNSUPPORTED
    assert lib.mxmoe_attention_workspace_bytes(C.byref(c), 16384, 1, 1024, 1, 0) == 0
    assert lib.mxmoe_attention_workspace_bytes(C.byref(cache(heads=1)), 16384, 1, 1023, 100, 0) > 0


@pytest.mark.parametrize("cap", [1e-31, 1e31, 1e-45])
def test_caps_out_of_range_are_refused(lib, cap):
    assert attend(lib, cap=cap) == M.ERR_INVALID_ARG


def test_attention_workspace(lib):
    need = lib.mxmoe_attention_workspace_bytes(C.byref(cache()), 3, 2, 4, 500, 4000)
    if need:
        assert attend(lib, width=500, plen=4000, wsb=need - 1) == M.ERR_WORKSPACE
        assert attend(lib, width=500, plen=4000, ws=None) == M.ERR_INVALID_ARG
        for other in (at(10), at(11), at(12), at(13), at(14), at(1), at(2), at(3), at(4)):
            assert attend(lib, width=500, plen=4000, ws=other) == M.ERR_INVALID_ARG
    for bad in ((-1, 1, 2, 4, 0), (1, 0, 2, 4, 0), (1, 1, 3, 4, 0), (1, 17, 2, 4, 0), (1, 1, 2, 1 << 26, 0)):
        assert lib.mxmoe_attention_workspace_bytes(C.byref(cache()), *bad) == 0


def test_binding_refuses_host_tensors():
    with pytest.raises(ValueError):
        M.KVCache(4, 2, 64, device="cpu")
    with pytest.raises(M.MxmoeError):
        M.KVCache(4, 2, 80, device="cpu")
