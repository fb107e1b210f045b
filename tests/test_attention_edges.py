"""Edges of the attention of a decode step, on the CPU: that the bounds of test_gpu_attention_edges tell
what they are for."""

from types import SimpleNamespace

import numpy as np
import pytest

from oracle import mxmoe_oracle as O
from paper_2505_05799_amd import mxmoe as M
from paper_2505_05799_amd import workloads as W
from tests import tolerance as TL


def rounded(a, act):
    """fp64 values to the nearest of the dtype"""
    return O.act_values(W.f64_to_act(np.asarray(a, dtype=np.float64), act), act)


def opposite_values(n, kv, dim, rows, qmax, act, first):
    """(q [rows, kv rows, dim], k, v [n, kv, dim]): two tokens whose values cancel but for some percent, so that the
    output's own rounding is small beside that of the weights; the other tokens have scores of -60 and values 0."""
    rng = np.random.default_rng(n + dim + rows)
    sign = np.where(rng.random((1, kv, dim)) < 0.5, -1.0, 1.0)
    size = rounded(rng.uniform(0.9, 1.1, (rows, 1, 1)), act)
    q = np.repeat(sign, 1, axis=0) * size                     # a score is size * what the key is made for
    x = np.full(n, -60.0)
    x[first], x[first + 1] = 0.5, -0.5
    k = rounded(sign * x[:, None, None] / dim ** 0.5, act)
    v = np.zeros((n, kv, dim))
    pattern = np.where(rng.random((kv, dim)) < 0.5, -1.0, 1.0)
    v[first], v[first + 1] = pattern, -pattern * np.e
    return q, k, rounded(v, act)


def parts_of(qmax, act):
    """What a weight is rounded by: half a step of the type of its product, twice where both parts are taken."""
    u = 2.0 ** -8 if act == "bf16" and qmax == 0 else 2.0 ** -11
    return u if qmax and act == "bf16" else u * u


def weight_bound(mass, ref, qmax, dim, act):
    """|out - ref| where two tokens hold the weight.  |x| <= 0.6: a score's fp32 sum of dim products, 2^-23 of their
    sum each, products by scales, the reference's difference and exp2 (8 * 2^-24 (1 + |x|)), in the numerator and in
    the normalizer; the weight's parts; sums of a few terms, the rows' meeting and the quotient, under 32 * 2^-24.
    What the other tokens add, n e^-60, and what lies under fp16's least, is below 2^-30."""
    d = dim * 2.0 ** -23 * 0.6 + 8 * TL.U32 * 1.6
    return TL.slot_bound(ref, (2 * d + parts_of(qmax, act) + 32 * TL.U32 + 2.0 ** -30) * mass, act)


@pytest.mark.parametrize("qmax,act", [(0, "bf16"), (0, "fp16"), (127, "fp16"), (448, "fp16")])
def test_the_bound_tells_one_part_of_a_weight_from_two(qmax, act):
    """Weights rounded once are past the bound, as two parts well inside it."""
    kv, dim, n, first = 2, 64, 70, 33
    q, k, v = opposite_values(n, kv, dim, 40, qmax, act, first)
    k, v = (O.cache_values(*O.cache_rows(r, qmax), qmax) for r in (k, v))
    ratio = {}
    for parts in (1, 2):
        worst = 0.0
        for r in range(40):
            ref, mass = O.attention(q[r:r + 1], k, v, [n], dim ** -0.5)
            for h in range(kv):
                x = (k[:, h] @ q[r, h]) * dim ** -0.5
                scale = np.abs(v[:, h]).max(axis=1) / qmax if qmax else np.ones(n)
                w = 2.0 ** 8 * np.exp(x - x[first]) * scale / scale[first]
                code = v[:, h] / np.where(scale > 0, scale, 1.0)[:, None]
                some = rounded(w, act)
                if parts == 2:
                    some = some + rounded(w - some, act)
                out = some @ code / (np.exp(x - x[first]).sum() * 2.0 ** 8 / scale[first])
                worst = max(worst, float((np.abs(rounded(out, act) - ref[0, h]) / weight_bound(mass, ref, qmax, dim, act)[0, h]).max()))
        ratio[parts] = worst
    assert ratio[1] > 2 and ratio[2] < 1, ratio


# ------------------------------------------------------------------ binding
@pytest.mark.parametrize("qmax", [0, 127, 448])
def test_a_cache_is_made(qmax, monkeypatch):
    """All of it but the GPU: the constructor's steps on memory that is none."""
    import torch
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    c = M.KVCache(4, 2, 64, page_size=32, qmax=qmax, device="meta")
    assert c.k.shape == c.v.shape == (4, 2, 2048) and c.t.qmax == qmax and c._dev == 0
    assert [t is not None for t in c.buffers()] == [True, True, qmax > 0, qmax > 0]


@pytest.mark.parametrize("name", ["k", "v", "k_scales", "v_scales", "t", "n_pages", "page_size", "qmax", "dtype"])
def test_a_cache_keeps_its_buffers(name):
    """The calls use the addresses that the descriptor was given: another tensor in a buffer's place would not be
    the one that they write, and the one that they write might be freed."""
    c = M.KVCache.__new__(M.KVCache)
    setattr(c, name, 1)
    with pytest.raises(AttributeError):
        setattr(c, name, 2)
    assert getattr(c, name) == 1


def test_sizes_past_32_bits_are_refused():
    """Not taken modulo 2^32."""
    import torch
    for k, size in enumerate((4, 2, 64, 64)):
        for by in (1 << 31, 1 << 32, 1 << 40):
            sizes = [4, 2, 64, 64]
            sizes[k] = size + by
            with pytest.raises(M.MxmoeError):
                M.KVCache(*sizes, device="cpu")
    with pytest.raises(M.MxmoeError):
        M.KVCache(4, 2, 64, qmax=127 + (1 << 32), device="cpu")
    cache = SimpleNamespace(_dev=0, dtype=torch.bfloat16, dim=64, page_size=64)
    q, n = torch.empty(1, 2, 64, dtype=torch.bfloat16, device="meta"), torch.empty(1, dtype=torch.int32, device="meta")
    pages = lambda *s: torch.empty(*s, dtype=torch.int32, device="meta")  # noqa: E731
    with pytest.raises(M.MxmoeError):
        M.attention_decode(cache, q, pages(1, (1 << 32) + 2), n)
    with pytest.raises(M.MxmoeError):
        M.attention_decode(cache, q, pages(1, 2), n, prefix=pages((1 << 26) + 1), prefix_len=(1 << 32) + 64)
