"""GPU parity of the attention of a decode step at the edges of its number range and in every launch
form, against the fp64 oracle.  Cases, bounds and helpers are those of test_gpu_attention."""

import numpy as np
import pytest

from oracle import mxmoe_oracle as O
from paper_2505_05799_amd import mxmoe as M
from tests.gpuhelp import torch_mod
from tests.test_attention_edges import opposite_values, weight_bound
from tests.test_gpu_attention import Case, down, i32, up

pytestmark = pytest.mark.gpu

# Launch forms: (sequences, kv heads, rows a kv head, own tokens, prefix).  own tokens fit 64 blocks: a workgroup of 8
# wavefronts (up to 256 items) or 4 to an item; more: the shared list; a short prefix is taken along by the
# items, a long one goes through LDS.  More than 16 rows (128 in LDS) make two fragments.
FORMS = {"item8": (3, 2, 4, 1500, 0), "item8, two": (3, 2, 20, 1500, 0), "item4": (150, 2, 4, 1500, 0),
         "item4, two": (150, 2, 20, 1500, 0), "list": (64, 2, 4, 3000, 0), "list, two": (64, 2, 20, 3000, 0),
         "fold": (8, 2, 4, 40, 1500), "lds": (20, 8, 4, 40, 6400), "lds, two": (128, 8, 4, 40, 6400)}


def steep(qmax, dim, form, period, gap, last, small):
    """Sequences over the same pages, whose scores are 0, `gap` and `gap` + `last` in turn, each for `period`
    blocks of 32 tokens; the values at `gap` are zeros, or 2^-110."""
    B, kv, group, own, prefix = FORMS[form]
    rng = np.random.default_rng(period)
    c = Case(7, [prefix + own], hq=group * kv, kv=kv, dim=dim, qmax=qmax, act="bf16", page=64, prefix=prefix, extra=0)
    at = c.slots(0)
    n = len(at)
    kind = np.arange(n) // (32 * period) % 3
    sign = np.where(rng.random((1, kv, dim)) < 0.5, -1.0, 1.0)
    x = np.choose(kind, [0.0, gap, gap + last])[:, None, None]
    k = O.round_to_act(sign * x / dim ** 0.5, "bf16")              # scale q . k = x for queries of that sign
    v = np.where(rng.random((n, kv, dim)) < 0.5, -1.0, 1.0) * np.choose(kind, [1.0, small, 1.0])[:, None, None]
    M.kv_append(c.cache, up(k, "bf16"), up(v, "bf16"), i32(at))
    c.k[at], c.v[at] = (O.cache_values(*O.cache_rows(r, qmax), qmax) for r in (k, v))
    c.q = np.repeat(np.repeat(sign, group, axis=1), B, axis=0)
    c.table = np.repeat(c.table, B, axis=0)
    c.lengths = prefix + own - np.arange(B) % 7
    return c


@pytest.mark.parametrize("last", [4.0, 16.0])
@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("qmax", [127, 448])
def test_large_weights_of_zero_values(qmax, form, last):
    """Weights that grow past 2^124 of those before, whose values are zeros (or so small that a value's scale times its
    weight stays small): they count in the sum, and the row is what its later tokens make of it."""
    period = 8 if form[:5] in ("item8", "fold") else 1     # (a wavefront takes every 8th block, every 4th, or all)
    for gap, small in ((75.5, 0.0), (76.3, 0.0), (76.3, 2.0 ** -110)):
        c = steep(qmax, 64, form, period, gap, last, small)
        c.check(c.run(), only=[0, 1, len(c.lengths) - 1], where=f"{form} {gap} {small}")


@pytest.mark.parametrize("act", ["bf16", "fp16"])
@pytest.mark.parametrize("qmax", [0, 127, 448])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("form", list(FORMS))
def test_both_parts_of_a_weight(form, dim, qmax, act):
    """Two tokens whose values cancel: what the rounding of the weights leaves, which the general bound allows one
    rounding, stays within that of both parts."""
    B, kv, group, own, prefix = FORMS[form]
    n = prefix + own
    c = Case(7, [n], hq=group * kv, kv=kv, dim=dim, qmax=qmax, act=act, page=64, prefix=prefix, extra=0)
    at = c.slots(0)
    rows = 16
    q, k, v = opposite_values(n, kv, dim, rows * group, qmax, act, n - 40 if prefix < 100 else 65)
    M.kv_append(c.cache, up(k, act), up(v, act), i32(at))
    c.k[at], c.v[at] = (O.cache_values(*O.cache_rows(r, qmax), qmax) for r in (k, v))
    # sequence b: rows b % 16 of a kv head
    q = q.reshape(rows, group, kv, dim).transpose(0, 2, 1, 3).reshape(rows, kv * group, dim)
    c.q = q[np.arange(B) % rows]
    c.table = np.repeat(c.table, B, axis=0)
    c.lengths = np.full(B, n)
    got = down(c.run())
    assert np.isfinite(got).all()
    for b in range(0, min(B, rows)):
        ref, mass = O.attention(c.q[b:b + 1], c.k[at], c.v[at], [n], c.scale)
        err, bound = np.abs(got[b] - ref[0]), weight_bound(mass, ref, qmax, dim, act)[0]
        assert np.all(err <= bound), (b, float((err / bound).max()))
