"""GPU parity of the attention of a decode step at the edges of its number range and in every launch
form, against the fp64 oracle.  Cases, bounds and helpers are those of test_gpu_attention."""

import numpy as np
import pytest

from oracle import mxmoe_oracle as O
from paper_2505_05799_amd import mxmoe as M
from tests.gpuhelp import torch_mod
from tests.test_attention_edges import opposite_values, rounded, weight_bound
from tests.test_gpu_attention import Case, down, exact_read, i32, up

pytestmark = pytest.mark.gpu

# Launch forms: (sequences, kv heads, rows a kv head, own tokens, prefix).  own tokens fit 64 blocks: a workgroup of 8
# wavefronts (up to 256 items) or 4 to an item; more: the shared list; a short prefix is taken along by the
# items, a long one goes through LDS.  More than 16 rows (128 in LDS) make two fragments.
FORMS = {"item8": (3, 2, 4, 1500, 0), "item8, two": (3, 2, 20, 1500, 0), "item4": (150, 2, 4, 1500, 0),
         "item4, two": (150, 2, 20, 1500, 0), "list": (64, 2, 4, 3000, 0), "list, two": (64, 2, 20, 3000, 0),
         "fold": (8, 2, 4, 40, 1500), "lds": (20, 2, 4, 40, 2700), "lds, two": (70, 2, 4, 40, 2700)}


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


# ------------------------------------------------------------------ what is masked, in every form
def spread(form, dim, qmax, act, seed=5):
    """Sequences of every length from half the form's own tokens on, two query tokens each, over the same pages (so
    that a token is past the end of some and seen by others), some that end inside the prefix; a table wider by a page."""
    B, kv, group, own, prefix = FORMS[form]
    c = Case(seed, [prefix + own], n_q=2, hq=max(1, group // 2) * kv, kv=kv, dim=dim, qmax=qmax, act=act, page=64, prefix=prefix)
    rng = np.random.default_rng(seed)
    c.q = c.q[:1] * rng.uniform(0.5, 1.5, (2 * B, 1, 1))
    c.q = rounded(c.q, act)
    c.table = np.repeat(c.table, B, axis=0)
    c.lengths = prefix + own - rng.integers(0, own // 2, B)
    c.lengths[0] = prefix + own
    if prefix:
        c.lengths[2:6] = prefix // 2 + 5, prefix // 2 + 6, prefix - 1, prefix
    return c


def poisoned(c, slots, what):
    torch = torch_mod()
    bad = torch.full((len(slots), c.kv, c.dim), what, dtype=c.cache.dtype, device="cuda")
    M.kv_append(c.cache, bad, bad, i32(slots))


def same_bits(a, b):
    torch = torch_mod()
    return bool(torch.equal(a.view(torch.int16), b.view(torch.int16)))


def compare(c, got, clean, hit, where):
    """Rows of tokens: those that `hit` names are not finite anywhere, the others as before, bit for bit."""
    torch = torch_mod()
    hit = torch.from_numpy(np.asarray(hit)).cuda()
    assert not torch.isfinite(got[hit]).any(), where
    assert same_bits(got[~hit], clean[~hit]), where


def seeing(c, at):
    """Whether each query token sees position `at`."""
    return (np.repeat(c.lengths, 2) - 2 + np.tile([0, 1], len(c.lengths))) >= at


@pytest.mark.parametrize("act", ["bf16", "fp16"])
@pytest.mark.parametrize("qmax", [0, 127, 448])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("form", list(FORMS))
def test_odd_values_in_every_form(form, dim, qmax, act):
    """Keys and values that are not finite, e4m3 NaN codes, pages outside the cache and lengths past the table: NaN or
    inf for the queries that see them, nothing for the others."""
    torch = torch_mod()
    c = spread(form, dim, qmax, act)
    n, prefix = int(c.lengths[0]), c.prefix_len
    slots = c.slots(0)
    clean = c.run()
    assert bool(torch.isfinite(clean).all())
    keep = [None if t is None else t.clone() for t in c.cache.buffers()]

    def restore():
        for t, k in zip(c.cache.buffers(), keep):
            if t is not None:
                t.copy_(k)

    ends = np.sort(c.lengths)
    places = [n - 1, int(ends[len(ends) // 2]) - 1, int(ends[0]) - 1, prefix + 13] + ([prefix // 2 + 5, prefix - 1] if prefix else [])
    for what in (float("nan"), float("inf")):
        for at in places:
            poisoned(c, slots[at:at + 1], what)
            compare(c, c.run(), clean, seeing(c, at), (what, at))
            restore()
        tail = np.setdiff1d(np.arange(c.cache.n_pages * c.page), slots)          # what no sequence has
        poisoned(c, tail, what)
        assert same_bits(c.run(), clean), what
        restore()
    if qmax == 448:                                # codes that kv_append does not write, from the eighth token of a page on
        first = prefix + (n - prefix) // c.page * c.page
        page, some = int(slots[first]) // c.page, i32(slots[first:first + 7])
        k, v = M.kv_read(c.cache, some)            # (rounded, and coded again)
        M.kv_append(c.cache, k, v, some)
        again = c.run()
        for t in c.cache.buffers():
            t[page].view(torch.uint8).fill_(0x7f)
        M.kv_append(c.cache, k, v, some)
        compare(c, c.run(), again, seeing(c, first + 7), "codes")
        restore()
    # a page outside the cache, for every second sequence
    at, table = (n - prefix) * 3 // 4 // c.page, c.table.copy()
    for id_ in (-1, c.cache.n_pages, 2 ** 31 - 1):
        c.table[::2, at] = id_
        hit = seeing(c, prefix + at * c.page) & np.repeat(np.arange(len(c.lengths)) % 2 == 0, 2)
        compare(c, c.run(), clean, hit, id_)
    c.table = table
    if prefix:
        pages = c.prefix.copy()
        c.prefix[len(pages) // 2] = c.cache.n_pages
        compare(c, c.run(), clean, seeing(c, len(pages) // 2 * c.page), "prefix")
        c.prefix = pages
    # lengths past the table: as empty places for all others (which decide where the shared list is cut)
    lengths = c.lengths.copy()
    c.lengths[1::3] = 0
    empty = c.run()
    assert not empty.reshape(len(lengths), 2, -1)[1::3].any()
    c.lengths[1::3] = prefix + c.table.shape[1] * c.page + 1 + np.arange(len(c.lengths[1::3])) % 2 * 10 ** 9
    past = np.zeros(len(lengths), bool)
    past[1::3] = True
    compare(c, c.run(), empty, np.repeat(past, 2), "past the table")


@pytest.mark.parametrize("act", ["bf16", "fp16"])
@pytest.mark.parametrize("qmax", [0, 127, 448])
def test_lengths_of_neighbours(qmax, act):
    """Where sequences share one list, the cuts between workgroups go by all lengths: a row may differ in rounding
    when a neighbour's length changes, and stays within its bound."""
    c = Case(23, [3000, 2500, 640, 0, 1], hq=4, kv=2, dim=64, qmax=qmax, act=act)
    c.check(c.run())
    for n in (1, 70, 2300):
        c.lengths = np.array([3000, n, 640, 0, 1])
        c.check(c.run(), where=f"{n}")


# ------------------------------------------------------------------ append
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("T,dim,qmax,rot", [(8192 + 5, 64, 448, 64), (8192 + 7, 128, 127, 128), (8192 + 3, 256, 0, 256),
                                            (16384 + 13, 64, 127, 32), (16384 + 9, 128, 448, 128), (16384 + 5, 256, 127, 128),
                                            (16384 + 15, 128, 0, 64)])
def test_append_workgroups_of_many_tokens(T, dim, qmax, rot, inter):
    """8 and 16 tokens to a workgroup, the last one filled in part: rows, codes and scales of single-token calls."""
    torch = torch_mod()
    g = torch.Generator(device="cuda").manual_seed(T)
    hq, kv = 5, 2
    make = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    x, w = make(T, hq + 2 * kv, dim), [make(dim) for _ in range(2)]
    pos = torch.randint(0, 90000, (T,), generator=g, device="cuda").to(torch.int32)
    freqs = torch.from_numpy(1e4 ** (-np.arange(rot // 2) / (rot // 2))).cuda()
    pages = -(-T // 64) + 1
    a, b = (M.KVCache(pages, kv, dim, page_size=64, act="bf16", qmax=qmax) for _ in range(2))
    slots = torch.arange(3, T + 3, device="cuda").to(torch.int32)

    def call(cache, s):
        return M.kv_append(cache, x[s, hq:hq + kv], x[s, hq + kv:], slots[s], q=x[s, :hq], q_weight=w[0], k_weight=w[1],
                           positions=pos[s], freqs=freqs, interleaved=inter)

    got = call(a, slice(0, T))
    some = sorted({*range(0, T, 997), *range(0, 17), *range(8180, 8193), *range(T - 33, T)})
    for t in some:
        assert same_bits(call(b, slice(t, t + 1))[0], got[t]), t
    at = slots[torch.tensor(some, device="cuda")]
    for g, h in zip(M.kv_read(a, at), M.kv_read(b, at)):
        assert same_bits(g, h)


@pytest.mark.parametrize("qmax", [0, 127])
@pytest.mark.parametrize("first", [-1, 64])
def test_runs_of_several_sequences(first, qmax):
    """A call that writes and reads several prompts, each from the beginning of a page on: runs that the call's blocks of
    32 tokens do not meet in step."""
    torch = torch_mod()
    rng = np.random.default_rng(8)
    kv, dim, page = 2, 128, 64
    lengths = [77, 1, 200, 33, 64, 130]
    at, slots = 1, []
    for n in lengths:
        slots.append(at * page + np.arange(n))
        at += -(-n // page)
    slots = np.concatenate(slots)
    slots[0] = first
    n = len(slots)
    cache = M.KVCache(at + 1, kv, dim, page_size=page, act="bf16", qmax=qmax)
    x, y = (rounded(rng.standard_normal((n, kv, dim)), "bf16") for _ in range(2))
    M.kv_append(cache, up(x, "bf16"), up(y, "bf16"), i32(slots))
    keep = slots >= 0
    for got, want in zip(M.kv_read(cache, i32(slots)), (x, y)):
        assert np.array_equal(down(got)[keep], exact_read(want, qmax, "bf16")[keep])
        assert not down(got)[~keep].any()
    others = np.setdiff1d(np.arange(cache.n_pages * page), slots)
    for got in M.kv_read(cache, i32(others)):
        assert not torch.any(got)
