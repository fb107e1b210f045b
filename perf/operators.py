"""The operators around the MoE block whose time this repository looks after.

* ``norm``: ``add_rms_norm``, the residual's addition and the RMS norm in front of a block
  or of a linear, with the normalized rows as 16-bit rows, as 8-bit codes with a scale per
  row, or both.
* ``linear``: ``linear_decode``, one packed linear on the few rows of a decode step: 4-bit
  weights with group scales on 16-bit rows, int8 and FP8 weights on rows that are encoded
  already.
* ``balance``: ``balance_loss``, the router's balance loss over a batch with the experts'
  counts and the gradient of the logits.

Shapes are those of ``workloads.CONFIGS`` (hidden sizes 2048, 3584 and 4096, 8 to 64 experts)
or generic.  The plain forms are elementary torch operations in 32 bits.  Sums of squares
and sums over tokens are taken in 64 bits: the norm's codes are whole steps, which a
different last bit of the row's factor would move.
"""

import math

import torch

own = False

DEV = "cuda"
ACT = {"bf16": torch.bfloat16, "fp16": torch.float16}
QMAX = {"int8": 127, "fp8": 448, "none": 0}
EPS = 1e-6


def listed():
    return [
        # one token of one stream in front of an int8 linear: latency
        dict(name="norm_token_int8", op="norm", rows=1, cols=2048, act="bf16", code="int8", residual=True, y=True, pad=0),
        # a decode batch; the block takes the 16-bit rows, an int8 linear the codes
        dict(name="norm_decode256_int8", op="norm", rows=256, cols=4096, act="fp16", code="int8", residual=True, y=True, pad=0),
        # rows that are a slice of wider ones, of an odd length: a head's part of a joint projection
        dict(name="norm_rows_odd", op="norm", rows=777, cols=1441, act="bf16", code="none", residual=False, y=True, pad=37),
        # a whole prefill in front of FP8 linears
        dict(name="norm_prefill_fp8", op="norm", rows=16384, cols=3584, act="bf16", code="fp8", residual=True, y=True, pad=0),
        # one token through a square projection
        dict(name="linear_token_w4", op="linear", scheme="w4g128", m=1, n=4096, k=4096, act="bf16", bias=False, pad=0),
        # a few streams through a small projection with a bias
        dict(name="linear_7_w4_bias", op="linear", scheme="w4g128", m=7, n=2064, k=1408, act="bf16", bias=True, pad=24),
        # one token through the widest linear of the configurations
        dict(name="linear_token_w4_wide", op="linear", scheme="w4g128", m=1, n=20480, k=3584, act="fp16", bias=False, pad=0),
        # a decode batch through an int8 linear whose rows the norm has encoded
        dict(name="linear_decode16_int8", op="linear", scheme="w8a8", m=16, n=5632, k=2048, act="bf16", bias=False, pad=0),
        # the largest batch of a decode step through the deepest linear
        dict(name="linear_decode64_fp8", op="linear", scheme="fp8", m=64, n=4096, k=14336, act="bf16", bias=False, pad=0),
        # a small step of a block with few experts
        dict(name="balance_64", op="balance", tokens=64, experts=8, top_k=2, masked=0.0),
        # an ordinary batch with padding
        dict(name="balance_4096_masked", op="balance", tokens=4096, experts=60, top_k=4, masked=0.2),
        # the batch of a large training step
        dict(name="balance_65536", op="balance", tokens=65536, experts=64, top_k=8, masked=0.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "linear", "balance"])
    if op == "norm":
        cols = _log_int(rng, 64, 16384)
        if rng.random() < 0.6:
            cols = max(8, cols // 8 * 8)
        code = rng.choice(["none", "int8", "fp8"])
        return dict(op="norm", rows=_log_int(rng, 1, min(16384, (1 << 25) // cols)), cols=cols, act=rng.choice(["bf16", "fp16"]),
                    code=code, residual=rng.random() < 0.7, y=code == "none" or rng.random() < 0.6,
                    pad=rng.choice([0, 0, 8, 13]))
    if op == "linear":
        k = 128 * _log_int(rng, 1, 112)
        n = 16 * _log_int(rng, 1, max(1, min(1280, 58_000_000 // k // 16)))
        return dict(op="linear", scheme=rng.choice(["w4g128", "w4g128", "w8a8", "fp8"]), m=_log_int(rng, 1, 64), n=n, k=k,
                    act=rng.choice(["bf16", "fp16"]), bias=rng.random() < 0.4, pad=rng.choice([0, 0, 16]))
    experts = _log_int(rng, 2, 512)
    return dict(op="balance", tokens=_log_int(rng, 1, min(65536, (1 << 22) // experts)), experts=experts,
                top_k=min(experts, rng.choice([1, 2, 4, 6, 8])), masked=rng.choice([0.0, 0.1, 0.5]))


# ------------------------------------------------------------------ inputs
def _rows(gen, m, cols, pad, act):
    """Rows of unit variance and a few large channels, a slice of wider rows where pad > 0."""
    x = torch.randn(m, cols + pad, generator=gen, device=DEV)
    x *= torch.where(torch.rand(cols + pad, generator=gen, device=DEV) < 0.005, 8.0, 1.0)
    return x.to(ACT[act])[:, :cols]


def _encode(y, code):
    """Codes and scales of 16-bit rows: amax, q / amax, amax / q and the products in 32 bits,
    codes to the nearest (ties to even).  Rows of zeros have scale 0."""
    v = y.float()
    amax = v.abs().amax(1)
    q = torch.full_like(amax, QMAX[code])  # a tensor: division by a plain number may be a product with 1 / it
    some = amax > 0
    inv = torch.where(some, q / amax, torch.zeros_like(amax))
    scales = torch.where(some, amax / q, torch.zeros_like(amax))
    v = (v * inv[:, None]).clamp(-QMAX[code], QMAX[code])
    if code == "int8":
        return v.round().to(torch.int8), scales
    codes = v.to(torch.float8_e4m3fn).view(torch.int8)
    return torch.where(codes == -128, torch.zeros_like(codes), codes), scales  # no negative zero


def _weights(gen, c):
    n, k = c["n"], c["k"]
    w = torch.randn(n, k, generator=gen, device=DEV) * 0.02
    if c["scheme"] == "w4g128":
        w = w.view(n, k // 128, 128)
        lo, hi = w.amin(2), w.amax(2)
        s = ((hi - lo) / 15).half()
        z = (-lo / s.float()).round().clamp(0, 15)
        q = ((w / s.float()[..., None]).round() + z[..., None]).clamp(0, 15)
        return q.to(torch.uint8).view(n, k), s, z.half()
    q, s = _encode(w, "int8" if c["scheme"] == "w8a8" else "fp8")
    return q if c["scheme"] == "w8a8" else q.view(torch.uint8), s, None


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    c, s = case, dict(case=case)
    if c["op"] == "norm":
        s["x"] = _rows(gen, c["rows"], c["cols"], c["pad"], c["act"])
        s["weight"] = (1 + 0.1 * torch.randn(c["cols"], generator=gen, device=DEV)).to(ACT[c["act"]])
        s["residual"] = _rows(gen, c["rows"], c["cols"], c["pad"], c["act"]) if c["residual"] else None
    elif c["op"] == "linear":
        s["codes"], s["scales"], s["zeros"] = _weights(gen, c)
        a = _rows(gen, c["m"], c["k"], c["pad"], c["act"])
        s["bias"] = torch.randn(c["n"], generator=gen, device=DEV).to(ACT[c["act"]]) if c["bias"] else None
        s["a"], s["a_scales"] = (a, None) if c["scheme"] == "w4g128" else _encode(a, "int8" if c["scheme"] == "w8a8" else "fp8")
        if own:  # the weights as a program keeps them: packed once
            from paper_2505_05799_amd import mxmoe as M
            from paper_2505_05799_amd import workloads as W
            scheme = {"w4g128": W.W4G128, "w8a8": W.W8A8, "fp8": W.FP8}[c["scheme"]]
            s["packed"] = M.PackedLinear(W.QLinear(scheme, c["n"], c["k"], s["codes"], s["scales"], s["zeros"]), c["act"])
    else:
        T, E, k = c["tokens"], c["experts"], c["top_k"]
        skew = -torch.log(1.0 + torch.randperm(E, generator=gen, device=DEV).float())
        s["logits"] = torch.randn(T, E, generator=gen, device=DEV) + skew
        s["ids"] = s["logits"].topk(k, 1).indices.to(torch.int32)
        s["mask"] = torch.rand(T, generator=gen, device=DEV) >= c["masked"] if c["masked"] else None
    return s


# -------------------------------------------------------------------- plain
def _plain_norm(s):
    c, act = s["case"], ACT[s["case"]["act"]]
    z = s["x"]
    if s["residual"] is not None:
        z = (z.float() + s["residual"].float()).to(act)
    ms = z.double().square().mean(1) + EPS
    r = (1.0 / ms.sqrt()).float()
    y = (z.float() * r[:, None] * s["weight"].float()).to(act)
    codes, scales = _encode(y, c["code"]) if c["code"] != "none" else (None, None)
    return y if c["y"] else None, z if s["residual"] is not None else None, codes, scales


def _plain_linear(s):
    c = s["case"]
    n, k = c["n"], c["k"]
    if c["scheme"] == "w4g128":
        q = s["codes"].float().view(n, k // 128, 128)
        w = ((q - s["zeros"].float()[..., None]) * s["scales"].float()[..., None]).view(n, k)
        out = s["a"].float() @ w.t()
    else:
        a, w = (s["a"].float(), s["codes"].float()) if c["scheme"] == "w8a8" else \
            (s["a"].view(torch.float8_e4m3fn).float(), s["codes"].view(torch.float8_e4m3fn).float())
        out = (a @ w.t()) * s["a_scales"][:, None] * s["scales"]
    if s["bias"] is not None:
        out = out + s["bias"].float()
    return out.to(ACT[c["act"]])


def _plain_balance(s):
    c, logits, ids = s["case"], s["logits"], s["ids"]
    T, E, k = c["tokens"], c["experts"], c["top_k"]
    p = torch.exp(logits - logits.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    kept = torch.ones(T, dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"]
    n = kept.sum().double()
    per = torch.where(n > 0, 1.0 / n, torch.zeros_like(n))  # no token kept: all zero
    counts = torch.zeros(E, dtype=torch.int32, device=DEV)
    counts.index_add_(0, ids.reshape(-1).long(), kept[:, None].expand(T, k).reshape(-1).to(torch.int32))
    f = counts.double() * per / k
    p = torch.where(kept[:, None], p, torch.zeros_like(p))
    probs = p.double().sum(0) * per
    loss = E * (f * probs).sum()
    f32 = f.float()
    grad = (E * per).float() * p * (f32 - (p * f32).sum(1, keepdim=True))
    return loss.float(), counts, probs.float(), grad


def _values(codes, scales, c):
    """8-bit codes as the values they stand for, in the rows' type; e4m3 bytes are values as
    they are (their scales are returned beside them)."""
    if codes is None:
        return None
    if c["code"] == "fp8":
        return codes.view(torch.float8_e4m3fn)
    return torch.mul(codes, scales[:, None], out=torch.empty(codes.shape, dtype=ACT[c["act"]], device=codes.device))


def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2505_05799_amd import mxmoe as M
        if c["op"] == "norm":
            y, z, codes, scales = M.add_rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS,
                                                 qmax=QMAX[c["code"]], want_y=c["y"])
        elif c["op"] == "linear":
            return {"out": M.linear_decode(s["packed"], s["a"], scales=s["a_scales"], bias=s["bias"])}
        else:
            loss, counts, probs, grad = M.balance_loss(s["logits"], s["ids"], token_mask=s["mask"])
    else:
        if c["op"] == "norm":
            y, z, codes, scales = _plain_norm(s)
        elif c["op"] == "linear":
            return {"out": _plain_linear(s)}
        else:
            loss, counts, probs, grad = _plain_balance(s)
    if c["op"] == "norm":
        return {"y": y, "sum": z, "values": _values(codes, scales, c), "scales": scales}
    return {"loss": loss, "counts": counts, "probs": probs, "grad": grad}


def work(case):
    c = case
    if c["op"] == "norm":
        e = c["rows"] * c["cols"]
        each = 2 + (4 if c["residual"] else 0) + (2 if c["y"] else 0) + (c["code"] != "none")
        rows = 4 * c["rows"] if c["code"] != "none" else 0
        return {"bytes": e * each + rows + 2 * c["cols"], "flops": e * (4 + 3 * (c["code"] != "none"))}
    if c["op"] == "linear":
        m, n, k = c["m"], c["n"], c["k"]
        w = n * k // 2 + n * (k // 128) * 4 if c["scheme"] == "w4g128" else n * k + 4 * n
        a = 2 * m * k if c["scheme"] == "w4g128" else m * k + 4 * m
        return {"bytes": w + a + 2 * m * n + (2 * n if c["bias"] else 0), "flops": 2 * m * n * k}
    T, E, k = c["tokens"], c["experts"], c["top_k"]
    return {"bytes": 8 * T * E + 4 * T * k + (T if c["masked"] else 0) + 8 * E + 4, "flops": 8 * T * E}


# -------------------------------------------------------------------- exact
def _fl32(v):
    return v.to(torch.float32).to(torch.float64)


def _exact_norm(s):
    """Products and quotients of 32-bit values formed in 64 bits and rounded where the
    definition rounds (the row's factor, each product, the 16-bit row the codes are of)."""
    c, act = s["case"], ACT[s["case"]["act"]]
    z = s["x"].double()
    if s["residual"] is not None:
        z = _fl32(z + s["residual"].double()).to(act).double()
    r = _fl32(torch.pow((z * z).sum(1) / c["cols"] + EPS, -0.5))
    y = _fl32(z * r[:, None]) * s["weight"].double()
    values = scales = None
    if c["code"] != "none":
        q = float(QMAX[c["code"]])
        y16 = _fl32(y).to(act).double()
        top = y16.abs().max(1).values
        safe = torch.where(top > 0, top, torch.ones_like(top))
        scales = torch.where(top > 0, _fl32(top / q), torch.zeros_like(top))
        v = _fl32(y16 * _fl32(q / safe)[:, None])
        if c["code"] == "int8":
            values = torch.round(v) * scales[:, None]
        else:  # the e4m3 grid: steps of 2^(e-3), 2^-9 at the least
            step = torch.exp2(torch.clamp(torch.floor(torch.log2(torch.clamp(v.abs(), min=2.0 ** -20))), min=-6) - 3)
            values = torch.clamp(torch.round(v / step) * step, -448, 448)
    return {"y": y if c["y"] else None, "sum": z if s["residual"] is not None else None, "values": values,
            "scales": scales}


def _exact_linear(s):
    c = s["case"]
    e4m3 = torch.tensor([(-1.0) ** (b >> 7) * ((b & 7) * 2.0 ** -9 if (b >> 3) & 15 == 0 else
                                              (8 + (b & 7)) * 2.0 ** (((b >> 3) & 15) - 10)) for b in range(256)],
                        dtype=torch.float64, device=DEV)
    out = torch.zeros(c["m"], c["n"], dtype=torch.float64, device=DEV)
    step = max(1, (1 << 25) // c["k"])
    if c["scheme"] == "fp8":
        a = e4m3[s["a"].view(torch.uint8).long()] * s["a_scales"].double()[:, None]
    else:
        a = s["a"].double() * (1.0 if s["a_scales"] is None else s["a_scales"].double()[:, None])
    for n0 in range(0, c["n"], step):  # in pieces of the channels: 64-bit weights are large
        at = slice(n0, min(n0 + step, c["n"]))
        q, sc = s["codes"][at], s["scales"][at].double()
        if c["scheme"] == "w4g128":
            w = (q.double() - s["zeros"][at].double().repeat_interleave(128, 1)) * sc.repeat_interleave(128, 1)
        else:
            w = (q.double() if c["scheme"] == "w8a8" else e4m3[q.long()]) * sc[:, None]
        out[:, at] = torch.mm(a, w.t().contiguous())
    return {"out": out if s["bias"] is None else out + s["bias"].double()}


def _exact_balance(s):
    c = s["case"]
    E, k = c["experts"], c["top_k"]
    keep = slice(None) if s["mask"] is None else s["mask"].nonzero()[:, 0]
    l, ids = s["logits"][keep].double(), s["ids"][keep]
    n = l.shape[0]
    grad = torch.zeros(c["tokens"], E, dtype=torch.float64, device=DEV)
    if n == 0:
        none = torch.zeros(E, dtype=torch.float64, device=DEV)
        return {"loss": none.sum(), "counts": none.int(), "probs": none, "grad": grad}
    p = torch.softmax(l, 1)
    counts = torch.bincount(ids.reshape(-1).long(), minlength=E)
    share = counts.double() / (n * k)
    mean = p.sum(0) / n
    grad[keep] = (E / n) * p * (share - torch.mv(p, share)[:, None])
    return {"loss": E * torch.dot(share, mean), "counts": counts.int(), "probs": mean, "grad": grad}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "linear": _exact_linear, "balance": _exact_balance}[case["op"]](s)
