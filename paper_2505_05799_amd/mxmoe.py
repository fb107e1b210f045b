"""ctypes binding of libmxmoe.so (C ABI in include/mxmoe.h).

Argument marshalling only: every step of the forward runs in the library's HIP
kernels.  PyTorch provides device memory and the current stream.  There is no
fallback: if the library is missing or a call fails, an exception is raised.
"""

from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import List, Optional, Sequence

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libmxmoe.so")

F16, BF16 = 0, 1
OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP = range(5)


class Scheme_t(C.Structure):
    _fields_ = [("w_bits", C.c_int32), ("a_bits", C.c_int32), ("w_group", C.c_int32),
                ("a_group", C.c_int32), ("symmetric", C.c_int32), ("fmt", C.c_int32)]


class Linear_t(C.Structure):
    _fields_ = [("n", C.c_int32), ("k", C.c_int32), ("s", Scheme_t)]


class Block_t(C.Structure):
    _fields_ = [("hidden", C.c_int32), ("ffn", C.c_int32), ("n_experts", C.c_int32),
                ("top_k", C.c_int32), ("n_shared", C.c_int32), ("ffn_shared", C.c_int32),
                ("act", C.c_int), ("scheme", C.POINTER(Scheme_t)), ("packed", C.POINTER(C.c_void_p))]


N_PHASES = 5
PHASE_NAMES = ("route_plan_xquant", "gemm_gate_up", "hquant", "gemm_down", "combine")


class ForwardOpts_t(C.Structure):
    _fields_ = [("expert_mask", C.POINTER(C.c_uint8)), ("reserved0", C.c_int32),
                ("skip_combine", C.c_int32), ("events", C.POINTER(C.c_void_p)),
                ("router_logits", C.c_void_p), ("renormalize", C.c_int32), ("shared_logits", C.c_void_p),
                ("shared_w", C.c_void_p), ("fp32_slots", C.c_int32), ("reserved1", C.c_int32)]


class KVCache_t(C.Structure):
    _fields_ = [("n_pages", C.c_int32), ("heads", C.c_int32), ("dim", C.c_int32), ("page_size", C.c_int32),
                ("act", C.c_int), ("qmax", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p), ("k_scales", C.c_void_p),
                ("v_scales", C.c_void_p)]


WS_FIELDS = ["status", "counts", "offsets", "sorted_pair", "inv", "plan", "xq8", "xs8", "xq4", "xs4",
             "h", "h_shared", "hq", "hs", "hq_shared", "hs_shared", "slots", "total", "plan_queue_cap",
             "plan_flat_cap", "partial", "partial_floats", "rsx", "rsh", "rsh_shared", "xq4g", "xs4g", "hsg",
             "hsg_shared", "xqmx", "xsmx", "hqmx", "hsmx", "hqmx_shared", "hsmx_shared", "router_ids", "router_w",
             "shared_w", "xqf8", "xsf8", "xqf6", "xsf6"]


class WsLayout_t(C.Structure):
    _fields_ = [(f, C.c_size_t) for f in WS_FIELDS]


EXPORTS = [
    "mxmoe_packed_bytes", "mxmoe_pack_weights", "mxmoe_unpack_weights", "mxmoe_route_workspace_bytes",
    "mxmoe_route_permute", "mxmoe_router_topk", "mxmoe_act_quant", "mxmoe_linear_workspace_bytes", "mxmoe_linear_forward",
    "mxmoe_block_table_bytes", "mxmoe_block_table_fill", "mxmoe_workspace_bytes", "mxmoe_moe_forward",
    "mxmoe_moe_forward_ex", "mxmoe_workspace_layout", "mxmoe_status_string", "mxmoe_version",
    "mxmoe_moe_forward_noalloc", "mxmoe_set_tile_costs", "mxmoe_get_tile_costs",
    "mxmoe_add_rms_norm", "mxmoe_linear_decode", "mxmoe_balance_workspace_bytes", "mxmoe_balance_loss",
    "mxmoe_kv_cache_bytes", "mxmoe_kv_scale_bytes", "mxmoe_kv_append", "mxmoe_kv_read",
    "mxmoe_attention_workspace_bytes", "mxmoe_attention_decode",
]
TILE_COST_SHAPE = (2, 11, 4, 4)     # [phase][scheme][configuration][a, bs, bu, h], MXMOE_TILE_COST_ENTRIES
NOALLOC_SCRATCH_BYTES = 128 << 20   # MXMOE_NOALLOC_SCRATCH_BYTES
DECODE_ROWS = 64                    # MXMOE_DECODE_ROWS
ATTENTION_QUERIES = 16              # MXMOE_ATTENTION_QUERIES

_lib = None


def load_library(path: str = LIB_PATH) -> C.CDLL:
    """Load libmxmoe.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2505_05799_amd.build`")
    lib = C.CDLL(path)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    PL, PB, PK = C.POINTER(Linear_t), C.POINTER(Block_t), C.POINTER(KVCache_t)
    sig = {
        "mxmoe_packed_bytes": (sz, [PL, C.c_int]),
        "mxmoe_pack_weights": (C.c_int, [PL, C.c_int, C.c_int, vp, vp, vp, vp, sz, vp]),
        "mxmoe_unpack_weights": (C.c_int, [PL, C.c_int, vp, vp, vp, vp, vp]),
        "mxmoe_route_workspace_bytes": (sz, [i32, i32, i32]),
        "mxmoe_route_permute": (C.c_int, [vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]),
        "mxmoe_router_topk": (C.c_int, [vp, i32, i32, i32, i32, vp, i32, vp, vp, vp, vp]),
        "mxmoe_act_quant": (C.c_int, [vp, C.c_int, i32, i32, i64, i32, vp, vp, vp]),
        "mxmoe_linear_workspace_bytes": (sz, [PL, i32]),
        "mxmoe_linear_forward": (C.c_int, [PL, C.c_int, vp, i32, vp, vp, vp, sz, vp]),
        "mxmoe_block_table_bytes": (sz, [PB]),
        "mxmoe_block_table_fill": (C.c_int, [PB, vp, sz]),
        "mxmoe_workspace_bytes": (sz, [PB, i32]),
        "mxmoe_moe_forward": (C.c_int, [PB, vp, i32, vp, vp, vp, vp, vp, sz, vp]),
        "mxmoe_moe_forward_ex": (C.c_int, [PB, vp, i32, vp, vp, vp, vp, vp, sz,
                                           C.POINTER(ForwardOpts_t), vp]),
        "mxmoe_workspace_layout": (C.c_int, [PB, i32, C.POINTER(WsLayout_t)]),
        "mxmoe_moe_forward_noalloc": (C.c_int, [PB, vp, i32, vp, vp, vp, vp, vp]),
        "mxmoe_status_string": (C.c_char_p, [C.c_int]),
        "mxmoe_version": (i32, []),
        "mxmoe_set_tile_costs": (C.c_int, [vp, i32]),
        "mxmoe_get_tile_costs": (C.c_int, [vp, i32]),
        "mxmoe_add_rms_norm": (C.c_int, [vp, i64, vp, i64, vp, C.c_int, i32, i32, C.c_double, vp, i64, vp, i64, i32, vp, vp,
                                         vp]),
        "mxmoe_linear_decode": (C.c_int, [PL, C.c_int, vp, i32, vp, i64, vp, vp, vp, i64, vp]),
        "mxmoe_balance_workspace_bytes": (sz, [i32, i32]),
        "mxmoe_balance_loss": (C.c_int, [vp, vp, vp, i32, i32, i32, C.c_float, vp, vp, vp, vp, vp, sz, vp]),
        "mxmoe_kv_cache_bytes": (sz, [PK]),
        "mxmoe_kv_scale_bytes": (sz, [PK]),
        "mxmoe_kv_append": (C.c_int, [PK, i32, vp, i64, i32, vp, i64, vp, i64, vp, vp, C.c_double, vp, vp, i32, i32, vp, vp, i64,
                                      vp]),
        "mxmoe_kv_read": (C.c_int, [PK, i32, vp, vp, vp, vp]),
        "mxmoe_attention_workspace_bytes": (sz, [PK, i32, i32, i32, i32, i32]),
        "mxmoe_attention_decode": (C.c_int, [PK, vp, i64, i32, i32, i32, vp, i32, vp, vp, i32, C.c_float, C.c_float, vp, i64, vp,
                                             sz, vp]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    _lib = lib
    # the run-time plan prices tiles with the profiled cost table when there is one
    from . import tile_cost
    if os.path.exists(tile_cost.DEFAULT_TABLE):
        set_tile_costs(tile_cost.CostTable.load().device_table())
    return lib


def set_tile_costs(table=None):
    """Install the run-time plan's tile cost table (int32 TILE_COST_SHAPE, ps),
    or the library's roofline default with None (mxmoe_set_tile_costs)."""
    lib = load_library()
    if table is None:
        _check(lib.mxmoe_set_tile_costs(None, 0), "mxmoe_set_tile_costs")
        return
    t = np.ascontiguousarray(table, dtype=np.int32)
    if t.shape != TILE_COST_SHAPE:
        raise ValueError(f"tile cost table of shape {t.shape}, expected {TILE_COST_SHAPE}")
    _check(lib.mxmoe_set_tile_costs(t.ctypes.data_as(C.c_void_p), t.size), "mxmoe_set_tile_costs")


def get_tile_costs() -> np.ndarray:
    """The tile cost table forwards use now (mxmoe_get_tile_costs)."""
    t = np.zeros(TILE_COST_SHAPE, dtype=np.int32)
    _check(load_library().mxmoe_get_tile_costs(t.ctypes.data_as(C.c_void_p), t.size), "mxmoe_get_tile_costs")
    return t


class MxmoeError(RuntimeError):
    def __init__(self, status: int, what: str):
        lib = load_library()
        super().__init__(f"{what}: {lib.mxmoe_status_string(status).decode()} (status {status})")
        self.status = status


def _check(status: int, what: str):
    if status != OK:
        raise MxmoeError(status, what)


def _torch():
    import torch
    return torch


def _stream_ptr(stream=None):
    torch = _torch()
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


def _ptr(t) -> C.c_void_p:
    return C.c_void_p(0 if t is None else t.data_ptr())


def scheme_t(s) -> Scheme_t:
    return Scheme_t(s.w_bits, s.a_bits, s.w_group, s.a_group, s.symmetric, getattr(s, "fmt", 0))


def act_code(act: str) -> int:
    return {"fp16": F16, "bf16": BF16}[act]


def _dev(arr: np.ndarray, device):
    """numpy -> device tensor with the same bytes (16-bit data travels as int16);
    a torch tensor is moved as it is."""
    torch = _torch()
    if isinstance(arr, torch.Tensor):
        return arr.contiguous().to(device)
    a = np.ascontiguousarray(arr)
    if a.dtype == np.uint16:
        a = a.view(np.int16)
    if a.dtype == np.float16:
        a = a.view(np.int16)
    return torch.from_numpy(a.copy()).to(device)


def act_tensor(x: np.ndarray, act: str, device="cuda"):
    """numpy activation storage (float16 or bf16 bits) -> torch tensor of the act dtype."""
    torch = _torch()
    t = _dev(x, device)
    return t.view(torch.float16 if act == "fp16" else torch.bfloat16)


def act_numpy(t, act: str) -> np.ndarray:
    """torch act tensor -> numpy storage (float16 array or bf16 bits)."""
    torch = _torch()
    a = t.detach().contiguous().view(torch.int16).cpu().numpy()
    return a.view(np.float16) if act == "fp16" else a.view(np.uint16)


def empty_aligned(nbytes: int, device="cuda"):
    torch = _torch()
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)


# --------------------------------------------------------------- packing
def operand_bytes(scheme, n: int, k: int):
    """Bytes the packer reads from (codes, scales, zeros) for a scheme (None: not read)."""
    s = scheme
    if s.w_bits == 16:
        return 2 * n * k, None, None
    if getattr(s, "fmt", 0) == 1:
        return n * k, n * (k // 32), None
    if s.a_bits == 16:
        return n * k, 2 * n * (k // 128), 2 * n * (k // 128)
    if s.w_group > 0:
        return n * k, 2 * n * (k // 128), None
    return n * k, 4 * n, None


def _nbytes(arr) -> int:
    if arr is None:
        return 0
    if hasattr(arr, "element_size"):
        return arr.numel() * arr.element_size()
    return np.asarray(arr).nbytes


def check_operands(q):
    """Raise ValueError unless the codes / scales / zeros of a QLinear hold at
    least the bytes the packer reads for its scheme (the packer takes raw
    pointers and cannot check their extent)."""
    want = operand_bytes(q.scheme, q.n, q.k)
    for name, arr, need in zip(("codes", "scales", "zeros"), (q.codes, q.scales, q.zeros), want):
        if need is not None and (arr is None or _nbytes(arr) < need):
            raise ValueError(f"{q.scheme.name} {q.n}x{q.k}: {name} hold {_nbytes(arr)} bytes, the packer reads {need}")


class PackedLinear:
    """One linear packed on the device (owns the packed buffer)."""

    def __init__(self, q, act: str, device="cuda", stream=None):
        lib = load_library()
        check_operands(q)
        self.q = q
        self.act = act
        self.L = Linear_t(q.n, q.k, scheme_t(q.scheme))
        nbytes = lib.mxmoe_packed_bytes(C.byref(self.L), act_code(act))
        if nbytes == 0:
            raise MxmoeError(ERR_UNSUPPORTED, f"packed_bytes({q.scheme.name} {q.n}x{q.k})")
        self.nbytes = nbytes
        self.buf = empty_aligned(nbytes, device)
        codes = _dev(q.codes, device)
        scales = _dev(q.scales, device) if q.scales is not None else None
        zeros = _dev(q.zeros, device) if q.zeros is not None else None
        _check(lib.mxmoe_pack_weights(C.byref(self.L), act_code(act), BF16, _ptr(codes), _ptr(scales),
                                      _ptr(zeros), _ptr(self.buf), nbytes, _stream_ptr(stream)),
               "mxmoe_pack_weights")
        self._keep = (codes, scales, zeros)   # alive until the pack kernel has run

    def release_sources(self):
        self._keep = None

    def unpack(self, stream=None):
        """Device unpack -> (codes, scales, zeros) as numpy arrays."""
        torch = _torch()
        lib = load_library()
        q = self.q
        s = q.scheme
        if s.w_bits == 16:
            codes = torch.empty((q.n, q.k), dtype=torch.int16, device=self.buf.device)
        else:
            codes = torch.empty((q.n, q.k), dtype=torch.uint8, device=self.buf.device)
        scales = zeros = None
        if s.w_bits < 16 and s.a_bits == 16:
            scales = torch.empty((q.n, q.k // 128), dtype=torch.int16, device=self.buf.device)
            zeros = torch.empty_like(scales)
        elif s.fmt == 1:                          # mxfp4: E8M0 bytes per 32
            scales = torch.empty((q.n, q.k // 32), dtype=torch.uint8, device=self.buf.device)
        elif s.w_bits < 16 and s.w_group > 0:     # w4a4-g128: fp16 group scales
            scales = torch.empty((q.n, q.k // 128), dtype=torch.int16, device=self.buf.device)
        elif s.w_bits < 16:
            scales = torch.empty(q.n, dtype=torch.float32, device=self.buf.device)
        _check(lib.mxmoe_unpack_weights(C.byref(self.L), act_code(self.act), _ptr(self.buf), _ptr(codes),
                                        _ptr(scales), _ptr(zeros), _stream_ptr(stream)),
               "mxmoe_unpack_weights")
        torch.cuda.synchronize()
        c = codes.cpu().numpy()
        if s.w_bits == 16:
            c = c.view(np.uint16)
        elif s.a_bits < 16 and s.fmt in (0, 3):
            c = c.view(np.int8)
        sc = None if scales is None else scales.cpu().numpy()
        if sc is not None and s.fmt == 0 and (s.a_bits == 16 or s.w_group > 0):
            sc = sc.view(np.float16)
        z = None if zeros is None else zeros.cpu().numpy().view(np.float16)
        return c, sc, z


def linear_forward(pl: PackedLinear, a, stream=None, return_ws: bool = False):
    """out = a W^T through the micro-kernels: int32 for w8a8/w4a4 (per channel,
    int8 or FP6 operands), else fp32 (fp8: scaled by s_a[m] s_w[n]).  return_ws: also return the
    workspace (its tile plan starts at offset 0)."""
    torch = _torch()
    lib = load_library()
    m = a.shape[0]
    s = pl.q.scheme
    raw_int = s.a_bits < 16 and s.a_group < 0 and getattr(s, "fmt", 0) in (0, 3)
    out = torch.empty((m, pl.q.n), dtype=torch.int32 if raw_int else torch.float32, device=a.device)
    wsb = lib.mxmoe_linear_workspace_bytes(C.byref(pl.L), m)
    ws = empty_aligned(wsb, a.device)
    _check(lib.mxmoe_linear_forward(C.byref(pl.L), act_code(pl.act), _ptr(pl.buf), m, _ptr(a.contiguous()),
                                    _ptr(out), _ptr(ws), wsb, _stream_ptr(stream)), "mxmoe_linear_forward")
    return (out, ws) if return_ws else out


# ------------------------------------------------- operators around the block
# (a decode step calls these once per layer: what they cost the host beside the
# launch is one pass of checks, the outputs' allocations and the call)
def _run_on(dev, stream, body, used):
    """body(stream handle) with GPU `dev` current, on `stream` (default: the GPU's
    current one); what body allocates belongs to that stream, and the tensors
    `used` are kept until its work on them is done."""
    torch = _torch()
    if stream is None:
        if dev == torch.cuda.current_device():
            return body(torch._C._cuda_getCurrentRawStream(dev))
        with torch.cuda.device(dev):
            return body(torch._C._cuda_getCurrentRawStream(dev))
    if stream.device.index != dev:
        raise ValueError(f"a stream of {stream.device} for tensors on GPU {dev}")
    with torch.cuda.stream(stream):
        out = body(stream.cuda_stream)
    for t in used:
        if t is not None:
            t.record_stream(stream)
    return out


def _dense(t, name, dtypes, shape, dev):
    """Raise ValueError unless t is a dense tensor of one of the dtypes, of the
    shape, on GPU `dev`; returns its address."""
    if t.dtype not in dtypes or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)} (strides {t.stride()}) on {t.device}, "
                         f"expected dense {dtypes} {tuple(shape)} on GPU {dev}")
    return t.data_ptr()


def _rows(t, name, dtypes, shape, dev):
    """The same for [rows, cols] tensors whose rows lie apart by any stride; returns
    the address and the row stride."""
    if t.dtype not in dtypes or t.shape != shape or t.get_device() != dev:
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)} on {t.device}, expected {dtypes} {tuple(shape)} on GPU {dev}")
    rows, cols = shape
    ld, one = t.stride()
    if (one != 1 and cols > 1) or (ld < cols and rows > 1):
        raise ValueError(f"{name}: strides {t.stride()}; rows of elements side by side, apart from each other, are expected")
    return t.data_ptr(), (ld if rows > 1 else max(cols, 1))


def _gpu_of(t, name):
    """Index of the GPU that holds a [rows, columns] tensor."""
    dev = t.get_device()
    if dev < 0 or t.dim() != 2:
        raise ValueError(f"{name}: a [rows, columns] tensor on a GPU is expected, got {tuple(t.shape)} on {t.device}")
    return dev


def add_rms_norm(x, weight, residual=None, eps: float = 1e-6, qmax: int = 0, want_y: bool = True, sum_out=None,
                 stream=None):
    """z = x + residual, y = RMS norm of z times weight, and y's 8-bit rows
    (mxmoe_add_rms_norm): returns (y, z, codes, scales).

    x, residual [rows, cols] fp16 or bf16, rows of any stride; weight [cols].
    z is None without a residual, else a new tensor or sum_out (which may be
    residual or x themselves); y is None with want_y=False.  qmax 127: int8 codes,
    448: FP8 e4m3 bytes in an int8 tensor, with fp32 scales per row (linear_decode
    takes them); 0: neither."""
    torch = _torch()
    lib = _lib or load_library()
    dev = _gpu_of(x, "x")
    dt = x.dtype
    if dt is torch.bfloat16:
        act = BF16
    elif dt is torch.float16:
        act = F16
    else:
        raise ValueError(f"x: {dt}, expected bfloat16 or float16")
    shape = x.shape
    rows, cols = shape
    own = (dt,)
    xp, ldx = _rows(x, "x", own, shape, dev)
    wp = _dense(weight, "weight", own, (cols,), dev)
    rp, ldr = (None, 0) if residual is None else _rows(residual, "residual", own, shape, dev)
    zp, ldz = None, cols
    if sum_out is not None:
        if residual is None:
            raise ValueError("sum_out: there is no sum without a residual")
        zp, ldz = _rows(sum_out, "sum_out", own, shape, dev)

    def body(s):
        d = x.device
        y = codes = scales = yp = cp = sp = None
        z, p = sum_out, zp
        if residual is not None and z is None:
            z = torch.empty(rows, cols, dtype=dt, device=d)
            p = z.data_ptr()
        if want_y:
            y = torch.empty(rows, cols, dtype=dt, device=d)
            yp = y.data_ptr()
        if qmax:
            codes = torch.empty(rows, cols, dtype=torch.int8, device=d)
            scales = torch.empty(rows, dtype=torch.float32, device=d)
            cp, sp = codes.data_ptr(), scales.data_ptr()
        st = lib.mxmoe_add_rms_norm(xp, ldx, rp, ldr, wp, act, rows, cols, eps, p, ldz, yp, cols, qmax, cp, sp, s)
        if st:
            raise MxmoeError(st, "mxmoe_add_rms_norm")
        return y, z, codes, scales

    return _run_on(dev, stream, body, (x, residual, weight, sum_out))


def linear_decode(pl: PackedLinear, a, scales=None, bias=None, out=None, stream=None):
    """out = a W^T + bias for at most DECODE_ROWS rows, in the activation dtype
    (mxmoe_linear_decode).  w4g128: a fp16 / bf16 [m, k]; w8a8 and fp8: a the
    codes [m, k] and scales [m] of act_quant or add_rms_norm.  Rows of any stride
    (copied if not 16-byte aligned)."""
    torch = _torch()
    lib = _lib or load_library()
    dev = _gpu_of(a, "a")
    q, buf = pl.q, pl.buf
    n, k, coded = q.n, q.k, q.scheme.a_bits < 16
    m = a.shape[0]
    act, dt = (BF16, torch.bfloat16) if pl.act == "bf16" else (F16, torch.float16)
    ap, lda = _rows(a, "a", (torch.int8, torch.uint8) if coded else (dt,), (m, k), dev)
    if buf.get_device() != dev:
        raise ValueError(f"a: on GPU {dev}, the packed weights on {buf.device}")
    if coded != (scales is not None):
        raise ValueError(f"{q.scheme.name}: scales are the rows' of 8-bit codes")
    sp = None if scales is None else _dense(scales, "scales", (torch.float32,), (m,), dev)
    bp = None if bias is None else _dense(bias, "bias", (dt,), (n,), dev)
    op, ldo = (None, n) if out is None else _rows(out, "out", (dt,), (m, n), dev)

    def body(s):
        rows, rp, ldr = a, ap, lda
        if rp % 16 or (m > 1 and ldr * (1 if coded else 2) % 16):
            rows = a.clone(memory_format=torch.contiguous_format)
            rp, ldr = rows.data_ptr(), k
        o, p = out, op
        if o is None:
            o = torch.empty(m, n, dtype=dt, device=a.device)
            p = o.data_ptr()
        st = lib.mxmoe_linear_decode(C.byref(pl.L), act, buf.data_ptr(), m, rp, ldr, sp, bp, p, ldo, s)
        if st:
            raise MxmoeError(st, "mxmoe_linear_decode")
        return o

    return _run_on(dev, stream, body, (a, scales, bias, out, buf))


def balance_loss(logits, topk_ids, alpha: float = 1.0, token_mask=None, want_grad: bool = True, stream=None):
    """Balance loss of the router (mxmoe_balance_loss): (loss [], counts int32
    [E], mean probabilities [E], gradient of the logits [T, E] or None).

    logits fp32 [T, E]; topk_ids int32 [T, k]; token_mask bool or uint8 [T], False
    for padding.  The returned tensors have no autograd graph, also where the logits
    have one: the gradient enters a backward pass as
    ``torch.autograd.backward([out, logits], [None, grad])``; alpha takes its
    factor."""
    torch = _torch()
    lib = _lib or load_library()
    dev = _gpu_of(logits, "logits")
    shape = logits.shape
    T, E = shape
    lp = _dense(logits, "logits", (torch.float32,), shape, dev)
    if topk_ids.dim() != 2:
        raise ValueError(f"topk_ids: shape {tuple(topk_ids.shape)}, expected [T, k]")
    k = topk_ids.shape[1]
    ip = _dense(topk_ids, "topk_ids", (torch.int32,), (T, k), dev)
    mp = None if token_mask is None else _dense(token_mask, "token_mask", (torch.bool, torch.uint8), (T,), dev)
    wsb = lib.mxmoe_balance_workspace_bytes(T, E)

    def body(s):
        d = logits.device
        counts = torch.empty(E, dtype=torch.int32, device=d)
        probs = torch.empty(E, dtype=torch.float32, device=d)
        loss = torch.empty((), dtype=torch.float32, device=d)
        grad = torch.empty(T, E, dtype=torch.float32, device=d) if want_grad else None
        ws = torch.empty(wsb, dtype=torch.uint8, device=d) if wsb else None
        st = lib.mxmoe_balance_loss(lp, ip, mp, T, E, k, alpha, counts.data_ptr(), probs.data_ptr(), loss.data_ptr(),
                                    grad.data_ptr() if want_grad else None, ws.data_ptr() if wsb else None, wsb, s)
        if st:
            raise MxmoeError(st, "mxmoe_balance_loss")
        return loss, counts, probs, grad

    return _run_on(dev, stream, body, (logits, topk_ids, token_mask))


# ------------------------------------------- attention of a decode step
class KVCache:
    """A paged cache of keys and values on one GPU (mxmoe_kv_cache): n_pages pages of
    page_size tokens, `heads` kv heads of `dim` elements.  qmax 0 keeps 16-bit rows of the
    activation dtype, 127 int8 codes and 448 FP8 e4m3 with an fp32 scale per token
    and head.  k, v [n_pages, heads, page_size * dim] and k_scales, v_scales [n_pages, heads,
    page_size] start as zeros; rows are in an order of their own inside a page
    (kv_append writes them, kv_read reads them), pages may be copied whole.  The calls use the
    buffers' addresses: contents change in place, attributes are not set again."""

    def __init__(self, n_pages: int, heads: int, dim: int, page_size: int = 64, act: str = "bf16", qmax: int = 0,
                 device="cuda"):
        torch = _torch()
        lib = load_library()
        self.n_pages, self.heads, self.dim, self.page_size, self.act, self.qmax = n_pages, heads, dim, page_size, act, qmax
        self.dtype = {"bf16": torch.bfloat16, "fp16": torch.float16}[act]
        self.t = KVCache_t(n_pages, heads, dim, page_size, act_code(act), qmax)
        # (the descriptor's fields would take larger numbers modulo 2^32)
        if max(n_pages, heads, dim, page_size, qmax) >> 31 > 0 or lib.mxmoe_kv_cache_bytes(C.byref(self.t)) == 0:
            raise MxmoeError(ERR_UNSUPPORTED, f"kv_cache({n_pages} pages of {page_size}, {heads} heads of {dim}, qmax {qmax})")
        rows = torch.int8 if qmax else self.dtype
        self.k, self.v = (torch.zeros(n_pages, heads, page_size * dim, dtype=rows, device=device) for _ in range(2))
        self.k_scales, self.v_scales = (torch.zeros(n_pages, heads, page_size, dtype=torch.float32, device=device) if qmax else None
                                        for _ in range(2))
        self.t.k, self.t.v = self.k.data_ptr(), self.v.data_ptr()
        if qmax:
            self.t.k_scales, self.t.v_scales = self.k_scales.data_ptr(), self.v_scales.data_ptr()
        self._ref = C.byref(self.t)
        self._dev = self.k.get_device()
        if self._dev < 0:
            raise ValueError(f"device {device}: a cache on a GPU is expected")

    def __setattr__(self, name, value):
        if name in self.__dict__:
            raise AttributeError(f"{name}: a cache keeps its buffers and sizes; copy into the buffers")
        super().__setattr__(name, value)

    def buffers(self):
        return self.k, self.v, self.k_scales, self.v_scales


def _heads(t, name, dtype, rows, heads, dim, dev):
    """Raise ValueError unless t is [rows, heads, dim] of the dtype on GPU `dev`, a
    token's heads side by side; returns its address and the tokens' stride."""
    if t.dtype is not dtype or t.shape != (rows, heads, dim) or t.get_device() != dev:
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)} on {t.device}, expected {dtype} {(rows, heads, dim)} on GPU {dev}")
    ld, hs, one = t.stride()
    if (one != 1 or (hs != dim and heads > 1) or (ld < heads * dim and rows > 1)) and rows:
        raise ValueError(f"{name}: strides {t.stride()}; a token's heads side by side, tokens apart from each other, are expected")
    return t.data_ptr(), (ld if rows > 1 else heads * dim)


def kv_append(cache: KVCache, k, v, slots, q=None, q_weight=None, k_weight=None, eps: float = 1e-6, positions=None,
              freqs=None, interleaved: bool = False, q_out=None, stream=None):
    """Keys and values of new tokens into the cache, normalized per head and rotated on
    the way, and the queries the same way (mxmoe_kv_append): returns the queries, a
    new tensor or q_out (which may be q itself), or None without q.

    k, v [tokens, heads, dim], q [tokens, q_heads, dim] in the cache's dtype, tokens of any
    stride (views of a joint projection); slots int32 [tokens], page * page_size + place
    (outside the cache: not kept); q_weight, k_weight [dim] or None for no norm;
    positions int32 [tokens] and freqs float64 [rot / 2], radians a position, or None for no
    rotation.  A slot must not come twice in a call.  32 and more tokens are fastest a sequence to a
    call (a run of slots).  The queries have no autograd graph, also where inputs have one."""
    torch = _torch()
    lib = _lib or load_library()
    dev, dt, kv, dim, i32 = cache._dev, cache.dtype, cache.heads, cache.dim, (torch.int32,)
    if k.dim() != 3:
        raise ValueError(f"k: shape {tuple(k.shape)}, expected [tokens, heads, dim]")
    n = k.shape[0]
    kp, ldk = _heads(k, "k", dt, n, kv, dim, dev)
    vp, ldv = _heads(v, "v", dt, n, kv, dim, dev)
    sp = _dense(slots, "slots", i32, (n,), dev)
    qp, ldq, hq, op, ldo = None, 0, 0, None, 0
    if q is None:
        if q_weight is not None or q_out is not None:
            raise ValueError("q_weight and q_out: there are no queries")
    else:
        if q.dim() != 3 or q.shape[1] == 0:
            raise ValueError(f"q: shape {tuple(q.shape)}, expected [tokens, q_heads, dim]")
        hq = q.shape[1]
        qp, ldq = _heads(q, "q", dt, n, hq, dim, dev)
        ldo = hq * dim
        if q_out is not None:
            op, ldo = _heads(q_out, "q_out", dt, n, hq, dim, dev)
    qw = None if q_weight is None else _dense(q_weight, "q_weight", (dt,), (dim,), dev)
    kw = None if k_weight is None else _dense(k_weight, "k_weight", (dt,), (dim,), dev)
    if (positions is None) != (freqs is None):
        raise ValueError("positions and freqs: a rotation needs both")
    pp = fp = None
    rot = 0
    if freqs is not None:
        rot = 2 * freqs.numel()
        pp = _dense(positions, "positions", i32, (n,), dev)
        fp = _dense(freqs, "freqs", (torch.float64,), (rot // 2,), dev)
        if rot == 0:
            pp = fp = None

    def body(s):
        o, p = q_out, op
        if q is not None and o is None:
            o = torch.empty(n, hq, dim, dtype=dt, device=q.device)
            p = o.data_ptr()
        st = lib.mxmoe_kv_append(cache._ref, n, qp, ldq, hq, kp, ldk, vp, ldv, qw, kw, eps, pp, fp, rot,
                                 1 if interleaved else 0, sp, p, ldo, s)
        if st:
            raise MxmoeError(st, "mxmoe_kv_append")
        return o

    return _run_on(dev, stream, body, stream and (q, k, v, slots, q_weight, k_weight, positions, freqs, q_out, *cache.buffers()))


def kv_read(cache: KVCache, slots, stream=None):
    """Rows of the cache back in its activation dtype (mxmoe_kv_read): (k, v), each [tokens,
    heads, dim]; slots int32 [tokens], zeros for one outside the cache.  Without autograd graph."""
    torch = _torch()
    lib = _lib or load_library()
    dev = cache._dev
    if slots.dim() != 1:
        raise ValueError(f"slots: shape {tuple(slots.shape)}, expected [tokens]")
    n = slots.shape[0]
    sp = _dense(slots, "slots", (torch.int32,), (n,), dev)

    def body(s):
        k = torch.empty(n, cache.heads, cache.dim, dtype=cache.dtype, device=slots.device)
        v = torch.empty_like(k)
        st = lib.mxmoe_kv_read(cache._ref, n, sp, k.data_ptr(), v.data_ptr(), s)
        if st:
            raise MxmoeError(st, "mxmoe_kv_read")
        return k, v

    return _run_on(dev, stream, body, stream and (slots, *cache.buffers()))


def attention_decode(cache: KVCache, q, table, lengths, prefix=None, prefix_len: int = 0, scale: Optional[float] = None,
                     softcap: float = 0.0, out=None, stream=None):
    """Attention of each sequence's last query tokens over its pages of the cache
    (mxmoe_attention_decode): [batch * n_q, q_heads, dim] in the cache's dtype.

    q [batch * n_q, q_heads, dim], sequence by sequence (n_q at most ATTENTION_QUERIES);
    table int32 [batch, width], pages of the positions from prefix_len on; lengths int32
    [batch], all tokens of a sequence (prefix and queries among them), 0 for padding; prefix
    int32 [ceil(prefix_len / page_size)], pages that every sequence begins with.  scale:
    1 / sqrt(dim) by default; softcap > 0 caps the scores.  The result has no autograd graph, also
    where q has one."""
    torch = _torch()
    lib = _lib or load_library()
    dev, dt, dim = cache._dev, cache.dtype, cache.dim
    if q.dim() != 3 or table.dim() != 2:
        raise ValueError(f"q {tuple(q.shape)}, table {tuple(table.shape)}: [batch * n_q, q_heads, dim] and [batch, width] are expected")
    batch, width = table.shape
    rows, hq = q.shape[0], q.shape[1]
    n_q = rows // batch if batch else 1
    if rows != batch * n_q or (batch and n_q == 0):
        raise ValueError(f"q: {rows} tokens for {batch} sequences")
    if max(width, prefix_len) >> 31 > 0:  # (the call would take them modulo 2^32)
        raise MxmoeError(ERR_UNSUPPORTED, f"attention_decode(width {width}, prefix_len {prefix_len})")
    qp, ldq = _heads(q, "q", dt, rows, hq, dim, dev)
    i32 = (torch.int32,)
    tp = _dense(table, "table", i32, (batch, width), dev)
    lp = _dense(lengths, "lengths", i32, (batch,), dev)
    pp = None
    if prefix is None:
        if prefix_len:
            raise ValueError(f"prefix_len {prefix_len} without prefix")
    else:
        pp = _dense(prefix, "prefix", i32, (-(-prefix_len // cache.page_size),), dev)
        pp = pp if prefix_len else None
    op, ldo = (None, hq * dim) if out is None else _heads(out, "out", dt, rows, hq, dim, dev)
    if scale is None:
        scale = dim ** -0.5
    wsb = lib.mxmoe_attention_workspace_bytes(cache._ref, batch, n_q, hq, width, prefix_len)

    def body(s):
        o, p = out, op
        if o is None:
            o = torch.empty(rows, hq, dim, dtype=dt, device=q.device)
            p = o.data_ptr()
        ws = torch.empty(wsb, dtype=torch.uint8, device=q.device) if wsb else None
        st = lib.mxmoe_attention_decode(cache._ref, qp, ldq, batch, n_q, hq, tp if width else None, width, lp, pp,
                                        prefix_len, scale, softcap, p, ldo, ws.data_ptr() if wsb else None, wsb, s)
        if st:
            raise MxmoeError(st, "mxmoe_attention_decode")
        return o

    return _run_on(dev, stream, body, stream and (q, table, lengths, prefix, out, *cache.buffers()))


# --------------------------------------------------------------- routing
def route_permute(topk_ids, E: int, stream=None):
    torch = _torch()
    lib = load_library()
    T, k = topk_ids.shape
    dev = topk_ids.device
    counts = torch.empty(E, dtype=torch.int32, device=dev)
    offsets = torch.empty(E + 1, dtype=torch.int32, device=dev)
    sp = torch.full((max(T * k, 1),), -7, dtype=torch.int32, device=dev)
    inv = torch.empty(max(T * k, 1), dtype=torch.int32, device=dev)
    status = torch.empty(1, dtype=torch.int32, device=dev)
    wsb = lib.mxmoe_route_workspace_bytes(T, k, E)
    ws = empty_aligned(wsb, dev)
    _check(lib.mxmoe_route_permute(_ptr(topk_ids.contiguous()), T, k, E, _ptr(counts), _ptr(offsets), _ptr(sp),
                                   _ptr(inv), _ptr(status), _ptr(ws), wsb, _stream_ptr(stream)),
           "mxmoe_route_permute")
    return {"counts": counts, "offsets": offsets, "sorted_pair": sp[: T * k], "inv": inv[: T * k],
            "status": status}


def router_topk(logits, k: int, renormalize: bool = False, shared_logits=None, stream=None):
    """Router front-end: (ids int32 [T,k], weights fp32 [T,k], shared gates fp32
    [T,n_shared] or None) from fp32 logits [T,E] (and shared-gate logits)."""
    torch = _torch()
    lib = load_library()
    T, E = logits.shape
    ids = torch.empty((T, k), dtype=torch.int32, device=logits.device)
    w = torch.empty((T, k), dtype=torch.float32, device=logits.device)
    n_sh = 0 if shared_logits is None else shared_logits.shape[1]
    shw = None if shared_logits is None else torch.empty((T, n_sh), dtype=torch.float32, device=logits.device)
    _check(lib.mxmoe_router_topk(_ptr(logits), T, E, k, 1 if renormalize else 0, _ptr(shared_logits), n_sh, _ptr(ids),
                                 _ptr(w), _ptr(shw), _stream_ptr(stream)), "mxmoe_router_topk")
    return ids, w, shw


def act_quant(a, act: str, qmax: int, stream=None):
    torch = _torch()
    lib = load_library()
    rows, cols = a.shape
    codes = torch.empty((rows, cols), dtype=torch.int8, device=a.device)
    scales = torch.empty(rows, dtype=torch.float32, device=a.device)
    _check(lib.mxmoe_act_quant(_ptr(a), act_code(act), rows, cols, a.stride(0), qmax, _ptr(codes), _ptr(scales),
                               _stream_ptr(stream)), "mxmoe_act_quant")
    return codes, scales


# --------------------------------------------------------------- block
class MoEBlock:
    """A packed MoE block on one GPU: weights, block table and workspace."""

    def __init__(self, block, device="cuda", T_max: Optional[int] = None, stream=None,
                 packed: Optional[List[List[PackedLinear]]] = None):
        """`packed`: already packed linears per expert (may repeat objects) instead
        of packing block.linears."""
        torch = _torch()
        lib = load_library()
        cfg = block.cfg
        self.cfg = cfg
        self.act = cfg.act
        self.device = device
        self.packed: List[List[PackedLinear]] = [list(ps) for ps in packed] if packed is not None else []
        if packed is None:
            for lins in block.linears:
                self.packed.append([PackedLinear(q, cfg.act, device, stream) for q in lins])
        G = cfg.E + cfg.n_shared
        if len(self.packed) != G:
            raise ValueError(f"{len(self.packed)} packed experts for a block of {G}")
        self._schemes = (Scheme_t * (3 * G))(*[scheme_t(p.q.scheme) for ps in self.packed for p in ps])
        self._ptrs = (C.c_void_p * (3 * G))(*[p.buf.data_ptr() for ps in self.packed for p in ps])
        self.B = Block_t(cfg.H, cfg.F, cfg.E, cfg.k, cfg.n_shared, cfg.F_shared if cfg.n_shared else 0,
                         act_code(cfg.act), C.cast(self._schemes, C.POINTER(Scheme_t)),
                         C.cast(self._ptrs, C.POINTER(C.c_void_p)))
        tb = lib.mxmoe_block_table_bytes(C.byref(self.B))
        if tb == 0:
            raise MxmoeError(ERR_UNSUPPORTED, "mxmoe_block_table_bytes")
        host = (C.c_uint8 * tb)()
        _check(lib.mxmoe_block_table_fill(C.byref(self.B), host, tb), "mxmoe_block_table_fill")
        self.table = torch.frombuffer(bytearray(host), dtype=torch.uint8).to(device)
        self.T_max = T_max or cfg.T
        self.ws_bytes = lib.mxmoe_workspace_bytes(C.byref(self.B), self.T_max)
        self.ws = empty_aligned(self.ws_bytes, device)
        torch.cuda.synchronize()
        for ps in self.packed:
            for p in ps:
                p.release_sources()

    def workspace_layout(self, T: int) -> dict:
        lay = WsLayout_t()
        _check(load_library().mxmoe_workspace_layout(C.byref(self.B), T, C.byref(lay)), "mxmoe_workspace_layout")
        return {f: getattr(lay, f) for f in WS_FIELDS}

    def forward(self, x, topk_ids, topk_w, y=None, expert_mask: Optional[Sequence[int]] = None,
                skip_combine: bool = False, events=None, stream=None, router_logits=None,
                renormalize: bool = False, shared_logits=None, shared_w=None, fp32_slots: bool = False):
        """topk_ids / topk_w may be None when router_logits (fp32 [T,E]) is
        given; the router's choice is then left in the workspace.
        fp32_slots: keep the weighted down rows in fp32 (default: rounded to
        the activation dtype); slot_dtype() says which the last call used."""
        torch = _torch()
        lib = load_library()
        T = x.shape[0]
        if T > self.T_max:
            raise ValueError(f"T={T} exceeds the workspace sized for {self.T_max} tokens")
        if y is None:
            y = torch.empty_like(x)
        opts = None
        self._fp32_slots = bool(fp32_slots)
        if (expert_mask is not None or skip_combine or events is not None or router_logits is not None
                or shared_w is not None or fp32_slots):
            o = ForwardOpts_t()
            o.fp32_slots = 1 if fp32_slots else 0
            o.router_logits = _ptr(router_logits)
            o.renormalize = 1 if renormalize else 0
            o.shared_logits = _ptr(shared_logits)
            o.shared_w = _ptr(shared_w)
            if events is not None:
                o.events = events.array
            if expert_mask is not None:
                self._mask = (C.c_uint8 * len(expert_mask))(*[1 if v else 0 for v in expert_mask])
                o.expert_mask = C.cast(self._mask, C.POINTER(C.c_uint8))
            o.skip_combine = 1 if skip_combine else 0
            opts = C.byref(o)
        st = lib.mxmoe_moe_forward_ex(C.byref(self.B), _ptr(self.table), T, _ptr(x), _ptr(topk_ids), _ptr(topk_w),
                                      _ptr(y), _ptr(self.ws), self.ws_bytes, opts, _stream_ptr(stream))
        _check(st, "mxmoe_moe_forward")
        return y

    def forward_noalloc(self, x, topk_ids, topk_w, y=None, stream=None):
        """The forward through mxmoe_moe_forward_noalloc (the library's own
        scratch array instead of this block's workspace)."""
        torch = _torch()
        lib = load_library()
        if y is None:
            y = torch.empty_like(x)
        st = lib.mxmoe_moe_forward_noalloc(C.byref(self.B), _ptr(self.table), x.shape[0], _ptr(x), _ptr(topk_ids),
                                           _ptr(topk_w), _ptr(y), _stream_ptr(stream))
        _check(st, "mxmoe_moe_forward_noalloc")
        return y

    def slot_dtype(self):
        """torch dtype of the slot rows the last forward wrote."""
        torch = _torch()
        if getattr(self, "_fp32_slots", False):
            return torch.float32
        return torch.bfloat16 if self.act == "bf16" else torch.float16

    def slot_rows(self, T: int):
        """The last forward's weighted down rows [T, k + n_shared, H] as a
        float32 numpy array (exact: a 16-bit slot widens without rounding)."""
        cfg = self.cfg
        n = T * (cfg.k + cfg.n_shared) * cfg.H
        v = self.ws_view("slots", self.slot_dtype(), n, T)
        return v.float().cpu().numpy().reshape(T, cfg.k + cfg.n_shared, cfg.H)

    def ws_view(self, field: str, dtype, count: int, T: int):
        """Typed view of an intermediate buffer inside the workspace (after a forward)."""
        off = self.workspace_layout(T)[field]
        if off == (1 << 64) - 1:
            return None
        torch = _torch()
        nbytes = count * torch.empty((), dtype=dtype).element_size()
        return self.ws[off: off + nbytes].view(dtype)


# --------------------------------------------------------------- HIP events
class PhaseEvents:
    """2 * N_PHASES hipEvents for MoEBlock.forward(events=...), via the HIP runtime."""

    def __init__(self):
        self.hip = C.CDLL("libamdhip64.so")
        self.hip.hipEventCreate.argtypes = [C.POINTER(C.c_void_p)]
        self.hip.hipEventElapsedTime.argtypes = [C.POINTER(C.c_float), C.c_void_p, C.c_void_p]
        self.hip.hipEventSynchronize.argtypes = [C.c_void_p]
        self.hip.hipEventDestroy.argtypes = [C.c_void_p]
        self.array = (C.c_void_p * (2 * N_PHASES))()
        for i in range(2 * N_PHASES):
            ev = C.c_void_p()
            if self.hip.hipEventCreate(C.byref(ev)) != 0:
                raise RuntimeError("hipEventCreate failed")
            self.array[i] = ev
        self.array = C.cast(self.array, C.POINTER(C.c_void_p))

    def elapsed_ms(self):
        """Per-phase durations (ms) of the last forward recorded with these events."""
        out = []
        self.hip.hipEventSynchronize(self.array[2 * N_PHASES - 1])
        for i in range(N_PHASES):
            t = C.c_float()
            if self.hip.hipEventElapsedTime(C.byref(t), self.array[2 * i], self.array[2 * i + 1]) != 0:
                raise RuntimeError("hipEventElapsedTime failed")
            out.append(float(t.value))
        return out

    def span_ms(self):
        """Duration (ms) of the whole last forward recorded with these events."""
        self.hip.hipEventSynchronize(self.array[2 * N_PHASES - 1])
        t = C.c_float()
        if self.hip.hipEventElapsedTime(C.byref(t), self.array[0], self.array[2 * N_PHASES - 1]) != 0:
            raise RuntimeError("hipEventElapsedTime failed")
        return float(t.value)

    def __del__(self):
        try:
            for i in range(2 * N_PHASES):
                self.hip.hipEventDestroy(self.array[i])
        except Exception:
            pass
