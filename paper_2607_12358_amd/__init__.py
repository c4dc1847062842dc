"""ACID-gated video-DiT denoise loop on AMD Instinct MI355X (gfx950).

Python face of libacid: each function marshals torch tensors (device memory)
and the current HIP stream into one C-ABI call.  All arithmetic runs in the
library's HIP kernels; there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import math
import struct
from typing import Iterable, Optional, Sequence

import numpy as np

from . import _lib as _L
from ._lib import (ACID_BF16, ACID_CACHE_APPLY, ACID_CACHE_STORE, ACID_EPI_BIAS,  # noqa: F401
                   ACID_EPI_BIAS_GELU, ACID_EPI_EULER, ACID_EPI_GATE_RESIDUAL, ACID_EPI_QKV,
                   ACID_EPI_QKV_GELU, ACID_BLOCK_PARALLEL, ACID_BLOCK_SEQUENTIAL,
                   ACID_F32, ACID_MODE_ACID, ACID_MODE_DICACHE, ACID_MODE_EASYCACHE,
                   ACID_MODE_NOCACHE, ACID_NORM_LAYER, ACID_NORM_NONE, ACID_NORM_RMS,
                   KERNEL_CLASSES, AcidError,
                   TRACE_DTYPE, check, lib)

__all__ = ["Model", "gate", "GateState", "gate_device_sequence", "cache_apply", "easycache_reuse", "attention", "linear",
           "ln_modulate", "linear_attention", "linear_attention_step", "linear_attention_workspace",
           "linear_w4", "quantize_w4", "w4_shapes", "residual_norm", "q_scale", "version", "AcidError", "KERNEL_CLASSES"]


def _torch():
    import torch
    return torch


def _stream(stream=None) -> int:
    torch = _torch()
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("expected a device tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return C.c_void_p(t.data_ptr())


def version() -> str:
    return lib().acid_version().decode()


def _torch_dtype(code):
    torch = _torch()
    return torch.bfloat16 if code == ACID_BF16 else torch.float32


# ------------------------------------------------------------------ gate


class GateState:
    """Algorithm 1's state (plain data, zero = initial)."""

    def __init__(self):
        self.c = _L.GateStateC()


def gate(state: GateState, tau_low: float, tau_high: float, delta: float, s_t: float,
         n_warmup: int = 1):
    """One step of the host gate. Returns (compute: bool, tau_used: float)."""
    p = _L.GateParamsC(tau_low, tau_high, delta, n_warmup)
    comp = C.c_int32()
    tau = C.c_double()
    check(lib().acid_gate(C.byref(state.c), C.byref(p), float(s_t), C.byref(comp), C.byref(tau)))
    return bool(comp.value), tau.value


def gate_device_sequence(signals, tau_low: float, tau_high: float, delta: float,
                         n_warmup: int = 1, device="cuda", stream=None) -> np.ndarray:
    """Algorithm 1 run by the device gate over a whole signal sequence (NaN
    where a step has no signal); returns the trace (waits for the GPU)."""
    torch = _torch()
    sig = np.ascontiguousarray(signals, dtype=np.float64)
    n = len(sig)
    p = _L.GateParamsC(tau_low, tau_high, delta, n_warmup)
    s_d = torch.from_numpy(sig).to(device)
    tsz = C.sizeof(_L.StepTraceC)
    tr_d = torch.zeros(max(n, 1) * tsz, dtype=torch.uint8, device=device)
    check(lib().acid_gate_device_sequence(C.byref(p), _ptr(s_d), n, _ptr(tr_d),
                                          _stream(stream)))
    raw = tr_d.cpu().numpy()  # waits for the stream
    tr = (_L.StepTraceC * max(n, 1))()
    C.memmove(tr, raw.ctypes.data, max(n, 1) * tsz)
    out = np.zeros(n, dtype=TRACE_DTYPE)
    for i in range(n):
        out[i] = (tr[i].compute, tr[i].gate_compute, tr[i].s, tr[i].sigma_sum_after,
                  tr[i].tau_used)
    return out


# ------------------------------------------------------------ components


def cache_apply(op: int, x, h_out, r, stream=None) -> None:
    n = x.numel()
    if h_out.numel() != n or r.numel() != n:
        raise ValueError("x, h_out and r must have the same number of elements")
    check(lib().acid_cache_apply(op, _ptr(x), _ptr(h_out), _ptr(r), n, _stream(stream)))


def easycache_reuse(x, x_prev, v, offset, dsigma: float, stream=None) -> None:
    """EasyCache's skipped step: v = x + offset; x_prev = x; x += dsigma v."""
    n = x.numel()
    if x_prev.numel() != n or v.numel() != n or offset.numel() != n:
        raise ValueError("x, x_prev, v and offset must have the same number of elements")
    check(lib().acid_easycache_reuse(_ptr(x), _ptr(x_prev), _ptr(v), _ptr(offset), n,
                                     float(dsigma), _stream(stream)))


def ln_modulate(x, shift, scale, out, stream=None) -> None:
    rows, hidden = x.shape
    code = ACID_BF16 if out.dtype == _torch().bfloat16 else ACID_F32
    check(lib().acid_ln_modulate(code, _ptr(x), rows, hidden, _ptr(shift), _ptr(scale),
                                 _ptr(out), _stream(stream)))


def attention(q, k, vt, o, stream=None, q_prescaled: bool = False) -> None:
    """q, k [heads, L, d]; vt [heads, d, vt_ld]; o [L, heads*d]; all bf16 or all fp32.
    q_prescaled: q holds Q * q_scale(d), as the QKV epilogue stores it with
    q_prescale=True (the model's own path)."""
    n_heads, L, d = q.shape
    code = ACID_BF16 if q.dtype == _torch().bfloat16 else ACID_F32
    check(lib().acid_attention(code, n_heads, L, d, _ptr(q), _ptr(k), _ptr(vt), vt.shape[2],
                               _ptr(o), int(bool(q_prescaled)), _stream(stream)))


def q_scale(d: int) -> float:
    """The float32 factor log2(e)/sqrt(d) a pre-scaled Q carries (the
    library's own constant, acid_q_scale)."""
    return float(lib().acid_q_scale(int(d)))


def linear(a, wt, kind: int, bias, gate=None, out=None, v_out=None, q=None, k=None, vt=None,
           n_heads=0, head_dim=0, dsigma=0.0, bias2=None, q_prescale=False,
           stream=None) -> None:
    """Fused GEMM y = a @ wt.T + bias with an epilogue (see include/acid.h).
    For ACID_EPI_QKV_GELU, out may be a row-strided view (unit column
    stride); its row stride is passed as out_ld."""
    M, K = a.shape
    N = wt.shape[0]
    code = ACID_BF16 if a.dtype == _torch().bfloat16 else ACID_F32
    e = _L.EpilogueArgsC()
    e.kind = kind
    e.bias = _ptr(bias)
    e.gate = _ptr(gate)
    e.bias2 = _ptr(bias2)
    if kind == _L.ACID_EPI_QKV_GELU and out is not None:
        if not out.is_cuda or out.stride(-1) != 1:
            raise ValueError("out must be a device tensor with unit column stride")
        e.out = C.c_void_p(out.data_ptr())
        e.out_ld = out.stride(0)
    else:
        e.out = _ptr(out)
    e.v_out = _ptr(v_out)
    e.q, e.k, e.vt = _ptr(q), _ptr(k), _ptr(vt)
    e.vt_ld = vt.shape[-1] if vt is not None else 0
    e.n_heads, e.head_dim, e.dsigma = n_heads, head_dim, dsigma
    e.q_prescale = int(bool(q_prescale))
    check(lib().acid_linear(code, M, N, K, _ptr(a), _ptr(wt), C.byref(e), _stream(stream)))


# ------------------------------------------------ linear-attention block
#
# A call for a few tokens is bound by the host, so tensors are looked at by the
# native module _binding, which calls _at and _rows_at below for those that are
# not as they have to be, and calls the library.


def _dtype_code(torch, t, name: str) -> int:
    dtype = t.dtype
    if dtype is torch.bfloat16:
        return ACID_BF16
    if dtype is torch.float32:
        return ACID_F32
    raise ValueError(f"{name}: expected bfloat16 or float32, got {t.dtype}")


def _device(t, name: str) -> int:
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{name}: expected a tensor on a GPU, got one on {t.device}")
    return dev


def _at(dev, name: str, t, shape: tuple, dtype) -> Optional[int]:
    """Address of t (or None): a contiguous tensor on GPU dev of this shape and type."""
    if t is None:
        return None
    if t.shape == shape and t.dtype is dtype and t.get_device() == dev and t.is_contiguous():
        return t.data_ptr()
    if t.get_device() != dev:
        raise ValueError(f"{name}: expected a tensor on GPU {dev}, got one on {t.device}")
    raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {shape}, "
                     f"got {t.dtype} {tuple(t.shape)} with strides {t.stride()}")


def _rows_at(dev, name: str, t, shape: tuple, dtype):
    """(address, row stride) of a matrix on GPU dev of this shape and type, of unit
    column stride; of one row the stride counts as whole 16 bytes."""
    if t.shape == shape and t.dtype is dtype and t.get_device() == dev:
        rows, cols = shape
        ld, unit = t.stride()
        if unit == 1 or cols == 1:
            if rows <= 1:
                return t.data_ptr(), (cols + 7) // 8 * 8
            if ld >= cols:
                return t.data_ptr(), ld
        raise ValueError(f"{name}: expected unit column stride and rows apart, got strides {t.stride()}")
    if t.get_device() != dev:
        raise ValueError(f"{name}: expected a tensor on GPU {dev}, got one on {t.device}")
    raise ValueError(f"{name}: expected {dtype} of shape {shape}, got {t.dtype} {tuple(t.shape)}")


_bound = None


def _native():
    """torch, and the native module, bound to it and to the library."""
    global _bound
    if _bound is None:
        torch = _torch()
        try:
            from . import _binding as N
        except ImportError as e:
            raise RuntimeError("_binding.so is missing: build it with "
                               "`python -m paper_2607_12358_amd.build`") from e
        N.bind(getattr(torch.Tensor, "__dlpack_c_exchange_api__", None), torch.Tensor, _at, _rows_at,
               ((torch.bfloat16, 4, 16), (torch.float32, 2, 32), (torch.int32, 0, 32), (torch.uint8, 1, 8)),
               {name: C.cast(getattr(lib(), name), C.c_void_p).value for name in _L._SIGS})
        _bound = torch, N, N.at, N.rows_at
    return _bound


def _on(torch, dev, stream, fn, *args) -> None:
    """fn(*args, stream) on GPU `dev`: the stream given, which has to be that
    device's, or its current one."""
    if stream is not None:
        if stream.device.index != dev:
            raise ValueError(f"stream of {stream.device} for tensors on GPU {dev}")
        raw = stream.cuda_stream
    else:
        raw = torch._C._cuda_getCurrentRawStream(dev)
    if dev != torch._C._cuda_getDevice():
        with torch.cuda.device(dev):  # what the null stream means
            status = fn(*args, raw)
    else:
        status = fn(*args, raw)
    if status:
        check(status)


def _scale(d: int) -> float:
    return d ** -0.5 if d else 1.0  # (no heads of 0: the library says so)


def linear_attention_workspace(n_seq: int, n_heads: int, seq_len: int, head_dim: int) -> int:
    """Bytes of workspace that are enough for linear_attention of these sizes."""
    return int(lib().acid_linear_attention_workspace_bytes(n_seq, n_heads, seq_len, head_dim))


def linear_attention(q, k, vt, slopes, o, state_in=None, state_out=None, lengths=None,
                     scale: Optional[float] = None, workspace=None, stream=None) -> None:
    """Causal linear attention, S_t = exp(-slope) S_{t-1} + k_t^T v_t and o_t =
    scale q_t S_t (scale defaults to 1/sqrt(d)).  q, k [n_seq, heads, L, d];
    vt [n_seq, heads, d, vt_ld]; o [n_seq, L, heads*d]; all bf16 or all fp32
    (attention's layouts; without the n_seq axis for one sequence).  slopes
    fp32 [heads]; states fp32 [n_seq, heads, d, d], state_out may be state_in
    (apart, shorter sequences take one launch and no workspace);
    lengths int32 [n_seq]: tokens of each sequence, its later rows of o are
    left as they are.  workspace: uint8 tensor of linear_attention_workspace
    bytes, kept by callers whose calls must not allocate; by default one is
    taken from torch's allocator for the call."""
    torch, N, at, rows_at = _native()
    if q.dim() not in (3, 4):
        raise ValueError("q: expected [heads, L, d] or [n_seq, heads, L, d]")
    code, dev, lead, dt = _dtype_code(torch, q, "q"), _device(q, "q"), tuple(q.shape[:-3]), q.dtype
    n_heads, L, d = q.shape[-3:]
    n_seq = lead[0] if lead else 1
    if vt.dim() != q.dim():
        raise ValueError("vt: expected as many axes as q")
    states, vt_ld = lead + (n_heads, d, d), vt.shape[-1]
    args = (at(dev, "q", q, lead + (n_heads, L, d), dt), at(dev, "k", k, lead + (n_heads, L, d), dt),
            at(dev, "vt", vt, lead + (n_heads, d, vt_ld), dt), vt_ld,
            at(dev, "slopes", slopes, (n_heads,), torch.float32),
            at(dev, "lengths", lengths, (n_seq,), torch.int32),
            at(dev, "state_in", state_in, states, torch.float32),
            at(dev, "state_out", state_out, states, torch.float32),
            _scale(d) if scale is None else scale,
            at(dev, "o", o, lead + (L, n_heads * d), dt))
    if workspace is None:
        in_place = args[6] is not None and args[6] == args[7]
        size = N.linear_attention_workspace_needed(code, n_seq, n_heads, L, d, in_place)
        if size:
            with torch.cuda.stream(stream):  # its memory goes back to that stream's pool
                workspace = torch.empty(size, dtype=torch.uint8, device=dev)
    else:
        size = workspace.numel()
    _on(torch, dev, stream, N.linear_attention, code, n_seq, n_heads, L, d, *args,
        None if workspace is None else at(dev, "workspace", workspace, (size,), torch.uint8), size)


def linear_attention_step(q, k, v, slopes, o, state, state_out=None, slots=None,
                          scale: Optional[float] = None, stream=None) -> None:
    """linear_attention's recurrence, one token a row.  q, k, v, o [rows,
    heads*d], unit column stride (columns of one projection's output will do);
    state fp32 [n_slots, heads, d, d], updated in place unless state_out is
    given; slots int32 [rows]: each row's state (default: its own index), any
    value outside [0, n_slots) marking a padding row that is left alone; rows
    of one slot are successive tokens, in row order (at most 65536 rows)."""
    torch, N, at, rows_at = _native()
    if state.dim() != 4:
        raise ValueError("state: expected [n_slots, heads, d, d]")
    if q.dim() != 2:
        raise ValueError("q: expected [rows, heads*d]")
    code, dev, dt = _dtype_code(torch, q, "q"), _device(state, "state"), q.dtype
    n_slots, n_heads, d = state.shape[:3]
    rows, states = q.shape[0], (n_slots, n_heads, d, d)
    shape = (rows, n_heads * d)
    state_at = at(dev, "state", state, states, torch.float32)
    _on(torch, dev, stream, N.linear_attention_step, code, rows, n_heads, d,
        *rows_at(dev, "q", q, shape, dt), *rows_at(dev, "k", k, shape, dt),
        *rows_at(dev, "v", v, shape, dt), at(dev, "slopes", slopes, (n_heads,), torch.float32),
        at(dev, "slots", slots, (rows,), torch.int32), n_slots, state_at,
        state_at if state_out is None else at(dev, "state_out", state_out, states, torch.float32),
        _scale(d) if scale is None else scale, *rows_at(dev, "o", o, shape, dt))


# acid_residual_norm_args, packed in a quarter of the time its ctypes form takes
_NORM_ARGS = struct.Struct("@PqPqPqPqiiiiPPPPPqff")
_NORMS = {"none": ACID_NORM_NONE, "layer": ACID_NORM_LAYER, "rms": ACID_NORM_RMS}


def residual_norm(h, y=None, h_out=None, out=None, res_scale: float = 1.0, post: str = "none",
                  post_weight=None, gate=None, pre: str = "layer", pre_weight=None, shift=None,
                  scale=None, rows_per_mod: int = 0, eps: float = 1e-6, stream=None) -> None:
    """Between two blocks, in one pass: h_out = res_scale h + gate (N_post(y)
    post_weight), then out = (N_pre(h_out) pre_weight) (1 + scale) + shift.
    h, h_out fp32 [rows, hidden] (h_out defaults to h, in place); y, out bf16
    or fp32, either may be None; norms "none", "layer" or "rms"; weights fp32
    [hidden]; gate, shift, scale fp32 [hidden], or [n_mod, hidden] with row r
    using row r // rows_per_mod.  Matrices may be row-strided."""
    torch, N, at, rows_at = _native()
    f32 = torch.float32
    if post not in _NORMS or pre not in _NORMS:
        raise ValueError(f"unknown norm {post if post not in _NORMS else pre!r}")
    if rows_per_mod < 0:
        raise ValueError("rows_per_mod < 0")
    if h.dim() != 2:
        raise ValueError("h: expected [rows, hidden]")
    if y is None and h_out is not None:
        raise ValueError("h_out without y")
    dev, shape = _device(h, "h"), tuple(h.shape)
    rows, hidden = shape
    n_mod = -(-rows // rows_per_mod) if rows_per_mod else 1
    nothing = (0, 0)

    def vector(name, t):
        one = t is not None and n_mod == 1 and t.dim() == 1
        return at(dev, name, t, (hidden,) if one else (n_mod, hidden), f32) or 0

    h_at = rows_at(dev, "h", h, shape, f32)
    a = _NORM_ARGS.pack(
        *h_at, *(nothing if y is None else rows_at(dev, "y", y, shape, y.dtype)),
        *(h_at if h_out is None else rows_at(dev, "h_out", h_out, shape, f32)),
        *(nothing if out is None else rows_at(dev, "out", out, shape, out.dtype)),
        0 if y is None else _dtype_code(torch, y, "y"), 0 if out is None else _dtype_code(torch, out, "out"),
        _NORMS[post], _NORMS[pre], at(dev, "post_weight", post_weight, (hidden,), f32) or 0,
        at(dev, "pre_weight", pre_weight, (hidden,), f32) or 0, vector("gate", gate),
        vector("shift", shift), vector("scale", scale), rows_per_mod, res_scale, eps)
    _on(torch, dev, stream, N.residual_norm, a, rows, hidden)


def w4_shapes(n: int, k: int, group: int = 128):
    """Shapes of the codes (uint8) and scales (fp32) of an [n outputs, k
    inputs] 4-bit weight; see include/acid.h for what they hold."""
    if n < 1 or k < 128 or k % 128 or group not in (32, 64, 128):
        raise ValueError("n >= 1, k a multiple of 128, group 32, 64 or 128")
    tiles = -(-n // 16)
    return (tiles, k // 128, 64, 16), (tiles, k // group, 16)


def _w4_at(torch, at, x, codes, scales, n: int, k: int):
    """(x's device, group, codes' address, scales' address)."""
    groups = scales.shape[1] if scales.dim() == 3 else 0
    if groups < 1 or k % groups or k % 128 or codes.dim() != 4:
        raise ValueError("codes, scales: see w4_shapes")
    tiles, dev = -(-n // 16), _device(x, "x")
    return (dev, k // groups, at(dev, "codes", codes, (tiles, k // 128, 64, 16), torch.uint8),
            at(dev, "scales", scales, (tiles, groups, 16), torch.float32))


def quantize_w4(w, codes, scales, stream=None) -> None:
    """codes, scales (w4_shapes) of the fp32 weight w [k inputs, n outputs]."""
    torch, N, at, rows_at = _native()
    if w.dim() != 2:
        raise ValueError("w: expected [k, n]")
    k, n = w.shape
    dev, group, c, s = _w4_at(torch, at, w, codes, scales, n, k)
    _on(torch, dev, stream, N.quantize_w4, at(dev, "w", w, (k, n), torch.float32), n, k, group,
        c, s)


def linear_w4(x, codes, scales, out, bias=None, gelu: bool = False, stream=None) -> None:
    """out = act(x w^T + bias) for few rows x [m, k] (bf16 or fp32) and 4-bit
    weights (quantize_w4); out [m, n] bf16 or fp32; bias fp32 [n].  x and out
    may be row-strided."""
    torch, N, at, rows_at = _native()
    if x.dim() != 2 or out.dim() != 2:
        raise ValueError("x and out: expected two axes")
    (m, k), n = x.shape, out.shape[1]
    dev, group, c, s = _w4_at(torch, at, x, codes, scales, n, k)
    _on(torch, dev, stream, N.linear_w4, _dtype_code(torch, x, "x"), m, n, k, group,
        *rows_at(dev, "x", x, (m, k), x.dtype), c, s,
        at(dev, "bias", bias, (n,), torch.float32),
        ACID_EPI_BIAS_GELU if gelu else ACID_EPI_BIAS, _dtype_code(torch, out, "out"),
        *rows_at(dev, "out", out, (m, n), out.dtype))


# ------------------------------------------------------------------ model


class Model:
    """A DiT stack bound to a caller-side (torch) weight arena and workspace."""

    def __init__(self, cfg, max_steps: int = 1, device="cuda"):
        torch = _torch()
        self.cfg = cfg
        self.c = _L.config_c(cfg)
        check(lib().acid_config_check(C.byref(self.c)))
        self.max_steps = max_steps
        wb = lib().acid_weights_bytes(C.byref(self.c))
        kb = lib().acid_workspace_bytes(C.byref(self.c), max_steps)
        self.arena = torch.empty(wb, dtype=torch.uint8, device=device)
        self.workspace = torch.empty(kb, dtype=torch.uint8, device=device)
        h = C.c_void_p()
        check(lib().acid_model_create(C.byref(self.c), _ptr(self.arena), _ptr(self.workspace),
                                      max_steps, C.byref(h)))
        self.h = h
        self.device = device
        self.dtype_code = self.c.dtype

    def __del__(self):
        try:
            if getattr(self, "h", None) and _L._lib is not None:
                _L._lib.acid_model_destroy(self.h)
                self.h = None
        except Exception:
            pass

    # -- weights ----------------------------------------------------------
    def tensor_count(self) -> int:
        return lib().acid_tensor_count(C.byref(self.c))

    def tensor_shape(self, tid: int):
        rank = C.c_int32()
        dims = (C.c_int64 * 2)()
        check(lib().acid_tensor_shape(C.byref(self.c), tid, C.byref(rank), dims))
        return tuple(dims[:rank.value])

    def load_tensor(self, tid: int, src, stream=None) -> None:
        """src: fp32 device tensor of the manifest shape [in, out]."""
        check(lib().acid_model_load_tensor(self.h, tid, _ptr(src), src.numel(), _stream(stream)))

    def load_tensor_host(self, tid: int, src: np.ndarray, stream=None) -> None:
        """src: fp32 host array of the manifest shape [in, out] (staged through
        the workspace; the call waits for the stream)."""
        a = np.ascontiguousarray(src, dtype=np.float32)
        check(lib().acid_model_load_tensor_host(self.h, tid, a.ctypes.data_as(C.c_void_p),
                                                a.size, _stream(stream)))

    def load_weights(self, tensors: Iterable) -> None:
        """tensors: iterable of (id, name, fp32 numpy array) in any order."""
        torch = _torch()
        for tid, _name, arr in tensors:
            src = torch.from_numpy(np.ascontiguousarray(arr, dtype=np.float32)).to(self.device)
            self.load_tensor(tid, src)
            torch.cuda.current_stream().synchronize()
            del src

    # -- the five calls ---------------------------------------------------
    def dit_step(self, x, sigma: float, text=None, v=None, resid=None, stream=None):
        torch = _torch()
        if v is None:
            v = torch.empty_like(x)
        check(lib().acid_dit_step(self.h, _ptr(x), float(sigma), _ptr(text), _ptr(v),
                                  _ptr(resid), _stream(stream)))
        return v

    def drift_signal(self, x, sigma: float, m_prev, m_cur, stream=None) -> float:
        s = C.c_double()
        check(lib().acid_drift_signal(self.h, _ptr(x), float(sigma), _ptr(m_prev), _ptr(m_cur),
                                      C.byref(s), _stream(stream)))
        return s.value

    def set_probe_blocks(self, n_probe: int) -> None:
        """DiCache probe depth (first n_probe blocks run on every step)."""
        check(lib().acid_model_set_probe_blocks(self.h, int(n_probe)))

    def l1_norms(self, a, b=None, c=None, stream=None):
        """(sum |a - b| or sum |a|, sum |c| or 0) in fp64, deterministic."""
        out = (C.c_double * 2)()
        check(lib().acid_l1_norms(self.h, _ptr(a), _ptr(b), _ptr(c), a.numel(), out,
                                  _stream(stream)))
        return out[0], out[1]

    def denoise_loop(self, x, sigmas: Sequence[float], text=None, mode: str = "acid",
                     tau_low: float = 0.05, tau_high: float = 0.2, delta: float = 0.01,
                     n_warmup: Optional[int] = None, forced_schedule=None,
                     stream=None, graph: bool = False,
                     trace: bool = True) -> Optional[np.ndarray]:
        """Runs the loop in place on x; returns the per-step trace.  mode is
        "nocache", "acid" (TeaCache's signal), "easycache" or "dicache"
        (probe depth: set_probe_blocks); n_warmup defaults to 1 (2 for
        "easycache").  graph=True runs the device-gate loop captured as a
        HIP graph (any mode); with trace=False it returns None without
        waiting for the GPU."""
        sig = np.ascontiguousarray(sigmas, dtype=np.float32)
        n = len(sig) - 1
        modes = {"acid": ACID_MODE_ACID, "nocache": ACID_MODE_NOCACHE,
                 "easycache": ACID_MODE_EASYCACHE, "dicache": ACID_MODE_DICACHE}
        if mode not in modes:
            raise ValueError(f"unknown mode {mode!r}")
        modec = modes[mode]
        if n_warmup is None:
            n_warmup = 2 if mode == "easycache" else 1
        p = _L.GateParamsC(tau_low, tau_high, delta, n_warmup)
        tr = (_L.StepTraceC * n)()
        forced = None
        if forced_schedule is not None:
            fs = np.ascontiguousarray(forced_schedule, dtype=np.uint8)
            forced = fs.ctypes.data_as(C.POINTER(C.c_uint8))
        fn = lib().acid_denoise_loop_graph if graph else lib().acid_denoise_loop
        check(fn(self.h, _ptr(x), sig.ctypes.data_as(C.POINTER(C.c_float)), n, _ptr(text),
                 modec, C.byref(p), forced, tr if trace else None, _stream(stream)))
        if not trace:
            return None
        out = np.zeros(n, dtype=TRACE_DTYPE)
        for i in range(n):
            out[i] = (tr[i].compute, tr[i].gate_compute, tr[i].s, tr[i].sigma_sum_after,
                      tr[i].tau_used)
        return out

    # -- components --------------------------------------------------------
    def timestep_modulation(self, sigmas, stream=None):
        torch = _torch()
        sig = np.ascontiguousarray(sigmas, dtype=np.float32)
        H, nb = self.cfg.hidden, self.cfg.n_blocks
        table = torch.empty((len(sig), 6 * nb + 2, H), dtype=torch.float32, device=self.device)
        check(lib().acid_timestep_modulation(self.h, sig.ctypes.data_as(C.POINTER(C.c_float)),
                                             len(sig), _ptr(table), _stream(stream)))
        return table

    def block_forward(self, block: int, mod6, h, stream=None) -> None:
        check(lib().acid_block_forward(self.h, block, _ptr(mod6), _ptr(h), _stream(stream)))

    # -- timing ------------------------------------------------------------
    def set_timing(self, enable: bool) -> None:
        check(lib().acid_model_set_timing(self.h, int(enable)))

    def reset_timing(self) -> None:
        check(lib().acid_model_reset_timing(self.h))

    def timing(self) -> dict:
        out = {}
        for i, name in enumerate(KERNEL_CLASSES):
            ms = C.c_double()
            n = C.c_int64()
            check(lib().acid_model_timing(self.h, i, C.byref(ms), C.byref(n)))
            out[name] = (ms.value, n.value)
        return out
