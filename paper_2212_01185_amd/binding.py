"""Thin ctypes binding over libpcc's C ABI (include/pcc.h): argument marshalling only.

PyTorch supplies device memory (``tensor.data_ptr()``) and the HIP stream
(``torch.cuda.current_stream().cuda_stream``); every step of the coding path
runs inside the library's kernels.  There is no fallback: if the shared object
has not been built, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# PCC_LIBRARY: another build of the same library, e.g. the measurement build with per-phase cycle counters
# (python -m paper_2212_01185_amd.build --out PATH -DPCC_PHASE_TIMING)
LIB_PATH = os.environ.get("PCC_LIBRARY") or os.path.join(_HERE, "libpcc.so")

PCC_OK = 0
PCC_E_ARG, PCC_E_BLOB, PCC_E_CAP, PCC_E_STREAM, PCC_E_HIP, PCC_E_INTERNAL, PCC_E_UNIMPL, PCC_E_SCRATCH = -1, -2, -3, -4, -5, -6, -7, -8
HEAD_OUTPUTS = 60          # of the 30-160-160-128-60 network; a Codec knows its own (head_outputs)

EXPORTS = (
    "pcc_create", "pcc_destroy", "pcc_stream_bound", "pcc_wavefront_steps", "pcc_model_info", "pcc_encode_probs", "pcc_encode",
    "pcc_decode", "pcc_decode_static", "pcc_decode_static_scratch_bytes", "pcc_cdf_tables", "pcc_copy_intervals", "pcc_set_profiling", "pcc_last_timings", "pcc_strerror",
    "pcc_contexts", "pcc_grouped_linear", "pcc_grouped_linear_grad_workspace_bytes", "pcc_grouped_linear_grad", "pcc_mixture_loss",
    "pcc_adamw_create", "pcc_adamw_destroy", "pcc_adamw_step",
    "pcc_layer_norm", "pcc_layer_norm_grad_workspace_bytes", "pcc_layer_norm_grad", "pcc_route", "pcc_route_grad",
    "pcc_expert_sort_workspace_bytes", "pcc_expert_sort", "pcc_expert_rows", "pcc_expert_join", "pcc_expert_join_grad", "pcc_dropout",
)
PCC_BF16, PCC_FP16, PCC_FP32 = 0, 1, 2
PCC_ACT_RELU, PCC_ACT_LEAKY, PCC_ACT_NONE = 0, 1, 2
PCC_MAX_EXPERTS, PCC_MAX_CHOICES = 1024, 16
STATE_BLOCK = 256          # elements of an 8-bit optimizer state that share a scale
TIMING_NAMES = ("encode_pixels", "encode_rans", "encode_scan", "encode_compact", "decode")

class _AdamwTensor(C.Structure):
    _fields_ = [(name, C.c_void_p) for name in ("d_param", "d_grad", "d_copy", "d_m", "d_v", "d_m_scale", "d_v_scale")] + [("n", C.c_size_t)]


class _AdamwHyper(C.Structure):
    _fields_ = [(name, C.c_double) for name in ("lr", "beta1", "beta2", "eps", "weight_decay")] + [("d_lr", C.c_void_p)]


_lib = None


def load():
    """Open libpcc.so (building it if no built library is present)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        from . import build as _build
        _build.build()
    L = C.CDLL(LIB_PATH)
    vp, sz, i32 = C.c_void_p, C.c_size_t, C.c_int
    L.pcc_create.argtypes = [C.POINTER(vp), vp, sz, i32]
    L.pcc_create.restype = i32
    L.pcc_destroy.argtypes = [vp]
    L.pcc_destroy.restype = None
    L.pcc_stream_bound.argtypes = [i32, i32, i32]
    L.pcc_stream_bound.restype = sz
    L.pcc_wavefront_steps.argtypes = [i32, i32, i32]
    L.pcc_wavefront_steps.restype = C.c_long
    L.pcc_model_info.argtypes = [vp, vp]
    L.pcc_model_info.restype = i32
    L.pcc_encode_probs.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp]
    L.pcc_encode_probs.restype = i32
    L.pcc_encode.argtypes = [vp, vp, i32, i32, i32, vp, sz, C.POINTER(sz), vp]
    L.pcc_encode.restype = i32
    L.pcc_decode.argtypes = [vp, vp, sz, i32, i32, i32, vp, vp]
    L.pcc_decode.restype = i32
    L.pcc_decode_static.argtypes = [vp, vp, sz, i32, i32, i32, vp, vp]
    L.pcc_decode_static.restype = i32
    L.pcc_decode_static_scratch_bytes.argtypes = [i32, i32, i32]
    L.pcc_decode_static_scratch_bytes.restype = sz
    L.pcc_cdf_tables.argtypes = [vp, vp, vp, sz, vp, vp]
    L.pcc_cdf_tables.restype = i32
    L.pcc_copy_intervals.argtypes = [vp, vp, sz, vp]
    L.pcc_copy_intervals.restype = i32
    L.pcc_set_profiling.argtypes = [vp, i32]
    L.pcc_set_profiling.restype = i32
    L.pcc_last_timings.argtypes = [vp, vp]
    L.pcc_last_timings.restype = i32
    L.pcc_contexts.argtypes = [vp, i32, i32, i32, i32, i32, vp, i32, sz, vp]
    L.pcc_contexts.restype = i32
    L.pcc_grouped_linear.argtypes = [vp, sz, vp, vp, vp, i32, sz, i32, i32, i32, i32, vp, i32, sz, vp]
    L.pcc_grouped_linear.restype = i32
    L.pcc_grouped_linear_grad_workspace_bytes.argtypes = [sz, i32, i32, i32]
    L.pcc_grouped_linear_grad_workspace_bytes.restype = sz
    L.pcc_grouped_linear_grad.argtypes = [vp, sz, vp, sz, vp, vp, i32, sz, i32, i32, i32, i32, vp, sz, vp, vp, vp, sz, vp]
    L.pcc_grouped_linear_grad.restype = i32
    L.pcc_mixture_loss.argtypes = [vp, sz, vp, vp, sz, i32, i32, C.c_float, vp, vp, i32, sz, vp]
    L.pcc_mixture_loss.restype = i32
    L.pcc_adamw_create.argtypes = [C.POINTER(vp), C.POINTER(_AdamwTensor), i32, i32, i32, i32, i32]
    L.pcc_adamw_create.restype = i32
    L.pcc_adamw_destroy.argtypes = [vp]
    L.pcc_adamw_destroy.restype = None
    L.pcc_adamw_step.argtypes = [vp, C.POINTER(_AdamwHyper), vp, vp]
    L.pcc_adamw_step.restype = i32
    L.pcc_layer_norm.argtypes = [vp, sz, vp, vp, vp, i32, sz, i32, C.c_float, i32, vp, i32, sz, vp, vp]
    L.pcc_layer_norm.restype = i32
    L.pcc_layer_norm_grad_workspace_bytes.argtypes = [sz, i32, i32]
    L.pcc_layer_norm_grad_workspace_bytes.restype = sz
    L.pcc_layer_norm_grad.argtypes = [vp, i32, sz, vp, sz, vp, vp, vp, i32, sz, i32, i32, vp, sz, vp, vp, vp, sz, vp]
    L.pcc_layer_norm_grad.restype = i32
    L.pcc_route.argtypes = [vp, sz, sz, i32, i32, i32, i32, vp, vp, vp]
    L.pcc_route.restype = i32
    L.pcc_route_grad.argtypes = [vp, vp, sz, vp, vp, sz, i32, i32, i32, i32, vp, sz, vp]
    L.pcc_route_grad.restype = i32
    L.pcc_expert_sort_workspace_bytes.argtypes = [sz, i32, i32]
    L.pcc_expert_sort_workspace_bytes.restype = sz
    L.pcc_expert_sort.argtypes = [vp, sz, i32, i32, vp, vp, vp, sz, vp]
    L.pcc_expert_sort.restype = i32
    L.pcc_expert_rows.argtypes = [vp, sz, vp, sz, i32, sz, i32, i32, vp, sz, vp]
    L.pcc_expert_rows.restype = i32
    L.pcc_expert_join.argtypes = [vp, sz, vp, vp, sz, i32, sz, i32, i32, vp, i32, sz, vp]
    L.pcc_expert_join.restype = i32
    L.pcc_expert_join_grad.argtypes = [vp, i32, sz, vp, sz, vp, vp, sz, i32, sz, i32, i32, vp, sz, vp, vp]
    L.pcc_expert_join_grad.restype = i32
    L.pcc_dropout.argtypes = [vp, sz, vp, sz, sz, i32, i32, C.c_double, C.c_uint64, vp, vp, i32, sz, vp]
    L.pcc_dropout.restype = i32
    L.pcc_strerror.argtypes = [i32]
    L.pcc_strerror.restype = C.c_char_p
    _lib = L
    return L


class PccError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__("%s: %s (%d)" % (what, pcc_strerror(code), code))
        self.code = code


def pcc_strerror(code: int) -> str:
    return load().pcc_strerror(code).decode()


def pcc_stream_bound(n: int, h: int, w: int) -> int:
    return int(load().pcc_stream_bound(n, h, w))


def pcc_wavefront_steps(h: int, w: int, delay: int = 2) -> int:
    return int(load().pcc_wavefront_steps(h, w, delay))


def _stream_handle():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check_img(img: torch.Tensor):
    if img.dtype != torch.uint8 or img.dim() != 4 or img.shape[3] != 3 or not img.is_cuda or not img.is_contiguous():
        raise ValueError("image must be a contiguous CUDA uint8 tensor [n, H, W, 3]")
    return int(img.shape[0]), int(img.shape[1]), int(img.shape[2])


class Codec:
    """Owns one pcc_ctx.  Methods mirror the C entry points one to one."""

    def __init__(self, blob: bytes, device: int = 0):
        self._h = C.c_void_p()
        self.device = device
        buf = C.create_string_buffer(blob, len(blob))
        rc = load().pcc_create(C.byref(self._h), buf, len(blob), device)
        if rc != PCC_OK:
            self._h = C.c_void_p()
            raise PccError(rc, "pcc_create")
        info = self.pcc_model_info()
        self.head_outputs, self.k, self.nbhd, self.delay, self.dist, self.n_layers = info

    def pcc_model_info(self):
        """(head outputs, K, neighbourhood size, delay, distribution id, layers) of the loaded network."""
        arr = (C.c_int * 6)()
        rc = load().pcc_model_info(self._h, arr)
        if rc != PCC_OK:
            raise PccError(rc, "pcc_model_info")
        return tuple(int(v) for v in arr)

    def close(self):
        if self._h and self._h.value:
            load().pcc_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def pcc_encode_probs(self, img: torch.Tensor, want_bits: bool = True):
        n, h, w = _check_img(img)
        params = torch.empty((n, h, w, self.head_outputs), dtype=torch.float32, device=img.device)
        bits = torch.empty((n, h, w), dtype=torch.float32, device=img.device) if want_bits else None
        rc = load().pcc_encode_probs(self._h, img.data_ptr(), n, h, w, params.data_ptr(),
                                     bits.data_ptr() if want_bits else None, _stream_handle())
        if rc != PCC_OK:
            raise PccError(rc, "pcc_encode_probs")
        return params, bits

    def pcc_encode(self, img: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
        """Returns the stream as a uint8 CUDA tensor view of exactly the written size."""
        n, h, w = _check_img(img)
        if out is None:
            out = torch.empty(pcc_stream_bound(n, h, w), dtype=torch.uint8, device=img.device)
        nbytes = C.c_size_t(0)
        rc = load().pcc_encode(self._h, img.data_ptr(), n, h, w, out.data_ptr(), out.numel(), C.byref(nbytes),
                               _stream_handle())
        if rc != PCC_OK:
            raise PccError(rc, "pcc_encode")
        return out[:nbytes.value]

    def pcc_decode(self, stream: torch.Tensor, n: int, h: int, w: int, out: torch.Tensor | None = None) -> torch.Tensor:
        if stream.dtype != torch.uint8 or not stream.is_cuda or not stream.is_contiguous():
            raise ValueError("stream must be a contiguous CUDA uint8 tensor")
        if out is None:
            out = torch.empty((n, h, w, 3), dtype=torch.uint8, device=stream.device)
        rc = load().pcc_decode(self._h, stream.data_ptr(), stream.numel(), n, h, w, out.data_ptr(), _stream_handle())
        if rc != PCC_OK:
            raise PccError(rc, "pcc_decode")
        return out

    def pcc_decode_static(self, stream: torch.Tensor, n: int, h: int, w: int, out: torch.Tensor) -> torch.Tensor:
        """pcc_decode with the mailbox in the library's static device array: allocates nothing (``out`` is required)."""
        if stream.dtype != torch.uint8 or not stream.is_cuda or not stream.is_contiguous():
            raise ValueError("stream must be a contiguous CUDA uint8 tensor")
        rc = load().pcc_decode_static(self._h, stream.data_ptr(), stream.numel(), n, h, w, out.data_ptr(), _stream_handle())
        if rc != PCC_OK:
            raise PccError(rc, "pcc_decode_static")
        return out

    def pcc_cdf_tables(self, params: torch.Tensor, rg: torch.Tensor) -> torch.Tensor:
        """params float32 [count, 12 K], rg uint8 [count, 2] -> uint32-valued int32 tensor [count, 3, 257]."""
        count = int(params.shape[0])
        assert params.dtype == torch.float32 and params.is_cuda and params.is_contiguous()
        assert params.shape[1] == self.head_outputs
        assert rg.dtype == torch.uint8 and rg.is_cuda and rg.is_contiguous() and tuple(rg.shape) == (count, 2)
        cq = torch.empty((count, 3, 257), dtype=torch.int32, device=params.device)
        rc = load().pcc_cdf_tables(self._h, params.data_ptr(), rg.data_ptr(), count, cq.data_ptr(), _stream_handle())
        if rc != PCC_OK:
            raise PccError(rc, "pcc_cdf_tables")
        return cq

    def pcc_set_profiling(self, enabled: bool) -> None:
        rc = load().pcc_set_profiling(self._h, 1 if enabled else 0)
        if rc != PCC_OK:
            raise PccError(rc, "pcc_set_profiling")

    def pcc_last_timings(self) -> dict:
        """Milliseconds per kernel of the last pcc_encode / pcc_decode (profiling must be on)."""
        arr = (C.c_float * len(TIMING_NAMES))()
        rc = load().pcc_last_timings(self._h, arr)
        if rc != PCC_OK:
            raise PccError(rc, "pcc_last_timings")
        return dict(zip(TIMING_NAMES, (float(v) for v in arr)))

    def pcc_copy_intervals(self, n: int, h: int, w: int, device=None) -> torch.Tensor:
        """(start | (freq-1) << 16) of every sub-pixel of the last pcc_encode: int32 tensor [n, H, W, 3]."""
        out = torch.empty((n, h, w, 3), dtype=torch.int32, device=device or ("cuda:%d" % self.device))
        rc = load().pcc_copy_intervals(self._h, out.data_ptr(), out.numel(), _stream_handle())
        if rc != PCC_OK:
            raise PccError(rc, "pcc_copy_intervals")
        return out


# ---- The operators of a training step ----
# Free functions: they launch on the current stream of their tensors' device.  Rows of tensors may be views with a longer stride.
# Autograd does not record them: tensors that require gradients are refused unless it is off.

_TYPES = {torch.bfloat16: PCC_BF16, torch.float16: PCC_FP16, torch.float32: PCC_FP32}


def _check(what: str, t, dtypes, shape, device=None, rows: bool = False):
    """A tensor argument: of one of `dtypes`, of `shape` (None: any size), on a GPU (`device`), contiguous or with `rows` a matrix
    whose rows are.  Returns the distance of its rows."""
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes or not _has_shape(t.shape, shape):
        raise ValueError("%s must be a tensor %s of %s" % (what, list("?" if s is None else s for s in shape), " or ".join(str(d) for d in dtypes)))
    if not t.is_cuda or (device is not None and t.device != device):
        raise ValueError("%s must be on %s" % (what, device or "a GPU"))
    if t.is_contiguous():
        return shape[1] or t.shape[1] if rows else 0
    if not rows:
        raise ValueError("%s must be contiguous" % what)
    n, width = t.shape
    apart, step = t.stride()
    if (width > 1 and step != 1) or (n > 1 and apart < width):
        raise ValueError("%s must have contiguous rows that do not overlap" % what)
    return apart if n > 1 else width


def _has_shape(have, shape) -> bool:
    if have == shape:
        return True
    if len(have) != len(shape):
        return False
    for n, s in zip(have, shape):
        if s is not None and s != n:
            return False
    return True


# The current stream's handle without an object around it, which took 2 of the 11 us of a small call.
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else lambda i: torch.cuda.current_stream(i).cuda_stream


def _call(what: str, device, *args) -> None:
    index = device.index
    call = getattr(_lib or load(), what)
    if torch.cuda.current_device() == index:
        rc = call(*args, _raw_stream(index))
    else:
        with torch.cuda.device(device):
            rc = call(*args, _raw_stream(index))
    if rc != PCC_OK:
        raise PccError(rc, what)


def _unrecorded(*tensors) -> None:
    """Refuses tensors whose gradients autograd is asked for: the operators' backward passes are calls of their own."""
    for t in tensors:
        if getattr(t, "requires_grad", False) and torch.is_grad_enabled():
            raise ValueError("autograd does not record these operators: call them under torch.no_grad() or on detached tensors")


def _ptr(t):
    return t.data_ptr() if t is not None else None


def pcc_contexts(img: torch.Tensor, nbhd: int = 10, delay: int = 2, width: int | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """Network inputs of all pixels of uint8 images [n, H, W, 3] as rows, bf16 [n H W, width]: 3 * nbhd values, then zeros.
    `width` is a multiple of eight by default, which the products read fastest."""
    n, h, w = _check_img(img)
    if out is not None:
        width = out.shape[1] if width is None and out.dim() == 2 else width
    elif width is None:
        width = -(-3 * nbhd // 8) * 8
    if out is None:
        out = torch.empty((n * h * w, width), dtype=torch.bfloat16, device=img.device)
    ld = _check("out", out, (torch.bfloat16,), (n * h * w, width), img.device, rows=True)
    _call("pcc_contexts", img.device, img.data_ptr(), n, h, w, nbhd, delay, out.data_ptr(), width, ld)
    return out


def _check_groups(x, w, offsets):
    ld = _check("x", x, (torch.bfloat16, torch.float16), (None, None), rows=True)
    _check("w", w, (x.dtype,), (None, None, x.shape[1]), x.device)
    groups, out = int(w.shape[0]), int(w.shape[1])
    _check("offsets", offsets, (torch.int64,), (groups + 1,), x.device)
    return ld, groups, out


def pcc_grouped_linear(x: torch.Tensor, w: torch.Tensor, bias: torch.Tensor | None, offsets: torch.Tensor, act: int = PCC_ACT_NONE,
                       out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None) -> torch.Tensor:
    """act(x_i w_g^T + bias_g) for rows offsets[g] <= i < offsets[g + 1] of each group g.  x [rows, in] and w [groups, out, in]
    bf16 or fp16, bias [groups, out] fp32, offsets [groups + 1] int64; the result has x's type or fp32.  Rows of no group are left
    as they are in `out`, and undefined in a new tensor."""
    _unrecorded(x, w, bias, out)
    ldx, groups, n_out = _check_groups(x, w, offsets)
    if bias is not None:
        _check("bias", bias, (torch.float32,), (groups, n_out), x.device)
    if out is None:
        out = torch.empty((x.shape[0], n_out), dtype=out_dtype or x.dtype, device=x.device)
    ldy = _check("out", out, (x.dtype, torch.float32) if out_dtype is None else (out_dtype,), (x.shape[0], n_out), x.device, rows=True)
    _call("pcc_grouped_linear", x.device, x.data_ptr(), ldx, w.data_ptr(), _ptr(bias), offsets.data_ptr(), groups, x.shape[0], x.shape[1],
          n_out, _TYPES[x.dtype], act, out.data_ptr(), _TYPES[out.dtype], ldy)
    return out


def pcc_grouped_linear_grad(dz: torch.Tensor, x: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor, x_act: int = PCC_ACT_NONE,
                            dx: torch.Tensor | None = None, want_dx: bool = True, dw: torch.Tensor | None = None,
                            db: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """(dx, dw, db) of pcc_grouped_linear.  dz [rows, out] is the gradient before the layer's activation; x_act the activation that
    made x: dx is the gradient before that one, the dz of the layer in front (None without want_dx).  dw [groups, out, in] and
    db [groups, out] are fp32.  Rows of no group are left as they are in `dx`, and undefined in a new tensor."""
    _unrecorded(dz, x, w, dx, dw, db)
    ldx, groups, n_out = _check_groups(x, w, offsets)
    rows, n_in = int(x.shape[0]), int(x.shape[1])
    lddz = _check("dz", dz, (x.dtype,), (rows, n_out), x.device, rows=True)
    if want_dx and dx is None:
        dx = torch.empty((rows, n_in), dtype=x.dtype, device=x.device)
    lddx = _check("dx", dx, (x.dtype,), (rows, n_in), x.device, rows=True) if want_dx else n_in
    dw = torch.empty(w.shape, dtype=torch.float32, device=x.device) if dw is None else dw
    db = torch.empty((groups, n_out), dtype=torch.float32, device=x.device) if db is None else db
    _check("dw", dw, (torch.float32,), tuple(w.shape), x.device)
    _check("db", db, (torch.float32,), (groups, n_out), x.device)
    if workspace is None:
        need = int((_lib or load()).pcc_grouped_linear_grad_workspace_bytes(rows, groups, n_in, n_out))
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    else:
        _check("workspace", workspace, (torch.uint8,), (None,), x.device)
    _call("pcc_grouped_linear_grad", x.device, dz.data_ptr(), lddz, x.data_ptr(), ldx, w.data_ptr(), offsets.data_ptr(), groups, rows, n_in,
          n_out, _TYPES[x.dtype], x_act, dx.data_ptr() if want_dx else None, lddx, dw.data_ptr(), db.data_ptr(),
          workspace.data_ptr(), workspace.numel())
    return (dx if want_dx else None), dw, db


def pcc_mixture_loss(params: torch.Tensor, rgb: torch.Tensor, dist: int = 0, scale: float = 1.0, weight: torch.Tensor | None = None,
                     want_grad: bool = True, grad_dtype: torch.dtype = torch.float32, grad: torch.Tensor | None = None):
    """(bits [count], gradient [count, 12 K]) of pixels rgb uint8 [count, 3] under head outputs params fp32 [count, 12 K]: the code
    length of Eq. (5) with the coder's one count for every level, and scale * weight times its gradient.  Pixels of weight 0 have 0."""
    _unrecorded(params, weight, grad)
    ldp = _check("params", params, (torch.float32,), (None, None), rows=True)
    count, outputs = int(params.shape[0]), int(params.shape[1])
    _check("rgb", rgb, (torch.uint8,), (count, 3), params.device)
    if weight is not None:
        _check("weight", weight, (torch.float32,), (count,), params.device)
    if outputs % 12:
        raise ValueError("params must have 12 K columns")
    bits = torch.empty(count, dtype=torch.float32, device=params.device)
    ldg = outputs
    if want_grad:
        if grad is None:
            grad = torch.empty((count, outputs), dtype=grad_dtype, device=params.device)
        ldg = _check("grad", grad, tuple(_TYPES), (count, outputs), params.device, rows=True)
    _call("pcc_mixture_loss", params.device, params.data_ptr(), ldp, rgb.data_ptr(), _ptr(weight), count, outputs // 12, dist, scale,
          bits.data_ptr(), grad.data_ptr() if want_grad else None, _TYPES[grad.dtype] if want_grad else PCC_FP32, ldg)
    return bits, (grad if want_grad else None)


# Layers round the grouped products.

_ANY = tuple(_TYPES)


def _made_or_checked(what: str, t, dtype, shape, device):
    """A contiguous result: a new tensor, or the one that was given."""
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _check(what, t, (dtype,), shape, device)
    return t


def _norm_groups(x, gamma, offsets):
    """(distance of x's rows, groups) of a layer norm; gamma and offsets may be None."""
    ldx = _check("x", x, _ANY, (None, None), rows=True)
    if offsets is not None:
        _check("offsets", offsets, (torch.int64,), (None,), x.device)
        groups = int(offsets.shape[0]) - 1
    else:
        groups = 1
    if gamma is not None:
        _check("gamma", gamma, (torch.float32,), (groups, int(x.shape[1])), x.device)
    return ldx, groups


def pcc_layer_norm(x: torch.Tensor, gamma: torch.Tensor | None = None, beta: torch.Tensor | None = None, offsets: torch.Tensor | None = None,
                   eps: float = 1e-5, out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None, stats: torch.Tensor | None = None,
                   want_stats: bool = True):
    """(y, stats) of the layer norm of the rows x [rows, features]; gamma, beta fp32 [groups, features] (None: 1 and 0), rows offsets[g] <= i <
    offsets[g + 1] have the g-th (offsets None: one group of all rows).  y has x's type, or a 16-bit one where x is fp32; stats fp32 [rows, 2], for
    the backward pass, are None without want_stats.  Rows of no group are left as they are in `out` and `stats`, and undefined in new tensors."""
    _unrecorded(x, gamma, beta, out, stats)
    ldx, groups = _norm_groups(x, gamma, offsets)
    rows, features = int(x.shape[0]), int(x.shape[1])
    if beta is not None:
        _check("beta", beta, (torch.float32,), (groups, features), x.device)
    ldy = features
    if out is None:
        out = torch.empty((rows, features), dtype=out_dtype or x.dtype, device=x.device)
    else:
        ldy = _check("out", out, (_ANY if x.dtype == torch.float32 else (x.dtype,)) if out_dtype is None else (out_dtype,), (rows, features), x.device,
                     rows=True)
    if stats is not None:
        _check("stats", stats, (torch.float32,), (rows, 2), x.device)
    elif want_stats:
        stats = torch.empty((rows, 2), dtype=torch.float32, device=x.device)
    _call("pcc_layer_norm", x.device, x.data_ptr(), ldx, _ptr(gamma), _ptr(beta), _ptr(offsets), groups, rows, features, eps, _TYPES[x.dtype],
          out.data_ptr(), _TYPES.get(out.dtype, -1), ldy, _ptr(stats))
    return out, stats


def pcc_layer_norm_grad(dy: torch.Tensor, x: torch.Tensor, stats: torch.Tensor, gamma: torch.Tensor | None = None, offsets: torch.Tensor | None = None,
                        dx: torch.Tensor | None = None, want_dx: bool = True, want_weights: bool = True, dgamma: torch.Tensor | None = None,
                        dbeta: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """(dx, dgamma, dbeta) of pcc_layer_norm: dx has x's type (None without want_dx), dgamma and dbeta fp32 [groups, features] (None without
    want_weights).  dy has y's type.  Rows of no group are left as they are in `dx`, and undefined in a new tensor."""
    _unrecorded(dy, x, stats, gamma, dx, dgamma, dbeta)
    ldx, groups = _norm_groups(x, gamma, offsets)
    rows, features = int(x.shape[0]), int(x.shape[1])
    lddy = _check("dy", dy, _ANY if x.dtype == torch.float32 else (x.dtype,), (rows, features), x.device, rows=True)
    _check("stats", stats, (torch.float32,), (rows, 2), x.device)
    lddx = features
    if want_dx and dx is None:
        dx = torch.empty((rows, features), dtype=x.dtype, device=x.device)
    elif want_dx:
        lddx = _check("dx", dx, (x.dtype,), (rows, features), x.device, rows=True)
    if want_weights:
        dgamma = _made_or_checked("dgamma", dgamma, torch.float32, (groups, features), x.device)
        dbeta = _made_or_checked("dbeta", dbeta, torch.float32, (groups, features), x.device)
        if workspace is None:
            need = int((_lib or load()).pcc_layer_norm_grad_workspace_bytes(rows, groups, features))
            workspace = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
        else:
            _check("workspace", workspace, (torch.uint8,), (None,), x.device)
    else:
        dgamma = dbeta = workspace = None
    _call("pcc_layer_norm_grad", x.device, dy.data_ptr(), _TYPES[dy.dtype], lddy, x.data_ptr(), ldx, stats.data_ptr(), _ptr(gamma), _ptr(offsets), groups,
          rows, features, _TYPES[x.dtype], dx.data_ptr() if want_dx else None, lddx, _ptr(dgamma), _ptr(dbeta), _ptr(workspace),
          workspace.numel() if workspace is not None else 0)
    return (dx if want_dx else None), dgamma, dbeta


def pcc_route(logits: torch.Tensor, k: int, over_all: bool = False, expert: torch.Tensor | None = None, weight: torch.Tensor | None = None):
    """(expert int32 [tokens, k], weight fp32 [tokens, k]): the experts with the k largest logits [tokens, experts] of each token, the largest first, and
    the softmax over them, or with over_all their part of the softmax over all.  A logit of -inf is never chosen: the choice is -1 then, its weight 0."""
    _unrecorded(logits, weight)
    ldl = _check("logits", logits, _ANY, (None, None), rows=True)
    if not 0 < k <= PCC_MAX_CHOICES:                # before results of k columns are made
        raise PccError(PCC_E_ARG, "pcc_route")
    tokens, experts = int(logits.shape[0]), int(logits.shape[1])
    expert = _made_or_checked("expert", expert, torch.int32, (tokens, k), logits.device)
    weight = _made_or_checked("weight", weight, torch.float32, (tokens, k), logits.device)
    _call("pcc_route", logits.device, logits.data_ptr(), ldl, tokens, experts, k, _TYPES[logits.dtype], int(over_all), expert.data_ptr(), weight.data_ptr())
    return expert, weight


def pcc_route_grad(dweight: torch.Tensor, logits: torch.Tensor, expert: torch.Tensor, weight: torch.Tensor, over_all: bool = False,
                   dlogits: torch.Tensor | None = None) -> torch.Tensor:
    """The logits' gradient, of their type, from that of the weights fp32 [tokens, k] and what pcc_route gave."""
    _unrecorded(dweight, logits, weight, dlogits)
    ldl = _check("logits", logits, _ANY, (None, None), rows=True)
    tokens, experts = int(logits.shape[0]), int(logits.shape[1])
    _check("expert", expert, (torch.int32,), (tokens, None), logits.device)
    k = int(expert.shape[1])
    _check("weight", weight, (torch.float32,), (tokens, k), logits.device)
    _check("dweight", dweight, (torch.float32,), (tokens, k), logits.device)
    lddl = experts
    if dlogits is None:
        dlogits = torch.empty((tokens, experts), dtype=logits.dtype, device=logits.device)
    else:
        lddl = _check("dlogits", dlogits, (logits.dtype,), (tokens, experts), logits.device, rows=True)
    _call("pcc_route_grad", logits.device, dweight.data_ptr(), logits.data_ptr(), ldl, expert.data_ptr(), weight.data_ptr(), tokens, experts, k,
          _TYPES[logits.dtype], int(over_all), dlogits.data_ptr(), lddl)
    return dlogits


def pcc_expert_sort(expert: torch.Tensor, experts: int, offsets: torch.Tensor | None = None, place: torch.Tensor | None = None,
                    workspace: torch.Tensor | None = None):
    """(offsets int64 [experts + 1], place int32 [tokens, k]): the rows of the choices expert int32 [tokens, k], sorted by expert and within one by
    token.  A choice outside 0..experts - 1 has place -1."""
    _check("expert", expert, (torch.int32,), (None, None))
    tokens, k = int(expert.shape[0]), int(expert.shape[1])
    if not 0 < experts <= PCC_MAX_EXPERTS:
        raise ValueError("experts must be 1 to %d" % PCC_MAX_EXPERTS)
    offsets = _made_or_checked("offsets", offsets, torch.int64, (experts + 1,), expert.device)
    place = _made_or_checked("place", place, torch.int32, (tokens, k), expert.device)
    if workspace is None:
        need = int((_lib or load()).pcc_expert_sort_workspace_bytes(tokens, k, experts))
        workspace = torch.empty(need, dtype=torch.uint8, device=expert.device) if need else None
    else:
        _check("workspace", workspace, (torch.uint8,), (None,), expert.device)
    _call("pcc_expert_sort", expert.device, expert.data_ptr(), tokens, k, experts, offsets.data_ptr(), place.data_ptr(), _ptr(workspace),
          workspace.numel() if workspace is not None else 0)
    return offsets, place


def _check_place(place, device):
    _check("place", place, (torch.int32,), (None, None), device)
    return int(place.shape[0]), int(place.shape[1])


def pcc_expert_rows(x: torch.Tensor, place: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    """Rows of each expert, one behind the other: out[place[t, j]] = x[t].  out [rows, features] has tokens * k rows by default; rows that no choice has
    are left as they are in `out`, and undefined in a new tensor.  (The gradient is pcc_expert_join without weights.)"""
    _unrecorded(x, out)
    ldx = _check("x", x, _ANY, (None, None), rows=True)
    tokens, k = _check_place(place, x.device)
    features = int(x.shape[1])
    if int(x.shape[0]) != tokens:
        raise ValueError("x and place must have one row for each token")
    ldr = features
    if out is None:
        out = torch.empty((tokens * k, features), dtype=x.dtype, device=x.device)
    else:
        ldr = _check("out", out, (x.dtype,), (None, features), x.device, rows=True)
    _call("pcc_expert_rows", x.device, x.data_ptr(), ldx, place.data_ptr(), tokens, k, out.shape[0], features, _TYPES[x.dtype], out.data_ptr(), ldr)
    return out


def pcc_expert_join(z: torch.Tensor, place: torch.Tensor, weight: torch.Tensor | None = None, out: torch.Tensor | None = None,
                    out_dtype: torch.dtype | None = None) -> torch.Tensor:
    """y[t] = sum over j of weight[t, j] z[place[t, j]] (None: weights of 1), summed in fp32.  z [rows, features]; y has its type or fp32."""
    _unrecorded(z, weight, out)
    ldz = _check("z", z, _ANY, (None, None), rows=True)
    tokens, k = _check_place(place, z.device)
    rows, features = int(z.shape[0]), int(z.shape[1])
    if weight is not None:
        _check("weight", weight, (torch.float32,), (tokens, k), z.device)
    ldy = features
    if out is None:
        out = torch.empty((tokens, features), dtype=out_dtype or z.dtype, device=z.device)
    else:
        ldy = _check("out", out, (z.dtype, torch.float32) if out_dtype is None else (out_dtype,), (tokens, features), z.device, rows=True)
    _call("pcc_expert_join", z.device, z.data_ptr(), ldz, place.data_ptr(), _ptr(weight), tokens, k, rows, features, _TYPES[z.dtype], out.data_ptr(),
          _TYPES.get(out.dtype, -1), ldy)
    return out


def pcc_expert_join_grad(dy: torch.Tensor, z: torch.Tensor, place: torch.Tensor, weight: torch.Tensor | None = None, dz: torch.Tensor | None = None,
                         want_dweight: bool = True, dweight: torch.Tensor | None = None):
    """(dz, dweight) of pcc_expert_join: dz has z's type, dweight fp32 [tokens, k] (None without want_dweight).  Rows that no choice has are left as they are
    in `dz`, and undefined in a new tensor."""
    _unrecorded(dy, z, weight, dz, dweight)
    ldz = _check("z", z, _ANY, (None, None), rows=True)
    tokens, k = _check_place(place, z.device)
    rows, features = int(z.shape[0]), int(z.shape[1])
    lddy = _check("dy", dy, (z.dtype, torch.float32), (tokens, features), z.device, rows=True)
    if weight is not None:
        _check("weight", weight, (torch.float32,), (tokens, k), z.device)
    lddz = features
    if dz is None:
        dz = torch.empty((rows, features), dtype=z.dtype, device=z.device)
    else:
        lddz = _check("dz", dz, (z.dtype,), (rows, features), z.device, rows=True)
    if want_dweight:
        dweight = _made_or_checked("dweight", dweight, torch.float32, (tokens, k), z.device)
    _call("pcc_expert_join_grad", z.device, dy.data_ptr(), _TYPES[dy.dtype], lddy, z.data_ptr(), ldz, place.data_ptr(), _ptr(weight), tokens, k, rows, features,
          _TYPES[z.dtype], dz.data_ptr(), lddz, dweight.data_ptr() if want_dweight else None)
    return dz, (dweight if want_dweight else None)


def pcc_dropout(x: torch.Tensor, p: float, seed: int, step: torch.Tensor | None = None, residual: torch.Tensor | None = None,
                out: torch.Tensor | None = None, out_dtype: torch.dtype | None = None) -> torch.Tensor:
    """residual + x / (1 - p) for the elements of x [rows, features] that are kept, residual (None: 0) for the others.  Which ones is a function of seed
    (64 bits), step (int64 [1] on the device, None: 0), row and column alone: the same call on the gradient is the backward pass.  p is taken to the
    nearest 1/65536.  The result has x's type, or one of the two is fp32; residual has the result's.  `out` may be x or residual."""
    _unrecorded(x, residual, out)
    ldx = _check("x", x, _ANY, (None, None), rows=True)
    shape, seed = (int(x.shape[0]), int(x.shape[1])), int(seed)
    if not 0 <= seed < 1 << 64:
        raise ValueError("seed must be a whole number of 64 bits")
    if step is not None:
        _check("step", step, (torch.int64,), (1,), x.device)
    ldy = shape[1]
    if out is None:
        out = torch.empty(shape, dtype=out_dtype or x.dtype, device=x.device)
    else:
        ldy = _check("out", out, (_ANY if x.dtype == torch.float32 else (x.dtype, torch.float32)) if out_dtype is None else (out_dtype,), shape, x.device, rows=True)
    ldr = _check("residual", residual, (out.dtype,), shape, x.device, rows=True) if residual is not None else shape[1]
    _call("pcc_dropout", x.device, x.data_ptr(), ldx, _ptr(residual), ldr, shape[0], shape[1], _TYPES[x.dtype], p, seed, _ptr(step), out.data_ptr(),
          _TYPES.get(out.dtype, -1), ldy)
    return out


class AdamW:
    """Owns one pcc_adamw plan: AdamW over lists of tensors, one launch a step.

    params fp32, grads all of one type (fp32, bf16, fp16), copies (16-bit copies of the new parameters) or None.  States are
    made here or handed in (a checkpoint's): m, v fp32, or with state_bits=8 torch.float8_e4m3fn codes of m and of the root of v
    with m_scale, v_scale fp32 [ceil(n / 256)].  `step` int64 [1] counts the steps on the device.  `lr_tensor` fp32 [1] on the
    device is read at every step in place of lr.

    The plan holds the tensors' addresses: gradients are written into the tensors given here (not allocated anew), and a graph that
    captured a step is replayed only while this object lives.  States in 8 bits have a scale for 256 elements of a tensor."""

    def __init__(self, params, grads, copies=None, state_bits: int = 32, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay: float = 0.01, step=None, m=None, v=None, m_scale=None, v_scale=None, lr_tensor=None):
        self._h = C.c_void_p()
        params, grads = list(params), list(grads)
        if not params or len(grads) != len(params) or (copies is not None and len(copies) != len(params)):
            raise ValueError("params, grads and copies must be lists of one length, not empty")
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        if not (betas[0] >= 0 and betas[0] < 1 and betas[1] >= 0 and betas[1] < 1 and (eps == 0 or eps >= 2.0 ** -126)):
            raise ValueError("betas must be in [0, 1), eps 0 or at least 2^-126")
        copies = [None] * len(params) if copies is None else list(copies)
        device = params[0].device
        state = torch.float32 if state_bits == 32 else torch.float8_e4m3fn
        blocks = [-(-p.numel() // STATE_BLOCK) for p in params]
        zeros = lambda n, dt: torch.zeros(n, dtype=torch.uint8 if dt == torch.float8_e4m3fn else dt, device=device).view(dt)  # noqa: E731
        self.m = [zeros(p.numel(), state) for p in params] if m is None else list(m)
        self.v = [zeros(p.numel(), state) for p in params] if v is None else list(v)
        self.m_scale = self.v_scale = None
        if state_bits == 8:
            self.m_scale = [zeros(b, torch.float32) for b in blocks] if m_scale is None else list(m_scale)
            self.v_scale = [zeros(b, torch.float32) for b in blocks] if v_scale is None else list(v_scale)
        self.step = torch.zeros(1, dtype=torch.int64, device=device) if step is None else step
        self.params, self.grads, self.copies, self.lr_tensor, self.device = params, grads, copies, lr_tensor, device
        self.lr, self.betas, self.eps, self.weight_decay, self.state_bits = lr, tuple(betas), eps, weight_decay, state_bits
        _check("step", self.step, (torch.int64,), (1,), device)
        if lr_tensor is not None:
            _check("lr_tensor", lr_tensor, (torch.float32,), (1,), device)
        copy_type = next((c.dtype for c in copies if c is not None), torch.bfloat16)
        for lists in (self.m, self.v) + ((self.m_scale, self.v_scale) if state_bits == 8 else ()):
            if len(lists) != len(params):
                raise ValueError("states must be lists as long as params")
        table = (_AdamwTensor * len(params))()
        for i, p in enumerate(params):
            _check("params[%d]" % i, p, (torch.float32,), tuple(p.shape), device)
            _check("grads[%d]" % i, grads[i], (grads[0].dtype,) if grads[0].dtype in _TYPES else tuple(_TYPES), tuple(p.shape), device)
            if copies[i] is not None:
                _check("copies[%d]" % i, copies[i], (copy_type,) if copy_type in (torch.bfloat16, torch.float16) else (torch.bfloat16, torch.float16),
                       tuple(p.shape), device)
            for name, s in (("m", self.m[i]), ("v", self.v[i])):
                if s.numel() != p.numel():
                    raise ValueError("%s[%d] must have as many elements as its parameter" % (name, i))
                _check("%s[%d]" % (name, i), s, (state,), tuple(s.shape), device)
            row = dict(d_param=p, d_grad=grads[i], d_copy=copies[i], d_m=self.m[i], d_v=self.v[i])
            if state_bits == 8:
                _check("m_scale[%d]" % i, self.m_scale[i], (torch.float32,), (blocks[i],), device)
                _check("v_scale[%d]" % i, self.v_scale[i], (torch.float32,), (blocks[i],), device)
                row.update(d_m_scale=self.m_scale[i], d_v_scale=self.v_scale[i])
            for name, tensor in row.items():
                setattr(table[i], name, _ptr(tensor))
            table[i].n = p.numel()
        rc = load().pcc_adamw_create(C.byref(self._h), table, len(params), _TYPES[grads[0].dtype], _TYPES[copy_type], state_bits, device.index)
        if rc != PCC_OK:
            self._h = C.c_void_p()
            raise PccError(rc, "pcc_adamw_create")

    def pcc_adamw_step(self) -> None:
        hyper = _AdamwHyper(self.lr, self.betas[0], self.betas[1], self.eps, self.weight_decay, _ptr(self.lr_tensor))
        _call("pcc_adamw_step", self.device, self._h, C.byref(hyper), self.step.data_ptr())

    def close(self):
        if self._h and self._h.value:
            load().pcc_adamw_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
