"""ctypes binding of libsurgeon.so: the same names as ``include/surgeon.h``.

Argument marshalling only — every step of the path runs in the library's CUDA kernels.  PyTorch
supplies device memory and the current stream.  There is no fallback: if the shared library is
missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os
import threading
from dataclasses import dataclass
from typing import Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# SURGEON_LIB names another build of the same library (the checked build libsurgeon_bounds.so)
LIB_PATH = os.environ.get("SURGEON_LIB") or os.path.join(_HERE, "libsurgeon.so")

SURGEON_OK = 0
SURGEON_ERR_INVALID_ARG = 1
SURGEON_ERR_BUFFER_TOO_SMALL = 2
SURGEON_ERR_DEGENERATE = 3
SURGEON_ERR_UNSUPPORTED = 4
SURGEON_ERR_CUDA = 5
SURGEON_ERR_TIMEOUT = 6
SURGEON_ERR_INTERNAL = 7
SURGEON_F32, SURGEON_BF16 = 0, 1
SURGEON_BLOCK = 128
PATH_TENSOR_CORE, PATH_FP32 = 0, 1


class SurgeonError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = int(status)
        super().__init__("%s: %s (status %d)" % (where, status_string(status), status))


class Header(C.Structure):
    _fields_ = [("threshold_key", C.c_uint32), ("status", C.c_uint32), ("n_keep", C.c_int64),
                ("n_greater", C.c_int64), ("tie_quota", C.c_int64)]


class Compressed(C.Structure):
    _fields_ = [("n", C.c_int64), ("dt", C.c_int32), ("reserved", C.c_int32),
                ("bitmap", C.c_void_p), ("values", C.c_void_p), ("block_offsets", C.c_void_p),
                ("header", C.c_void_p)]


class Gradient(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("out", C.c_void_p), ("n", C.c_int64), ("dt", C.c_int32), ("reserved", C.c_int32)]


class LayerDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("kind", "batch", "c_in", "h", "w", "c_out", "kh", "kw",
                                         "stride", "pad", "path", "groups")]


_lib = None
# Short calls marshalled in C++ (pyext/calls.cpp): each returns the library's status, or None for a call that is not its
# ordinary case, which then goes through the checks below.  None if the module has not been built: every call does.
_calls = None


def _bind_calls(l):
    global _calls
    try:
        from . import _calls as module
    except ImportError:
        return
    module.bind(*(C.cast(f, C.c_void_p).value for f in (l.surgeon_layer_norm, l.surgeon_layer_norm_grad, l.surgeon_linear,
                                                        l.surgeon_linear_grad, l.surgeon_gradient_norm, l.surgeon_clip_gradients)))
    _calls = module


def lib():
    """The loaded shared library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                "libsurgeon.so is missing at %s: build it with "
                "`python -m paper_2503_20354_b200.build` (there is no CPU fallback)" % LIB_PATH)
        l = C.CDLL(LIB_PATH)
        l.surgeon_layer_ratios.restype = C.c_int
        l.surgeon_layer_ratios.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
        l.surgeon_layer_ratios_rule.restype = C.c_int
        l.surgeon_layer_ratios_rule.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int, C.c_double,
                                                C.c_void_p]
        l.surgeon_gradient_importance.restype = C.c_int
        l.surgeon_gradient_importance.argtypes = [C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p,
                                                  C.c_size_t, C.c_void_p]
        l.surgeon_compact_sizes.restype = C.c_int
        l.surgeon_compact_sizes.argtypes = [C.c_int64, C.c_int, C.c_double, C.c_void_p, C.c_void_p,
                                            C.c_void_p, C.c_void_p, C.c_void_p]      # int64 and size_t: 8 bytes each
        l.surgeon_prune_compact.restype = C.c_int
        l.surgeon_prune_compact.argtypes = [C.c_void_p, C.c_int64, C.c_int, C.c_double,
                                            C.POINTER(Compressed), C.c_void_p, C.c_size_t, C.c_void_p]
        l.surgeon_prune_compact_flags.restype = C.c_int
        l.surgeon_prune_compact_flags.argtypes = [C.c_void_p, C.c_int64, C.c_int, C.c_double, C.c_uint32,
                                                  C.POINTER(Compressed), C.c_void_p, C.c_size_t, C.c_void_p]
        l.surgeon_prune_compact_static.restype = C.c_int
        l.surgeon_prune_compact_static.argtypes = [C.c_void_p, C.c_int64, C.c_int, C.c_double,
                                                   C.POINTER(Compressed), C.c_void_p]
        l.surgeon_weight_grad_workspace.restype = C.c_size_t
        l.surgeon_weight_grad_workspace.argtypes = [C.POINTER(LayerDesc)]
        l.surgeon_weight_grad.restype = C.c_int
        l.surgeon_weight_grad.argtypes = [C.POINTER(Compressed), C.POINTER(LayerDesc), C.c_void_p,
                                          C.c_void_p, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]
        l.surgeon_weight_grad_flags.restype = C.c_int
        l.surgeon_weight_grad_flags.argtypes = [C.POINTER(Compressed), C.POINTER(LayerDesc), C.c_void_p, C.c_void_p,
                                                C.c_int32, C.c_uint32, C.c_void_p, C.c_size_t, C.c_void_p]
        P, I64, I32, F64 = C.c_void_p, C.c_int64, C.c_int32, C.c_double
        l.surgeon_layer_norm.restype = C.c_int
        l.surgeon_layer_norm.argtypes = [P, I64, I32, C.c_int, P, P, F64, P, P, P]
        l.surgeon_layer_norm_grad_workspace.restype = C.c_size_t
        l.surgeon_layer_norm_grad_workspace.argtypes = [I64, I32]
        l.surgeon_layer_norm_grad.restype = C.c_int
        l.surgeon_layer_norm_grad.argtypes = [P, P, I64, I32, C.c_int, C.c_int, P, P, P, P, P, P, I32, P, C.c_size_t, P]
        D = C.POINTER(LayerDesc)
        l.surgeon_linear_workspace.restype = C.c_size_t
        l.surgeon_linear_workspace.argtypes = [D]
        l.surgeon_linear.restype = C.c_int
        l.surgeon_linear.argtypes = [D, P, P, P, C.c_int, P, C.c_int, P, P, P, C.c_size_t, P]
        l.surgeon_linear_grad_workspace.restype = C.c_size_t
        l.surgeon_linear_grad_workspace.argtypes = [D]
        l.surgeon_linear_grad.restype = C.c_int
        l.surgeon_linear_grad.argtypes = [D, P, C.c_int, P, P, C.c_int, C.c_int, P, P, P, I32, P, C.c_size_t, P]
        l.surgeon_gradient_norm_workspace.restype = C.c_size_t
        l.surgeon_gradient_norm_workspace.argtypes = [I32]
        l.surgeon_gradient_norm.restype = C.c_int
        l.surgeon_gradient_norm.argtypes = [P, I32, P, P, P, C.c_size_t, P]
        l.surgeon_clip_gradients.restype = C.c_int
        l.surgeon_clip_gradients.argtypes = [P, I32, F64, P, P, P, C.c_size_t, P]
        l.surgeon_decompress.restype = C.c_int
        l.surgeon_decompress.argtypes = [C.POINTER(Compressed), C.c_void_p, C.c_void_p]
        l.surgeon_launch_count.restype = C.c_uint64
        l.surgeon_launch_count.argtypes = []
        l.surgeon_status_string.restype = C.c_char_p
        l.surgeon_status_string.argtypes = [C.c_int]
        _bind_calls(l)
        _lib = l
    return _lib


def status_string(status: int) -> str:
    return lib().surgeon_status_string(int(status)).decode()


def surgeon_launch_count() -> int:
    """Kernels launched by the library in this process so far."""
    return int(lib().surgeon_launch_count())


def _check(status: int, where: str, allow=()):
    if status != SURGEON_OK and status not in allow:
        raise SurgeonError(status, where)
    return status


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    if stream is not None:
        return stream.cuda_stream
    # the raw handle: a Stream object, made only to be asked for it, costs 3 us of a call's 10
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _scratch(nbytes: int, device, stream: Optional[torch.cuda.Stream]) -> torch.Tensor:
    """A scratch tensor made here (the caller passed none).  It is dropped when the call returns,
    while the kernels that use it are still queued on ``stream``: the allocator is told, so that
    the block is not handed out again before they are done."""
    t = torch.empty(max(int(nbytes), 16), dtype=torch.uint8, device=device)
    if stream is not None:
        t.record_stream(stream)
    return t


def dtype_code(t: torch.dtype) -> int:
    if t == torch.float32:
        return SURGEON_F32
    if t == torch.bfloat16:
        return SURGEON_BF16
    raise TypeError("activation dtype must be float32 or bfloat16, got %s" % t)


# ---------------------------------------------------------------------------------------------
# surgeon_layer_ratios (Eq. 5-7) and surgeon_compact_sizes (Algorithm 1: prune step): host arithmetic
# ---------------------------------------------------------------------------------------------

def surgeon_layer_ratios(gi, lam, allow_degenerate: bool = False) -> np.ndarray:
    """Per-layer pruning ratios from Gradient Importance ``gi`` and activation sizes ``lam``."""
    g = np.ascontiguousarray(gi, dtype=np.float64)
    m = np.ascontiguousarray(lam, dtype=np.float64)
    if g.ndim != 1 or g.shape != m.shape:
        raise ValueError("gi and lam must be 1-D and of equal length")
    out = np.empty_like(g)
    st = lib().surgeon_layer_ratios(g.ctypes.data, m.ctypes.data, int(g.size), out.ctypes.data)
    _check(st, "surgeon_layer_ratios", allow=(SURGEON_ERR_DEGENERATE,) if allow_degenerate else ())
    return out


SURGEON_RULE_BOTH, SURGEON_RULE_NO_GRADIENT, SURGEON_RULE_NO_MEMORY, SURGEON_RULE_STATIC = 0, 1, 2, 3
SURGEON_GI_WORKSPACE_BYTES = 8192


def surgeon_layer_ratios_rule(gi, lam, rule: int, static_ratio: float = 0.0,
                              allow_degenerate: bool = False) -> np.ndarray:
    """The ratio rule with one factor left out ("w/o G", "w/o M") or a global static ratio."""
    g = None if gi is None else np.ascontiguousarray(gi, dtype=np.float64)
    m = None if lam is None else np.ascontiguousarray(lam, dtype=np.float64)
    ref = g if g is not None else m
    if ref is None or ref.ndim != 1 or (g is not None and m is not None and g.shape != m.shape):
        raise ValueError("gi and lam must be 1-D and of equal length (one of them may be None)")
    out = np.empty(ref.shape, dtype=np.float64)
    st = lib().surgeon_layer_ratios_rule(None if g is None else g.ctypes.data,
                                         None if m is None else m.ctypes.data, int(ref.size),
                                         int(rule), float(static_ratio), out.ctypes.data)
    _check(st, "surgeon_layer_ratios_rule",
           allow=(SURGEON_ERR_DEGENERATE,) if allow_degenerate else ())
    return out


def surgeon_gradient_importance(dw: torch.Tensor, out: Optional[torch.Tensor] = None,
                                workspace: Optional[torch.Tensor] = None,
                                stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Eq. 4 on the device: a one-element float64 tensor holding sqrt(mean(dw^2))."""
    if not dw.is_cuda or not dw.is_contiguous() or dw.dtype != torch.float32:
        raise ValueError("dw must be a contiguous fp32 CUDA tensor")
    if out is None:
        out = torch.empty(1, dtype=torch.float64, device=dw.device)
    if workspace is None:
        workspace = _scratch(SURGEON_GI_WORKSPACE_BYTES, dw.device, stream)
    st = lib().surgeon_gradient_importance(dw.data_ptr() if dw.numel() else None, dw.numel(),
                                           out.data_ptr(), workspace.data_ptr(),
                                           workspace.numel() * workspace.element_size(),
                                           _stream_ptr(stream))
    _check(st, "surgeon_gradient_importance")
    return out


@dataclass
class CompactSizes:
    n_keep: int
    bitmap_bytes: int
    values_bytes: int
    offsets_bytes: int
    workspace_bytes: int


class _SizesOut(threading.local):
    """Where the C call puts its five numbers, one place per thread (made once: five ctypes objects
    and references per call cost more than the call)."""

    def __init__(self):
        self.words = (C.c_int64 * 5)()
        a = C.addressof(self.words)
        self.at = tuple(a + 8 * i for i in range(5))


_sizes_out = _SizesOut()


def surgeon_compact_sizes(n: int, dt: int, ratio: float) -> CompactSizes:
    out = _sizes_out
    st = lib().surgeon_compact_sizes(int(n), int(dt), float(ratio), *out.at)
    if st != SURGEON_OK:
        _check(st, "surgeon_compact_sizes")
    return CompactSizes(*out.words)


# ---------------------------------------------------------------------------------------------
# The compressed store and surgeon_prune_compact (Algorithm 1: prune and decompose steps)
# ---------------------------------------------------------------------------------------------

class CompressedActivation:
    """Device buffers of one compressed activation plus the C struct that points at them."""

    def __init__(self, n: int, dt: int, ratio: float, device, sizes: Optional[CompactSizes] = None,
                 _blank: bool = False):
        # _blank: a call that writes the header follows, so it need not be zeroed (a kernel launch)
        s = sizes or surgeon_compact_sizes(n, dt, ratio)
        self.n, self.dt, self.ratio, self._sizes = int(n), int(dt), float(ratio), s
        self.bitmap = torch.empty(max(s.bitmap_bytes // 4, 1), dtype=torch.int32, device=device)
        vt = torch.float32 if dt == SURGEON_F32 else torch.bfloat16
        self.values = torch.empty(max(s.n_keep, 1), dtype=vt, device=device)
        self.block_offsets = torch.empty(s.offsets_bytes // 4, dtype=torch.int32, device=device)
        self.header = (torch.empty if _blank else torch.zeros)(4, dtype=torch.int64, device=device)
        self.c = Compressed(self.n, self.dt, 0, self.bitmap.data_ptr(), self.values.data_ptr(),
                            self.block_offsets.data_ptr(), self.header.data_ptr())

    @property
    def sizes(self) -> CompactSizes:
        """Sizes at the store's present ratio (a call that changes the ratio leaves them to be asked for)."""
        if self._sizes is None:
            self._sizes = surgeon_compact_sizes(self.n, self.dt, self.ratio)
        return self._sizes

    def _now_at(self, ratio: float):
        if ratio != self.ratio:
            self.ratio, self._sizes = ratio, None

    def _fits(self, ratio: float) -> bool:
        # (a buffer for every element, as for ratios that change from batch to batch, fits any ratio)
        room = self.values.numel()
        return room >= self.n or room >= surgeon_compact_sizes(self.n, self.dt, ratio).n_keep

    @property
    def n_keep(self) -> int:
        return self.sizes.n_keep

    @property
    def stored_bytes(self) -> int:
        """Bytes of the cached form: packed values + 1 bit per element + block offsets."""
        return self.sizes.values_bytes + self.sizes.bitmap_bytes + self.sizes.offsets_bytes

    def read_header(self) -> Header:
        """Synchronising device->host read of the 32-byte result header."""
        raw = self.header.cpu().numpy().tobytes()
        return Header.from_buffer_copy(raw)

    def to_numpy(self):
        """Host copies for comparison: (bitmap uint32, values, offsets uint32, Header)."""
        nw = (self.n + 31) // 32
        bitmap = self.bitmap[:nw].cpu().numpy().view(np.uint32)
        hdr = self.read_header()
        vals = self.values[: int(hdr.n_keep)].cpu()    # the stored count (= n_keep unless zeros are dropped)
        vals = vals.view(torch.int16).numpy().view(np.uint16) if self.dt == SURGEON_BF16 else vals.numpy()
        offs = self.block_offsets[: self.sizes.offsets_bytes // 4].cpu().numpy().view(np.uint32)
        return bitmap, vals, offs, hdr


SURGEON_STORE_DROP_ZEROS = 1
SURGEON_SHARE_GPU = 2
SURGEON_DEBUG_STALL_BARRIER = 0x80000000


def surgeon_prune_compact(x: torch.Tensor, ratio: float, out: Optional[CompressedActivation] = None,
                          workspace: Optional[torch.Tensor] = None,
                          stream: Optional[torch.cuda.Stream] = None,
                          flags: int = 0) -> CompressedActivation:
    """Prune ``x`` (CUDA tensor, fp32 or bf16, contiguous) at ``ratio`` into a compressed store.
    ``flags=SURGEON_STORE_DROP_ZEROS``: kept zeros get no bit and no value (the header's n_keep
    is then the stored count; ``out.sizes.n_keep`` stays the upper bound the buffers are sized for).
    ``flags=SURGEON_SHARE_GPU``: other streams' calls run at the same time, so this one takes a part of
    the GPU; a call that is sent to another stream than the current one says so by that."""
    if not x.is_cuda or not x.is_contiguous():
        raise ValueError("x must be a contiguous CUDA tensor")
    dt = dtype_code(x.dtype)
    n = x.numel()
    ratio = float(ratio)
    if out is None:
        out = CompressedActivation(n, dt, ratio, x.device, _blank=True)
    elif out.n != n or out.dt != dt or not out._fits(ratio):
        raise ValueError("output store does not fit this tensor / ratio")
    if workspace is None:
        workspace = _scratch(surgeon_compact_sizes(n, dt, ratio).workspace_bytes, x.device, stream)
    at = _stream_ptr(stream)
    if stream is not None and at != torch._C._cuda_getCurrentRawStream(stream.device_index):
        flags |= SURGEON_SHARE_GPU
    st = lib().surgeon_prune_compact_flags(x.data_ptr(), n, dt, ratio, int(flags), C.byref(out.c),
                                           workspace.data_ptr(),
                                           workspace.numel() * workspace.element_size(), at)
    if st != SURGEON_OK:
        _check(st, "surgeon_prune_compact")
    out._now_at(ratio)
    return out


SURGEON_STATIC_MAX_N = 1 << 22


def surgeon_prune_compact_static(x: torch.Tensor, ratio: float, out: CompressedActivation,
                                 stream: Optional[torch.cuda.Stream] = None) -> CompressedActivation:
    """``surgeon_prune_compact`` without a workspace, for callers that must not allocate device
    memory (a hook running while the allocator is locked, a frozen memory pool): the scratch is
    a fixed array inside the library.  ``out`` must already exist and be large enough for this
    ratio (build it once with ``CompressedActivation(n, dt, 0.0, device)``); this function
    creates no tensor.  Tensors of more than ``SURGEON_STATIC_MAX_N`` elements are refused.
    Calls on one GPU share the scratch, so they must not overlap in time."""
    if not x.is_cuda or not x.is_contiguous():
        raise ValueError("x must be a contiguous CUDA tensor")
    dt = dtype_code(x.dtype)
    n = x.numel()
    if n > SURGEON_STATIC_MAX_N:
        raise SurgeonError(SURGEON_ERR_UNSUPPORTED, "surgeon_prune_compact_static: %d elements "
                           "exceed the built-in scratch (limit %d)" % (n, SURGEON_STATIC_MAX_N))
    ratio = float(ratio)
    if out.n != n or out.dt != dt or not out._fits(ratio):
        raise ValueError("output store does not fit this tensor / ratio")
    st = lib().surgeon_prune_compact_static(x.data_ptr(), n, dt, ratio, C.byref(out.c),
                                            _stream_ptr(stream))
    _check(st, "surgeon_prune_compact_static")
    out._now_at(ratio)
    return out


def surgeon_decompress(act: CompressedActivation, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Dense flat tensor rebuilt from the store (test utility; Algorithm 1: Reshape step)."""
    vt = torch.float32 if act.dt == SURGEON_F32 else torch.bfloat16
    out = torch.empty(max(act.n, 1), dtype=vt, device=act.bitmap.device)
    if stream is not None:
        out.record_stream(stream)
    st = lib().surgeon_decompress(C.byref(act.c), out.data_ptr(), _stream_ptr(stream))
    _check(st, "surgeon_decompress")
    return out[: act.n]


# ---------------------------------------------------------------------------------------------
# surgeon_weight_grad (Algorithm 1: Reshape and gradient steps, Eq. 2)
# ---------------------------------------------------------------------------------------------

def layer_desc(layer, path: int) -> LayerDesc:
    """LayerDesc from any object with kind/batch/c_in/h/w/c_out/kh/kw/stride/pad attributes."""
    return LayerDesc(layer.kind, layer.batch, layer.c_in, layer.h, layer.w, layer.c_out, layer.kh,
                     layer.kw, layer.stride, layer.pad, int(path), int(getattr(layer, "groups", 1)))


def surgeon_weight_grad_workspace(desc: LayerDesc) -> int:
    return int(lib().surgeon_weight_grad_workspace(C.byref(desc)))


def surgeon_weight_grad(act: CompressedActivation, desc: LayerDesc, grad_out: torch.Tensor,
                        dw: Optional[torch.Tensor] = None, accumulate: bool = False,
                        workspace: Optional[torch.Tensor] = None,
                        stream: Optional[torch.cuda.Stream] = None, flags: int = 0) -> torch.Tensor:
    """dW of the layer from the compressed activation and fp32 ``grad_out``; returns ``dw``.
    ``flags=SURGEON_SHARE_GPU``: other streams' calls run at the same time, so a small layer is cut into
    fewer parts (its sums are grouped otherwise, which is why a ``stream`` argument does not imply it)."""
    if grad_out.dtype != torch.float32 or not grad_out.is_cuda or not grad_out.is_contiguous():
        raise ValueError("grad_out must be a contiguous fp32 CUDA tensor")
    if dw is None:
        if accumulate:
            raise ValueError("accumulate needs an existing dw")
        shape = (desc.c_out, desc.c_in // max(desc.groups, 1), desc.kh, desc.kw) if desc.kind == 1 else (desc.c_out, desc.c_in)
        dw = torch.empty(shape, dtype=torch.float32, device=grad_out.device)
    if workspace is None:
        workspace = _scratch(surgeon_weight_grad_workspace(desc), grad_out.device, stream)
    st = lib().surgeon_weight_grad_flags(C.byref(act.c), C.byref(desc), grad_out.data_ptr(), dw.data_ptr(),
                                         1 if accumulate else 0, int(flags), workspace.data_ptr(),
                                         workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    _check(st, "surgeon_weight_grad")
    return dw


# ---------------------------------------------------------------------------------------------
# The layers around the store: what produces the activations (Eq. 1) and carries the gradient back
# (Eq. 2, first line), and the list of gradients that a step ends with
# ---------------------------------------------------------------------------------------------

def _operand(t: Optional[torch.Tensor], name: str, device: int, shape, dtype):
    """Checks one tensor of a call (None: left out) and returns its address.  ``device``: the current one."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        _refuse(t, name, device, shape, dtype)
    return t.data_ptr()


def _refuse(t: torch.Tensor, name: str, device: int, shape, dtype):
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("%s must be a contiguous CUDA tensor" % name)
    if t.get_device() != device:
        raise ValueError("%s is on %s, which is not the current device" % (name, t.device))
    if t.shape != shape:
        raise ValueError("%s must have the shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    raise ValueError("%s must be %s, got %s" % (name, dtype, t.dtype))


def _new(shape, dtype, device, stream: Optional[torch.cuda.Stream]) -> torch.Tensor:
    """A tensor made here for kernels on ``stream``, from that stream's part of the allocator's memory:
    a block of the current stream's may still be in use there."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _work(workspace: Optional[torch.Tensor], need, dev: int, stream: Optional[torch.cuda.Stream]):
    """Address and size of a call's scratch; where the caller passed none it is made here, of ``need()`` bytes."""
    if workspace is None:
        workspace = _new(max(int(need()), 16), torch.uint8, torch.device("cuda", dev), stream)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        _refuse(workspace, "workspace", dev, workspace.shape, workspace.dtype)
    return workspace.data_ptr(), workspace.nbytes


_TYPES = {torch.float32: SURGEON_F32, torch.bfloat16: SURGEON_BF16}


def _rows(t: torch.Tensor, name: str):
    """Shape, rows and channels of a tensor whose channels are its last dimension."""
    shape = t.shape
    if not shape or shape[-1] == 0:
        raise ValueError("%s must have channels in its last dimension" % name)
    return shape, t.numel() // shape[-1], shape[-1]


def surgeon_layer_norm(x: torch.Tensor, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None,
                       eps: float = 1e-5, out: Optional[torch.Tensor] = None, stats: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Layer norm over the last dimension of ``x`` (fp32 or bf16); returns ``out``, which may be ``x``.
    ``gamma``, ``beta``: fp32.  ``stats``: an fp32 tensor [2, rows] that receives the means and the reciprocal
    standard deviations for ``surgeon_layer_norm_grad``."""
    if _calls is not None and stream is None and out is not None:
        st = _calls.layer_norm(x, gamma, beta, eps, out, stats)
        if st is not None:
            if st != SURGEON_OK:
                _check(st, "surgeon_layer_norm")
            return out
    shape, rows, channels = _rows(x, "x")
    dev, dt, f32, vector = torch._C._cuda_getDevice(), x.dtype, torch.float32, (channels,)
    code = _TYPES.get(dt)
    if code is None:
        dtype_code(dt)
    if out is None:
        out = _new(shape, dt, x.device, stream)
    st = lib().surgeon_layer_norm(_operand(x, "x", dev, shape, dt), rows, channels, code,
                                  _operand(gamma, "gamma", dev, vector, f32), _operand(beta, "beta", dev, vector, f32), eps,
                                  _operand(out, "out", dev, shape, dt), _operand(stats, "stats", dev, (2, rows), f32),
                                  _stream_ptr(stream))
    if st != SURGEON_OK:
        _check(st, "surgeon_layer_norm")
    return out


def surgeon_layer_norm_grad_workspace(rows: int, channels: int) -> int:
    return int(lib().surgeon_layer_norm_grad_workspace(int(rows), int(channels)))


def surgeon_layer_norm_grad(x: torch.Tensor, dy: torch.Tensor, gamma: Optional[torch.Tensor], stats: torch.Tensor,
                            residual_grad: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None,
                            dgamma: Optional[torch.Tensor] = None, dbeta: Optional[torch.Tensor] = None,
                            accumulate: bool = False, workspace: Optional[torch.Tensor] = None,
                            stream: Optional[torch.cuda.Stream] = None, want_dx: bool = True) -> Optional[torch.Tensor]:
    """Backward pass of ``surgeon_layer_norm``; returns ``dx`` (of dy's type, made here if None; None with
    ``want_dx=False``).  ``residual_grad`` (dy's shape and type) is added to it; ``dx`` may be ``dy`` or
    ``residual_grad``.  ``dgamma``, ``dbeta``: fp32, written (``accumulate=True``: added to) where given."""
    if _calls is not None and stream is None and dx is not None and workspace is not None and want_dx:
        st = _calls.layer_norm_grad(x, dy, gamma, stats, residual_grad, dx, dgamma, dbeta, accumulate, workspace)
        if st is not None:
            if st != SURGEON_OK:
                _check(st, "surgeon_layer_norm_grad")
            return dx
    shape, rows, channels = _rows(x, "x")
    dev, f32, vector, gt = torch._C._cuda_getDevice(), torch.float32, (channels,), dy.dtype
    if not want_dx:
        if dx is not None:
            raise ValueError("dx given, but not wanted")
    elif dx is None:
        dx = _new(shape, gt, dy.device, stream)
    ws = None, 0
    if dgamma is not None or dbeta is not None:
        ws = _work(workspace, lambda: surgeon_layer_norm_grad_workspace(rows, channels), dev, stream)
    st = lib().surgeon_layer_norm_grad(_operand(x, "x", dev, shape, x.dtype), _operand(dy, "dy", dev, shape, gt), rows, channels,
                                       dtype_code(x.dtype), dtype_code(gt), _operand(gamma, "gamma", dev, vector, f32),
                                       _operand(stats, "stats", dev, (2, rows), f32),
                                       _operand(residual_grad, "residual_grad", dev, shape, gt),
                                       _operand(dx, "dx", dev, shape, gt), _operand(dgamma, "dgamma", dev, vector, f32),
                                       _operand(dbeta, "dbeta", dev, vector, f32), 1 if accumulate else 0, *ws,
                                       _stream_ptr(stream))
    if st != SURGEON_OK:
        _check(st, "surgeon_layer_norm_grad")
    return dx


SURGEON_ACT_NONE, SURGEON_ACT_RELU, SURGEON_ACT_GELU = 0, 1, 2


def linear_desc(rows: int, c_in: int, c_out: int) -> LayerDesc:
    """The descriptor of a linear layer on ``rows`` rows, tensor-core path (as ``layer_desc`` makes it of a layer)."""
    return LayerDesc(0, int(rows), int(c_in), 1, 1, int(c_out), 1, 1, 1, 0, PATH_TENSOR_CORE, 1)


def surgeon_linear_workspace(desc: LayerDesc) -> int:
    return int(lib().surgeon_linear_workspace(C.byref(desc)))


def surgeon_linear(desc: LayerDesc, x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None,
                   act: int = SURGEON_ACT_NONE, residual: Optional[torch.Tensor] = None,
                   out: Optional[torch.Tensor] = None, pre: Optional[torch.Tensor] = None,
                   out_dtype: torch.dtype = torch.bfloat16, workspace: Optional[torch.Tensor] = None,
                   stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """act(x W^T + bias) + residual; returns ``out`` (made here as ``out_dtype`` if None; it may be ``residual``).
    ``x`` [rows, c_in], ``weight`` [c_out, c_in]: bf16; ``bias``: fp32; ``residual``: of the output's type.
    ``pre``: a bf16 tensor [rows, c_out] that receives x W^T + bias for ``surgeon_linear_grad``."""
    if _calls is not None and stream is None and out is not None and workspace is not None:
        st = _calls.linear(desc, x, weight, bias, act, residual, out, pre, workspace)
        if st is not None:
            if st != SURGEON_OK:
                _check(st, "surgeon_linear")
            return out
    rows, ci, co = desc.batch, desc.c_in, desc.c_out
    dev, b16, shape = torch._C._cuda_getDevice(), torch.bfloat16, (rows, co)
    if out is None:
        out = _new(shape, out_dtype, x.device, stream)
    dt = out.dtype
    ws = _work(workspace, lambda: surgeon_linear_workspace(desc), dev, stream)
    st = lib().surgeon_linear(desc, _operand(x, "x", dev, (rows, ci), b16), _operand(weight, "weight", dev, (co, ci), b16),
                              _operand(bias, "bias", dev, (co,), torch.float32), act,
                              _operand(residual, "residual", dev, shape, dt), dtype_code(dt),
                              _operand(out, "out", dev, shape, dt), _operand(pre, "pre", dev, shape, b16), *ws,
                              _stream_ptr(stream))
    if st != SURGEON_OK:
        _check(st, "surgeon_linear")
    return out


def surgeon_linear_grad_workspace(desc: LayerDesc) -> int:
    return int(lib().surgeon_linear_grad_workspace(C.byref(desc)))


def surgeon_linear_grad(desc: LayerDesc, dy: torch.Tensor, weight: Optional[torch.Tensor], pre: Optional[torch.Tensor] = None,
                        act: int = SURGEON_ACT_NONE, dx: Optional[torch.Tensor] = None, dz: Optional[torch.Tensor] = None,
                        dbias: Optional[torch.Tensor] = None, accumulate: bool = False,
                        workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None,
                        want_dx: bool = True) -> Optional[torch.Tensor]:
    """Backward pass of ``surgeon_linear`` but for the weights' gradient; returns ``dx`` (bf16 if made here; bf16 or
    fp32 if given; None with ``want_dx=False``).  ``dy`` [rows, c_out]: fp32 or bf16.  ``dz``: fp32 [rows, c_out], receives
    dy act'(pre), the ``grad_out`` of ``surgeon_weight_grad``.  ``dbias``: fp32, written (``accumulate=True``: added to)."""
    if _calls is not None and stream is None and dx is not None and workspace is not None and want_dx:
        st = _calls.linear_grad(desc, dy, weight, pre, act, dx, dz, dbias, accumulate, workspace)
        if st is not None:
            if st != SURGEON_OK:
                _check(st, "surgeon_linear_grad")
            return dx
    rows, ci, co = desc.batch, desc.c_in, desc.c_out
    dev, b16, f32, shape, gt = torch._C._cuda_getDevice(), torch.bfloat16, torch.float32, (rows, co), dy.dtype
    if not want_dx:
        if dx is not None:
            raise ValueError("dx given, but not wanted")
    elif dx is None:
        dx = _new((rows, ci), b16, dy.device, stream)
    xt = b16 if dx is None else dx.dtype
    ws = _work(workspace, lambda: surgeon_linear_grad_workspace(desc), dev, stream)
    st = lib().surgeon_linear_grad(desc, _operand(dy, "dy", dev, shape, gt), dtype_code(gt),
                                   _operand(weight, "weight", dev, (co, ci), b16), _operand(pre, "pre", dev, shape, b16), act,
                                   dtype_code(xt), _operand(dx, "dx", dev, (rows, ci), xt), _operand(dz, "dz", dev, shape, f32),
                                   _operand(dbias, "dbias", dev, (co,), f32), 1 if accumulate else 0, *ws, _stream_ptr(stream))
    if st != SURGEON_OK:
        _check(st, "surgeon_linear_grad")
    return dx


class GradientList:
    """A list of gradients (fp32 or bf16, contiguous) and where their clipped values go (``outs``; None: in place),
    as the C array that the two calls below take.  The tensors are kept alive, and must not be reallocated."""

    def __init__(self, grads, outs=None):
        self.grads = tuple(grads)                    # (as many as the array below has entries, for good)
        self.outs = self.grads if outs is None else tuple(outs)
        if len(self.outs) != len(self.grads):
            raise ValueError("%d outputs for %d gradients" % (len(self.outs), len(self.grads)))
        self.device = self.grads[0].device if self.grads else None
        entries = []
        for i, (g, o) in enumerate(zip(self.grads, self.outs)):
            for t, what in ((g, "gradient"), (o, "output")):
                if not t.is_cuda or not t.is_contiguous() or t.device != self.device:
                    raise ValueError("%s %d must be a contiguous CUDA tensor on the device of the first" % (what, i))
            if o.dtype != g.dtype or o.shape != g.shape:
                raise ValueError("output %d must have its gradient's shape and type" % i)
            entries.append((g.data_ptr() or None, o.data_ptr() or None, g.numel(), dtype_code(g.dtype), 0))
        self.c = (Gradient * max(len(entries), 1))(*entries)
        self.address = C.addressof(self.c)

    def __len__(self):
        return len(self.grads)


def surgeon_gradient_norm_workspace(grads) -> int:
    """Scratch bytes for a ``GradientList`` (or any sequence as long)."""
    return int(lib().surgeon_gradient_norm_workspace(len(grads)))


def _list_call(grads, norm, gi, workspace, stream, new_gi):
    lst = grads if isinstance(grads, GradientList) else GradientList(grads)
    dev, f64, n = torch._C._cuda_getDevice(), torch.float64, len(lst.grads)
    if lst.device is not None and lst.device.index != dev:
        raise ValueError("the gradients are on %s, which is not the current device" % lst.device)
    if norm is None:
        norm = _new(1, f64, torch.device("cuda", dev), stream)
    if gi is None and new_gi:
        gi = _new(n, f64, torch.device("cuda", dev), stream)
    ws = _work(workspace, lambda: surgeon_gradient_norm_workspace(lst), dev, stream)
    return (lst, norm, gi, (_operand(norm, "norm", dev, (1,), f64), _operand(gi, "gi", dev, (n,), f64), *ws, _stream_ptr(stream)))


def _list_fast(grads, max_norm, norm, gi, workspace):
    if type(grads) is not GradientList or grads.device is None:
        return None
    return _calls.gradients(grads.address, len(grads.grads), grads.device.index, max_norm, norm, gi, workspace)


def surgeon_gradient_norm(grads, norm: Optional[torch.Tensor] = None, gi: Optional[torch.Tensor] = None,
                          workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """``(norm, gi)`` of a ``GradientList`` or a sequence of gradients: the global norm (one float64 on the device)
    and every tensor's Gradient Importance (Eq. 4, float64), as the ratio rule takes them."""
    if _calls is not None and stream is None and norm is not None and gi is not None and workspace is not None:
        st = _list_fast(grads, None, norm, gi, workspace)
        if st is not None:
            if st != SURGEON_OK:
                _check(st, "surgeon_gradient_norm")
            return norm, gi
    lst, norm, gi, args = _list_call(grads, norm, gi, workspace, stream, True)
    st = lib().surgeon_gradient_norm(lst.address, len(lst.grads), *args)
    if st != SURGEON_OK:
        _check(st, "surgeon_gradient_norm")
    return norm, gi


def surgeon_clip_gradients(grads, max_norm: float, norm: Optional[torch.Tensor] = None, gi: Optional[torch.Tensor] = None,
                           workspace: Optional[torch.Tensor] = None,
                           stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Scales the gradients by min(1, max_norm / (norm + 1e-6)) into their outputs (a sequence: in place) and returns the
    norm before.  An infinite or NaN norm leaves them as they are.  ``gi``: receives Eq. 4 of each, if given."""
    if _calls is not None and stream is None and norm is not None and workspace is not None:
        st = _list_fast(grads, max_norm, norm, gi, workspace)
        if st is not None:
            if st != SURGEON_OK:
                _check(st, "surgeon_clip_gradients")
            return norm
    lst, norm, gi, args = _list_call(grads, norm, gi, workspace, stream, False)
    st = lib().surgeon_clip_gradients(lst.address, len(lst.grads), max_norm, *args)
    if st != SURGEON_OK:
        _check(st, "surgeon_clip_gradients")
    return norm
