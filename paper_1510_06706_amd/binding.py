"""ctypes binding of libznn.so: same names as include/znn.h, argument marshalling only.

Tensors are torch CUDA tensors (device memory and streams come from torch);
every compute step runs inside the library.  There is no fallback: if the
library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Sequence, Tuple

# torch ships its own HIP runtime: loaded before the library, which then binds to the same runtime instance (one process, one
# runtime) instead of a second copy.
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libznn.so")

ZNN_OK, ZNN_EINVAL, ZNN_EUNSUPPORTED, ZNN_EWORKSPACE, ZNN_EHIP = 0, -1, -2, -3, -4
ZNN_DIRECT, ZNN_FFT, ZNN_AUTO = 0, 1, 2
ZNN_PASS_FWD, ZNN_PASS_BWD, ZNN_PASS_WGRAD = 0, 1, 2
MODES = {"direct": ZNN_DIRECT, "fft": ZNN_FFT, "auto": ZNN_AUTO}

EXPORTS = [
    "znn_plan_create", "znn_plan_destroy", "znn_plan_mode", "znn_plan_fft_extents",
    "znn_plan_workspace_bytes", "znn_plan_spectra_bytes", "znn_conv_prepare_kernels",
    "znn_conv_release_kernels", "znn_conv3d_fwd", "znn_conv3d_bwd", "znn_conv3d_wgrad",
    "znn_maxfilter3d_fwd", "znn_maxfilter3d_bwd", "znn_transfer_fwd", "znn_transfer_bwd",
    "znn_bias_grad", "znn_square_loss_grad", "znn_sgd_update", "znn_autotune_workspace_bytes",
    "znn_autotune", "znn_last_error", "znn_trace_enable", "znn_trace_collect",
    "znn_plan_memo_bytes", "znn_conv_set_memo", "znn_conv3d_wgrad_memo",
    "znn_maxfilter3d_sparse_fwd", "znn_maxfilter3d_sparse_bwd", "znn_maxpool3d_fwd", "znn_maxpool3d_bwd",
    "znn_transfer_fn_fwd", "znn_transfer_fn_bwd", "znn_cross_entropy_loss_grad",
    "znn_autotune_round_workspace_bytes", "znn_autotune_round", "znn_accumulate",
    "znn_plan_set_spectra_layout", "znn_plan_spectra_layout", "znn_plan_tiles", "znn_conv3d_fwd_static",
    "znn_program_create", "znn_program_destroy", "znn_program_scratch_bytes", "znn_program_run",
    "znn_plan_set_round_memory",
    "znn_random_advance", "znn_dropout", "znn_layernorm_workspace_bytes", "znn_layernorm_fwd", "znn_layernorm_bwd",
    "znn_residual_norm_fwd", "znn_residual_norm_bwd",
    "znn_gated_workspace_bytes", "znn_gated_fwd", "znn_gated_bwd",
    "znn_recurrence_workspace_bytes", "znn_recurrence_fwd", "znn_recurrence_bwd",
]
STATIC_SCRATCH_BYTES = 32 * 1024 * 1024
SPECTRA_LAYOUTS = {"auto": 0, "full": 1, "folded": 2}
STRATEGIES = ("direct", "fft", "fft_memo")
TRANSFER_FNS = {"rectify": 0, "logistic": 1, "tanh": 2}
GATE_FNS = {"rectify": 0, "logistic": 1, "tanh": 2, "silu": 3, "gelu": 4}
NORM_EPS = 1e-5


class Vec3(ctypes.Structure):
    _fields_ = [("z", ctypes.c_int32), ("y", ctypes.c_int32), ("x", ctypes.c_int32)]


class ConvDesc(ctypes.Structure):
    _fields_ = [("fan_in", ctypes.c_int32), ("fan_out", ctypes.c_int32), ("image", Vec3),
                ("kernel", Vec3), ("sparsity", Vec3), ("mode", ctypes.c_int32)]


class Op(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("stream", ctypes.c_int32), ("fn", ctypes.c_int32), ("loss", ctypes.c_int32),
                ("maps", ctypes.c_int32), ("n", Vec3), ("window", Vec3), ("sparsity", Vec3),
                ("buf", ctypes.c_int32 * 8), ("plan", ctypes.c_void_p)]


class TraceRecord(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 56), ("ms", ctypes.c_float)]


class RoundReport(ctypes.Structure):
    _fields_ = [("ms", ctypes.c_float * 3), ("bytes", ctypes.c_uint64 * 3), ("chosen", ctypes.c_int32)]


class ZnnError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__("znn error %d: %s" % (code, message))
        self.code = code


_lib = None


def lib():
    """Loads libznn.so (raises if it is missing: there is no other compute path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libznn.so is not built: run `python -m paper_1510_06706_amd.build` "
                               "(or __graft_entry__.build()) first")
        L = ctypes.CDLL(LIB_PATH)
        vp, sz, i32, i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_int64
        L.znn_last_error.restype = ctypes.c_char_p
        L.znn_plan_create.argtypes = [ctypes.POINTER(ConvDesc), ctypes.POINTER(vp)]
        L.znn_plan_destroy.argtypes = [vp]
        L.znn_plan_destroy.restype = None
        L.znn_plan_mode.argtypes = [vp, ctypes.POINTER(i32)]
        L.znn_plan_fft_extents.argtypes = [vp, ctypes.POINTER(Vec3)]
        L.znn_plan_workspace_bytes.argtypes = [vp, i32, ctypes.POINTER(sz)]
        L.znn_plan_spectra_bytes.argtypes = [vp, ctypes.POINTER(sz)]
        L.znn_plan_set_spectra_layout.argtypes = [vp, i32]
        L.znn_plan_spectra_layout.argtypes = [vp, ctypes.POINTER(i32)]
        L.znn_plan_tiles.argtypes = [vp, ctypes.POINTER(Vec3), ctypes.POINTER(Vec3)]
        L.znn_conv_prepare_kernels.argtypes = [vp, vp, vp, sz, vp, sz, vp]
        L.znn_conv_release_kernels.argtypes = [vp]
        for name in ("znn_conv3d_fwd", "znn_conv3d_bwd", "znn_conv3d_wgrad"):
            getattr(L, name).argtypes = [vp, vp, vp, vp, vp, sz, vp]
        L.znn_conv3d_fwd_static.argtypes = [vp, vp, vp, vp, vp]
        L.znn_maxfilter3d_fwd.argtypes = [i32, Vec3, Vec3, vp, vp, vp, vp]
        L.znn_maxfilter3d_bwd.argtypes = [i32, Vec3, Vec3, vp, vp, vp, vp]
        L.znn_maxfilter3d_sparse_fwd.argtypes = [i32, Vec3, Vec3, Vec3, vp, vp, vp, vp]
        L.znn_maxfilter3d_sparse_bwd.argtypes = [i32, Vec3, Vec3, Vec3, vp, vp, vp, vp]
        L.znn_maxpool3d_fwd.argtypes = [i32, Vec3, Vec3, vp, vp, vp, vp]
        L.znn_maxpool3d_bwd.argtypes = [i32, Vec3, Vec3, vp, vp, vp, vp]
        L.znn_transfer_fn_fwd.argtypes = [i32, i32, i64, vp, vp, vp, vp]
        L.znn_transfer_fn_bwd.argtypes = [i32, i32, i64, vp, vp, vp, vp]
        L.znn_cross_entropy_loss_grad.argtypes = [i64, vp, vp, vp, vp]
        L.znn_transfer_fwd.argtypes = [i32, i64, vp, vp, vp, vp]
        L.znn_transfer_bwd.argtypes = [i32, i64, vp, vp, vp, vp]
        L.znn_bias_grad.argtypes = [i32, i64, vp, vp, vp]
        L.znn_square_loss_grad.argtypes = [i64, vp, vp, vp, vp]
        L.znn_accumulate.argtypes = [i64, vp, vp, vp]
        L.znn_sgd_update.argtypes = [i64, ctypes.c_float, vp, vp, vp]
        L.znn_autotune_workspace_bytes.argtypes = [ctypes.POINTER(ConvDesc), ctypes.POINTER(sz)]
        L.znn_autotune.argtypes = [ctypes.POINTER(ConvDesc), vp, sz, vp, ctypes.POINTER(i32),
                                   ctypes.POINTER(ctypes.c_float * 3 * 2)]
        L.znn_autotune_round_workspace_bytes.argtypes = [ctypes.POINTER(ConvDesc), ctypes.POINTER(sz)]
        L.znn_autotune_round.argtypes = [ctypes.POINTER(ConvDesc), ctypes.c_uint64, vp, sz, vp,
                                         ctypes.POINTER(RoundReport)]
        L.znn_plan_memo_bytes.argtypes = [vp, ctypes.POINTER(sz)]
        L.znn_conv_set_memo.argtypes = [vp, vp, sz]
        L.znn_conv3d_wgrad_memo.argtypes = [vp, vp, vp, sz, vp]
        L.znn_trace_enable.argtypes = [i32]
        L.znn_trace_collect.argtypes = [ctypes.POINTER(TraceRecord), i32, ctypes.POINTER(i32)]
        L.znn_plan_set_round_memory.argtypes = [vp, sz]
        L.znn_program_create.argtypes = [ctypes.POINTER(Op), i32, i32, i32, ctypes.POINTER(vp)]
        L.znn_program_destroy.argtypes = [vp]
        L.znn_program_destroy.restype = None
        L.znn_program_scratch_bytes.argtypes = [vp, ctypes.POINTER(sz)]
        L.znn_program_run.argtypes = [vp, ctypes.POINTER(vp), vp, sz, ctypes.c_float, ctypes.POINTER(vp)]
        u32, f32, f64 = ctypes.c_uint32, ctypes.c_float, ctypes.c_double
        L.znn_random_advance.argtypes = [vp, vp]
        L.znn_dropout.argtypes = [i64, i64, f64, vp, u32, vp, vp, vp]
        L.znn_layernorm_workspace_bytes.argtypes = [i64, i64, i32, ctypes.POINTER(sz)]
        L.znn_layernorm_fwd.argtypes = [i64, i64, i32, f32] + [vp] * 6
        L.znn_layernorm_bwd.argtypes = [i64, i64, i32] + [vp] * 8 + [sz, vp]
        L.znn_residual_norm_fwd.argtypes = [i64, i64, i32, f32, f64, vp, u32] + [vp] * 8
        L.znn_residual_norm_bwd.argtypes = [i64, i64, i32, f64, vp, u32] + [vp] * 10 + [sz, vp]
        L.znn_gated_workspace_bytes.argtypes = [i32, i32, i64, i32, i32, ctypes.POINTER(sz)]
        L.znn_gated_fwd.argtypes = [i32, i32, i32, i64, i32] + [vp] * 6 + [sz, vp]
        L.znn_gated_bwd.argtypes = [i32, i32, i32, i64, i32] + [vp] * 8 + [sz, vp]
        L.znn_recurrence_workspace_bytes.argtypes = [i64, i64, i64, ctypes.POINTER(sz)]
        L.znn_recurrence_fwd.argtypes = [i64, i64, i64, i32] + [vp] * 5 + [sz, vp]
        L.znn_recurrence_bwd.argtypes = [i64, i64, i64, i32] + [vp] * 9 + [sz, vp]
        for name in EXPORTS:
            if name not in ("znn_last_error", "znn_plan_destroy", "znn_program_destroy"):
                getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def last_error() -> str:
    return lib().znn_last_error().decode()


def _check(rc: int):
    if rc != ZNN_OK:
        raise ZnnError(rc, last_error())


def _v3(t: Sequence[int]) -> Vec3:
    return Vec3(int(t[0]), int(t[1]), int(t[2]))


def make_desc(fan_in, fan_out, image, kernel, mode="direct", sparsity=(1, 1, 1)) -> ConvDesc:
    m = MODES[mode] if isinstance(mode, str) else int(mode)
    return ConvDesc(int(fan_in), int(fan_out), _v3(image), _v3(kernel), _v3(sparsity), m)


def _stream_ptr(stream=None):
    """The stream's handle; without one that of torch's current stream (0.3 us; 2.7 as a ``torch.cuda.Stream``)."""
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) if stream is None else stream.cuda_stream


def _ptr(t, dtype=None):
    """Device pointer of a contiguous CUDA tensor (None -> NULL), as the integer that ctypes takes for a pointer."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("tensor must live on the GPU")
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError("tensor must be %s, got %s" % (dtype, t.dtype))
    return t.data_ptr()


class Plan:
    """Owner of a znn_plan; methods mirror the C entry points."""

    def __init__(self, fan_in, fan_out, image, kernel, mode="direct", sparsity=(1, 1, 1)):
        self.desc = make_desc(fan_in, fan_out, image, kernel, mode, sparsity)
        self.f, self.fo = int(fan_in), int(fan_out)
        self.n, self.k = tuple(int(v) for v in image), tuple(int(v) for v in kernel)
        self.s = tuple(int(v) for v in sparsity)
        self.o = tuple(n - s * (k - 1) for n, k, s in zip(self.n, self.k, self.s))
        self._in, self._out, self._ker = (self.f,) + self.n, (self.fo,) + self.o, (self.fo, self.f) + self.k
        self._h = ctypes.c_void_p(0)
        self._ws = None
        self._spectra = None
        self._memo = None
        self.revision = 0           # counts the changes that a program made of the plan does not see
        _check(lib().znn_plan_create(ctypes.byref(self.desc), ctypes.byref(self._h)))

    def close(self):
        if self._h:
            lib().znn_plan_destroy(self._h)
            self._h = ctypes.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def mode(self) -> int:
        m = ctypes.c_int32(-1)
        _check(lib().znn_plan_mode(self._h, ctypes.byref(m)))
        return m.value

    @property
    def fft_extents(self) -> Tuple[int, int, int]:
        v = Vec3()
        _check(lib().znn_plan_fft_extents(self._h, ctypes.byref(v)))
        return (v.z, v.y, v.x)

    def workspace_bytes(self, which: int) -> int:
        b = ctypes.c_size_t(0)
        _check(lib().znn_plan_workspace_bytes(self._h, which, ctypes.byref(b)))
        return b.value

    def spectra_bytes(self) -> int:
        b = ctypes.c_size_t(0)
        _check(lib().znn_plan_spectra_bytes(self._h, ctypes.byref(b)))
        return b.value

    def set_spectra_layout(self, layout: str):
        """'auto', 'full' (the kernel transforms themselves) or 'folded' (half spectra)."""
        _check(lib().znn_plan_set_spectra_layout(self._h, SPECTRA_LAYOUTS[layout]))
        self.revision += 1

    def set_round_memory(self, nbytes: int):
        """Bounds what rounds as one program hold of this layer beside the workspace of its passes."""
        _check(lib().znn_plan_set_round_memory(self._h, int(nbytes)))
        self.revision += 1

    @property
    def spectra_layout(self) -> str:
        v = ctypes.c_int32(-1)
        _check(lib().znn_plan_spectra_layout(self._h, ctypes.byref(v)))
        return {1: "full", 2: "folded"}[v.value]

    @property
    def tiles(self):
        """(transform lengths, tiles) per axis of the FFT method on overlapping tiles, None on whole volumes."""
        m, t = Vec3(), Vec3()
        _check(lib().znn_plan_tiles(self._h, ctypes.byref(m), ctypes.byref(t)))
        return ((m.z, m.y, m.x), (t.z, t.y, t.x)) if m.x else None

    def _workspace(self, which: int, device):
        """Grows (never shrinks) a torch byte buffer used as the caller workspace."""
        need = self.workspace_bytes(which)
        if need == 0:
            return None, 0
        if self._ws is None or self._ws.numel() < need + 256:
            self._ws = None
            self._ws = torch.empty(need + 256, dtype=torch.uint8, device=device)
        base = self._ws.data_ptr()
        aligned = (base + 255) & ~255
        return aligned, need

    def prepare_kernels(self, w, stream=None):
        """Transforms all kernels once; the spectra stay resident in a buffer this object owns."""
        need = self.spectra_bytes()
        buf = getattr(self, "_spectra", None)
        if buf is None or buf.numel() != need + 256 or buf.device != w.device:
            buf = torch.empty(need + 256, dtype=torch.uint8, device=w.device)
        aligned = (buf.data_ptr() + 255) & ~255
        ws, wsb = self._workspace(ZNN_PASS_FWD, w.device)
        _check(lib().znn_conv_prepare_kernels(self._h, _ptr(w, torch.float32), ctypes.c_void_p(aligned), need,
                                              ws, wsb, _stream_ptr(stream)))
        self._spectra = buf

    def memo_bytes(self) -> int:
        b = ctypes.c_size_t(0)
        _check(lib().znn_plan_memo_bytes(self._h, ctypes.byref(b)))
        return b.value

    def enable_memo(self, device="cuda:0"):
        """Attaches a buffer (owned by this object) in which fwd / bwd leave their node spectra."""
        need = self.memo_bytes()
        buf = torch.empty(need + 256, dtype=torch.uint8, device=device)
        aligned = (buf.data_ptr() + 255) & ~255
        _check(lib().znn_conv_set_memo(self._h, ctypes.c_void_p(aligned), need))
        self._memo = buf

    def disable_memo(self):
        _check(lib().znn_conv_set_memo(self._h, ctypes.c_void_p(0), 0))
        self._memo = None

    def wgrad_memo(self, gw=None, device="cuda:0", stream=None):
        """Kernel gradient of the tensors given to the last fwd and bwd, from their memoized spectra."""
        if gw is None:
            gw = torch.empty((self.fo, self.f) + self.k, dtype=torch.float32, device=device)
        assert tuple(gw.shape) == (self.fo, self.f) + self.k
        ws, wsb = self._workspace(ZNN_PASS_WGRAD, gw.device)
        _check(lib().znn_conv3d_wgrad_memo(self._h, _ptr(gw, torch.float32), ws, wsb, _stream_ptr(stream)))
        return gw

    def release_kernels(self):
        _check(lib().znn_conv_release_kernels(self._h))
        self._spectra = None

    def fwd(self, inp, w, out=None, stream=None):
        assert inp.shape == self._in, inp.shape
        if w is not None:
            assert w.shape == self._ker, w.shape
        if out is None:
            out = torch.empty(self._out, dtype=torch.float32, device=inp.device)
        assert out.shape == self._out
        ws, wsb = self._workspace(ZNN_PASS_FWD, inp.device)
        _check(lib().znn_conv3d_fwd(self._h, _ptr(inp, torch.float32), _ptr(w, torch.float32),
                                    _ptr(out, torch.float32), ws, wsb, _stream_ptr(stream)))
        return out

    def fwd_static(self, inp, w, out, stream=None):
        """znn_conv3d_fwd_static: the forward pass with the library's built-in scratch array; this
        wrapper allocates nothing either (the caller passes `out`)."""
        assert inp.shape == self._in, inp.shape
        assert out.shape == self._out
        _check(lib().znn_conv3d_fwd_static(self._h, _ptr(inp, torch.float32), _ptr(w, torch.float32),
                                           _ptr(out, torch.float32), _stream_ptr(stream)))
        return out

    def bwd(self, gout, w, gin=None, stream=None):
        assert gout.shape == self._out, gout.shape
        if w is not None:
            assert w.shape == self._ker, w.shape
        if gin is None:
            gin = torch.empty(self._in, dtype=torch.float32, device=gout.device)
        assert gin.shape == self._in
        ws, wsb = self._workspace(ZNN_PASS_BWD, gout.device)
        _check(lib().znn_conv3d_bwd(self._h, _ptr(gout, torch.float32), _ptr(w, torch.float32),
                                    _ptr(gin, torch.float32), ws, wsb, _stream_ptr(stream)))
        return gin

    def wgrad(self, inp, gout, gw=None, stream=None):
        assert inp.shape == self._in, inp.shape
        assert gout.shape == self._out, gout.shape
        if gw is None:
            gw = torch.empty(self._ker, dtype=torch.float32, device=inp.device)
        assert gw.shape == self._ker
        ws, wsb = self._workspace(ZNN_PASS_WGRAD, inp.device)
        _check(lib().znn_conv3d_wgrad(self._h, _ptr(inp, torch.float32), _ptr(gout, torch.float32),
                                      _ptr(gw, torch.float32), ws, wsb, _stream_ptr(stream)))
        return gw


def maxfilter3d_fwd(inp, win, sparsity=(1, 1, 1), stream=None):
    maps, n = inp.shape[0], tuple(inp.shape[1:])
    o = tuple(a - s * (b - 1) for a, b, s in zip(n, win, sparsity))
    if min(o) < 1:
        o = (0, 0, 0)
    out = torch.empty((maps,) + o, dtype=torch.float32, device=inp.device)
    idx = torch.empty((maps,) + o, dtype=torch.int32, device=inp.device)
    if tuple(sparsity) == (1, 1, 1):
        _check(lib().znn_maxfilter3d_fwd(maps, _v3(n), _v3(win), _ptr(inp, torch.float32), _ptr(out), _ptr(idx),
                                         _stream_ptr(stream)))
    else:
        _check(lib().znn_maxfilter3d_sparse_fwd(maps, _v3(n), _v3(win), _v3(sparsity), _ptr(inp, torch.float32),
                                                _ptr(out), _ptr(idx), _stream_ptr(stream)))
    return out, idx


def maxfilter3d_bwd(gout, idx, n, win, sparsity=(1, 1, 1), stream=None):
    maps = gout.shape[0]
    gin = torch.empty((maps,) + tuple(n), dtype=torch.float32, device=gout.device)
    if tuple(sparsity) == (1, 1, 1):
        _check(lib().znn_maxfilter3d_bwd(maps, _v3(n), _v3(win), _ptr(gout, torch.float32), _ptr(idx, torch.int32),
                                         _ptr(gin), _stream_ptr(stream)))
    else:
        _check(lib().znn_maxfilter3d_sparse_bwd(maps, _v3(n), _v3(win), _v3(sparsity), _ptr(gout, torch.float32),
                                                _ptr(idx, torch.int32), _ptr(gin), _stream_ptr(stream)))
    return gin


def maxpool3d_fwd(inp, p, stream=None):
    maps, n = inp.shape[0], tuple(inp.shape[1:])
    o = tuple(a // b if b > 0 else 0 for a, b in zip(n, p))
    out = torch.empty((maps,) + o, dtype=torch.float32, device=inp.device)
    idx = torch.empty((maps,) + o, dtype=torch.int32, device=inp.device)
    _check(lib().znn_maxpool3d_fwd(maps, _v3(n), _v3(p), _ptr(inp, torch.float32), _ptr(out), _ptr(idx),
                                   _stream_ptr(stream)))
    return out, idx


def maxpool3d_bwd(gout, idx, n, p, stream=None):
    maps = gout.shape[0]
    gin = torch.empty((maps,) + tuple(n), dtype=torch.float32, device=gout.device)
    _check(lib().znn_maxpool3d_bwd(maps, _v3(n), _v3(p), _ptr(gout, torch.float32), _ptr(idx, torch.int32),
                                   _ptr(gin), _stream_ptr(stream)))
    return gin


def transfer_fwd(x, bias, fn="rectify", stream=None):
    y = torch.empty_like(x)
    maps = x.shape[0]
    if fn == "rectify":
        _check(lib().znn_transfer_fwd(maps, x.numel() // maps, _ptr(x, torch.float32), _ptr(bias, torch.float32),
                                      _ptr(y), _stream_ptr(stream)))
    else:
        _check(lib().znn_transfer_fn_fwd(TRANSFER_FNS[fn], maps, x.numel() // maps, _ptr(x, torch.float32),
                                         _ptr(bias, torch.float32), _ptr(y), _stream_ptr(stream)))
    return y


def transfer_bwd(gy, y, fn="rectify", stream=None):
    gx = torch.empty_like(gy)
    maps = gy.shape[0]
    if fn == "rectify":
        _check(lib().znn_transfer_bwd(maps, gy.numel() // maps, _ptr(gy, torch.float32), _ptr(y, torch.float32),
                                      _ptr(gx), _stream_ptr(stream)))
    else:
        _check(lib().znn_transfer_fn_bwd(TRANSFER_FNS[fn], maps, gy.numel() // maps, _ptr(gy, torch.float32),
                                         _ptr(y, torch.float32), _ptr(gx), _stream_ptr(stream)))
    return gx


def bias_grad(g, stream=None):
    maps = g.shape[0]
    gb = torch.empty((maps,), dtype=torch.float32, device=g.device)
    _check(lib().znn_bias_grad(maps, g.numel() // maps, _ptr(g, torch.float32), _ptr(gb), _stream_ptr(stream)))
    return gb


def square_loss_grad(out, target, stream=None):
    g = torch.empty_like(out)
    _check(lib().znn_square_loss_grad(out.numel(), _ptr(out, torch.float32), _ptr(target, torch.float32),
                                      _ptr(g), _stream_ptr(stream)))
    return g


def cross_entropy_loss_grad(out, target, stream=None):
    g = torch.empty_like(out)
    _check(lib().znn_cross_entropy_loss_grad(out.numel(), _ptr(out, torch.float32), _ptr(target, torch.float32),
                                             _ptr(g), _stream_ptr(stream)))
    return g


def loss_grad(out, target, loss="square", stream=None):
    if loss == "square":
        return square_loss_grad(out, target, stream)
    if loss == "cross_entropy":
        return cross_entropy_loss_grad(out, target, stream)
    raise ValueError(loss)


def accumulate(y, x, stream=None):
    """y += x (node sum of a computation graph)."""
    assert y.shape == x.shape
    _check(lib().znn_accumulate(y.numel(), _ptr(x, torch.float32), _ptr(y, torch.float32), _stream_ptr(stream)))
    return y


def sgd_update(p, g, eta, stream=None):
    _check(lib().znn_sgd_update(p.numel(), float(eta), _ptr(g, torch.float32), _ptr(p, torch.float32),
                                _stream_ptr(stream)))
    return p


# ---------------------------------------------------------------- dropout, layer norm, residual join
# Arrays are tensors [rows, ...] with all dimensions behind the first as their columns: images [map][z][y][x] with axis 0
# (every voxel over the maps), rows of features with axis 1.
def random_state(seed, device="cuda:0"):
    """{seed, round} on the device: what dropout goes by.  ``random_advance`` behind a round makes the next one drop others."""
    seed = int(seed) & 0xFFFFFFFFFFFFFFFF
    return torch.tensor([seed - (1 << 64) if seed >> 63 else seed, 0], dtype=torch.int64, device=device)


def random_advance(state, stream=None):
    _check(lib().znn_random_advance(_state_ptr(state), _stream_ptr(stream)))
    return state


def _state_ptr(state):
    if state is not None and state.numel() != 2:
        raise ValueError("a random state holds two numbers")
    return _ptr(state, torch.int64)


def _site(site):
    """The calls of a round are told apart by 32 bits, of which ctypes would cut the rest off."""
    if not 0 <= site < 1 << 32:
        raise ValueError("a site has 32 bits, got %r" % (site,))
    return site


def _extents(x, axis, *params):
    """(rows, columns, positions of the norm) of an array whose parameters are checked."""
    rows = x.shape[0] if x.dim() else 0
    if rows < 1:
        raise ValueError("expected an array [rows, ...], got %s" % (tuple(x.shape),))
    cols = x.numel() // rows
    if axis == 0:
        n, positions = rows, cols
    elif axis == 1:
        n, positions = cols, rows
    else:
        raise ValueError("axis must be 0 or 1, got %r" % (axis,))
    for p in params:
        if p.numel() != n:
            raise ValueError("expected %d parameters, got %d" % (n, p.numel()))
    return rows, cols, positions


def _same_shape(t, *others):
    for o in others:
        if o is not None and o.shape != t.shape:
            raise ValueError("expected shape %s, got %s" % (tuple(t.shape), tuple(o.shape)))


def dropout(x, p, state=None, site=0, stream=None):
    """x / (1 - p) where an element is kept, 0 elsewhere; on a gradient, with the same state and site, the Jacobian."""
    if stream is not None:          # what is made belongs to the stream that works on it
        with torch.cuda.stream(stream):
            return dropout(x, p, state, site)
    rows, cols, _ = _extents(x, 0)
    y = torch.empty_like(x)
    _check(lib().znn_dropout(rows, cols, p, _state_ptr(state), _site(site), _ptr(x, torch.float32), y.data_ptr(), _stream_ptr()))
    return y


def layernorm_fwd(x, w, b, eps=NORM_EPS, axis=0, stats=True, stream=None):
    """(y, stats): stats, for ``layernorm_bwd``, holds mean and 1 / deviation of every position (None if not asked for)."""
    if stream is not None:          # what is made belongs to the stream that works on it
        with torch.cuda.stream(stream):
            return layernorm_fwd(x, w, b, eps, axis, stats)
    rows, cols, positions = _extents(x, axis, w, b)
    y = torch.empty_like(x)
    kept = x.new_empty((2, positions)) if stats else None
    _check(lib().znn_layernorm_fwd(rows, cols, axis, eps, _ptr(x, torch.float32), _ptr(w, torch.float32), _ptr(b, torch.float32),
                                   y.data_ptr(), _ptr(kept), _stream_ptr()))
    return y, kept


@functools.lru_cache(maxsize=1024)
def layernorm_workspace_bytes(rows, cols, axis):
    b = ctypes.c_size_t(0)
    _check(lib().znn_layernorm_workspace_bytes(rows, cols, axis, ctypes.byref(b)))
    return b.value


def _norm_workspace(x, rows, cols, axis):
    """(tensor that holds it, aligned address, bytes)"""
    need = layernorm_workspace_bytes(rows, cols, axis)
    if not need:
        return None, None, 0
    ws = x.new_empty(need // 4 + 64)
    return ws, (ws.data_ptr() + 255) & ~255, need


def layernorm_bwd(gy, x, w, stats, axis=0, stream=None):
    """(gx, gw, gb) from the input and the statistics of the forward pass."""
    if stream is not None:          # what is made belongs to the stream that works on it
        with torch.cuda.stream(stream):
            return layernorm_bwd(gy, x, w, stats, axis)
    rows, cols, positions = _extents(x, axis, w)
    _same_shape(x, gy)
    if stats.numel() != 2 * positions:
        raise ValueError("expected statistics of %d positions, got %s" % (positions, tuple(stats.shape)))
    gx, gw, gb = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
    ws, at, need = _norm_workspace(x, rows, cols, axis)
    _check(lib().znn_layernorm_bwd(rows, cols, axis, _ptr(gy, torch.float32), _ptr(x, torch.float32), _ptr(w, torch.float32),
                                   _ptr(stats, torch.float32), gx.data_ptr(), gw.data_ptr(), gb.data_ptr(), at, need, _stream_ptr()))
    return gx, gw, gb


def residual_norm_fwd(h, x, w, b, p=0.0, state=None, site=0, eps=NORM_EPS, axis=0, stats=True, stream=None):
    """(r, y, stats) with r = x + dropout(h), y = layernorm(r): the end of a residual branch in one pass."""
    if stream is not None:          # what is made belongs to the stream that works on it
        with torch.cuda.stream(stream):
            return residual_norm_fwd(h, x, w, b, p, state, site, eps, axis, stats)
    rows, cols, positions = _extents(x, axis, w, b)
    _same_shape(x, h)
    r, y = torch.empty_like(x), torch.empty_like(x)
    kept = x.new_empty((2, positions)) if stats else None
    _check(lib().znn_residual_norm_fwd(rows, cols, axis, eps, p, _state_ptr(state), _site(site), _ptr(h, torch.float32),
                                       _ptr(x, torch.float32), _ptr(w, torch.float32), _ptr(b, torch.float32), r.data_ptr(),
                                       y.data_ptr(), _ptr(kept), _stream_ptr()))
    return r, y, kept


def residual_norm_bwd(gy, gr, r, w, stats, p=0.0, state=None, site=0, axis=0, stream=None):
    """(gx, gh, gw, gb): gradients of x, h and the parameters.  gr, the gradient that reaches r beside the norm, may be
    None.  Where p is 0, gh is gx."""
    if stream is not None:          # what is made belongs to the stream that works on it
        with torch.cuda.stream(stream):
            return residual_norm_bwd(gy, gr, r, w, stats, p, state, site, axis)
    rows, cols, positions = _extents(r, axis, w)
    _same_shape(r, gy, gr)
    if stats.numel() != 2 * positions:
        raise ValueError("expected statistics of %d positions, got %s" % (positions, tuple(stats.shape)))
    gx, gw, gb = torch.empty_like(r), torch.empty_like(w), torch.empty_like(w)
    gh = torch.empty_like(r) if p != 0 else None
    ws, at, need = _norm_workspace(r, rows, cols, axis)
    _check(lib().znn_residual_norm_bwd(rows, cols, axis, p, _state_ptr(state), _site(site), _ptr(gy, torch.float32),
                                       _ptr(gr, torch.float32), _ptr(r, torch.float32), _ptr(w, torch.float32), _ptr(stats, torch.float32), gx.data_ptr(),
                                       _ptr(gh), gw.data_ptr(), gb.data_ptr(), at, need, _stream_ptr()))
    return gx, gx if gh is None else gh, gw, gb


# ---------------------------------------------------------------- gated unit, gated recurrence
def _take_workspace(like, need):
    """(tensor that holds it, aligned address, bytes)"""
    if not need:
        return None, None, 0
    ws = like.new_empty(need // 4 + 64)
    return ws, (ws.data_ptr() + 255) & ~255, need


def _operands(*tensors):
    """(device pointers of fp32 tensors, None -> NULL, handle of the current stream).  Tensors have to live on the current device: the
    call runs on a stream of it."""
    pointers = []
    for t in tensors:
        if t is None:
            pointers.append(None)
            continue
        if not (t.is_cuda and t.dtype is torch.float32 and t.is_contiguous()):
            _ptr(t, torch.float32)          # says what is wrong
        if not pointers:
            device = torch._C._cuda_getDevice()
        if t.get_device() != device:
            raise ValueError("tensor lives on device %d, the current one is %d" % (t.get_device(), device))
        pointers.append(t.data_ptr())
    return pointers, torch._C._cuda_getCurrentRawStream(device)


def _gate_number(fn):
    number = GATE_FNS.get(fn)
    if number is None:
        raise ValueError("a gate function is one of %s, got %r" % (", ".join(GATE_FNS), fn))
    return number


def _gated_extents(x, w, axis):
    """(f, f', positions) of x with its features along ``axis`` and w [2 f', f], which may have axes of extent 1 behind these."""
    if axis != 0 and axis != 1:
        raise ValueError("axis must be 0 or 1, got %r" % (axis,))
    shape, ws, count = x.shape, w.shape, x.numel()
    if not shape or count < 1:
        raise ValueError("expected an array of features, got %s" % (tuple(shape),))
    f = shape[-axis]
    if len(ws) < 2 or ws[1] != f or ws[0] % 2 or w.numel() != ws[0] * f:
        raise ValueError("expected weights [2 f', %d], got %s" % (f, tuple(ws)))
    if f >> 31 or ws[0] >> 31:          # ctypes would cut them off
        raise ValueError("%d to %d features are too many" % (f, ws[0] // 2))
    return f, ws[0] // 2, count // f


def _gated_like(x, axis, features):
    return x.new_empty((features,) + x.shape[1:] if axis == 0 else x.shape[:-1] + (features,))


def _expect_shape(t, shape, what):
    if tuple(t.shape) != tuple(shape):
        raise ValueError("expected %s of shape %s, got %s" % (what, tuple(shape), tuple(t.shape)))


@functools.lru_cache(maxsize=1024)
def gated_workspace_bytes(f, fo, positions, axis, which):
    b = ctypes.c_size_t(0)
    _check(lib().znn_gated_workspace_bytes(f, fo, positions, axis, which, ctypes.byref(b)))
    return b.value


def gated_fwd(x, w, b=None, fn="silu", axis=0, kept=True, stream=None):
    """(y, kept) with y = fn(u) v, [u; v] = w x + b over the features of x: its first dimension (axis 0, images) or its last one
    (axis 1, rows of features).  kept, for ``gated_bwd``, holds u and v (None if not asked for)."""
    if stream is not None:          # what is made belongs to the stream that works on it
        with torch.cuda.stream(stream):
            return gated_fwd(x, w, b, fn, axis, kept)
    number = _gate_number(fn)
    f, fo, positions = _gated_extents(x, w, axis)
    if b is not None and b.numel() != 2 * fo:
        raise ValueError("expected %d biases, got %d" % (2 * fo, b.numel()))
    operands, on = _operands(x, w, b)
    y = _gated_like(x, axis, fo)
    both = _gated_like(x, axis, 2 * fo) if kept else None
    ws, at, need = _take_workspace(x, gated_workspace_bytes(f, fo, positions, axis, ZNN_PASS_FWD))
    _check(lib().znn_gated_fwd(number, f, fo, positions, axis, *operands, y.data_ptr(), both.data_ptr() if kept else None, at, need, on))
    return y, both


def gated_bwd(gy, x, w, kept, fn="silu", axis=0, bias=True, need_gx=True, stream=None):
    """(gx, gw, gb) from the input and what the forward pass kept; gb is None without ``bias``, gx without ``need_gx``."""
    if stream is not None:          # what is made belongs to the stream that works on it
        with torch.cuda.stream(stream):
            return gated_bwd(gy, x, w, kept, fn, axis, bias, need_gx)
    number = _gate_number(fn)
    f, fo, positions = _gated_extents(x, w, axis)
    outer = (lambda n: (n,) + x.shape[1:]) if axis == 0 else (lambda n: x.shape[:-1] + (n,))
    _expect_shape(gy, outer(fo), "a gradient")
    _expect_shape(kept, outer(2 * fo), "kept values")
    operands, on = _operands(gy, x, w, kept)
    gx, gw = torch.empty_like(x) if need_gx else None, torch.empty_like(w)
    gb = w.new_empty(2 * fo) if bias else None
    ws, at, need = _take_workspace(x, gated_workspace_bytes(f, fo, positions, axis, ZNN_PASS_BWD))
    _check(lib().znn_gated_bwd(number, f, fo, positions, axis, *operands, _ptr(gx), gw.data_ptr(), _ptr(gb), at, need, on))
    return gx, gw, gb


def _line_extents(z, dim, h0, *others):
    """(outer, length, inner) of the lines along a dimension; h0 has a state for each of them, or is None."""
    shape = z.shape
    if not -len(shape) <= dim < len(shape):
        raise ValueError("an array of %d dimensions has no dimension %r" % (len(shape), dim))
    count = z.numel()
    if count < 1:
        raise ValueError("expected an array of lines, got %s" % (tuple(shape),))
    _same_shape(z, *others)
    dim %= len(shape)
    if h0 is not None and h0.shape != shape[:dim] + shape[dim + 1:]:
        raise ValueError("expected one state for every line along dimension %d of %s, got %s" % (dim, tuple(shape), tuple(h0.shape)))
    outer = 1
    for n in shape[:dim]:
        outer *= n
    return outer, shape[dim], count // (outer * shape[dim])


def _expect_apart(results, operands):
    """Pieces of a line are read and written side by side: a result that shares memory with anything else would be read half changed."""
    spans = [(t.data_ptr(), t.data_ptr() + 4 * t.numel()) for t in results + operands if t is not None]
    for i, (first, end) in enumerate(spans[:sum(t is not None for t in results)]):
        if any(first < other_end and other < end for other, other_end in spans[i + 1:]):
            raise ValueError("a result needs memory of its own")


@functools.lru_cache(maxsize=1024)
def recurrence_workspace_bytes(outer, length, inner):
    b = ctypes.c_size_t(0)
    _check(lib().znn_recurrence_workspace_bytes(outer, length, inner, ctypes.byref(b)))
    return b.value


def recurrence_fwd(z, x, h0=None, dim=-1, reverse=False, out=None, stream=None):
    """h with h_t = f_t h_(t-1) + (1 - f_t) x_t, f = logistic(z), along a dimension, from the state h0 (the shape without that
    dimension; None: zeros).  One step of a running sequence is a call on one step, with the last state as h0.  ``out`` (optional) receives h, in
    memory of its own."""
    if stream is not None:          # what is made belongs to the stream that works on it
        with torch.cuda.stream(stream):
            return recurrence_fwd(z, x, h0, dim, reverse, out)
    outer, length, inner = _line_extents(z, dim, h0, x, out)
    if out is not None:
        _expect_apart((out,), (z, x, h0))
    (zp, xp, sp, _), on = _operands(z, x, h0, out)
    h = torch.empty_like(z) if out is None else out
    ws, at, need = _take_workspace(z, recurrence_workspace_bytes(outer, length, inner))
    _check(lib().znn_recurrence_fwd(outer, length, inner, bool(reverse), zp, xp, sp, h.data_ptr(), at, need, on))
    return h


def recurrence_bwd(gh, z, x, h, h0=None, dim=-1, reverse=False, gz=None, gx=None, stream=None):
    """(gz, gx, gh0) from the gradient of every h and the forward pass's operands and result; gh0 is None without h0.  ``gz`` and ``gx``
    (optional) receive these, in memory of their own."""
    if stream is not None:          # what is made belongs to the stream that works on it
        with torch.cuda.stream(stream):
            return recurrence_bwd(gh, z, x, h, h0, dim, reverse, gz, gx)
    outer, length, inner = _line_extents(z, dim, h0, gh, x, h, gz, gx)
    if gz is not None or gx is not None:
        _expect_apart((gz, gx), (gh, z, x, h, h0))
    operands, on = _operands(gh, z, x, h, h0, gz, gx)
    gz = torch.empty_like(z) if gz is None else gz
    gx = torch.empty_like(x) if gx is None else gx
    gh0 = None if h0 is None else torch.empty_like(h0)
    ws, at, need = _take_workspace(z, recurrence_workspace_bytes(outer, length, inner))
    _check(lib().znn_recurrence_bwd(outer, length, inner, bool(reverse), *operands[:5], gz.data_ptr(), gx.data_ptr(), _ptr(gh0), at, need, on))
    return gz, gx, gh0


def autotune_workspace_bytes(desc: ConvDesc) -> int:
    b = ctypes.c_size_t(0)
    _check(lib().znn_autotune_workspace_bytes(ctypes.byref(desc), ctypes.byref(b)))
    return b.value


def autotune(fan_in, fan_out, image, kernel, device="cuda:0", stream=None, sparsity=(1, 1, 1)):
    """Returns (chosen mode, ms[method][pass]) and caches the choice for mode='auto' plans."""
    desc = make_desc(fan_in, fan_out, image, kernel, "auto", sparsity)
    need = autotune_workspace_bytes(desc)
    buf = torch.empty(need + 256, dtype=torch.uint8, device=device)
    aligned = (buf.data_ptr() + 255) & ~255
    chosen = ctypes.c_int32(-1)
    ms = (ctypes.c_float * 3 * 2)()
    _check(lib().znn_autotune(ctypes.byref(desc), ctypes.c_void_p(aligned), need, _stream_ptr(stream),
                              ctypes.byref(chosen), ctypes.byref(ms)))
    return chosen.value, [[ms[m][p] for p in range(3)] for m in range(2)]


def autotune_round(fan_in, fan_out, image, kernel, memory_budget=None, sparsity=(1, 1, 1), device="cuda:0",
                   stream=None):
    """Times a whole training round of the layer as direct / FFT / FFT with memoized spectra,
    leaving out what exceeds ``memory_budget`` bytes (None = no limit).  Returns
    (chosen strategy name, {name: ms}, {name: bytes})."""
    desc = make_desc(fan_in, fan_out, image, kernel, "auto", sparsity)
    b = ctypes.c_size_t(0)
    _check(lib().znn_autotune_round_workspace_bytes(ctypes.byref(desc), ctypes.byref(b)))
    budget = (1 << 62) if memory_budget is None else int(memory_budget)
    buf = torch.empty(b.value + 256, dtype=torch.uint8, device=device)
    aligned = (buf.data_ptr() + 255) & ~255
    rep = RoundReport()
    _check(lib().znn_autotune_round(ctypes.byref(desc), budget, ctypes.c_void_p(aligned), b.value,
                                    _stream_ptr(stream), ctypes.byref(rep)))
    return (STRATEGIES[rep.chosen], {n: float(rep.ms[i]) for i, n in enumerate(STRATEGIES)},
            {n: int(rep.bytes[i]) for i, n in enumerate(STRATEGIES)})


def trace_enable(on: bool):
    _check(lib().znn_trace_enable(1 if on else 0))


def trace_collect(capacity: int = 4096):
    """[(kernel role, ms)] of every launch recorded since the last call, in launch order."""
    buf = (TraceRecord * capacity)()
    n = ctypes.c_int32(0)
    _check(lib().znn_trace_collect(buf, capacity, ctypes.byref(n)))
    return [(buf[i].name.decode(), float(buf[i].ms)) for i in range(min(n.value, capacity))]
