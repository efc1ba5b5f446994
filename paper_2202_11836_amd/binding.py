"""Thin ctypes binding of the C ABI of libskystage.so: the encoder stage
(include/stage.h), the attention operators (include/attn.h), layer norm
(include/norm.h), rotary positions (include/rotary.h), AdamW (include/adamw.h) and
the host-side layer allocator (include/alloc.h).

Argument marshalling only: torch tensors supply device memory and the HIP
stream (torch.cuda.current_stream()); every step of the stage runs in the
HIP kernels of libskystage.so.  There is no fallback: if the library is not
built, loading fails with an error.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libskystage.so")

STAGE_OK, STAGE_EINVAL, STAGE_ESTATE, STAGE_ENOMEM, STAGE_EHIP = range(5)
STAGE_F32, STAGE_BF16 = 0, 1
PARAM_NAMES = ("W_qkv", "b_qkv", "W_o", "b_o", "g1", "be1",
               "W_1", "b_1", "W_2", "b_2", "g2", "be2")
SAVED_NAMES = ("X", "QKV", "CTX", "H1", "GD", "G")  # GD = GELU'(U)
KIND_PARAM, KIND_GRAD, KIND_SAVED, KIND_RECORDED_GRAD = 0, 1, 2, 3
STATUS_NAMES = {0: "OK", 1: "EINVAL", 2: "ESTATE", 3: "ENOMEM", 4: "EHIP"}

ALLOC_OK, ALLOC_EINVAL, ALLOC_ENOFIT = range(3)
ALLOC_CT_PER_LAYER, ALLOC_CT_PER_DEVICE = 0, 1
ALLOC_STATUS_NAMES = {0: "OK", 1: "EINVAL", 2: "ENOFIT"}

EXPORTED = ("alloc_coarse", "alloc_fine", "alloc_workloads", "stage_init", "stage_init_units",
            "stage_set_stream", "stage_forward", "stage_backward", "stage_param",
            "stage_grad", "stage_set_param", "stage_read", "stage_tensor_bytes",
            "stage_trace_site", "stage_trace_mask", "stage_trace_read", "stage_site_count",
            "stage_site_name", "stage_device_bytes", "stage_memory_model",
            "stage_memory_model_units", "stage_mfma_peak", "stage_record_grads",
            "stage_backward_noalloc", "stage_set_relpos", "stage_relpos", "stage_set_rotary",
            "stage_forward_cross", "stage_backward_cross",
            "stage_last_error", "stage_destroy")

EXPORTED_ATTN = ("attn_relpos_init", "attn_relpos_bucket", "attn_workspace", "attn_forward",
                 "attn_backward", "attn_last_error")

EXPORTED_OPS = ("layer_norm_workspace", "layer_norm_forward", "layer_norm_backward",
                "layer_norm_last_error", "rotary_init", "rotary_init_freqs", "rotary_forward",
                "rotary_backward", "rotary_last_error", "adamw_init", "adamw_step", "adamw_destroy",
                "adamw_last_error")

_lib = None


class AllocError(RuntimeError):
    def __init__(self, status: int, pi=None):
        super().__init__(ALLOC_STATUS_NAMES.get(status, str(status)))
        self.status = status
        self.pi = pi  # last partition index (ENOFIT)


class StageError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


class _RelPos(ctypes.Structure):  # attn_relpos
    _fields_ = [("num_buckets", ctypes.c_int), ("max_distance", ctypes.c_int),
                ("bidirectional", ctypes.c_int), ("reach", ctypes.c_int),
                ("n_borders", ctypes.c_int), ("border", ctypes.c_int * 128)]


# attn_shape: dtype, batch, seq_q, seq_k, heads, kv_heads, causal, scale and the
# strides of q, k, v, out, dout, dq, dk, dv
_ATTN_SHAPE = struct.Struct("@7if24q")


class _RotaryFreqs(ctypes.Structure):  # rotary_freqs
    _fields_ = [("rot_dim", ctypes.c_int), ("interleaved", ctypes.c_int),
                ("amplitude", ctypes.c_float), ("turns", ctypes.c_double * 32)]


class _AdamWTensor(ctypes.Structure):  # adamw_tensor
    _fields_ = [(n, ctypes.c_void_p) for n in ("param", "grad", "m", "v", "m_scale", "v_scale",
                                               "master")] + \
               [("numel", ctypes.c_int64), ("dtype", ctypes.c_int), ("grad_dtype", ctypes.c_int),
                ("state_bits", ctypes.c_int), ("weight_decay", ctypes.c_float),
                ("lr_scale", ctypes.c_float)]


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libskystage.so and declare the C signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is not built; run __graft_entry__.build() first")
    # torch ships its own HIP runtime (same soname as /opt/rocm's).  Load it
    # first so that the library binds to the runtime that owns torch's
    # device memory and streams, never to a second copy in the process.
    import torch  # noqa: F401
    lib = ctypes.CDLL(path)
    vp, i32, i64, u64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_uint64, ctypes.c_size_t
    lib.stage_init.argtypes = [i32, i32, i32, i32, u64, i32, vp, ctypes.POINTER(vp)]
    lib.stage_init.restype = i32
    lib.stage_init_units.argtypes = [i32, i32, i32, i32, i32, u64, i32, vp, ctypes.POINTER(vp)]
    lib.stage_init_units.restype = i32
    lib.stage_set_stream.argtypes = [vp, vp]
    lib.stage_set_stream.restype = i32
    lib.stage_forward.argtypes = [vp, vp, vp, i32, i32, vp]
    lib.stage_forward.restype = i32
    lib.stage_backward.argtypes = [vp, vp, vp]
    lib.stage_backward.restype = i32
    lib.stage_backward_noalloc.argtypes = [vp, vp, vp]
    lib.stage_backward_noalloc.restype = i32
    lib.stage_param.argtypes = [vp, i32, i32, ctypes.POINTER(vp), ctypes.POINTER(i64), ctypes.POINTER(i32)]
    lib.stage_param.restype = i32
    lib.stage_grad.argtypes = [vp, i32, i32, ctypes.POINTER(vp), ctypes.POINTER(i64)]
    lib.stage_grad.restype = i32
    lib.stage_set_param.argtypes = [vp, i32, i32, vp, sz]
    lib.stage_set_param.restype = i32
    lib.stage_read.argtypes = [vp, i32, i32, i32, vp, sz]
    lib.stage_read.restype = i32
    lib.stage_tensor_bytes.argtypes = [vp, i32, i32, i32]
    lib.stage_tensor_bytes.restype = sz
    lib.stage_trace_site.argtypes = [vp, i32]
    lib.stage_trace_site.restype = i32
    lib.stage_trace_mask.argtypes = [vp, u64]
    lib.stage_trace_mask.restype = i32
    lib.stage_trace_read.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(ctypes.c_double)]
    lib.stage_trace_read.restype = i32
    lib.stage_site_count.argtypes = []
    lib.stage_site_count.restype = i32
    lib.stage_site_name.argtypes = [i32]
    lib.stage_site_name.restype = ctypes.c_char_p
    lib.stage_last_error.argtypes = [vp]
    lib.stage_last_error.restype = ctypes.c_char_p
    lib.stage_destroy.argtypes = [vp]
    lib.stage_destroy.restype = None
    lib.stage_device_bytes.argtypes = [vp, ctypes.POINTER(i64)]
    lib.stage_device_bytes.restype = i32
    lib.stage_memory_model.argtypes = [i32, i32, i32, i32, i32, i32, ctypes.POINTER(i64),
                                       ctypes.POINTER(i64)]
    lib.stage_memory_model.restype = i32
    lib.stage_memory_model_units.argtypes = [i32, i32, i32, i32, i32, i32, ctypes.POINTER(i64),
                                             ctypes.POINTER(i64), ctypes.POINTER(i64)]
    lib.stage_memory_model_units.restype = i32
    lib.stage_mfma_peak.argtypes = [vp, i32, ctypes.POINTER(ctypes.c_double),
                                    ctypes.POINTER(ctypes.c_double)]
    lib.stage_mfma_peak.restype = i32
    lib.stage_record_grads.argtypes = [vp, i32]
    lib.stage_record_grads.restype = i32
    lib.stage_set_relpos.argtypes = [vp, i32, i32]
    lib.stage_set_relpos.restype = i32
    lib.stage_relpos.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(i64)]
    lib.stage_relpos.restype = i32
    lib.stage_set_rotary.argtypes = [vp, ctypes.POINTER(_RotaryFreqs)]
    lib.stage_set_rotary.restype = i32
    lib.stage_forward_cross.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp]
    lib.stage_forward_cross.restype = i32
    lib.stage_backward_cross.argtypes = [vp, vp, vp, vp]
    lib.stage_backward_cross.restype = i32
    dp, ip = ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i32)
    lib.alloc_coarse.argtypes = [i32, i32, dp, dp, ip, ip]
    lib.alloc_coarse.restype = i32
    lib.alloc_fine.argtypes = [i32, i32, dp, dp, dp, dp, dp, i32, ip, ip]
    lib.alloc_fine.restype = i32
    lib.alloc_workloads.argtypes = [i32, i32, dp, dp, dp, ip, i32, dp]
    lib.alloc_workloads.restype = i32
    rp, sh = ctypes.POINTER(_RelPos), ctypes.c_char_p  # (attn_shape: packed bytes)
    lib.attn_relpos_init.argtypes = [i32, i32, i32, rp]
    lib.attn_relpos_init.restype = i32
    lib.attn_relpos_bucket.argtypes = [rp, i64]
    lib.attn_relpos_bucket.restype = i32
    lib.attn_workspace.argtypes = [sh, rp, i32, ctypes.POINTER(sz)]
    lib.attn_workspace.restype = i32
    lib.attn_forward.argtypes = [sh, rp] + [vp] * 9 + [sz, vp]
    lib.attn_forward.restype = i32
    lib.attn_backward.argtypes = [sh, rp] + [vp] * 14 + [sz, vp]
    lib.attn_backward.restype = i32
    lib.attn_last_error.argtypes = []
    lib.attn_last_error.restype = ctypes.c_char_p
    dbl, fr = ctypes.c_double, ctypes.POINTER(_RotaryFreqs)
    lib.rotary_init.argtypes = [i32, i32, dbl, i32, dbl, i32, dbl, dbl, dbl, fr]
    lib.rotary_init.restype = i32
    lib.rotary_init_freqs.argtypes = [i32, i32, dp, dbl, fr]
    lib.rotary_init_freqs.restype = i32
    lib.adamw_init.argtypes = [ctypes.POINTER(_AdamWTensor), i32, vp, ctypes.POINTER(vp)]
    lib.adamw_init.restype = i32
    lib.adamw_destroy.argtypes = [vp]
    lib.adamw_destroy.restype = None
    for f in (lib.rotary_last_error, lib.layer_norm_last_error, lib.adamw_last_error):
        f.argtypes = []
        f.restype = ctypes.c_char_p
    # (the other calls of the three are marshalled by csrc/py/ops_call.cpp)
    _lib = lib
    return lib


def _check(handle, status: int):
    if status != STAGE_OK:
        msg = ""
        if handle:
            raw = load_library().stage_last_error(handle)
            msg = raw.decode() if raw else ""
        raise StageError(status, msg)


def _current_stream():
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


# ---------------------------------------------------------------------------
# Same names as the C ABI (argument marshalling only)
# ---------------------------------------------------------------------------

def stage_init(L: int, hidden: int, heads: int, ffn: int, seed: int, dtype: int,
               stream=None) -> ctypes.c_void_p:
    lib = load_library()
    out = ctypes.c_void_p()
    st = lib.stage_init(L, hidden, heads, ffn, seed, dtype,
                        stream if stream is not None else _current_stream(), ctypes.byref(out))
    if st != STAGE_OK:
        raise StageError(st, "stage_init: " + (lib.stage_last_error(None) or b"").decode())
    return out


def stage_init_units(first_unit: int, n_units: int, hidden: int, heads: int, ffn: int, seed: int,
                     dtype: int, stream=None) -> ctypes.c_void_p:
    lib = load_library()
    out = ctypes.c_void_p()
    st = lib.stage_init_units(first_unit, n_units, hidden, heads, ffn, seed, dtype,
                              stream if stream is not None else _current_stream(),
                              ctypes.byref(out))
    if st != STAGE_OK:
        raise StageError(st, "stage_init_units: " + (lib.stage_last_error(None) or b"").decode())
    return out


def stage_set_stream(handle, stream) -> None:
    _check(handle, load_library().stage_set_stream(handle, stream))


def stage_forward(handle, x, key_mask, batch: int, seq: int, y) -> None:
    _check(handle, load_library().stage_forward(handle, _ptr(x), _ptr(key_mask), batch, seq, _ptr(y)))


def stage_backward(handle, dy, dx) -> None:
    _check(handle, load_library().stage_backward(handle, _ptr(dy), _ptr(dx)))


def stage_backward_noalloc(handle, dy, dx) -> None:
    _check(handle, load_library().stage_backward_noalloc(handle, _ptr(dy), _ptr(dx)))


def stage_set_relpos(handle, num_buckets: int, max_distance: int) -> None:
    _check(handle, load_library().stage_set_relpos(handle, num_buckets, max_distance))


def stage_relpos(handle):
    """(table pointer, gradient pointer, elements) of the relative position bias."""
    t, g, n = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_int64()
    _check(handle, load_library().stage_relpos(handle, ctypes.byref(t), ctypes.byref(g),
                                               ctypes.byref(n)))
    return t.value, g.value, n.value


def stage_set_rotary(handle, freqs) -> None:
    """freqs: a Rotary's c, or None."""
    _check(handle, load_library().stage_set_rotary(handle, None if freqs is None else ctypes.byref(freqs)))


def stage_forward_cross(handle, x, memory, key_mask, batch: int, seq: int, mem_seq: int, y) -> None:
    _check(handle, load_library().stage_forward_cross(handle, _ptr(x), _ptr(memory), _ptr(key_mask),
                                                      batch, seq, mem_seq, _ptr(y)))


def stage_backward_cross(handle, dy, dx, dmemory) -> None:
    _check(handle, load_library().stage_backward_cross(handle, _ptr(dy), _ptr(dx), _ptr(dmemory)))


def stage_param(handle, layer: int, which: int):
    p, n, d = ctypes.c_void_p(), ctypes.c_int64(), ctypes.c_int()
    _check(handle, load_library().stage_param(handle, layer, which, ctypes.byref(p), ctypes.byref(n),
                                              ctypes.byref(d)))
    return p.value, n.value, d.value


def stage_grad(handle, layer: int, which: int):
    p, n = ctypes.c_void_p(), ctypes.c_int64()
    _check(handle, load_library().stage_grad(handle, layer, which, ctypes.byref(p), ctypes.byref(n)))
    return p.value, n.value


def stage_set_param(handle, layer: int, which: int, src) -> None:
    nbytes = src.numel() * src.element_size()
    _check(handle, load_library().stage_set_param(handle, layer, which, src.data_ptr(), nbytes))


def stage_read(handle, kind: int, layer: int, which: int, dst) -> None:
    nbytes = dst.numel() * dst.element_size()
    _check(handle, load_library().stage_read(handle, kind, layer, which, dst.data_ptr(), nbytes))


def stage_record_grads(handle, on: int) -> None:
    _check(handle, load_library().stage_record_grads(handle, int(on)))


def stage_tensor_bytes(handle, kind: int, layer: int, which: int) -> int:
    return load_library().stage_tensor_bytes(handle, kind, layer, which)


def stage_trace_site(handle, site: int) -> None:
    _check(handle, load_library().stage_trace_site(handle, site))


def stage_trace_mask(handle, mask: int) -> None:
    _check(handle, load_library().stage_trace_mask(handle, mask))


def stage_trace_read(handle):
    n, ms = ctypes.c_int(), ctypes.c_double()
    _check(handle, load_library().stage_trace_read(handle, ctypes.byref(n), ctypes.byref(ms)))
    return n.value, ms.value


def stage_site_count() -> int:
    return load_library().stage_site_count()


def stage_site_name(site: int) -> str:
    return load_library().stage_site_name(site).decode()


def stage_device_bytes(handle) -> int:
    v = ctypes.c_int64(0)
    _check(handle, load_library().stage_device_bytes(handle, ctypes.byref(v)))
    return v.value


def stage_memory_model(hidden: int, heads: int, ffn: int, batch: int, seq: int, dtype: int):
    """(per_layer, shared) device bytes of a stage after a forward of batch x seq."""
    a, b = ctypes.c_int64(0), ctypes.c_int64(0)
    _check(None, load_library().stage_memory_model(hidden, heads, ffn, batch, seq, dtype,
                                                   ctypes.byref(a), ctypes.byref(b)))
    return a.value, b.value


def stage_memory_model_units(hidden: int, heads: int, ffn: int, batch: int, seq: int, dtype: int):
    """(attn_unit, ffn_unit, shared) device bytes per half-layer unit."""
    a, b, c = ctypes.c_int64(0), ctypes.c_int64(0), ctypes.c_int64(0)
    _check(None, load_library().stage_memory_model_units(hidden, heads, ffn, batch, seq, dtype,
                                                         ctypes.byref(a), ctypes.byref(b),
                                                         ctypes.byref(c)))
    return a.value, b.value, c.value


def stage_mfma_peak(iters: int = 20000, stream=None):
    """(TFLOP/s, GHz): achievable dense bf16 MFMA rate and the shader clock
    held meanwhile, on the current device and stream."""
    t, g = ctypes.c_double(0.0), ctypes.c_double(0.0)
    st = stream if stream is not None else _current_stream()
    _check(None, load_library().stage_mfma_peak(st, iters, ctypes.byref(t), ctypes.byref(g)))
    return t.value, g.value


def stage_last_error(handle) -> str:
    raw = load_library().stage_last_error(handle)
    return raw.decode() if raw else ""


def stage_destroy(handle) -> None:
    if handle:
        load_library().stage_destroy(handle)


# ---------------------------------------------------------------------------
# Convenience wrapper
# ---------------------------------------------------------------------------

class _DeviceFloats:
    """Memory of a stage (fp32, or any type of numpy's) for torch.as_tensor; the tensor keeps the
    stage alive."""

    def __init__(self, stage, ptr, shape, typestr="<f4"):
        self.stage = stage
        self.__cuda_array_interface__ = {"data": (ptr, False), "shape": shape, "typestr": typestr,
                                         "strides": None, "version": 2}


class Stage:
    """One stage of L encoder layers on the current GPU, or, with
    first_unit / n_units, of the half-layer units [first_unit, first_unit +
    n_units) (unit 2j: attention half of layer j, unit 2j+1: its
    feed-forward half; L is then the number of layers they touch)."""

    def __init__(self, L: Optional[int], hidden: int, heads: int, ffn: int, seed: int = 0,
                 dtype: str = "bf16", first_unit: int = 0, n_units: Optional[int] = None):
        import torch
        self.hidden, self.heads, self.ffn = hidden, heads, ffn
        self._cross = None  # shapes of x and memory of the latest forward, if of cross attention
        self._tables = 0  # relative position tables that there have been
        self.dtype_name = dtype
        self.code = STAGE_BF16 if dtype == "bf16" else STAGE_F32
        self.torch_dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        if n_units is None:
            self.first_unit, self.n_units = 0, 2 * L
            self.handle = stage_init(L, hidden, heads, ffn, seed, self.code)
        else:
            self.first_unit, self.n_units = first_unit, n_units
            self.handle = stage_init_units(first_unit, n_units, hidden, heads, ffn, seed, self.code)
            L = (first_unit + n_units - 1) // 2 - first_unit // 2 + 1
        self.L = L

    def _sync_stream(self):
        stage_set_stream(self.handle, _current_stream())

    def forward(self, x, key_mask=None, out=None):
        import torch
        B, S, h = x.shape
        assert h == self.hidden and x.dtype == self.torch_dtype and x.is_cuda and x.is_contiguous()
        if key_mask is not None:
            assert key_mask.dtype == torch.uint8 and key_mask.shape == (B, S) and key_mask.is_contiguous()
        y = torch.empty_like(x) if out is None else out
        self._cross = None
        self._sync_stream()
        stage_forward(self.handle, x, key_mask, B, S, y)
        return y

    def backward(self, dy, out=None):
        import torch
        assert dy.dtype == self.torch_dtype and dy.is_cuda and dy.is_contiguous()
        dx = torch.empty_like(dy) if out is None else out
        self._sync_stream()
        stage_backward(self.handle, dy, dx)
        return dx

    def backward_noalloc(self, dy, out):
        """Backward with the partial results in the library's static
        scratch (stage_backward_noalloc); out must be given."""
        import torch
        assert dy.dtype == self.torch_dtype and dy.is_cuda and dy.is_contiguous()
        assert out is not None and out.dtype == dy.dtype and out.shape == dy.shape
        self._sync_stream()
        stage_backward_noalloc(self.handle, dy, out)
        return out

    def set_relpos(self, num_buckets: int, max_distance: int = 128):
        """Give the self attention of the stage's layers one relative position bias
        (both directions; a table of zeros), or take it out (num_buckets 0)."""
        self._sync_stream()
        self._tables += 1  # (the earlier one is gone, whatever comes of this)
        stage_set_relpos(self.handle, num_buckets, max_distance)

    def _relpos_view(self, which: int):
        import torch
        t, g, n = stage_relpos(self.handle)
        return torch.as_tensor(_DeviceFloats(self, (t, g)[which], (n // self.heads, self.heads)),
                               device="cuda")

    def relpos_table(self):
        """The bias table [num_buckets, heads], fp32, in the stage's own memory (to read
        and to update in place, until the next set_relpos)."""
        return self._relpos_view(0)

    def relpos_grad(self):
        """Its gradient of the latest backward, in the stage's own memory."""
        return self._relpos_view(1)

    def set_rotary(self, rotary):
        """Turn the queries and keys of the stage's self attention by their positions (a Rotary),
        or no longer (None)."""
        stage_set_rotary(self.handle, None if rotary is None else rotary.c)

    def _view(self, ptr, which: int, bf16: bool):
        """The stage's own memory of a parameter or gradient as a tensor."""
        import torch
        t = torch.as_tensor(_DeviceFloats(self, ptr, self._param_shape(which), "<i2" if bf16 else "<f4"),
                            device="cuda")
        if t.data_ptr() != ptr:
            raise StageError(STAGE_ESTATE, "the stage is not of the current device")
        return t.view(torch.bfloat16) if bf16 else t

    def adamw(self, weight_decay=0.01, state_bits=32, **kw):
        """An AdamW over the stage's parameters (with the bias table, where there is one) and their
        gradients of the latest backward, where they lie; its step() goes behind backward().
        weight_decay and 8-bit states are the matrices'; other arguments as AdamW's.  It is of use
        until the next set_relpos and until close()."""
        if not self.handle:
            raise StageError(STAGE_ESTATE, "the stage is closed")
        params, grads, decay, bits, names = [], [], [], [], []
        for layer in range(self.L):
            for which, name in enumerate(PARAM_NAMES):
                try:
                    p, _, d = stage_param(self.handle, layer, which)
                except StageError:  # of the half that the stage does not hold
                    continue
                matrix = len(self._param_shape(which)) == 2
                params.append(self._view(p, which, d == STAGE_BF16))
                grads.append(self._view(stage_grad(self.handle, layer, which)[0], which, False))
                decay.append(weight_decay if matrix else 0.0)
                bits.append(state_bits if matrix else 32)
                names.append((layer, name))
        try:
            table, grad = self.relpos_table(), self.relpos_grad()
        except StageError:
            pass
        else:
            params.append(table)
            grads.append(grad)
            decay.append(0.0)
            bits.append(32)
            names.append((None, "relpos_table"))
        return _StageAdamW(self, names, params, grads, weight_decay=decay, state_bits=bits, **kw)

    def forward_cross(self, x, memory, key_mask=None, out=None):
        """Cross attention of x [batch, seq, hidden] over memory [batch, mem_seq,
        hidden] (a stage of one attention half)."""
        import torch
        B, S, h = x.shape
        assert h == self.hidden and x.dtype == self.torch_dtype and x.is_cuda and x.is_contiguous()
        assert memory.dim() == 3 and memory.shape[0] == B and memory.shape[2] == h
        assert memory.dtype == x.dtype and memory.device == x.device and memory.is_contiguous()
        M = memory.shape[1]
        if key_mask is not None:
            assert key_mask.dtype == torch.uint8 and key_mask.shape == (B, M) and key_mask.is_contiguous()
        y = torch.empty_like(x) if out is None else out
        assert y.shape == x.shape and y.dtype == x.dtype and y.device == x.device and y.is_contiguous()
        self._cross = None
        self._sync_stream()
        stage_forward_cross(self.handle, x, memory, key_mask, B, S, M, y)
        self._cross = x.shape, memory.shape
        return y

    def backward_cross(self, dy, out=None, out_memory=None):
        """(dx, dmemory) of the latest forward_cross."""
        import torch
        assert dy.dtype == self.torch_dtype and dy.is_cuda and dy.is_contiguous()
        dx = torch.empty_like(dy) if out is None else out
        # (without a context the library refuses the call)
        x_shape, mem_shape = self._cross or (dy.shape, (0, 0, self.hidden))
        dmem = torch.empty(mem_shape, dtype=dy.dtype, device=dy.device) if out_memory is None else out_memory
        assert dy.shape == x_shape
        for t, shape in ((dx, x_shape), (dmem, mem_shape)):
            assert t.shape == shape and t.dtype == dy.dtype and t.device == dy.device and t.is_contiguous()
        self._sync_stream()
        stage_backward_cross(self.handle, dy, dx, dmem)
        return dx, dmem

    def _param_shape(self, which: int):
        h, f = self.hidden, self.ffn
        return {0: (3 * h, h), 1: (3 * h,), 2: (h, h), 3: (h,), 4: (h,), 5: (h,), 6: (f, h),
                7: (f,), 8: (h, f), 9: (h,), 10: (h,), 11: (h,)}[which]

    def param(self, layer: int, which: int):
        import torch
        _, n, d = stage_param(self.handle, layer, which)
        dt = torch.bfloat16 if d == STAGE_BF16 else torch.float32
        out = torch.empty(self._param_shape(which), dtype=dt, device="cuda")
        self._sync_stream()
        stage_read(self.handle, KIND_PARAM, layer, which, out)
        return out

    def grad(self, layer: int, which: int):
        import torch
        out = torch.empty(self._param_shape(which), dtype=torch.float32, device="cuda")
        self._sync_stream()
        stage_read(self.handle, KIND_GRAD, layer, which, out)
        return out

    def set_param(self, layer: int, which: int, value):
        import torch
        _, n, d = stage_param(self.handle, layer, which)
        dt = torch.bfloat16 if d == STAGE_BF16 else torch.float32
        v = value.to(dtype=dt).contiguous()
        assert v.numel() == n
        self._sync_stream()
        stage_set_param(self.handle, layer, which, v)

    def saved(self, layer: int, which: int, tokens: int):
        import torch
        width = {0: self.hidden, 1: (1 if self._cross else 3) * self.hidden, 2: self.hidden,
                 3: self.hidden, 4: self.ffn, 5: self.ffn}[which]
        out = torch.empty((tokens, width), dtype=self.torch_dtype, device="cuda")
        self._sync_stream()
        stage_read(self.handle, KIND_SAVED, layer, which, out)
        return out

    def record_grads(self, on: bool = True):
        """Record the gradient reaching each layer's output in later
        backward passes (from the next forward on)."""
        stage_record_grads(self.handle, 1 if on else 0)

    def recorded_grad(self, layer: int, tokens: int):
        """fp32 [tokens, hidden] gradient that reached `layer`'s output in
        the latest backward."""
        import torch
        out = torch.empty((tokens, self.hidden), dtype=torch.float32, device="cuda")
        self._sync_stream()
        stage_read(self.handle, KIND_RECORDED_GRAD, layer, 0, out)
        return out

    def trace(self, site_names):
        """Trace every launch of the named kernel site(s) (None: off)."""
        if site_names is None:
            site_names = []
        elif isinstance(site_names, str):
            site_names = [site_names]
        names = [stage_site_name(i) for i in range(stage_site_count())]
        mask = 0
        for n in site_names:
            mask |= 1 << names.index(n)
        self._sync_stream()
        stage_trace_mask(self.handle, mask)

    def device_bytes(self) -> int:
        return stage_device_bytes(self.handle)

    def trace_read(self):
        """(launches, total_ms) of the traced site since trace() / the last read."""
        self._sync_stream()
        return stage_trace_read(self.handle)

    def close(self):
        if getattr(self, "handle", None):
            stage_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---------------------------------------------------------------------------
# Attention operators (include/attn.h)
# ---------------------------------------------------------------------------
def _attn_check(status: int) -> None:
    if status != STAGE_OK:
        raise StageError(status, (load_library().attn_last_error() or b"").decode())


class RelPos:
    """Buckets of a relative position bias (attn_relpos): num_buckets over both
    directions (bidirectional), or for the keys at or before a query only;
    distances from max_distance on share the last one."""

    def __init__(self, num_buckets: int = 32, max_distance: int = 128, bidirectional: bool = True):
        self.num_buckets, self.max_distance = int(num_buckets), int(max_distance)
        self.bidirectional = bool(bidirectional)
        self.c = _RelPos()
        _attn_check(load_library().attn_relpos_init(self.num_buckets, self.max_distance,
                                                    int(self.bidirectional), ctypes.byref(self.c)))
        self.ref, self.addr = ctypes.byref(self.c), ctypes.addressof(self.c)

    def __reduce__(self):  # (a copy holds buckets of its own)
        return RelPos, (self.num_buckets, self.max_distance, self.bidirectional)

    def bucket(self, distance: int) -> int:
        """Bucket of key position - query position."""
        return load_library().attn_relpos_bucket(ctypes.byref(self.c), int(distance))


_attn_module = None


def _attn_setup():
    """csrc/py/attn_call.cpp, which checks and marshals the tensors of a call."""
    global _attn_module
    import torch
    lib = load_library()
    try:
        from . import _attn_call
    except ImportError as e:
        raise RuntimeError("_attn_call is not built; run __graft_entry__.build() first "
                           "(it needs Python's headers)") from e
    _attn_call.setup(*(ctypes.cast(f, ctypes.c_void_p).value
                       for f in (lib.attn_workspace, lib.attn_forward, lib.attn_backward,
                                 lib.attn_last_error)),
                     StageError, torch.bfloat16, torch.float32, torch.uint8, torch.int32,
                     torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream,
                     lambda n, dev: torch.empty(n, dtype=torch.uint8, device=dev))
    _attn_module = _attn_call
    return _attn_module


def _attn_on(dev, fn, *args):
    """The call again, on the device that it gave as the tensors' own."""
    import torch
    with torch.cuda.device(dev):
        return fn(*args)


def attn_forward(q, k, v, key_mask=None, scale=None, causal=False, q_pos=None, relpos=None,
                 table=None, out=None, lse=None):
    """Attention of q [batch, seq_q, heads, 64] over k, v [batch, seq_k, kv_heads, 64]
    (fp32 or bf16, any strides that leave a head's 64 values side by side):
    returns out, shaped like q, and lse [batch, heads, seq_q] fp32, which
    attn_backward takes.

    key_mask   uint8 [batch, seq_k], 1 = attend (None: every key)
    scale      of the scores (None: 1 / 8)
    causal     query i sees the keys at positions up to i + q_pos
    q_pos      int32 [batch], position of query 0 on the key axis (None: 0)
    relpos, table   a RelPos and its fp32 [num_buckets, heads] biases
    out, lse   where to write

    A query without a key gets zeros and lse = -inf.  Runs on the current stream
    of q's device."""
    fn = (_attn_module or _attn_setup()).forward
    r = fn(q, k, v, key_mask, scale, causal, q_pos, relpos, table, out, lse)
    return r if r.__class__ is tuple else _attn_on(r, fn, q, k, v, key_mask, scale, causal, q_pos,
                                                   relpos, table, out, lse)


def attn_backward(q, k, v, out, lse, dout, key_mask=None, scale=None, causal=False, q_pos=None,
                  relpos=None, table=None, dq=None, dk=None, dv=None, dtable=None):
    """Gradients of <out, dout> for attn_forward's arguments, out and lse: returns
    dq, dk, dv and dtable (None without a table), written where given.  dtable=False
    leaves the table's gradient out (a table that is not trained): None is returned."""
    fn = (_attn_module or _attn_setup()).backward
    r = fn(q, k, v, out, lse, dout, key_mask, scale, causal, q_pos, relpos, table, dq, dk, dv, dtable)
    return r if r.__class__ is tuple else _attn_on(r, fn, q, k, v, out, lse, dout, key_mask, scale,
                                                   causal, q_pos, relpos, table, dq, dk, dv, dtable)


# ---------------------------------------------------------------------------
# Layer norm (include/norm.h), rotary positions (include/rotary.h), AdamW (include/adamw.h)
# ---------------------------------------------------------------------------
_ops_module = None


def _ops_setup():
    """csrc/py/ops_call.cpp, which checks and marshals the tensors of a call."""
    global _ops_module
    import torch
    lib = load_library()
    try:
        from . import _ops_call
    except ImportError as e:
        raise RuntimeError("_ops_call is not built; run __graft_entry__.build() first "
                           "(it needs Python's and torch's headers)") from e
    _ops_call.setup(*(ctypes.cast(f, ctypes.c_void_p).value
                      for f in (lib.layer_norm_workspace, lib.layer_norm_forward,
                                lib.layer_norm_backward, lib.layer_norm_last_error,
                                lib.rotary_forward, lib.rotary_backward, lib.rotary_last_error,
                                lib.adamw_step, lib.adamw_last_error)),
                    StageError, torch.bfloat16, torch.float32, torch.uint8, torch.int32,
                    torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream,
                    lambda n, dev: torch.empty(n, dtype=torch.uint8, device=dev))
    _ops_module = _ops_call
    return _ops_module


def layer_norm_forward(x, gamma=None, beta=None, residual=None, eps=1e-12, out=None, total=None,
                       mean=None, rstd=None):
    """Layer norm over the last dimension of x (fp32 or bf16, rows that may lie apart): returns
    out, total, mean and rstd, of which layer_norm_backward takes the last three.

    gamma, beta   fp32 [width] (None: 1 and 0)
    residual      added to x first; total is then that sum, as it is stored, else x
    out, total, mean, rstd   where to write; out and total may be x or residual

    Runs on the current stream of x's device."""
    fn = (_ops_module or _ops_setup()).norm_forward
    r = fn(x, gamma, beta, residual, eps, out, total, mean, rstd)
    return r if r.__class__ is tuple else _attn_on(r, fn, x, gamma, beta, residual, eps, out, total,
                                                   mean, rstd)


def layer_norm_backward(dy, total, gamma, mean, rstd, dtotal=None, dx=None, dgamma=None, dbeta=None):
    """Gradients of <out, dy> + <total, dtotal> for layer_norm_forward's total, mean and rstd:
    returns dx (x's and the residual's), dgamma and dbeta (fp32), written where given; dx may be
    dy, dtotal or total.  False for one of them leaves it out: None is returned in its place."""
    fn = (_ops_module or _ops_setup()).norm_backward
    r = fn(dy, total, gamma, mean, rstd, dtotal, dx, dgamma, dbeta)
    return r if r.__class__ is tuple else _attn_on(r, fn, dy, total, gamma, mean, rstd, dtotal, dx,
                                                   dgamma, dbeta)


class Rotary:
    """Frequencies of rotary positions (rotary_freqs): the first rot_dim of a head's 64 values
    turn in pairs, (i, rot_dim / 2 + i) (layout "half") or (2 i, 2 i + 1) ("interleaved"), pair i
    by base^(-2 i / rot_dim) a position, all times amplitude.

    scaling   for contexts `factor` times those of original_len positions: "linear" (positions
              squeezed), "base" (a larger base) or "parts" (pairs that make fewer than `low`
              turns in original_len squeezed, those of more than `high` not, others in part)
    freqs     rot_dim / 2 frequencies of the caller's instead, in radians a position"""

    LAYOUTS = ("half", "interleaved")
    SCALINGS = (None, "linear", "base", "parts")

    def __init__(self, rot_dim: int = 64, base: float = 10000.0, layout: str = "half", scaling=None,
                 factor: float = 1.0, original_len: int = 0, low: float = 1.0, high: float = 32.0,
                 amplitude: float = 1.0, freqs=None):
        self._args = (rot_dim, base, layout, scaling, factor, original_len, low, high, amplitude,
                      None if freqs is None else tuple(float(f) for f in freqs))
        freqs = self._args[-1]
        if layout not in self.LAYOUTS:
            raise StageError(STAGE_EINVAL, f"layout must be one of {self.LAYOUTS}")
        if scaling not in self.SCALINGS:
            raise StageError(STAGE_EINVAL, f"scaling must be one of {self.SCALINGS}")
        if freqs is not None and (scaling is not None or len(freqs) != rot_dim // 2):
            raise StageError(STAGE_EINVAL, "freqs takes rot_dim / 2 frequencies and no scaling")
        self.rot_dim, self.layout, self.amplitude = int(rot_dim), layout, float(amplitude)
        self.c = _RotaryFreqs()
        lib, inter = load_library(), self.LAYOUTS.index(layout)
        if freqs is None:
            st = lib.rotary_init(self.rot_dim, inter, base, self.SCALINGS.index(scaling), factor,
                                 int(original_len), low, high, amplitude, ctypes.byref(self.c))
        else:
            st = lib.rotary_init_freqs(self.rot_dim, inter, (ctypes.c_double * max(len(freqs), 1))(*freqs),
                                       amplitude, ctypes.byref(self.c))
        if st != STAGE_OK:
            raise StageError(st, (lib.rotary_last_error() or b"").decode())
        self.addr = ctypes.addressof(self.c)

    def __reduce__(self):  # (a copy holds frequencies of its own)
        return Rotary, self._args


def rotary_forward(rotary, q, k=None, pos=None, q_out=None, k_out=None):
    """q [batch, seq, heads, 64] and k [batch, seq, kv_heads, 64] (fp32 or bf16, any strides
    that leave a head's 64 values side by side) turned by their positions: returns q_out and
    k_out (None without k), written where given; q_out may be q and k_out k.

    pos   int32 [batch], position of token 0 of each sequence, or [batch, seq], of each token
          (None: 0, 1, ...)

    Runs on the current stream of q's device."""
    fn = (_ops_module or _ops_setup()).rotary
    r = fn(False, rotary, q, k, pos, q_out, k_out)
    return r if r.__class__ is tuple else _attn_on(r, fn, False, rotary, q, k, pos, q_out, k_out)


def rotary_backward(rotary, dq, dk=None, pos=None, q_out=None, k_out=None):
    """Gradients of rotary_forward's q and k from those of its outputs, dq and dk (turned back,
    times the same amplitude), with the same rotary and pos: returns both, written where given."""
    fn = (_ops_module or _ops_setup()).rotary
    r = fn(True, rotary, dq, dk, pos, q_out, k_out)
    return r if r.__class__ is tuple else _attn_on(r, fn, True, rotary, dq, dk, pos, q_out, k_out)


class AdamW:
    """AdamW over many tensors at once (adamw.h): step() updates params, each with the gradient
    in grads, in place, in one launch (two with max_norm).

    params, grads   lists of contiguous fp32 or bf16 tensors of one GPU; the gradients' memory
                    is read by every step.  A step is refused once one of the tensors (or of
                    the states) is of other memory (its .data set, its module cast): make
                    another AdamW then, of this one's .state
    eps             1e-30 or more
    weight_decay, lr_scale   a number, or one for each tensor
    state_bits      32 or 8, or a list of them: fp32 states, or e4m3 and e5m2 with a scale for
                    each 256 elements
    master          bf16 parameters have fp32 copies that take the updates (False: none, the
                    parameters are rounded at random in proportion)
    state           the states to go on with (another AdamW's .state, say), held in place; None:
                    new ones

    Steps of one AdamW go one after the other; a captured step counts on with each replay, for which
    the AdamW has to be there still, and open.  Autograd's version counters do not see a step: a
    backward pass that needs a parameter's earlier value takes the new one, where after an in-place
    operation of torch's it were refused.

    state: a dict of lists, an entry for each tensor: "exp_avg", "exp_avg_sq" (fp32, or
    float8_e4m3fn and float8_e5m2), "exp_avg_scale", "exp_avg_sq_scale" (8 bits: fp32, one for
    256 elements, else None), "master" (fp32 or None); and "steps", int64 [1] on the GPU."""

    LISTS = ("exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale", "master")

    def __init__(self, params, grads, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, lr_scale=1.0,
                 state_bits=32, master=True, state=None):
        import torch
        self.handle = None
        self.params, self.grads, n = list(params), list(grads), len(params)
        self.betas, self.eps = (float(betas[0]), float(betas[1])), float(eps)
        self.device = self.params[0].device if n else torch.device("cuda", torch.cuda.current_device())

        def each(name, v):
            v = list(v) if isinstance(v, (list, tuple)) else [v] * n
            if len(v) != n:
                raise StageError(STAGE_EINVAL, f"{name}: {len(v)} values for {n} tensors")
            return v

        decay, scale = each("weight_decay", weight_decay), each("lr_scale", lr_scale)
        self.state_bits = [int(b) for b in each("state_bits", state_bits)]
        if len(self.grads) != n:
            raise StageError(STAGE_EINVAL, f"{len(self.grads)} gradients for {n} tensors")
        if any(b not in (8, 32) for b in self.state_bits):
            raise StageError(STAGE_EINVAL, "state_bits must be 32 or 8")
        types = (torch.float32, torch.bfloat16)
        for i, (p, g) in enumerate(zip(self.params, self.grads)):
            self._fits(f"params[{i}]", p, p.shape, types)
            self._fits(f"grads[{i}]", g, p.shape, types)
        self.state = self._new_state(bool(master)) if state is None else self._given_state(state)
        self.norm = torch.zeros(1, device=self.device)
        self._make(decay, scale)
        self._hold()

    def _hold(self):
        """The handle has addresses: their memory stays, whatever becomes of the lists or of a tensor's
        .data, and step() looks at the tensors themselves, whether they still are of that memory."""
        lists = [self.params, self.grads] + [self.state[n] for n in self.LISTS] + [[self.state["steps"]]]
        given = tuple(t for ts in lists for t in ts if t is not None)
        self._held, places = (_ops_module or _ops_setup()).hold(given)
        self._given = given, places

    def _name(self, t):
        """Of one of the tensors given."""
        for n, ts in [("params", self.params), ("grads", self.grads)] + [(n, self.state[n]) for n in self.LISTS]:
            for i, x in enumerate(ts):
                if x is t:
                    return f"{n}[{i}]"
        return "steps" if t is self.state["steps"] else "a tensor"

    def _fits(self, name, t, shape, types):
        if t.dtype not in types or t.device != self.device or not t.is_cuda or not t.is_contiguous() or \
                tuple(t.shape) != tuple(shape):
            raise StageError(STAGE_EINVAL, f"{name} must be contiguous {' or '.join(map(str, types))} "
                                           f"{list(shape)} on {self.device}")

    def _types(self, i):
        """(type and shape of each state of tensor i or None) by name."""
        import torch
        p, eight = self.params[i], self.state_bits[i] == 8
        blocks = ((p.numel() + 255) // 256,)
        return {"exp_avg": (torch.float8_e4m3fn if eight else torch.float32, p.shape),
                "exp_avg_sq": (torch.float8_e5m2 if eight else torch.float32, p.shape),
                "exp_avg_scale": (torch.float32, blocks) if eight else None,
                "exp_avg_sq_scale": (torch.float32, blocks) if eight else None,
                "master": (torch.float32, p.shape) if p.dtype == torch.bfloat16 else None}

    def _new_state(self, master):
        import torch
        s = {n: [] for n in self.LISTS}
        for i, p in enumerate(self.params):
            for n, t in self._types(i).items():
                if t is None or (n == "master" and not master):
                    s[n].append(None)
                elif n == "master":
                    s[n].append(p.detach().float())
                else:
                    s[n].append(torch.zeros(t[1], device=self.device).to(t[0]))
        s["steps"] = torch.zeros(1, dtype=torch.int64, device=self.device)
        return s

    def _given_state(self, state):
        import torch
        s = {n: list(state[n]) for n in self.LISTS}
        s["steps"] = state["steps"]
        self._fits("steps", s["steps"], (1,), (torch.int64,))
        for n in self.LISTS:
            if len(s[n]) != len(self.params):
                raise StageError(STAGE_EINVAL, f"{n}: {len(s[n])} entries for {len(self.params)} tensors")
        for i in range(len(self.params)):
            for n, t in self._types(i).items():
                if t is None or (n == "master" and s[n][i] is None):
                    if s[n][i] is not None:
                        raise StageError(STAGE_EINVAL, f"{n}[{i}] must be None")
                elif s[n][i] is None:
                    raise StageError(STAGE_EINVAL, f"{n}[{i}] is missing")
                else:
                    self._fits(f"{n}[{i}]", s[n][i], t[1], (t[0],))
        return s

    def _make(self, decay, scale):
        import torch
        code = {torch.float32: STAGE_F32, torch.bfloat16: STAGE_BF16}
        table = (_AdamWTensor * max(len(self.params), 1))()
        for i, (p, g) in enumerate(zip(self.params, self.grads)):
            m, v, ms, vs, w = (self.state[n][i] for n in self.LISTS)
            table[i] = _AdamWTensor(_ptr(p), _ptr(g), _ptr(m), _ptr(v), _ptr(ms), _ptr(vs), _ptr(w), p.numel(),
                                    code[p.dtype], code[g.dtype], self.state_bits[i], decay[i], scale[i])
        out, lib = ctypes.c_void_p(), load_library()
        with torch.cuda.device(self.device):
            st = lib.adamw_init(table, len(self.params), _ptr(self.state["steps"]), ctypes.byref(out))
        if st != STAGE_OK:
            raise StageError(st, (lib.adamw_last_error() or b"").decode())
        self.handle = out.value

    def step(self, lr, max_norm=None):
        """One step at rate lr (a number, or fp32 [1] on the GPU that the step reads, so that a
        captured one follows it) on the current stream.  max_norm: gradients are clipped by their
        global norm; returns that norm before clipping (fp32 [1] on the GPU, the same tensor for
        every step), else None.  With max_norm a step whose norm is not finite changes nothing."""
        fn, dev = (_ops_module or _ops_setup()).adamw, self.device.index
        a = (self.handle or 0, dev, lr, self.betas[0], self.betas[1], self.eps, max_norm, self.norm, *self._given)
        r = fn(*a)
        if r.__class__ is tuple:
            raise StageError(STAGE_EINVAL,
                             f"{self._name(self._given[0][r[0]])} has other memory than when the AdamW was made")
        if r is not None:
            _attn_on(r, fn, *a)
        return None if max_norm is None else self.norm

    def reset_master(self):
        """The master copies as the parameters now are (after something else changed those)."""
        for p, w in zip(self.params, self.state["master"]):
            if w is not None:
                w.copy_(p.detach())

    def __reduce__(self):  # (two of one handle would both free it)
        raise TypeError("an AdamW is not copied or pickled: make another one, of copies of its .state")

    def close(self):
        if getattr(self, "handle", None):
            load_library().adamw_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class _StageAdamW(AdamW):
    """Of a stage's parameters: names[i] is the (layer, name) of params[i]."""

    def __init__(self, stage, names, params, grads, **kw):
        self.stage, self.names, self._tables = stage, names, stage._tables
        super().__init__(params, grads, **kw)

    def _of_use(self):
        if not self.stage.handle:
            raise StageError(STAGE_ESTATE, "the stage is closed")
        if self.stage._tables != self._tables:
            raise StageError(STAGE_ESTATE, "the stage's bias table is another one since")

    def step(self, lr, max_norm=None):
        self._of_use()
        return super().step(lr, max_norm)

    def reset_master(self):
        self._of_use()
        super().reset_master()


# ---------------------------------------------------------------------------
# Layer allocator (host code; include/alloc.h)
# ---------------------------------------------------------------------------
def _dvec(v):
    v = [float(x) for x in v]
    return (ctypes.c_double * max(len(v), 1))(*v), len(v)


def _ivec(v, n=None):
    v = [int(x) for x in v] if v is not None else [0] * n
    return (ctypes.c_int * max(len(v), 1))(*v)


def alloc_coarse(lm, dm):
    """Algorithm 1: returns (pi, sweeps); raises AllocError (with .pi, the
    last partition index, for ENOFIT)."""
    a_lm, L = _dvec(lm)
    a_dm, D = _dvec(dm)
    pi = _ivec(None, D + 1)
    n = ctypes.c_int(0)
    st = load_library().alloc_coarse(L, D, a_lm, a_dm, pi, ctypes.byref(n))
    if st != ALLOC_OK:
        raise AllocError(st, list(pi) if st == ALLOC_ENOFIT else None)
    return list(pi), n.value


def alloc_fine(dt, dm, ct, lf, lm, pi, max_iter: int):
    """Algorithm 2 from partition pi: returns (tuned pi, rounds)."""
    a_dt, D = _dvec(dt)
    a_dm, _ = _dvec(dm)
    a_ct, _ = _dvec(ct)
    a_lf, L = _dvec(lf)
    a_lm, _ = _dvec(lm)
    p = _ivec(pi)
    if len(pi) != D + 1 or len(dm) != D or len(ct) != D or len(lm) != L:
        raise AllocError(ALLOC_EINVAL)
    n = ctypes.c_int(0)
    st = load_library().alloc_fine(L, D, a_dt, a_dm, a_ct, a_lf, a_lm, int(max_iter), p,
                                   ctypes.byref(n))
    if st != ALLOC_OK:
        raise AllocError(st)
    return list(p), n.value


def alloc_workloads(dt, ct, lf, pi, mode: int = ALLOC_CT_PER_LAYER):
    """Workload of every device under partition pi."""
    a_dt, D = _dvec(dt)
    a_ct, _ = _dvec(ct)
    a_lf, L = _dvec(lf)
    if len(pi) != D + 1 or len(ct) != D:
        raise AllocError(ALLOC_EINVAL)
    out = (ctypes.c_double * D)()
    st = load_library().alloc_workloads(L, D, a_dt, a_ct, a_lf, _ivec(pi), int(mode), out)
    if st != ALLOC_OK:
        raise AllocError(st)
    return list(out)
