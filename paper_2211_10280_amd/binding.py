"""ctypes binding of libtensair.so -- argument marshalling only.

Every function here has the name of the C entry point it forwards to
(``include/tensair.h``); PyTorch supplies device memory and the stream, nothing
else.  There is no CPU fallback: if the shared library is missing, ``lib()``
raises.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtensair.so")

F32, BF16, FP8 = 0, 1, 2
OK, EINVAL, ECAPACITY, EHIP, EDATA = 0, -1, -2, -3, -4
MAX_PEERS = 31
MAX_VOCAB = (1 << 28) - 64
MAX_DENSE = 1 << 33
STATIC_MAX_VOCAB = 1 << 21
STATIC_MAX_PEERS = 15
RESAMPLE_NEGATIVES = 1
STOCHASTIC_ROUNDING = 2

SYMBOLS = [
    "tensair_workspace_bytes", "tensair_capacity_in", "tensair_capacity_out", "tensair_model_init",
    "tensair_model_rebind", "tensair_model_alias", "tensair_pair_count", "tensair_sgns_grad",
    "tensair_dasgd_apply", "tensair_step", "tensair_status", "tensair_model_destroy",
    "tensair_last_error", "tensair_profile", "tensair_profile_read", "tensair_copy_probe",
    "tensair_prefetch", "tensair_grad_add", "tensair_dense_apply", "tensair_lookup",
    "tensair_cosine_difference", "tensair_grad_pack", "tensair_dasgd_apply_packed", "tensair_step_packed",
    "tensair_dasgd_apply_static", "tensair_stream_probe", "tensair_aligned_row_stride",
    "tensair_embed", "tensair_embed_workspace_bytes", "tensair_embed_grad", "tensair_embed_grad_dense",
    "tensair_softmax_workspace_bytes", "tensair_softmax_loss", "tensair_softmax_grad",
    "tensair_adamw_workspace_bytes", "tensair_adamw_init", "tensair_adamw_step", "tensair_adamw_step_at", "tensair_adamw_destroy",
    "tensair_norm", "tensair_norm_workspace_bytes", "tensair_norm_grad", "tensair_dropout",
    "tensair_recur_state_rows", "tensair_recur_workspace_bytes", "tensair_recur", "tensair_recur_grad", "tensair_recur_step",
    "tensair_sample_workspace_bytes", "tensair_sample",
]

PROFILE_TAGS = {1: "keys", 2: "forward", 3: "sort", 4: "segments", 5: "reduce_in", 6: "reduce_out",
                8: "apply_index", 9: "apply_update", 11: "add_index", 12: "add_rows", 14: "pack"}


class TensairError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"libtensair error {code}: {msg}")
        self.code = code


class Config(C.Structure):
    _fields_ = [("vocab", C.c_int64), ("dim", C.c_int32), ("row_stride", C.c_int32),
                ("dtype", C.c_int32), ("window", C.c_int32), ("negatives", C.c_int32),
                ("max_centers", C.c_int32), ("max_peers", C.c_int32), ("worker_id", C.c_uint32),
                ("seed", C.c_uint64), ("flags", C.c_uint32)]


class SparseRows(C.Structure):
    _fields_ = [("capacity", C.c_int64), ("n_rows", C.c_void_p), ("row_ids", C.c_void_p),
                ("row_grads", C.c_void_p)]


class SparseGrad(C.Structure):
    _fields_ = [("in_", SparseRows), ("out", SparseRows)]


class AdamwTensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("m_scale", C.c_void_p), ("v_scale", C.c_void_p), ("param_copy", C.c_void_p),
                ("n", C.c_int64), ("param_dtype", C.c_int32), ("grad_dtype", C.c_int32), ("weight_decay", C.c_float)]


_lib = None


def lib():
    """The loaded shared library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2211_10280_amd.build` "
                "(there is no fallback path)")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, u32 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint32
        L.tensair_aligned_row_stride.argtypes = [i32, i32]
        L.tensair_aligned_row_stride.restype = i32
        L.tensair_workspace_bytes.argtypes = [C.POINTER(Config)]
        L.tensair_workspace_bytes.restype = C.c_size_t
        L.tensair_capacity_in.argtypes = [C.POINTER(Config), i32]
        L.tensair_capacity_in.restype = i64
        L.tensair_capacity_out.argtypes = [C.POINTER(Config), i32]
        L.tensair_capacity_out.restype = i64
        L.tensair_model_init.argtypes = [C.POINTER(vp), C.POINTER(Config), vp, vp, C.c_int, vp, vp,
                                         C.c_size_t, vp]
        L.tensair_model_init.restype = C.c_int
        L.tensair_model_rebind.argtypes = [vp, vp, vp, u32]
        L.tensair_model_rebind.restype = C.c_int
        L.tensair_model_alias.argtypes = [vp, vp, vp]
        L.tensair_model_alias.restype = C.c_int
        L.tensair_pair_count.argtypes = [vp, i64, i64, i32]
        L.tensair_pair_count.restype = i64
        L.tensair_sgns_grad.argtypes = [vp, vp, i64, i64, i32, u32, C.POINTER(SparseGrad), vp, vp, vp, vp, vp]
        L.tensair_sgns_grad.restype = C.c_int
        L.tensair_dasgd_apply.argtypes = [vp, C.POINTER(SparseGrad), C.POINTER(SparseGrad), i32,
                                          C.c_float, vp]
        L.tensair_dasgd_apply.restype = C.c_int
        L.tensair_step.argtypes = [vp, vp, i64, i64, i32, u32, C.POINTER(SparseGrad), i32, C.c_float,
                                   C.POINTER(SparseGrad), vp, vp]
        L.tensair_step.restype = C.c_int
        L.tensair_prefetch.argtypes = [vp, vp, i64, i64, i32, u32, vp]
        L.tensair_prefetch.restype = C.c_int
        L.tensair_grad_add.argtypes = [vp, C.POINTER(SparseGrad), C.POINTER(SparseGrad), C.POINTER(SparseGrad), vp]
        L.tensair_grad_add.restype = C.c_int
        L.tensair_dense_apply.argtypes = [vp, i32, i64, C.POINTER(vp), i32, C.c_float, vp]
        L.tensair_dense_apply.restype = C.c_int
        L.tensair_lookup.argtypes = [vp, i32, vp, i64, vp, vp]
        L.tensair_lookup.restype = C.c_int
        L.tensair_cosine_difference.argtypes = [vp, vp, i32, i64, i32, i32, vp, vp]
        L.tensair_cosine_difference.restype = C.c_int
        # a packed gradient has the layout of a sparse one (its rows are bfloat16 instead of fp32)
        L.tensair_grad_pack.argtypes = [vp, C.POINTER(SparseGrad), C.POINTER(SparseGrad), vp]
        L.tensair_grad_pack.restype = C.c_int
        L.tensair_dasgd_apply_packed.argtypes = L.tensair_dasgd_apply.argtypes
        L.tensair_dasgd_apply_packed.restype = C.c_int
        L.tensair_step_packed.argtypes = [vp, vp, i64, i64, i32, u32, C.POINTER(SparseGrad), i32, C.c_float,
                                          C.POINTER(SparseGrad), C.POINTER(SparseGrad), vp, vp]
        L.tensair_step_packed.restype = C.c_int
        L.tensair_dasgd_apply_static.argtypes = [vp, vp, i64, i32, i32, i32, C.POINTER(SparseGrad),
                                                 C.POINTER(SparseGrad), i32, C.c_float, vp, vp]
        L.tensair_dasgd_apply_static.restype = C.c_int
        L.tensair_status.argtypes = [vp, vp]
        L.tensair_status.restype = C.c_int
        L.tensair_model_destroy.argtypes = [vp]
        L.tensair_model_destroy.restype = C.c_int
        L.tensair_profile.argtypes = [vp, C.c_int]
        L.tensair_profile.restype = C.c_int
        L.tensair_profile_read.argtypes = [vp, vp, vp, i32]
        L.tensair_profile_read.restype = C.c_int
        L.tensair_copy_probe.argtypes = [vp, vp, C.c_size_t, vp]
        L.tensair_copy_probe.restype = C.c_int
        L.tensair_stream_probe.argtypes = [vp, vp, C.c_size_t, i32, vp]
        L.tensair_stream_probe.restype = C.c_int
        f32, sz = C.c_float, C.c_size_t
        L.tensair_embed.argtypes = [vp, i32, i64, i32, i64, vp, i64, f32, vp, i32, i64, vp, vp]
        L.tensair_embed.restype = C.c_int
        L.tensair_embed_workspace_bytes.argtypes = [i64, i32, i64]
        L.tensair_embed_workspace_bytes.restype = sz
        L.tensair_embed_grad.argtypes = [vp, i64, vp, i32, i64, i64, i32, f32, C.POINTER(SparseRows), vp, sz, vp, vp]
        L.tensair_embed_grad.restype = C.c_int
        L.tensair_embed_grad_dense.argtypes = [vp, i64, vp, i32, i64, i64, i32, f32, vp, i32, i64, i32, vp, sz, vp, vp]
        L.tensair_embed_grad_dense.restype = C.c_int
        L.tensair_softmax_workspace_bytes.argtypes = [i64, i64, i32, i32, i32]
        L.tensair_softmax_workspace_bytes.restype = sz
        L.tensair_softmax_loss.argtypes = [vp, i64, vp, i64, i32, i64, i64, i32, vp, i32, f32, vp, vp, vp, sz, vp, vp]
        L.tensair_softmax_loss.restype = C.c_int
        L.tensair_softmax_grad.argtypes = [vp, i64, vp, i64, i32, i64, i64, i32, vp, i32, f32, vp, vp, vp, i64, vp, i64,
                                           vp, sz, vp, vp]
        L.tensair_softmax_grad.restype = C.c_int
        L.tensair_adamw_workspace_bytes.argtypes = [C.POINTER(AdamwTensor), i32, i32]
        L.tensair_adamw_workspace_bytes.restype = sz
        L.tensair_adamw_init.argtypes = [C.POINTER(vp), C.POINTER(AdamwTensor), i32, i32, vp, sz, vp]
        L.tensair_adamw_init.restype = C.c_int
        L.tensair_adamw_step.argtypes = [vp, C.c_double, i64, C.c_double, C.c_double, C.c_double, vp, vp]
        L.tensair_adamw_step.restype = C.c_int
        L.tensair_adamw_step_at.argtypes = [vp, vp, vp, C.c_double, C.c_double, C.c_double, vp, vp]
        L.tensair_adamw_step_at.restype = C.c_int
        L.tensair_adamw_destroy.argtypes = [vp]
        L.tensair_adamw_destroy.restype = C.c_int
        u64, f64 = C.c_uint64, C.c_double
        L.tensair_norm.argtypes = [vp, i32, i64, i64, i32, vp, vp, f32, vp, i32, i64, vp, vp, vp]
        L.tensair_norm.restype = C.c_int
        L.tensair_norm_workspace_bytes.argtypes = [i64, i32]
        L.tensair_norm_workspace_bytes.restype = sz
        L.tensair_norm_grad.argtypes = [vp, i32, i64, vp, i32, i64, i64, i32, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp, sz, vp]
        L.tensair_norm_grad.restype = C.c_int
        L.tensair_dropout.argtypes = [vp, i32, i64, i64, i32, f64, u64, u32, i64, vp, vp, i64, vp, i32, i64, vp]
        L.tensair_dropout.restype = C.c_int
        L.tensair_recur_state_rows.argtypes = [i64]
        L.tensair_recur_state_rows.restype = i64
        L.tensair_recur_workspace_bytes.argtypes = [i64, i32]
        L.tensair_recur_workspace_bytes.restype = sz
        L.tensair_recur.argtypes = [vp, i64, vp, i64, i32, i64, i32, vp, i64, vp, vp, i64, vp, vp, vp, sz, vp, vp]
        L.tensair_recur.restype = C.c_int
        L.tensair_recur_grad.argtypes = [vp, i64, vp, i64, i32, i64, i32, vp, i64, vp, vp, vp, i64, vp, vp, i64, vp, i64, vp, vp, sz, vp, vp]
        L.tensair_recur_grad.restype = C.c_int
        L.tensair_recur_step.argtypes = [vp, i64, vp, i64, i32, i64, i32, vp, i64, vp, i64, vp, i64, vp, vp]
        L.tensair_recur_step.restype = C.c_int
        L.tensair_sample_workspace_bytes.argtypes = [i64, i64]
        L.tensair_sample_workspace_bytes.restype = sz
        L.tensair_sample.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp]
        L.tensair_sample.restype = C.c_int
        L.tensair_last_error.argtypes = []
        L.tensair_last_error.restype = C.c_char_p
        _lib = L
    return _lib


def _check(rc):
    if rc != 0:
        raise TensairError(rc, lib().tensair_last_error().decode())


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


# the current stream's handle without a Stream object (which takes 3 us a call), where torch has it: the name is private
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream=None):
    if stream is None and _raw_stream is not None:
        return C.c_void_p(_raw_stream(torch.cuda.current_device()))
    return C.c_void_p((stream if stream is not None else torch.cuda.current_stream()).cuda_stream)


# ---------------------------------------------------------------- device buffers
class GradBuffers:
    """Device memory of one tensair_sparse_grad (caller-owned, as the ABI asks)."""

    ROWS = torch.float32

    def __init__(self, cap_in: int, cap_out: int, dim: int, device="cuda"):
        self.dim = dim
        self.n_rows = torch.zeros(2, dtype=torch.int32, device=device)     # [in, out]
        self.in_ids = torch.empty(max(cap_in, 1), dtype=torch.int32, device=device)
        self.in_rows = torch.empty((max(cap_in, 1), dim), dtype=self.ROWS, device=device)
        self.out_ids = torch.empty(max(cap_out, 1), dtype=torch.int32, device=device)
        self.out_rows = torch.empty((max(cap_out, 1), dim), dtype=self.ROWS, device=device)
        self.cap_in, self.cap_out = cap_in, cap_out
        self.c = SparseGrad()
        self.c.in_ = SparseRows(cap_in, self.n_rows.data_ptr(), self.in_ids.data_ptr(), self.in_rows.data_ptr())
        self.c.out = SparseRows(cap_out, self.n_rows.data_ptr() + 4, self.out_ids.data_ptr(),
                                self.out_rows.data_ptr())

    def sizes(self):
        n = self.n_rows.cpu()
        return int(n[0]), int(n[1])

    def to_host(self):
        """((ids_in, rows_in), (ids_out, rows_out)) as numpy arrays trimmed to n_rows."""
        ui, uo = self.sizes()
        return ((self.in_ids[:ui].cpu().numpy(), self.in_rows[:ui].cpu().numpy()),
                (self.out_ids[:uo].cpu().numpy(), self.out_rows[:uo].cpu().numpy()))

    def ids_to_host(self):
        """(ids_in, ids_out) as numpy arrays trimmed to n_rows (the rows stay on the device)."""
        ui, uo = self.sizes()
        return self.in_ids[:ui].cpu().numpy(), self.out_ids[:uo].cpu().numpy()

    def load(self, ids_in, rows_in, ids_out, rows_out):
        """Fill from host arrays (e.g. a gradient received from a peer)."""
        ui, uo = len(ids_in), len(ids_out)
        assert ui <= self.cap_in and uo <= self.cap_out
        self.in_ids[:ui] = torch.from_numpy(np.ascontiguousarray(ids_in, dtype=np.int32)).to(self.in_ids.device)
        self.out_ids[:uo] = torch.from_numpy(np.ascontiguousarray(ids_out, dtype=np.int32)).to(self.in_ids.device)
        if ui:
            self.in_rows[:ui] = torch.from_numpy(np.ascontiguousarray(rows_in, dtype=np.float32)).to(self.in_ids.device)
        if uo:
            self.out_rows[:uo] = torch.from_numpy(np.ascontiguousarray(rows_out, dtype=np.float32)).to(self.in_ids.device)
        self.n_rows.copy_(torch.tensor([ui, uo], dtype=torch.int32))


class PackedBuffers(GradBuffers):
    """Device memory of one tensair_packed_grad: the same, with bfloat16 rows (kept as int16 bits)."""
    ROWS = torch.int16

    def to_host(self):
        (ii, ri), (io, ro) = super().to_host()
        return (ii, ri.view(np.uint16)), (io, ro.view(np.uint16))

    def load(self, ids_in, bits_in, ids_out, bits_out):
        """Fill from host arrays; the rows are uint16 bfloat16 bits."""
        ui, uo = len(ids_in), len(ids_out)
        assert ui <= self.cap_in and uo <= self.cap_out
        dev = self.in_ids.device
        self.in_ids[:ui] = torch.from_numpy(np.ascontiguousarray(ids_in, dtype=np.int32)).to(dev)
        self.out_ids[:uo] = torch.from_numpy(np.ascontiguousarray(ids_out, dtype=np.int32)).to(dev)
        if ui:
            self.in_rows[:ui] = torch.from_numpy(np.ascontiguousarray(bits_in, dtype=np.uint16).view(np.int16)).to(dev)
        if uo:
            self.out_rows[:uo] = torch.from_numpy(np.ascontiguousarray(bits_out, dtype=np.uint16).view(np.int16)).to(dev)
        self.n_rows.copy_(torch.tensor([ui, uo], dtype=torch.int32))


# ---------------------------------------------------------------- C entry points, same names
def tensair_aligned_row_stride(dim: int, dtype: int) -> int:
    n = lib().tensair_aligned_row_stride(dim, dtype)
    if n < 0:
        raise TensairError(EINVAL, "aligned_row_stride: bad dim or dtype")
    return n


def tensair_workspace_bytes(cfg: Config) -> int:
    n = lib().tensair_workspace_bytes(C.byref(cfg))
    if n == 0:
        raise TensairError(EINVAL, lib().tensair_last_error().decode())
    return n


def tensair_capacity_in(cfg: Config, n_centers: int) -> int:
    return lib().tensair_capacity_in(C.byref(cfg), n_centers)


def tensair_capacity_out(cfg: Config, n_centers: int) -> int:
    return lib().tensair_capacity_out(C.byref(cfg), n_centers)


def tensair_model_init(cfg: Config, w_in, w_out, fill_tables: bool, unigram_counts: np.ndarray,
                       workspace, stream=None):
    counts = np.ascontiguousarray(unigram_counts, dtype=np.uint64)
    h = C.c_void_p()
    _check(lib().tensair_model_init(C.byref(h), C.byref(cfg), _ptr(w_in), _ptr(w_out), int(fill_tables),
                                    counts.ctypes.data_as(C.c_void_p), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _stream(stream)))
    return h


def tensair_model_rebind(h, w_in, w_out, worker_id: int):
    _check(lib().tensair_model_rebind(h, _ptr(w_in), _ptr(w_out), worker_id))


def tensair_model_alias(h, vocab: int):
    thr = np.zeros(vocab, dtype=np.uint32)
    alias = np.zeros(vocab, dtype=np.int32)
    _check(lib().tensair_model_alias(h, thr.ctypes.data_as(C.c_void_p), alias.ctypes.data_as(C.c_void_p)))
    return thr, alias


def tensair_pair_count(h, n_tokens: int, center_begin: int, n_centers: int) -> int:
    p = lib().tensair_pair_count(h, n_tokens, center_begin, n_centers)
    if p < 0:
        raise TensairError(EINVAL, lib().tensair_last_error().decode())
    return p


def tensair_sgns_grad(h, tokens, center_begin: int, n_centers: int, epoch: int, grad: GradBuffers,
                      mean_loss=None, negatives_dbg=None, seg_offsets_in=None, seg_offsets_out=None,
                      stream=None):
    _check(lib().tensair_sgns_grad(h, _ptr(tokens), tokens.numel(), center_begin, n_centers, epoch,
                                   C.byref(grad.c), _ptr(mean_loss), _ptr(negatives_dbg),
                                   _ptr(seg_offsets_in), _ptr(seg_offsets_out), _stream(stream)))


def _peer_array(peers):
    arr = (SparseGrad * max(len(peers), 1))()
    for i, p in enumerate(peers):
        arr[i] = p.c
    return arr


def tensair_dasgd_apply(h, own, peers, lr: float, stream=None):
    arr = _peer_array(peers)
    _check(lib().tensair_dasgd_apply(h, C.byref(own.c) if own is not None else None, arr, len(peers),
                                     C.c_float(lr), _stream(stream)))


def tensair_dasgd_apply_static(w_in, w_out, dim: int, own, peers, lr: float, status=None, stream=None):
    """w_in, w_out: [vocab, row_stride] tables of the same dtype; status: int32 tensor of one element or None."""
    dt = F32 if w_in.dtype == torch.float32 else BF16
    arr = _peer_array(peers)
    _check(lib().tensair_dasgd_apply_static(_ptr(w_in), _ptr(w_out), w_in.shape[0], dim, w_in.shape[1], dt,
                                            C.byref(own.c) if own is not None else None, arr, len(peers),
                                            C.c_float(lr), _ptr(status), _stream(stream)))


def tensair_step(h, tokens, center_begin: int, n_centers: int, epoch: int, peers, lr: float,
                 own_out: GradBuffers, mean_loss=None, stream=None):
    arr = _peer_array(peers)
    _check(lib().tensair_step(h, _ptr(tokens), tokens.numel(), center_begin, n_centers, epoch, arr,
                              len(peers), C.c_float(lr), C.byref(own_out.c), _ptr(mean_loss),
                              _stream(stream)))


def tensair_grad_pack(h, g: GradBuffers, out: PackedBuffers, stream=None):
    _check(lib().tensair_grad_pack(h, C.byref(g.c), C.byref(out.c), _stream(stream)))


def tensair_dasgd_apply_packed(h, own, peers, lr: float, stream=None):
    arr = _peer_array(peers)
    _check(lib().tensair_dasgd_apply_packed(h, C.byref(own.c) if own is not None else None, arr, len(peers),
                                            C.c_float(lr), _stream(stream)))


def tensair_step_packed(h, tokens, center_begin: int, n_centers: int, epoch: int, peers, lr: float,
                        own_out: GradBuffers, own_msg_out=None, mean_loss=None, stream=None):
    arr = _peer_array(peers)
    _check(lib().tensair_step_packed(h, _ptr(tokens), tokens.numel(), center_begin, n_centers, epoch, arr,
                                     len(peers), C.c_float(lr), C.byref(own_out.c),
                                     C.byref(own_msg_out.c) if own_msg_out is not None else None, _ptr(mean_loss),
                                     _stream(stream)))


def tensair_prefetch(h, tokens, center_begin: int, n_centers: int, epoch: int, stream=None):
    _check(lib().tensair_prefetch(h, _ptr(tokens), tokens.numel(), center_begin, n_centers, epoch,
                                  _stream(stream)))


def tensair_grad_add(h, a: GradBuffers, b: GradBuffers, out: GradBuffers, stream=None):
    _check(lib().tensair_grad_add(h, C.byref(a.c), C.byref(b.c), C.byref(out.c), _stream(stream)))


def tensair_dense_apply(theta, grads, lr: float, stream=None):
    """theta: 1-D float32 or bfloat16 tensor; grads: list of float32 tensors of the same length."""
    dt = F32 if theta.dtype == torch.float32 else BF16
    arr = (C.c_void_p * max(len(grads), 1))(*[g.data_ptr() for g in grads])
    _check(lib().tensair_dense_apply(_ptr(theta), dt, theta.numel(), arr, len(grads), C.c_float(lr),
                                     _stream(stream)))


def tensair_lookup(h, table: int, ids, out, stream=None):
    _check(lib().tensair_lookup(h, table, _ptr(ids), ids.numel(), _ptr(out), _stream(stream)))


def tensair_cosine_difference(a, b, dim: int, diff, stream=None):
    """a, b: [vocab, row_stride] tables of the same dtype; diff: float32 [vocab]."""
    dt = F32 if a.dtype == torch.float32 else BF16
    _check(lib().tensair_cosine_difference(_ptr(a), _ptr(b), dt, a.shape[0], dim, a.shape[1], _ptr(diff),
                                           _stream(stream)))


# ---- a table as the input and output layer of a model
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float8_e4m3fn: FP8}


def _dtype(t, what):
    """The C dtype of a tensor or torch dtype; EINVAL for one that no entry point takes."""
    code = _DTYPES.get(t if isinstance(t, torch.dtype) else t.dtype)
    if code is None:
        raise TensairError(EINVAL, f"{what}: unknown dtype")
    return code


# The smallest calls below take the GPU less time than Python takes to check and pass their arguments: plain numbers instead of
# C objects, every attribute of a tensor asked for once (tensair_embed of 64 words, GPU and all: 7.4 -> 6.1 us a call).
def _matrix(t, rows, dim, what):
    """(address, C dtype, row stride) of a [rows, >= dim] tensor whose rows are contiguous."""
    shape, stride, code = t.shape, t.stride(), _DTYPES.get(t.dtype)
    if len(shape) != 2 or shape[0] != rows or shape[1] < dim or (stride[1] != 1 and shape[1] > 1):
        raise TensairError(EINVAL, f"{what}: expected {rows} contiguous rows of at least {dim} elements")
    if code is None:
        raise TensairError(EINVAL, f"{what}: unknown dtype")
    return t.data_ptr(), code, stride[0] if rows > 1 else max(stride[0], shape[1])


def _vector(t, n, dtype, what):
    """The address of a contiguous one-dimensional tensor of n elements."""
    if t.dtype is not dtype or t.shape != (n,) or not t.is_contiguous():
        raise TensairError(EINVAL, f"{what}: expected {n} contiguous elements of {dtype}")
    return t.data_ptr()


def _ids(t, what="ids"):
    return _vector(t, t.numel(), torch.int32, what)


def _device(t, *others):
    """The number of the GPU that a tensor is on, and all others (None: not given): the kernels take addresses as they are."""
    dev = t.get_device()
    if dev < 0:
        raise TensairError(EINVAL, "a tensor is not on a GPU")
    for x in others:
        if x is not None and x.get_device() != dev:
            raise TensairError(EINVAL, "the tensors are not on one GPU")
    return dev


def _word(t, dtype=torch.int32, what="status"):
    """The address of a status word or a scale, or None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() < 1:
        raise TensairError(EINVAL, f"{what}: expected an element of {dtype}")
    return t.data_ptr()


def _bytes(workspace):
    """The bytes of a workspace, a tensor of any type."""
    if not workspace.is_contiguous():
        raise TensairError(EINVAL, "workspace: expected a contiguous tensor")
    return workspace.numel() * workspace.element_size()


def _on(dev, stream):
    """The handle of `stream`, by default the current one of the GPU of that number."""
    return _raw_stream(dev) if stream is None and _raw_stream is not None else _stream(stream)


class RowBuffers:
    """Device memory of one tensair_sparse_rows, one table's half of a gradient message."""

    def __init__(self, capacity: int, dim: int, device="cuda"):
        self.n_rows = torch.zeros(1, dtype=torch.int32, device=device)
        self.row_ids = torch.empty(max(capacity, 1), dtype=torch.int32, device=device)
        self.rows = torch.empty((max(capacity, 1), dim), dtype=torch.float32, device=device)

    def __iter__(self):
        return iter((self.n_rows, self.row_ids, self.rows))

    def to_host(self):
        """(ids, rows) as numpy arrays trimmed to n_rows."""
        n = int(self.n_rows.item())
        return self.row_ids[:n].cpu().numpy(), self.rows[:n].cpu().numpy()


def tensair_embed(table, dim: int, ids, out, scale=1.0, status=None, stream=None):
    """table: [vocab, >= dim] float32 or bfloat16; ids: int32 [n]; out: [n, >= dim] float32 or bfloat16."""
    n, dev = ids.numel(), _device(table, ids, out, status)
    tp, td, ts = _matrix(table, table.shape[0], dim, "table")
    op, od, os_ = _matrix(out, n, dim, "out")
    rc = (_lib or lib()).tensair_embed(tp, td, table.shape[0], dim, ts, _ids(ids), n, scale, op, od, os_, _word(status), _on(dev, stream))
    if rc:
        _check(rc)


def tensair_embed_workspace_bytes(vocab: int, dim: int, n: int) -> int:
    nbytes = lib().tensair_embed_workspace_bytes(vocab, dim, n)
    if nbytes == 0:
        raise TensairError(EINVAL, lib().tensair_last_error().decode())
    return nbytes


def tensair_embed_grad(ids, d_out, dim: int, vocab: int, grad, workspace, scale=1.0, status=None, stream=None):
    """grad: RowBuffers, or (n_rows int32 [1], row_ids int32 [capacity], rows float32 [capacity, dim])."""
    n_rows, row_ids, rows = grad
    n, cap, dev = ids.numel(), row_ids.numel(), _device(d_out, ids, n_rows, row_ids, rows, workspace, status)
    dp, dd, ds = _matrix(d_out, n, dim, "d_out")
    if rows.dtype != torch.float32 or tuple(rows.shape) != (cap, dim) or not rows.is_contiguous():
        raise TensairError(EINVAL, f"grad: expected contiguous float32 rows of shape ({cap}, {dim})")
    c = SparseRows(cap, _vector(n_rows, 1, torch.int32, "n_rows"), _ids(row_ids, "row_ids"), rows.data_ptr())
    rc = (_lib or lib()).tensair_embed_grad(_ids(ids), n, dp, dd, ds, vocab, dim, scale, C.byref(c), workspace.data_ptr(),
                                    _bytes(workspace), _word(status), _on(dev, stream))
    if rc:
        _check(rc)


def tensair_embed_grad_dense(ids, d_out, dim: int, grad, workspace, scale=1.0, accumulate=False, status=None, stream=None):
    """grad: [vocab, >= dim] float32 or bfloat16, overwritten or, with accumulate, added to."""
    n, vocab, dev = ids.numel(), grad.shape[0], _device(d_out, ids, grad, workspace, status)
    dp, dd, ds = _matrix(d_out, n, dim, "d_out")
    gp, gd, gs = _matrix(grad, vocab, dim, "grad")
    rc = (_lib or lib()).tensair_embed_grad_dense(_ids(ids), n, dp, dd, ds, vocab, dim, scale, gp, gd, gs, int(accumulate), workspace.data_ptr(),
                                          _bytes(workspace), _word(status), _on(dev, stream))
    if rc:
        _check(rc)


def tensair_softmax_workspace_bytes(n: int, vocab: int, dim: int, dtype, with_grad: bool) -> int:
    """dtype: torch.float32 or torch.bfloat16."""
    nbytes = lib().tensair_softmax_workspace_bytes(n, vocab, dim, _dtype(dtype, "dtype"), int(with_grad))
    if nbytes == 0:
        raise TensairError(EINVAL, lib().tensair_last_error().decode())
    return nbytes


def tensair_softmax_loss(hidden, table, dim: int, labels, loss, lse, workspace, scale=1.0, ignore_label=-1, status=None, stream=None):
    """hidden: [n, >= dim], table: [vocab, >= dim] of one type; labels: int32 [n]; loss, lse: float32 [n]."""
    n, vocab = labels.numel(), table.shape[0]
    dev = _device(table, hidden, labels, loss, lse, workspace, status)
    hp, hd, hs = _matrix(hidden, n, dim, "hidden")
    tp, td, ts = _matrix(table, vocab, dim, "table")
    if hd != td:
        raise TensairError(EINVAL, "hidden and table must have one type")
    rc = (_lib or lib()).tensair_softmax_loss(hp, hs, tp, ts, td, n, vocab, dim, _ids(labels, "labels"), ignore_label, scale,
                                      _vector(loss, n, torch.float32, "loss"), _vector(lse, n, torch.float32, "lse"), workspace.data_ptr(),
                                      _bytes(workspace), _word(status), _on(dev, stream))
    if rc:
        _check(rc)


def tensair_softmax_grad(hidden, table, dim: int, labels, lse, d_loss, d_hidden, d_table, workspace, scale=1.0, ignore_label=-1,
                         status=None, stream=None):
    """lse: as tensair_softmax_loss gave it; d_loss: float32 [n]; d_hidden, d_table: like hidden and table, or None."""
    n, vocab = labels.numel(), table.shape[0]
    dev = _device(table, hidden, labels, lse, d_loss, d_hidden, d_table, workspace, status)
    hp, hd, hs = _matrix(hidden, n, dim, "hidden")
    tp, td, ts = _matrix(table, vocab, dim, "table")
    dhp, dhd, dhs = _matrix(d_hidden, n, dim, "d_hidden") if d_hidden is not None else (None, td, dim)
    dtp, dtd, dts = _matrix(d_table, vocab, dim, "d_table") if d_table is not None else (None, td, dim)
    if not hd == td == dhd == dtd:
        raise TensairError(EINVAL, "hidden, table and their gradients must have one type")
    rc = (_lib or lib()).tensair_softmax_grad(hp, hs, tp, ts, td, n, vocab, dim, _ids(labels, "labels"), ignore_label, scale,
                                      _vector(lse, n, torch.float32, "lse"), _vector(d_loss, n, torch.float32, "d_loss"), dhp, dhs, dtp, dts,
                                      workspace.data_ptr(), _bytes(workspace), _word(status), _on(dev, stream))
    if rc:
        _check(rc)


def _adamw_tensors(tensors):
    """(C array, state dtype) of a list of dicts: param, grad, m, v, for 8-bit states m_scale and v_scale, and on request
    param_copy (bfloat16) and weight_decay."""
    arr = (AdamwTensor * max(len(tensors), 1))()
    state = None
    for k, t in enumerate(tensors):
        n, s = t["param"].numel(), _dtype(t["m"], f"tensor {k}: m")
        if state is None:
            state = s
        scales = [t.get("m_scale"), t.get("v_scale")] if s == FP8 else []
        if s == BF16 or s != state or t["v"].dtype != t["m"].dtype:
            raise TensairError(EINVAL, f"tensor {k}: all states are float32 or all float8_e4m3fn")
        if any(x is None for x in scales):
            raise TensairError(EINVAL, f"tensor {k}: 8-bit states need scales")
        groups = -(-n // 256)
        for name, x, size in [(w, t[w], n) for w in ("grad", "m", "v")] + [("scales", x, groups) for x in scales] + \
                ([("param_copy", t["param_copy"], n)] if t.get("param_copy") is not None else []):
            if x.numel() != size or not x.is_contiguous():
                raise TensairError(EINVAL, f"tensor {k}: {name}: expected {size} contiguous elements")
        if not t["param"].is_contiguous() or any(x.dtype != torch.float32 for x in scales) or \
                (t.get("param_copy") is not None and t["param_copy"].dtype != torch.bfloat16):
            raise TensairError(EINVAL, f"tensor {k}: param must be contiguous, scales float32, param_copy bfloat16")
        a = arr[k]
        a.param, a.grad, a.m, a.v = (t[w].data_ptr() for w in ("param", "grad", "m", "v"))
        a.m_scale, a.v_scale = (x.data_ptr() for x in scales) if scales else (None, None)
        a.param_copy = t["param_copy"].data_ptr() if t.get("param_copy") is not None else None
        a.n, a.param_dtype, a.grad_dtype = n, _dtype(t["param"], f"tensor {k}: param"), _dtype(t["grad"], f"tensor {k}: grad")
        a.weight_decay = t.get("weight_decay", 0.0)
    return arr, F32 if state is None else state


# `c`: what _adamw_tensors makes of the tensors, where the caller has it (half a millisecond for a hundred of them)
def tensair_adamw_workspace_bytes(tensors, c=None) -> int:
    arr, state = c or _adamw_tensors(tensors)
    nbytes = lib().tensair_adamw_workspace_bytes(arr, len(tensors), state)
    if nbytes == 0:
        raise TensairError(EINVAL, lib().tensair_last_error().decode())
    return nbytes


def tensair_adamw_init(tensors, workspace, stream=None, c=None):
    arr, state = c or _adamw_tensors(tensors)
    h = C.c_void_p()
    dev = _device(workspace, *(t[w] for t in tensors for w in ("param", "grad", "m", "v", "m_scale", "v_scale", "param_copy") if t.get(w) is not None))
    _check(lib().tensair_adamw_init(C.byref(h), arr, len(tensors), state, _ptr(workspace), _bytes(workspace), _on(dev, stream)))
    return h


def tensair_adamw_step(h, lr: float, step: int, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=None, stream=None):
    """grad_scale: float32 tensor of one element that the gradients are multiplied by, or None."""
    if grad_scale is not None:
        _device(grad_scale)
    _check(lib().tensair_adamw_step(h, lr, step, beta1, beta2, eps, _word(grad_scale, torch.float32, "grad_scale"), _stream(stream)))


def tensair_adamw_step_at(h, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=None, stream=None):
    """lr: float64 tensor, step: int64 tensor of one element each, read when the work runs (in a graph: at every replay)."""
    dev = _device(lr, step, grad_scale)
    _check(lib().tensair_adamw_step_at(h, _word(lr, torch.float64, "lr"), _word(step, torch.int64, "step"), beta1, beta2, eps,
                                       _word(grad_scale, torch.float32, "grad_scale"), _on(dev, stream)))


def tensair_adamw_destroy(h):
    _check(lib().tensair_adamw_destroy(h))


class AdamW:
    """Owns the handle and the workspace of an optimizer over a list of tensors and keeps the tensors alive (their gradients are
    read where they are when this is made)."""

    def __init__(self, tensors, stream=None):
        self.h = None
        self.tensors = [dict(t) for t in tensors]
        c = _adamw_tensors(self.tensors)
        nbytes = tensair_adamw_workspace_bytes(self.tensors, c)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.tensors[0]["param"].device)
        self.h = tensair_adamw_init(self.tensors, self.workspace, stream, c)

    def step(self, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=None, stream=None):
        """lr and step: numbers or, for a step that is recorded into a graph, float64 and int64 tensors of one element on the GPU."""
        if isinstance(step, torch.Tensor):
            _device(self.workspace, step)
            return tensair_adamw_step_at(self.h, lr, step, beta1, beta2, eps, grad_scale, stream)
        rc = _lib.tensair_adamw_step(self.h, lr, step, beta1, beta2, eps, _word(grad_scale, torch.float32, "grad_scale"),
                                     _on(_device(self.workspace, grad_scale), stream))
        if rc:
            _check(rc)

    def close(self):
        if self.h is not None:
            tensair_adamw_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- what lies between a table's two ends in a model of word sequences, and behind them
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _launch(dev, call, *args):
    """A call whose kernels go to the GPU of that number, whichever is the current one."""
    if _current_device() == dev:
        rc = call(*args)
    else:
        with torch.cuda.device(dev):
            rc = call(*args)
    if rc:
        _check(rc)


def _floats(t, shape, what):
    """The address of contiguous float32 elements of that shape, or None."""
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.shape != shape or not t.is_contiguous():
        raise TensairError(EINVAL, f"{what}: expected contiguous float32 elements of shape {shape}")
    return t.data_ptr()


def tensair_norm(x, dim: int, weight, bias, out, mean=None, rstd=None, eps=1e-5, stream=None):
    """x, out: [n, >= dim] float32 or bfloat16; weight, bias: float32 [dim] or None; mean, rstd: float32 [n] or both None."""
    n, dev = x.shape[0], _device(x, weight, bias, out, mean, rstd)
    xp, xd, xs = _matrix(x, n, dim, "x")
    op, od, os_ = _matrix(out, n, dim, "out")
    _launch(dev, (_lib or lib()).tensair_norm, xp, xd, xs, n, dim, _floats(weight, (dim,), "weight"), _floats(bias, (dim,), "bias"), eps, op, od, os_,
            _floats(mean, (n,), "mean"), _floats(rstd, (n,), "rstd"), _on(dev, stream))


def tensair_norm_workspace_bytes(n: int, dim: int) -> int:
    nbytes = lib().tensair_norm_workspace_bytes(n, dim)
    if nbytes == 0:
        raise TensairError(EINVAL, lib().tensair_last_error().decode())
    return nbytes


def tensair_norm_grad(d_out, x, dim: int, weight, mean, rstd, d_x, d_weight=None, d_bias=None, workspace=None, d_add=None, stream=None):
    """d_out: [n, >= dim]; x, d_x, d_add (or None): of one type; mean, rstd: as tensair_norm gave them; d_weight, d_bias: float32 [dim] or None (not
    wanted; with neither no workspace is needed)."""
    n, dev = x.shape[0], _device(x, d_out, weight, mean, rstd, d_x, d_weight, d_bias, workspace, d_add)
    dp, dd, ds = _matrix(d_out, n, dim, "d_out")
    xp, xd, xs = _matrix(x, n, dim, "x")
    dxp, dxd, dxs = _matrix(d_x, n, dim, "d_x")
    ap, ad, as_ = _matrix(d_add, n, dim, "d_add") if d_add is not None else (None, xd, dim)
    if not xd == dxd == ad:
        raise TensairError(EINVAL, "x, d_x and d_add must have one type")
    ws = (workspace.data_ptr(), _bytes(workspace)) if workspace is not None else (None, 0)
    _launch(dev, (_lib or lib()).tensair_norm_grad, dp, dd, ds, xp, xd, xs, n, dim, _floats(weight, (dim,), "weight"), _vector(mean, n, torch.float32, "mean"),
            _vector(rstd, n, torch.float32, "rstd"), ap, as_, dxp, dxs, _floats(d_weight, (dim,), "d_weight"), _floats(d_bias, (dim,), "d_bias"), *ws,
            _on(dev, stream))


def tensair_dropout(x, dim: int, out, p: float, seed: int, layer=0, step=0, residual=None, stream=None):
    """x, out: [n, >= dim] float32 or bfloat16; residual: like out, or None; step: a number or, for a call that is recorded into a graph, an int64 tensor
    of one element on the GPU."""
    n, at = x.shape[0], step if isinstance(step, torch.Tensor) else None
    dev = _device(x, out, residual, at)
    xp, xd, xs = _matrix(x, n, dim, "x")
    op, od, os_ = _matrix(out, n, dim, "out")
    rp, rd, rs = _matrix(residual, n, dim, "residual") if residual is not None else (None, od, dim)
    if rd != od:
        raise TensairError(EINVAL, "residual and out must have one type")
    _launch(dev, (_lib or lib()).tensair_dropout, xp, xd, xs, n, dim, p, seed, layer, 0 if at is not None else step, _word(at, torch.int64, "step"), rp, rs, op, od,
            os_, _on(dev, stream))


def tensair_recur_state_rows(n: int) -> int:
    rows = lib().tensair_recur_state_rows(n)
    if rows < 0:
        raise TensairError(EINVAL, lib().tensair_last_error().decode())
    return rows


def tensair_recur_workspace_bytes(n: int, dim: int) -> int:
    nbytes = lib().tensair_recur_workspace_bytes(n, dim)
    if nbytes == 0:
        raise TensairError(EINVAL, lib().tensair_last_error().decode())
    return nbytes


def _recur_inputs(x, gate, dim, offsets, states):
    n, n_seq = x.shape[0], offsets.numel() - 1
    xp, xd, xs = _matrix(x, n, dim, "x")
    gp, gd, gs = _matrix(gate, n, dim, "gate")
    if xd != gd:
        raise TensairError(EINVAL, "x and gate must have one type")
    if n_seq < 0:
        raise TensairError(EINVAL, "offsets: expected one more than there are sequences")
    sp = None if states is None else _floats(states, (tensair_recur_state_rows(n), dim), "states")
    return n, n_seq, xd, (xp, xs, gp, gs, xd, n, dim, _ids(offsets, "offsets"), n_seq), sp


def tensair_recur(x, gate, dim: int, offsets, out, workspace, h0=None, h_last=None, states=None, status=None, stream=None):
    """x, gate, out: [n, >= dim] of one type; offsets: int32 [sequences + 1]; h0, h_last: float32 [sequences, dim] or None; states: float32
    [tensair_recur_state_rows(n), dim] or None (no gradient is wanted)."""
    dev = _device(x, gate, offsets, out, workspace, h0, h_last, states, status)
    n, n_seq, code, head, sp = _recur_inputs(x, gate, dim, offsets, states)
    op, od, os_ = _matrix(out, n, dim, "out")
    if od != code:
        raise TensairError(EINVAL, "x, gate and out must have one type")
    _launch(dev, (_lib or lib()).tensair_recur, *head, _floats(h0, (n_seq, dim), "h0"), op, os_, _floats(h_last, (n_seq, dim), "h_last"), sp,
            workspace.data_ptr(), _bytes(workspace), _word(status), _on(dev, stream))


def tensair_recur_grad(x, gate, dim: int, offsets, states, d_out, d_x, d_gate, workspace, h0=None, d_last=None, d_h0=None, status=None, stream=None):
    """states: as tensair_recur gave them; d_out, d_x, d_gate: like x; d_last, d_h0: float32 [sequences, dim] or None."""
    dev = _device(x, gate, offsets, states, d_out, d_x, d_gate, workspace, h0, d_last, d_h0, status)
    n, n_seq, code, head, sp = _recur_inputs(x, gate, dim, offsets, states)
    dp, dd, ds = _matrix(d_out, n, dim, "d_out")
    xp, xd, xs = _matrix(d_x, n, dim, "d_x")
    gp, gd, gs = _matrix(d_gate, n, dim, "d_gate")
    if not code == dd == xd == gd:
        raise TensairError(EINVAL, "x, gate and their gradients must have one type")
    _launch(dev, (_lib or lib()).tensair_recur_grad, *head, _floats(h0, (n_seq, dim), "h0"), sp, dp, ds, _floats(d_last, (n_seq, dim), "d_last"), xp, xs, gp, gs,
            _floats(d_h0, (n_seq, dim), "d_h0"), workspace.data_ptr(), _bytes(workspace), _word(status), _on(dev, stream))


def tensair_recur_step(x, gate, dim: int, state, out=None, slots=None, status=None, stream=None):
    """x, gate, out (or None): [n, >= dim] of one type; state: float32 [slots, >= dim], updated; slots: int32 [n], the rows of state, or None (row i)."""
    n, dev = x.shape[0], _device(x, gate, state, out, slots, status)
    xp, xd, xs = _matrix(x, n, dim, "x")
    gp, gd, gs = _matrix(gate, n, dim, "gate")
    sp, sd, ss = _matrix(state, state.shape[0], dim, "state")
    op, od, os_ = _matrix(out, n, dim, "out") if out is not None else (None, xd, dim)
    if not xd == gd == od or sd != F32:
        raise TensairError(EINVAL, "x, gate and out must have one type, state float32")
    _launch(dev, (_lib or lib()).tensair_recur_step, xp, xs, gp, gs, xd, n, dim, _vector(slots, n, torch.int32, "slots") if slots is not None else None,
            state.shape[0], sp, ss, op, os_, _word(status), _on(dev, stream))


def tensair_sample_workspace_bytes(n: int, vocab: int) -> int:
    nbytes = lib().tensair_sample_workspace_bytes(n, vocab)
    if nbytes == 0:
        raise TensairError(EINVAL, lib().tensair_last_error().decode())
    return nbytes


def tensair_sample(logits, vocab: int, u, words, workspace, temperature=None, top_k=None, top_p=None, min_p=None, prob=None, status=None, stream=None):
    """logits: [n, >= vocab] float32 or bfloat16; u: float32 [n]; words: int32 [n]; temperature, top_p, min_p: float32 [n], top_k: int32 [n], each or None;
    prob: float32 [n] or None."""
    n, dev = logits.shape[0], _device(logits, u, words, workspace, temperature, top_k, top_p, min_p, prob, status)
    zp, zd, zs = _matrix(logits, n, vocab, "logits")
    _launch(dev, (_lib or lib()).tensair_sample, zp, zd, zs, n, vocab, _floats(temperature, (n,), "temperature"),
            _vector(top_k, n, torch.int32, "top_k") if top_k is not None else None, _floats(top_p, (n,), "top_p"), _floats(min_p, (n,), "min_p"),
            _vector(u, n, torch.float32, "u"), _vector(words, n, torch.int32, "words"), _floats(prob, (n,), "prob"), workspace.data_ptr(), _bytes(workspace),
            _word(status), _on(dev, stream))


def tensair_status(h, stream=None):
    _check(lib().tensair_status(h, _stream(stream)))


def tensair_profile(h, level: int):
    _check(lib().tensair_profile(h, level))


def tensair_profile_read(h, max_records: int = 65536):
    """[(tag name, milliseconds), ...] since the previous read."""
    tags = np.zeros(max_records, dtype=np.int32)
    ms = np.zeros(max_records, dtype=np.float32)
    n = lib().tensair_profile_read(h, tags.ctypes.data_as(C.c_void_p), ms.ctypes.data_as(C.c_void_p), max_records)
    if n < 0:
        raise TensairError(n, lib().tensair_last_error().decode())
    return [(PROFILE_TAGS.get(int(tags[i]), str(int(tags[i]))), float(ms[i])) for i in range(n)]


def tensair_copy_probe(dst, src, nbytes: int, stream=None):
    _check(lib().tensair_copy_probe(_ptr(dst), _ptr(src), nbytes, _stream(stream)))


def tensair_stream_probe(dst, src, nbytes: int, mode: int, stream=None):
    _check(lib().tensair_stream_probe(_ptr(dst), _ptr(src), nbytes, mode, _stream(stream)))


def tensair_model_destroy(h):
    _check(lib().tensair_model_destroy(h))


# ---------------------------------------------------------------- convenience owner of the buffers
class Model:
    """Owns the device memory a tensair_model needs (tables, workspace) and forwards to the
    C entry points.  No arithmetic happens here."""

    def __init__(self, vocab, dim, dtype, window, negatives, max_centers, max_peers, seed,
                 unigram_counts, worker_id=0, row_stride=None, tables=None, device="cuda", flags=0):
        self.cfg = Config(vocab, dim, row_stride or dim, dtype, window, negatives, max_centers,
                          max_peers, worker_id, seed, flags)
        tdt = torch.float32 if dtype == F32 else torch.bfloat16
        if tables is None:
            self.w_in = torch.empty((vocab, self.cfg.row_stride), dtype=tdt, device=device)
            self.w_out = torch.empty((vocab, self.cfg.row_stride), dtype=tdt, device=device)
            fill = True
        else:
            self.w_in, self.w_out = tables
            fill = False
        nbytes = tensair_workspace_bytes(self.cfg)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.h = tensair_model_init(self.cfg, self.w_in, self.w_out, fill, unigram_counts, self.workspace)
        self.device = device

    def grad_buffers(self, n_centers=None) -> GradBuffers:
        n = self.cfg.max_centers if n_centers is None else n_centers
        return GradBuffers(tensair_capacity_in(self.cfg, n), tensair_capacity_out(self.cfg, n),
                           self.cfg.dim, self.device)

    def rebind(self, w_in, w_out, worker_id):
        tensair_model_rebind(self.h, w_in, w_out, worker_id)

    def alias(self):
        return tensair_model_alias(self.h, self.cfg.vocab)

    def pair_count(self, n_tokens, begin, n):
        return tensair_pair_count(self.h, n_tokens, begin, n)

    def sgns_grad(self, tokens, begin, n, epoch, grad, **kw):
        tensair_sgns_grad(self.h, tokens, begin, n, epoch, grad, **kw)

    def dasgd_apply(self, own, peers, lr):
        tensair_dasgd_apply(self.h, own, peers, lr)

    def step(self, tokens, begin, n, epoch, peers, lr, own_out, mean_loss=None):
        tensair_step(self.h, tokens, begin, n, epoch, peers, lr, own_out, mean_loss)

    def grad_pack(self, g, out):
        tensair_grad_pack(self.h, g, out)

    def dasgd_apply_packed(self, own, peers, lr):
        tensair_dasgd_apply_packed(self.h, own, peers, lr)

    def step_packed(self, tokens, begin, n, epoch, peers, lr, own_out, own_msg_out=None, mean_loss=None):
        tensair_step_packed(self.h, tokens, begin, n, epoch, peers, lr, own_out, own_msg_out, mean_loss)

    def packed_buffers(self, n_centers=None) -> PackedBuffers:
        n = self.cfg.max_centers if n_centers is None else n_centers
        return PackedBuffers(tensair_capacity_in(self.cfg, n), tensair_capacity_out(self.cfg, n),
                             self.cfg.dim, self.device)

    def lookup(self, table, ids, out):
        tensair_lookup(self.h, table, ids, out)

    def grad_add(self, a, b, out):
        tensair_grad_add(self.h, a, b, out)

    def prefetch(self, tokens, begin, n, epoch):
        tensair_prefetch(self.h, tokens, begin, n, epoch)

    def status(self):
        tensair_status(self.h)

    def close(self):
        if self.h is not None:
            tensair_model_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
