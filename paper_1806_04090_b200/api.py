"""Thin Python binding of the C ABI in ``include/atomo.h`` (argument marshalling only).

Every step of the encode / decode path runs in the CUDA library; PyTorch is used for device
memory and streams.  There is no CPU fallback: if the shared library is missing or no CUDA
device is present, the calls raise.
"""
from __future__ import annotations

import ctypes
import functools
import operator
import os
import struct
from dataclasses import dataclass, field
from typing import List, Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("ATOMO_B200_LIB", os.path.join(_HERE, "libatomo_b200.so"))

KIND_SPECTRAL = 0
KIND_ENTRYWISE = 1
EW_EXPLICIT, EW_COMPACT = 0, 1      # entry-wise payload formats
EW_TILE = 4096                       # elements per tile of the entry-wise offset table
STATUS_NAMES = ["OK", "INVALID_ARG", "BUDGET", "CAPACITY", "NONFINITE", "NOT_CONVERGED", "TIMEOUT", "CUDA",
                "PAYLOAD"]
STAGES = ["gram", "eig", "sample", "backproject", "ew_reduce", "ew_pack", "decode"]

# every symbol include/atomo.h declares
EXPORTS = [
    "atomo_create", "atomo_destroy", "atomo_last_cuda_error", "atomo_payload_bytes_spectral",
    "atomo_payload_bytes_entrywise", "atomo_encode_spectral", "atomo_encode_entrywise", "atomo_decode",
    "atomo_payload_read_headers", "atomo_payload_status", "atomo_set_profiling", "atomo_get_stage_times",
    "atomo_set_eig_params", "atomo_set_eig_mode", "atomo_set_sigma_refinement", "atomo_set_gram_path", "atomo_set_persistent_eig", "atomo_last_eig_scheme", "atomo_decode_spectral_static", "atomo_decode_average", "atomo_lq_budget",
    "atomo_payload_bytes_entrywise_compact", "atomo_set_entrywise_format", "atomo_get_stage_totals",
    "atomo_set_tridiag_ctas", "atomo_limit_tridiag_route", "atomo_limit_workspace", "atomo_measure_fma_peak", "atomo_encode_spectral_from_svd", "atomo_get_table_uploads",
    "atomo_set_entrywise_launch",
    "atomo_get_entrywise_list_chunks",
    "atomo_grad_norm_workspace_bytes", "atomo_grad_norm", "atomo_adamw", "atomo_embedding", "atomo_embedding_workspace_bytes",
    "atomo_embedding_backward", "atomo_layer_norm", "atomo_layer_norm_workspace_bytes", "atomo_layer_norm_backward",
]
TYPE_CODES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}   # atomo_type
STATE_BLOCK = 32                     # elements of an 8-bit optimiser state that share a power of two


class AtomoError(RuntimeError):
    def __init__(self, code: int, where: str, detail: str = ""):
        name = STATUS_NAMES[code] if 0 <= code < len(STATUS_NAMES) else str(code)
        super().__init__(f"{where}: ATOMO_ERR_{name}" + (f" ({detail})" if detail else ""))
        self.code = code


class _Mat(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_int32), ("cols", ctypes.c_int32), ("ld", ctypes.c_int64)]


class _Vec(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("n", ctypes.c_int64)]


class _Debug(ctypes.Structure):
    _fields_ = [("sigma", ctypes.c_void_p), ("prob", ctypes.c_void_p), ("mask_words", ctypes.c_void_p),
                ("short_vecs", ctypes.c_void_p)]


class _Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("n", ctypes.c_int64), ("type", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class _AdamWTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("exp_avg", ctypes.c_void_p), ("exp_avg_sq", ctypes.c_void_p), ("exp_avg_scale", ctypes.c_void_p),
                ("exp_avg_sq_scale", ctypes.c_void_p), ("master", ctypes.c_void_p), ("n", ctypes.c_int64), ("weight_decay", ctypes.c_float),
                ("type", ctypes.c_int32)]


class _AdamWArgs(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double), ("step", ctypes.c_int64),
                ("seed", ctypes.c_uint64), ("scale", ctypes.c_void_p), ("state_bits", ctypes.c_int32), ("grad_type", ctypes.c_int32)]


class PayloadHeader(ctypes.Structure):
    _fields_ = [("magic", ctypes.c_uint32), ("version", ctypes.c_uint32), ("kind", ctypes.c_uint32),
                ("n_layers", ctypes.c_uint32), ("total_bytes", ctypes.c_uint64), ("seed", ctypes.c_uint64),
                ("step", ctypes.c_uint64), ("s", ctypes.c_double), ("ew_format", ctypes.c_uint64), ("ew_sat_cap", ctypes.c_uint64)]


class LayerHeader(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("k_cap", ctypes.c_uint32), ("k", ctypes.c_uint32),
                ("n_sat", ctypes.c_uint32), ("status", ctypes.c_uint32), ("c", ctypes.c_float),
                ("sweeps", ctypes.c_uint32), ("off_idx", ctypes.c_uint64), ("off_val", ctypes.c_uint64),
                ("off_short", ctypes.c_uint64), ("off_long", ctypes.c_uint64), ("l1", ctypes.c_double)]


assert ctypes.sizeof(PayloadHeader) == 64 and ctypes.sizeof(LayerHeader) == 80

_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libatomo_b200.so (no CUDA call is made by loading)."""
    global _lib
    if _lib is not None and path == LIB_PATH:
        return _lib
    if not os.path.exists(path):
        raise FileNotFoundError(
            f"{path} not found: build it with `python -m paper_1806_04090_b200.build` (there is no CPU fallback)")
    lib = ctypes.CDLL(path)
    vp, i32, i64, u64, dbl = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_double
    lib.atomo_create.argtypes = [ctypes.POINTER(vp), ctypes.c_int]
    lib.atomo_destroy.argtypes = [vp]
    lib.atomo_last_cuda_error.argtypes = [vp]
    lib.atomo_last_cuda_error.restype = ctypes.c_char_p
    lib.atomo_payload_bytes_spectral.argtypes = [ctypes.POINTER(i32), ctypes.POINTER(i32), i32, i32]
    lib.atomo_payload_bytes_spectral.restype = i64
    lib.atomo_payload_bytes_entrywise.argtypes = [ctypes.POINTER(i64), i32, i64]
    lib.atomo_payload_bytes_entrywise.restype = i64
    lib.atomo_payload_bytes_entrywise_compact.argtypes = [ctypes.POINTER(i64), i32, i64, i64]
    lib.atomo_payload_bytes_entrywise_compact.restype = i64
    lib.atomo_set_entrywise_format.argtypes = [vp, i32, i64]
    lib.atomo_set_entrywise_launch.argtypes = [vp, i32]
    lib.atomo_get_entrywise_list_chunks.argtypes = [vp, i32, ctypes.POINTER(ctypes.c_uint32), ctypes.POINTER(ctypes.c_uint32)]
    lib.atomo_encode_spectral.argtypes = [vp, ctypes.POINTER(_Mat), i32, dbl, u64, u64, i32, vp, i64,
                                          ctypes.POINTER(_Debug), vp]
    lib.atomo_encode_entrywise.argtypes = [vp, ctypes.POINTER(_Vec), i32, dbl, u64, u64, i64, vp, i64,
                                           ctypes.POINTER(_Debug), vp]
    lib.atomo_decode.argtypes = [vp, i32, vp, ctypes.POINTER(i64), ctypes.POINTER(i64), ctypes.POINTER(vp), i32, vp]
    lib.atomo_decode_average.argtypes = [vp, i32, ctypes.POINTER(vp), i32, ctypes.POINTER(i64), ctypes.POINTER(i64),
                                         ctypes.POINTER(vp), i32, vp]
    lib.atomo_lq_budget.argtypes = [vp, ctypes.POINTER(_Vec), i32, dbl, ctypes.POINTER(dbl), vp]
    lib.atomo_payload_read_headers.argtypes = [vp, vp, i32, ctypes.POINTER(PayloadHeader),
                                               ctypes.POINTER(LayerHeader), vp]
    lib.atomo_payload_status.argtypes = [vp, vp, i32, ctypes.POINTER(i32), ctypes.POINTER(i32), vp]
    lib.atomo_set_profiling.argtypes = [vp, ctypes.c_int]
    lib.atomo_get_stage_times.argtypes = [vp, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(i64)]
    lib.atomo_get_stage_totals.argtypes = [vp, ctypes.POINTER(dbl), ctypes.POINTER(i64), ctypes.POINTER(i64)]
    lib.atomo_set_eig_params.argtypes = [vp, i32, ctypes.c_float]
    lib.atomo_set_eig_mode.argtypes = [vp, i32]
    lib.atomo_set_sigma_refinement.argtypes = [vp, i32]
    lib.atomo_set_gram_path.argtypes = [vp, i32]
    lib.atomo_set_persistent_eig.argtypes = [vp, i32]
    lib.atomo_last_eig_scheme.argtypes = [vp]
    lib.atomo_set_tridiag_ctas.argtypes = [vp, i32]
    lib.atomo_limit_tridiag_route.argtypes = [vp, i32, i32]
    lib.atomo_limit_workspace.argtypes = [vp, i64]
    lib.atomo_get_table_uploads.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(i64)]
    lib.atomo_encode_spectral_from_svd.argtypes = [vp, ctypes.POINTER(_Mat), i32, ctypes.POINTER(vp), ctypes.POINTER(vp),
                                                   ctypes.c_double, u64, u64, i32, vp, i64, ctypes.POINTER(_Debug), vp]
    lib.atomo_measure_fma_peak.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_double)]
    lib.atomo_decode_spectral_static.argtypes = [ctypes.c_int, vp, ctypes.POINTER(i64), ctypes.POINTER(i64),
                                                 ctypes.POINTER(vp), i32, vp]
    # (descriptors of these are packed bytes: filling ctypes structures takes longer than a kernel launch)
    lib.atomo_grad_norm_workspace_bytes.argtypes = [vp, i32]
    lib.atomo_grad_norm_workspace_bytes.restype = i64
    lib.atomo_grad_norm.argtypes = [vp, vp, i32, dbl, vp, vp, i64, vp]
    lib.atomo_adamw.argtypes = [vp, vp, vp, i32, vp, vp]
    lib.atomo_embedding.argtypes = [vp, vp, i32, i64, i64, i64, vp, i32, i64, dbl, vp, i64, vp, vp]
    lib.atomo_embedding_workspace_bytes.argtypes = [i64, i64, i64]
    lib.atomo_embedding_workspace_bytes.restype = i64
    lib.atomo_embedding_backward.argtypes = [vp, vp, i32, i64, vp, i32, i64, i64, i64, dbl, i64, vp, i64, i32, vp, vp, i64, vp]
    lib.atomo_layer_norm.argtypes = [vp, vp, i32, i64, i64, i64, vp, vp, i32, dbl, vp, i64, vp, vp, vp]
    lib.atomo_layer_norm_workspace_bytes.argtypes = [i64, i64]
    lib.atomo_layer_norm_workspace_bytes.restype = i64
    lib.atomo_layer_norm_backward.argtypes = [vp, vp, i64, vp, i64, i32, i64, i64, vp, i32, vp, vp, vp, i64, vp, vp, vp, i64, vp]
    if path == LIB_PATH:
        _lib = lib
    return lib


@functools.lru_cache(maxsize=256)
def _dims(shapes: tuple):
    """(rows, cols) of the layers as the C arrays a decode takes; nobody writes to them."""
    n = len(shapes)
    return (ctypes.c_int64 * n)(*[int(r) for r, _ in shapes]), (ctypes.c_int64 * n)(*[int(c) for _, c in shapes])


@functools.lru_cache(maxsize=256)
def _payload_bytes(kind: int, shapes: tuple, k_cap: int, compact: bool, sat_cap: int) -> int:
    """The payload sizes below for shapes seen before (a training step encodes the same shapes every time)."""
    if kind == KIND_SPECTRAL:
        return payload_bytes_spectral(shapes, k_cap)
    lengths = [c for _, c in shapes]
    return payload_bytes_entrywise_compact(lengths, k_cap, sat_cap) if compact else payload_bytes_entrywise(lengths, k_cap)


def payload_bytes_spectral(shapes: Sequence[Sequence[int]], k_cap: int) -> int:
    lib = load_library()
    n = len(shapes)
    rows = (ctypes.c_int32 * n)(*[int(s[0]) for s in shapes])
    cols = (ctypes.c_int32 * n)(*[int(s[1]) for s in shapes])
    return int(lib.atomo_payload_bytes_spectral(rows, cols, n, int(k_cap)))


def payload_bytes_entrywise(lengths: Sequence[int], k_cap: int) -> int:
    lib = load_library()
    n = len(lengths)
    arr = (ctypes.c_int64 * n)(*[int(x) for x in lengths])
    return int(lib.atomo_payload_bytes_entrywise(arr, n, int(k_cap)))


def payload_bytes_entrywise_compact(lengths: Sequence[int], k_cap: int, sat_cap: int) -> int:
    lib = load_library()
    n = len(lengths)
    arr = (ctypes.c_int64 * n)(*[int(x) for x in lengths])
    return int(lib.atomo_payload_bytes_entrywise_compact(arr, n, int(k_cap), int(sat_cap)))


def measure_fma_peak(device: int = 0, fp64: bool = False) -> float:
    """Measured FMA rate of the GPU in TFLOP/s (fp32 or fp64), see atomo_measure_fma_peak."""
    out = ctypes.c_double(0.0)
    rc = load_library().atomo_measure_fma_peak(int(device), 1 if fp64 else 0, ctypes.byref(out))
    if rc != 0:
        raise AtomoError(rc, "atomo_measure_fma_peak")
    return float(out.value)


_ADAMW_ARGS = struct.Struct("=ddddqQQii").pack          # _AdamWArgs
_T, _dtype_of = torch.Tensor, operator.attrgetter("dtype")


# autograd's check of saved tensors sees what a call writes through a raw pointer only when told (takes tensors; those of inference mode are left out)
_written = torch._C._increment_version


def _no_graph(*tensors) -> None:
    """Refuses tensors that autograd would follow through a call: the operators record no graph, and a gradient would end there without a word."""
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise RuntimeError("the operators record no autograd graph, but one of the tensors requires a gradient: detach it, or make the call under "
                                   "torch.no_grad() or in the methods of a torch.autograd.Function")


def default_k_cap(s: float, n_atoms: int) -> int:
    """k is a sum of independent Bernoulli draws with mean <= s: s + 8 sqrt(s) + 8 is never reached."""
    return int(min(n_atoms, np.ceil(s + 8.0 * np.sqrt(max(float(s), 0.0)) + 8.0)))


@dataclass
class Debug:
    """Optional per-atom outputs (device tensors) for parity checks."""
    sigma: Optional[torch.Tensor] = None
    prob: Optional[torch.Tensor] = None
    mask_words: Optional[torch.Tensor] = None
    short_vecs: Optional[torch.Tensor] = None
    atom_offsets: List[int] = field(default_factory=list)
    word_offsets: List[int] = field(default_factory=list)
    sq_offsets: List[int] = field(default_factory=list)

    def layer_mask(self, l: int, n_atoms: int) -> np.ndarray:
        w0 = self.word_offsets[l]
        words = self.mask_words[w0: w0 + (n_atoms + 31) // 32].cpu().numpy().astype(np.uint32)
        bits = np.unpackbits(words.view(np.uint8), bitorder="little")
        return bits[:n_atoms].astype(bool)

    def layer_prob(self, l: int, n_atoms: int) -> np.ndarray:
        a0 = self.atom_offsets[l]
        return self.prob[a0: a0 + n_atoms].cpu().numpy()

    def layer_sigma(self, l: int, n_atoms: int) -> np.ndarray:
        a0 = self.atom_offsets[l]
        return self.sigma[a0: a0 + n_atoms].cpu().numpy()

    def layer_short(self, l: int, r: int) -> np.ndarray:
        o = self.sq_offsets[l]
        return self.short_vecs[o: o + r * r].cpu().numpy().reshape(r, r)


@dataclass
class Payload:
    """A device payload plus the host-side facts needed to decode it."""
    buf: torch.Tensor            # uint8, device
    kind: int
    shapes: List[tuple]          # (rows, cols) per layer; entry-wise: (1, n)
    k_cap: int
    ctx: "Atomo"
    ew_format: int = 0           # entry-wise: EW_EXPLICIT or EW_COMPACT
    sat_cap: int = 0             # compact entry-wise: capacity of the saturated list

    @property
    def n_layers(self) -> int:
        return len(self.shapes)

    def headers(self):
        return self.ctx.read_headers(self)

    def layer_arrays(self, l: int, hdrs=None):
        """Host copies of one layer's kept atoms (test / inspection helper)."""
        _, lh = hdrs if hdrs is not None else self.headers()
        h = lh[l]
        k = int(h.k)
        raw = self.buf

        def view(off, count, dtype):
            nbytes = count * 4
            return raw[off: off + nbytes].cpu().numpy().view(dtype)

        if self.kind == KIND_ENTRYWISE and self.ew_format == EW_COMPACT:
            # expand the compact form to the explicit (idx, val) pair: entries carry the index inside their tile
            # and the sign of +-c; the saturated atoms sit in a list of their own
            n = self.shapes[l][1]
            n_sat = int(h.n_sat)
            k_list = k - n_sat
            n_tiles = (n + EW_TILE - 1) // EW_TILE
            ent = raw[h.off_idx: h.off_idx + 2 * k_list].cpu().numpy().view(np.uint16).astype(np.int64)
            table = view(h.off_short, n_tiles + 1, np.uint32).astype(np.int64)
            tile_of = np.searchsorted(table[1:], np.arange(k_list), side="right")
            idx_u = tile_of * EW_TILE + (ent & (EW_TILE - 1))
            val_u = np.where(ent & 0x8000, -np.float32(h.c), np.float32(h.c)).astype(np.float32)
            idx_s = view(h.off_long, n_sat, np.uint32).astype(np.int64)
            val_s = view(h.off_val, n_sat, np.float32)
            idx = np.concatenate([idx_u, idx_s])
            val = np.concatenate([val_u, val_s])
            order = np.argsort(idx, kind="stable")
            return dict(k=k, idx=idx[order].astype(np.uint32), val=val[order].astype(np.float32),
                        n_sat_kept=n_sat, table=table)
        idx = view(h.off_idx, k, np.uint32).copy()
        val = view(h.off_val, k, np.float32).copy()
        if self.kind == KIND_ENTRYWISE:
            return dict(k=k, idx=idx, val=val)
        rows, cols = self.shapes[l]
        r, L = min(rows, cols), max(rows, cols)
        short = view(h.off_short, k * r, np.float32).reshape(k, r).copy()
        long_ = view(h.off_long, k * L, np.float32).reshape(k, L).copy()
        U, V = (short, long_) if rows <= cols else (long_, short)
        return dict(k=k, idx=idx, coef=val, U=U.T.copy(), V=V.T.copy())


def atomo_decode_spectral_static(payload: "Payload", out: Sequence[torch.Tensor], device: Optional[int] = None,
                                 stream: Optional[torch.cuda.Stream] = None) -> List[torch.Tensor]:
    """Spectral decode that allocates nothing on the device: for processes whose framework
    allocator owns the whole GPU, or that cannot take cudaMalloc's device-wide synchronisation
    where they decode.  The caller supplies the output tensors; the layers' descriptors travel as
    kernel arguments (limits: 64 layers, 8192 output tiles of 64 x 1024), so calls share no state.  Every output must be a contiguous
    fp32 CUDA tensor on the payload's device with exactly rows * cols elements: the kernel writes all
    of them through the raw pointer, so anything else is refused here, before the C call."""
    lib = load_library()
    if payload.kind != KIND_SPECTRAL:
        raise ValueError("atomo_decode_spectral_static decodes spectral payloads only")
    n = payload.n_layers
    if len(out) != n:
        raise ValueError("one output tensor per layer is required (this call does not allocate)")
    dev = payload.buf.device.index if device is None else int(device)
    for l, (o, (r_, c_)) in enumerate(zip(out, payload.shapes)):
        if not (isinstance(o, torch.Tensor) and o.is_cuda and o.device.index == dev and o.dtype == torch.float32
                and o.is_contiguous() and o.numel() == int(r_) * int(c_)):
            raise ValueError(f"output {l}: a contiguous fp32 CUDA tensor on device {dev} with {int(r_) * int(c_)} elements is required")
    rows = (ctypes.c_int64 * n)(*[r for r, _ in payload.shapes])
    cols = (ctypes.c_int64 * n)(*[c for _, c in payload.shapes])
    ptrs = (ctypes.c_void_p * n)(*[o.data_ptr() for o in out])
    s = stream if stream is not None else torch.cuda.current_stream()
    rc = lib.atomo_decode_spectral_static(dev, ctypes.c_void_p(payload.buf.data_ptr()), rows, cols, ptrs, n,
                                          ctypes.c_void_p(s.cuda_stream))
    if rc != 0:
        raise AtomoError(rc, "atomo_decode_spectral_static",
                         "batch exceeds the limits (64 layers / 8192 tiles)" if rc == 3 else "")
    return list(out)


def _rows(t: torch.Tensor, cols: int, what: str):
    """(rows, leading dimension) of a tensor seen as a matrix over its last dimension; its rows must lie at one distance."""
    shape, stride = t.shape, t.stride()
    if len(shape) == 0 or shape[-1] != cols or (cols > 1 and stride[-1] != 1):
        raise ValueError(f"{what}: a tensor with {cols} values in its last dimension, of unit stride, is required")
    if t.is_contiguous():
        return t.numel() // max(cols, 1), cols
    if len(shape) == 1:
        return 1, cols
    rows, ld = shape[-2], stride[-2] if shape[-2] > 1 else cols
    for n, s in zip(reversed(shape[:-2]), reversed(stride[:-2])):
        if rows > 1 and n > 1 and s != rows * ld:
            raise ValueError(f"{what}: its rows do not lie at one distance")
        if n > 1 and rows == 1:
            ld = s
        rows *= n
    if rows > 1 and ld < cols:
        raise ValueError(f"{what}: its rows overlap")
    return rows, max(ld, cols)


class AdamWState:
    """Parameters and their optimiser states as atomo_adamw takes them.

    params: contiguous CUDA tensors of one device, fp32, bf16 or fp16.  State in 32 bits: exp_avg and exp_avg_sq are fp32 tensors of as many
    elements.  State in 8 bits: float8_e4m3fn tensors of as many elements, with exp_avg_scale and exp_avg_sq_scale of one
    float8_e8m0fnu number for each 32 elements.  master: fp32 copies that are updated instead of the parameters, which then receive them
    rounded (None, or a list in which single entries may be None).  weight_decay: one number, or one per parameter.
    The object keeps the tensors and their memory and describes it once: they are updated in place.  A parameter that was given other memory since
    (p.data = ..., a module moved or cast) is refused by the call; states must not be given other memory.  `AdamWState.zeros(params, bits=...)` makes the states of a new run."""

    def __init__(self, params: Sequence[torch.Tensor], exp_avg: Sequence[torch.Tensor], exp_avg_sq: Sequence[torch.Tensor],
                 exp_avg_scale: Optional[Sequence[torch.Tensor]] = None, exp_avg_sq_scale: Optional[Sequence[torch.Tensor]] = None,
                 master: Optional[Sequence[Optional[torch.Tensor]]] = None, weight_decay=0.01):
        n = len(params)
        if n == 0:
            raise ValueError("at least one parameter is required")
        if (exp_avg_scale is None) != (exp_avg_sq_scale is None):
            raise ValueError("both states have scales, or neither")
        self.bits = 32 if exp_avg_scale is None else 8
        self.params, self.exp_avg, self.exp_avg_sq = list(params), list(exp_avg), list(exp_avg_sq)
        self.exp_avg_scale = [None] * n if exp_avg_scale is None else list(exp_avg_scale)
        self.exp_avg_sq_scale = [None] * n if exp_avg_sq_scale is None else list(exp_avg_sq_scale)
        self.master = [None] * n if master is None else list(master)
        self.weight_decay = [float(weight_decay)] * n if isinstance(weight_decay, (int, float)) else [float(w) for w in weight_decay]
        lists = (self.exp_avg, self.exp_avg_sq, self.exp_avg_scale, self.exp_avg_sq_scale, self.master, self.weight_decay)
        if any(len(x) != n for x in lists):
            raise ValueError("one state, scale, master copy and weight decay per parameter is required")
        if any(not (w >= 0.0 and np.isfinite(w)) for w in self.weight_decay):
            raise ValueError("weight decays are finite and not negative")
        state = torch.float32 if self.bits == 32 else torch.float8_e4m3fn
        dev, desc, ranges = self.params[0].device, [], []
        self.lengths = []
        for i, (p, m, v, ms, vs, w) in enumerate(zip(self.params, *lists[:5])):
            size = p.numel()
            blocks = -(-size // STATE_BLOCK)
            parts = [("parameter", p, size, None), ("exp_avg", m, size, state), ("exp_avg_sq", v, size, state)]
            if self.bits == 8:
                parts += [("exp_avg_scale", ms, blocks, torch.float8_e8m0fnu), ("exp_avg_sq_scale", vs, blocks, torch.float8_e8m0fnu)]
            if w is not None:
                parts.append(("master copy", w, size, torch.float32))
            for name, t, count, kind in parts:
                if not (isinstance(t, torch.Tensor) and t.is_cuda and t.device == dev and t.is_contiguous() and t.numel() == count
                        and (t.dtype in TYPE_CODES if kind is None else t.dtype == kind)):
                    raise ValueError(f"{name} {i}: a contiguous CUDA tensor on {dev} with {count} elements of "
                                     f"{'fp32, bf16 or fp16' if kind is None else kind} is required")
                if count:
                    ranges.append((t.data_ptr(), t.data_ptr() + count * t.element_size()))
            desc.append((p.data_ptr(), m.data_ptr(), v.data_ptr(), None if ms is None else ms.data_ptr(), None if vs is None else vs.data_ptr(),
                         None if w is None else w.data_ptr(), size, self.weight_decay[i], TYPE_CODES[p.dtype]))
            self.lengths.append(size)
        ranges.sort()
        if any(a[1] > b[0] for a, b in zip(ranges, ranges[1:])):
            raise ValueError("parameters and states must not overlap")
        self.device = dev
        self._desc = (_AdamWTensor * n)(*desc)
        # what the description names stays allocated, also where one of the tensors is given other memory
        self._memory = [t.detach() for part in lists[:5] + (self.params,) for t in part if t is not None]
        self._addresses = [d[0] for d in desc]
        self._pack = struct.Struct("=%dQ" % n).pack

    @classmethod
    def zeros(cls, params: Sequence[torch.Tensor], bits: int = 32, master: bool = False, weight_decay=0.01) -> "AdamWState":
        """The state of a run that has made no step.  master: keep fp32 copies of the parameters that are not fp32."""
        if bits not in (8, 32):
            raise ValueError("states have 8 or 32 bits")
        kind = torch.float32 if bits == 32 else torch.float8_e4m3fn
        moments = [[torch.zeros(p.numel(), dtype=torch.uint8 if bits == 8 else kind, device=p.device).view(kind) for p in params] for _ in range(2)]
        scales = [[torch.zeros(-(-p.numel() // STATE_BLOCK), dtype=torch.uint8, device=p.device).view(torch.float8_e8m0fnu) for p in params]
                  for _ in range(2)] if bits == 8 else [None, None]
        copies = [p.detach().float().clone() if p.dtype != torch.float32 else None for p in params] if master else None
        return cls(params, moments[0], moments[1], scales[0], scales[1], copies, weight_decay)


class Atomo:
    """One library context bound to a CUDA device."""

    def __init__(self, device: int = 0):
        if not torch.cuda.is_available():
            raise RuntimeError("atomo: no CUDA device available (the library has no CPU fallback)")
        self.lib = load_library()
        self.device = int(device)
        self._torch_device = torch.device("cuda", self.device)
        torch.cuda.init()
        h = ctypes.c_void_p()
        rc = self.lib.atomo_create(ctypes.byref(h), self.device)
        self._h = h
        self._ew_format, self._ew_sat_cap = EW_EXPLICIT, 0
        if rc != 0:
            raise AtomoError(rc, "atomo_create", self._cuda_error())
        # tensors that new ones are made after (cheaper than naming type and device each time)
        self._floats = torch.empty(1, dtype=torch.float32, device=self._torch_device)
        self._bytes = torch.empty(1, dtype=torch.uint8, device=self._torch_device)

    def _cuda_error(self) -> str:
        try:
            return (self.lib.atomo_last_cuda_error(self._h) or b"").decode()
        except Exception:  # pragma: no cover
            return ""

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self.lib.atomo_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int, where: str):
        if rc != 0:
            raise AtomoError(rc, where, self._cuda_error() if rc == 7 else "")

    @staticmethod
    def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
        # (the stream's handle without a Stream object, which takes as long as a kernel launch)
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()) if stream is None else stream.cuda_stream

    def _make_debug(self, n_atoms: Sequence[int], spectral: bool, want_short: bool, dev, want_prob: bool = True) -> Debug:
        a_off = np.concatenate([[0], np.cumsum(n_atoms)]).astype(np.int64)
        w_off = np.concatenate([[0], np.cumsum([(n + 31) // 32 for n in n_atoms])]).astype(np.int64)
        sq_off = np.concatenate([[0], np.cumsum([n * n for n in n_atoms])]).astype(np.int64)
        d = Debug(atom_offsets=a_off.tolist(), word_offsets=w_off.tolist(), sq_offsets=sq_off.tolist())
        if want_prob:
            d.prob = torch.zeros(int(a_off[-1]), dtype=torch.float32, device=dev)
        d.mask_words = torch.zeros(int(w_off[-1]), dtype=torch.int32, device=dev)
        if spectral:
            d.sigma = torch.zeros(int(a_off[-1]), dtype=torch.float32, device=dev)
            if want_short:
                d.short_vecs = torch.zeros(int(sq_off[-1]), dtype=torch.float32, device=dev)
        return d

    @staticmethod
    def _debug_struct(d: Optional[Debug]):
        if d is None:
            return None
        ptr = lambda t: ctypes.c_void_p(t.data_ptr()) if t is not None else None
        return _Debug(ptr(d.sigma), ptr(d.prob), ptr(d.mask_words), ptr(d.short_vecs))

    # ------------------------------------------------------------------------------------------
    def atomo_encode_spectral(self, layers: Sequence[torch.Tensor], s: float, seed: int, step: int = 0,
                              k_cap: Optional[int] = None, payload: Optional[torch.Tensor] = None,
                              debug: bool = False, debug_short: bool = False,
                              stream: Optional[torch.cuda.Stream] = None):
        """Spectral ATOMO over a batch of 2-D fp32 CUDA tensors.  Returns (Payload, Debug | None)."""
        n = len(layers)
        desc, shapes = [], []
        for g in layers:
            if not (g.is_cuda and g.dtype == torch.float32 and g.dim() == 2 and g.stride(1) == 1):
                raise ValueError("layers must be 2-D fp32 CUDA tensors with unit column stride")
            m, c = g.shape
            desc.append((g.data_ptr(), m, c, g.stride(0) if m > 1 else c))
            shapes.append((m, c))
        mats = (_Mat * n)(*desc)
        if k_cap is None:
            k_cap = default_k_cap(s, max(min(r, c) for r, c in shapes))
        nbytes = _payload_bytes(KIND_SPECTRAL, tuple(shapes), int(k_cap), False, 0)
        if nbytes < 0:
            raise AtomoError(1, "atomo_payload_bytes_spectral")
        dev = layers[0].device
        if payload is None:
            payload = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        dbg = self._make_debug([min(r, c) for r, c in shapes], True, debug_short, dev) if (debug or debug_short) else None
        ds = self._debug_struct(dbg)
        rc = self.lib.atomo_encode_spectral(self._h, mats, n, float(s), int(seed), int(step), int(k_cap),
                                            payload.data_ptr(), payload.numel(),
                                            ctypes.byref(ds) if ds is not None else None, self._stream_ptr(stream))
        self._check(rc, "atomo_encode_spectral")
        return Payload(payload, KIND_SPECTRAL, shapes, int(k_cap), self), dbg

    def atomo_encode_spectral_from_svd(self, layers: Sequence[torch.Tensor], sigma: Sequence[torch.Tensor],
                                       short_vecs: Sequence[torch.Tensor], s: float, seed: int, step: int = 0,
                                       k_cap: Optional[int] = None, debug: bool = True,
                                       stream: Optional[torch.cuda.Stream] = None):
        """Test entry point: the path downstream of the SVD for a decomposition given by the caller.  sigma[l]: r
        fp32 values, descending; short_vecs[l]: r x r fp32, row i = the unit short-side vector of atom i."""
        n = len(layers)
        mats = (_Mat * n)()
        shapes = []
        for i, g in enumerate(layers):
            if not (g.is_cuda and g.dtype == torch.float32 and g.dim() == 2 and g.is_contiguous()):
                raise ValueError("layers must be contiguous 2-D fp32 CUDA tensors")
            r = min(g.shape)
            for t, want in ((sigma[i], r), (short_vecs[i], r * r)):
                if not (t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() and t.numel() == want):
                    raise ValueError("sigma / short_vecs must be contiguous fp32 CUDA tensors of r and r * r elements")
            mats[i] = _Mat(g.data_ptr(), g.shape[0], g.shape[1], g.shape[1])
            shapes.append((int(g.shape[0]), int(g.shape[1])))
        if k_cap is None:
            k_cap = default_k_cap(s, max(min(r, c) for r, c in shapes))
        payload = torch.empty(payload_bytes_spectral(shapes, k_cap), dtype=torch.uint8, device=layers[0].device)
        dbg = self._make_debug([min(r, c) for r, c in shapes], True, False, layers[0].device) if debug else None
        ds = self._debug_struct(dbg)
        sp = (ctypes.c_void_p * n)(*[t.data_ptr() for t in sigma])
        vp_ = (ctypes.c_void_p * n)(*[t.data_ptr() for t in short_vecs])
        rc = self.lib.atomo_encode_spectral_from_svd(self._h, mats, n, sp, vp_, float(s), int(seed), int(step), int(k_cap),
                                                     payload.data_ptr(), payload.numel(),
                                                     ctypes.byref(ds) if ds is not None else None, self._stream_ptr(stream))
        self._check(rc, "atomo_encode_spectral_from_svd")
        return Payload(payload, KIND_SPECTRAL, shapes, int(k_cap), self), dbg

    def atomo_encode_entrywise(self, vecs: Sequence[torch.Tensor], s: float, seed: int, step: int = 0,
                               k_cap: Optional[int] = None, payload: Optional[torch.Tensor] = None,
                               debug=False, stream: Optional[torch.cuda.Stream] = None):
        """Entry-wise ATOMO over a batch of flat fp32 CUDA tensors.  Returns (Payload, Debug | None).
        The payload format is the one last chosen with set_entrywise_format (explicit by default).
        debug: True = probabilities and mask words, "mask" = the mask words alone (asking for the probabilities makes
        the one-kernel form read every vector twice)."""
        n = len(vecs)
        desc, shapes = [], []
        for g in vecs:
            if not (g.is_cuda and g.dtype == torch.float32 and g.is_contiguous()):
                raise ValueError("vectors must be contiguous fp32 CUDA tensors")
            length = g.numel()
            desc.append((g.data_ptr(), length))
            shapes.append((1, length))
        arr = (_Vec * n)(*desc)
        if k_cap is None:
            k_cap = default_k_cap(s, max(c for _, c in shapes))
        nbytes = _payload_bytes(KIND_ENTRYWISE, tuple(shapes), int(k_cap), self._ew_format == EW_COMPACT, self._ew_sat_cap)
        if nbytes < 0:
            raise AtomoError(1, "atomo_payload_bytes_entrywise")
        dev = vecs[0].device
        if payload is None:
            payload = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        dbg = self._make_debug([c for _, c in shapes], False, False, dev, want_prob=(debug != "mask")) if debug else None
        ds = self._debug_struct(dbg)
        rc = self.lib.atomo_encode_entrywise(self._h, arr, n, float(s), int(seed), int(step), int(k_cap),
                                             payload.data_ptr(), payload.numel(),
                                             ctypes.byref(ds) if ds is not None else None, self._stream_ptr(stream))
        self._check(rc, "atomo_encode_entrywise")
        return Payload(payload, KIND_ENTRYWISE, shapes, int(k_cap), self, self._ew_format, self._ew_sat_cap), dbg

    def atomo_decode(self, payload: Payload, out: Optional[Sequence[torch.Tensor]] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> List[torch.Tensor]:
        """Dense fp32 gradients from a payload (one tensor per layer)."""
        n = payload.n_layers
        dev = payload.buf.device
        if out is None:
            out = [torch.empty(r * c, dtype=torch.float32, device=dev).view((c,) if payload.kind == KIND_ENTRYWISE else (r, c))
                   for r, c in payload.shapes]
        rows, cols = _dims(tuple(payload.shapes))
        ptrs = (ctypes.c_void_p * n)(*[o.data_ptr() for o in out])
        rc = self.lib.atomo_decode(self._h, payload.kind, payload.buf.data_ptr(), rows, cols, ptrs, n,
                                   self._stream_ptr(stream))
        self._check(rc, "atomo_decode")
        return list(out)

    # ------------------------------------------------------------------------------------------
    def atomo_decode_average(self, payloads: Sequence[Payload], out: Optional[Sequence[torch.Tensor]] = None,
                             stream: Optional[torch.cuda.Stream] = None) -> List[torch.Tensor]:
        """Mean of the dense gradients of several payloads of the same shapes (the workers' payloads after an
        all-gather), one tensor per layer, in one pass over the output."""
        if len(payloads) == 0:
            raise ValueError("atomo_decode_average needs at least one payload")
        first = payloads[0]
        for p in payloads[1:]:
            if p.kind != first.kind or list(p.shapes) != list(first.shapes):
                raise ValueError("payloads of one average must share kind and shapes")
        n = first.n_layers
        dev = first.buf.device
        if out is None:
            out = [torch.empty(r * c, dtype=torch.float32, device=dev).view((c,) if first.kind == KIND_ENTRYWISE else (r, c))
                   for r, c in first.shapes]
        rows, cols = _dims(tuple(first.shapes))
        ptrs = (ctypes.c_void_p * n)(*[o.data_ptr() for o in out])
        pays = (ctypes.c_void_p * len(payloads))(*[p.buf.data_ptr() for p in payloads])
        rc = self.lib.atomo_decode_average(self._h, first.kind, pays, len(payloads), rows, cols, ptrs, n,
                                           self._stream_ptr(stream))
        self._check(rc, "atomo_decode_average")
        return list(out)

    def atomo_lq_budget(self, vecs: Sequence[torch.Tensor], q: float, stream: Optional[torch.cuda.Stream] = None) -> List[float]:
        """s = ||g||_1 / ||g||_q per vector (Section 4: q = 2 is QSGD's budget, q = inf TernGrad's)."""
        n = len(vecs)
        arr = (_Vec * n)()
        for i, v in enumerate(vecs):
            if v.dtype != torch.float32 or not v.is_cuda or not v.is_contiguous():
                raise ValueError("vectors must be contiguous fp32 CUDA tensors")
            arr[i].data = v.data_ptr(); arr[i].n = v.numel()
        out = (ctypes.c_double * n)()
        self._check(self.lib.atomo_lq_budget(self._h, arr, n, float(q), out, self._stream_ptr(stream)), "atomo_lq_budget")
        return [float(x) for x in out]

    # ---- operators on either side of the exchange ---------------------------------------------
    # They record no autograd graph: the embedding, the layer norm and their gradients refuse tensors that require a gradient where one would be recorded.
    # (Small calls take as long as their host side: what is a C call on a tensor, an allocation or a ctypes object is counted here.)
    def _on(self, stream: torch.cuda.Stream, call, *args):
        """A call with `stream` current, so that what it allocates belongs to that stream too."""
        if stream.device_index != self.device:
            raise ValueError(f"the stream belongs to device {stream.device_index}, the context to device {self.device}")
        with torch.cuda.stream(stream):
            return call(*args)

    def _own_stream(self) -> int:
        """The current stream of the context's device (whatever device is current)."""
        return torch._C._cuda_getCurrentRawStream(self.device)

    def _scratch(self, nbytes: int) -> torch.Tensor:
        """A workspace for one call: torch's allocator keeps it from other work until this stream is done with it, also in a captured graph."""
        return self._bytes.new_empty(nbytes)

    def _operand(self, t, what: str, types=TYPE_CODES) -> torch.Tensor:
        if not (isinstance(t, torch.Tensor) and t.get_device() == self.device and t.dtype in types):
            raise ValueError(f"{what}: a CUDA tensor on device {self.device} of type {', '.join(str(x) for x in types)} is required")
        return t

    def atomo_grad_norm(self, grads: Sequence[torch.Tensor], max_norm: float = float("inf"), out: Optional[torch.Tensor] = None,
                        stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """Two fp32 numbers on the device: the 2-norm over all elements of all gradients, and min(1, max_norm / (norm + 1e-6)), the factor
        that clips them (NaN where the norm is not finite), as atomo_adamw takes them.  Gradients: contiguous fp32, bf16 or fp16."""
        if stream is not None:
            return self._on(stream, self.atomo_grad_norm, grads, max_norm, out)
        device, n = self.device, len(grads)
        desc = []                                        # of _Tensor; the type's high half is the reserved word
        if n <= 4:
            for g in grads:
                desc += (g.data_ptr(), g.numel(), TYPE_CODES.get(g.dtype))
                if desc[-1] is None or g.get_device() != device or not g.is_contiguous():
                    desc = None
                    break
        else:                                            # (of a method mapped over a long list a call takes two thirds of one in a loop)
            codes = [TYPE_CODES.get(k) for k in map(_dtype_of, grads)]
            desc = [0] * (3 * n)
            desc[0::3], desc[1::3], desc[2::3] = map(_T.data_ptr, grads), map(_T.numel, grads), codes
            if None in codes or not all(map(_T.is_contiguous, grads)) or any(map(device.__ne__, map(_T.get_device, grads))):
                desc = None
        if desc is None:
            raise ValueError(f"gradients must be contiguous fp32, bf16 or fp16 tensors on CUDA device {device}")
        if out is None:
            out = self._floats.new_empty(2)
        elif not (out.get_device() == device and out.dtype == torch.float32 and out.numel() == 2 and out.is_contiguous()):
            raise ValueError(f"out: two fp32 numbers on CUDA device {device} are required")
        else:
            _written((out,))
        s = self._own_stream()
        packed = struct.pack("=%dq" % (3 * n), *desc)
        nbytes = self.lib.atomo_grad_norm_workspace_bytes(packed, n)
        if nbytes < 0:
            raise AtomoError(1, "atomo_grad_norm_workspace_bytes")
        ws = self._scratch(nbytes) if nbytes else None
        self._check(self.lib.atomo_grad_norm(self._h, packed, n, max_norm, out.data_ptr(), ws.data_ptr() if nbytes else None, nbytes, s), "atomo_grad_norm")
        return out

    def atomo_adamw(self, state: AdamWState, grads: Sequence[torch.Tensor], lr: float, step: int, beta1: float = 0.9, beta2: float = 0.999,
                    eps: float = 1e-8, seed: int = 0, scale: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
        """One AdamW step (decoupled weight decay) over all parameters of `state`, in place.  grads: one contiguous tensor per parameter, all of
        one type.  step counts from 1.  scale: what atomo_grad_norm returned; its second number multiplies the gradients, and where it
        is not finite nothing is updated.  seed: of the stochastic rounding of 8-bit states.  (An eps below 3.6e-12 / sqrt(1 - beta2^step), zero among them, is served
        exactly too, with 8-bit states at half the speed.)"""
        if stream is not None:
            return self._on(stream, self.atomo_adamw, state, grads, lr, step, beta1, beta2, eps, seed, scale)
        n, device = len(state.lengths), self.device
        if len(grads) != n:
            raise ValueError(f"{n} gradients are required")
        if state.device.index != device:
            raise ValueError(f"the parameters are on {state.device}, the context on device {device}")
        if list(map(_T.data_ptr, state.params)) != state._addresses:
            raise ValueError("a parameter was given other memory since its AdamWState was made: make one of the parameters as they are, with the same states")
        kind = grads[0].dtype
        if not (kind in TYPE_CODES and set(map(_dtype_of, grads)) == {kind} and set(map(_T.get_device, grads)) == {device} and list(map(_T.numel, grads)) == state.lengths
                and all(map(_T.is_contiguous, grads))):
            raise ValueError(f"gradients must be contiguous tensors on CUDA device {device}, of one type (fp32, bf16 or fp16), with as many elements as their parameters")
        if scale is not None and not (scale.get_device() == device and scale.dtype == torch.float32 and scale.numel() == 2 and scale.is_contiguous()):
            raise ValueError(f"scale: two fp32 numbers on CUDA device {device} are required")
        args = _ADAMW_ARGS(lr, beta1, beta2, eps, step, seed & 0xFFFFFFFFFFFFFFFF, 0 if scale is None else scale.data_ptr(), state.bits, TYPE_CODES[kind])
        rc = self.lib.atomo_adamw(self._h, state._desc, state._pack(*map(_T.data_ptr, grads)), n, args, self._own_stream())
        _written(state.params)
        self._check(rc, "atomo_adamw")

    def _status(self, status: Optional[torch.Tensor]):
        if status is None:
            return None
        if not (status.get_device() == self.device and status.dtype == torch.int32 and status.numel() == 1):
            raise ValueError(f"status: one int32 number on CUDA device {self.device} is required")
        return status.data_ptr()

    def _ids(self, ids: torch.Tensor) -> int:
        if not (isinstance(ids, torch.Tensor) and ids.get_device() == self.device and ids.is_contiguous() and ids.dtype in (torch.int32, torch.int64)):
            raise ValueError(f"ids: a contiguous int32 or int64 tensor on CUDA device {self.device} is required")
        return 8 if ids.dtype == torch.int64 else 4

    def atomo_embedding(self, table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, out: Optional[torch.Tensor] = None,
                        status: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """scale * table[ids], of shape ids.shape + (cols,).  An id outside the table gives a row of zeros and raises `status` (one int32, set to
        zero by the caller) to ATOMO_ERR_INVALID_ARG.  out must not overlap the table."""
        if stream is not None:
            return self._on(stream, self.atomo_embedding, table, ids, scale, out, status)
        kind = self._operand(table, "table").dtype
        _no_graph(table, out)
        if table.dim() != 2:
            raise ValueError("table: a matrix is required")
        rows, cols = table.shape
        ld = cols if table.is_contiguous() else _rows(table, cols, "table")[1]
        width = self._ids(ids)
        n = ids.numel()
        if out is None:
            out = table.new_empty((n, cols)) if ids.dim() == 1 else table.new_empty((*ids.shape, cols))
            ld_out = cols
        else:
            n_out, ld_out = _rows(self._operand(out, "out", (kind,)), cols, "out")
            if n_out != n:
                raise ValueError(f"out: {n} rows are required")
            _written((out,))
        rc = self.lib.atomo_embedding(self._h, table.data_ptr(), TYPE_CODES[kind], rows, cols, ld, ids.data_ptr(), width, n, scale, out.data_ptr(), ld_out,
                                      self._status(status) if status is not None else None, self._own_stream())
        self._check(rc, "atomo_embedding")
        return out

    def atomo_embedding_backward(self, ids: torch.Tensor, grad: torch.Tensor, rows: int, scale: float = 1.0, padding_idx: int = -1,
                                 out: Optional[torch.Tensor] = None, accumulate: bool = False, status: Optional[torch.Tensor] = None,
                                 stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """The gradient of a table of `rows` rows, fp32: row v is scale times the sum of grad over the tokens of id v, in the order of the
        tokens.  grad: ids.shape + (cols,).  out: a matrix to write to, or with accumulate=True to add to.  Tokens of padding_idx (-1: none) are left out."""
        if stream is not None:
            return self._on(stream, self.atomo_embedding_backward, ids, grad, rows, scale, padding_idx, out, accumulate, status)
        code = TYPE_CODES[self._operand(grad, "grad").dtype]
        _no_graph(grad, out)
        width = self._ids(ids)
        if grad.dim() < 1 or grad.shape[:-1] != ids.shape:
            raise ValueError("grad: the shape of ids with one more dimension is required")
        n, cols = ids.numel(), grad.shape[-1]
        ld = cols if grad.is_contiguous() else _rows(grad, cols, "grad")[1] if n and cols else max(cols, 1)
        if out is None:
            if accumulate:
                raise ValueError("accumulate needs out")
            out = self._floats.new_empty((rows, cols))
            ld_out = cols
        else:
            n_out, ld_out = _rows(self._operand(out, "out", (torch.float32,)), cols, "out")
            if n_out != rows:
                raise ValueError(f"out: {rows} rows are required")
            _written((out,))
        s = self._own_stream()
        nbytes = self.lib.atomo_embedding_workspace_bytes(n, rows, cols)
        if nbytes < 0:
            raise AtomoError(1, "atomo_embedding_workspace_bytes")
        ws = self._scratch(nbytes) if nbytes else None
        rc = self.lib.atomo_embedding_backward(self._h, ids.data_ptr(), width, n, grad.data_ptr(), code, ld, rows, cols, scale, padding_idx, out.data_ptr(), ld_out,
                                               1 if accumulate else 0, self._status(status), ws.data_ptr() if nbytes else None, nbytes, s)
        self._check(rc, "atomo_embedding_backward")
        return out

    def _weight(self, weight, cols: int, what: str):
        """(pointer, type) of a layer norm's weight or bias, which may be None."""
        if weight is None:
            return None, None
        kind = self._operand(weight, what).dtype
        if weight.numel() != cols or not weight.is_contiguous():
            raise ValueError(f"{what}: a contiguous tensor of {cols} elements is required")
        return weight.data_ptr(), kind

    def atomo_layer_norm(self, x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
                         out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
        """Layer norm over the last dimension: (y, mean, rstd), y of x's type and shape, mean and rstd in fp32 with one value per row.  out may
        be x."""
        if stream is not None:
            return self._on(stream, self.atomo_layer_norm, x, weight, bias, eps, out)
        kind = self._operand(x, "x").dtype
        _no_graph(x, weight, bias, out)
        shape = x.shape
        cols = shape[-1] if shape else 0
        w, wkind = self._weight(weight, cols, "weight")
        b, bkind = self._weight(bias, cols, "bias")
        if w is not None and b is not None and wkind is not bkind:
            raise ValueError("weight and bias must have one type")
        rows, ld = (x.numel() // max(cols, 1), cols) if x.is_contiguous() else _rows(x, cols, "x")
        if out is None:
            out, ld_out = (torch.empty_like(x) if ld == cols else torch.empty(shape, dtype=kind, device=x.device)), cols
        else:
            if self._operand(out, "out", (kind,)).shape != shape:
                raise ValueError("out: the shape of x is required")
            ld_out = cols if out.is_contiguous() else _rows(out, cols, "out")[1]
            _written((out,))
        lines = rows if len(shape) == 2 else shape[:-1]
        mean, rstd = self._floats.new_empty(lines), self._floats.new_empty(lines)
        rc = self.lib.atomo_layer_norm(self._h, x.data_ptr(), TYPE_CODES[kind], rows, cols, ld, w, b, TYPE_CODES[wkind or bkind or kind], eps, out.data_ptr(), ld_out,
                                       mean.data_ptr(), rstd.data_ptr(), self._own_stream())
        self._check(rc, "atomo_layer_norm")
        return out, mean, rstd

    def atomo_layer_norm_backward(self, dy: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], mean: torch.Tensor, rstd: torch.Tensor,
                                  out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
        """(dx, dweight, dbias) of atomo_layer_norm: dx of x's type, dweight and dbias in fp32, whatever the weight's type.  out (for dx) may
        be dy or x."""
        if stream is not None:
            return self._on(stream, self.atomo_layer_norm_backward, dy, x, weight, mean, rstd, out)
        kind = self._operand(x, "x").dtype
        self._operand(dy, "dy", (kind,))
        _no_graph(dy, x, weight, out)
        shape = x.shape
        cols = shape[-1] if shape else 0
        if dy.shape != shape:
            raise ValueError("dy: the shape of x is required")
        rows, ld = (x.numel() // max(cols, 1), cols) if x.is_contiguous() else _rows(x, cols, "x")
        ld_dy = cols if dy.is_contiguous() else _rows(dy, cols, "dy")[1]
        for name, t in (("mean", mean), ("rstd", rstd)):
            if t.dtype != torch.float32 or t.get_device() != self.device or t.numel() != rows or not t.is_contiguous():
                raise ValueError(f"{name}: {rows} contiguous fp32 numbers on CUDA device {self.device} are required")
        w, wkind = self._weight(weight, cols, "weight")
        if out is None:
            out, ld_dx = (torch.empty_like(x) if ld == cols else torch.empty(shape, dtype=kind, device=x.device)), cols
        else:
            if self._operand(out, "out", (kind,)).shape != shape:
                raise ValueError("out: the shape of x is required")
            ld_dx = cols if out.is_contiguous() else _rows(out, cols, "out")[1]
            _written((out,))
        dweight, dbias = self._floats.new_empty(cols), self._floats.new_empty(cols)
        s = self._own_stream()
        nbytes = self.lib.atomo_layer_norm_workspace_bytes(rows, cols)
        if nbytes < 0:
            raise AtomoError(1, "atomo_layer_norm_workspace_bytes")
        ws = self._scratch(nbytes) if nbytes else None
        rc = self.lib.atomo_layer_norm_backward(self._h, dy.data_ptr(), ld_dy, x.data_ptr(), ld, TYPE_CODES[kind], rows, cols, w, TYPE_CODES[wkind or kind], mean.data_ptr(), rstd.data_ptr(),
                                                out.data_ptr(), ld_dx, dweight.data_ptr(), dbias.data_ptr(), ws.data_ptr() if nbytes else None, nbytes, s)
        self._check(rc, "atomo_layer_norm_backward")
        return out, dweight, dbias

    def read_headers(self, payload: Payload, stream: Optional[torch.cuda.Stream] = None):
        gh = PayloadHeader()
        lh = (LayerHeader * payload.n_layers)()
        rc = self.lib.atomo_payload_read_headers(self._h, ctypes.c_void_p(payload.buf.data_ptr()), payload.n_layers,
                                                 ctypes.byref(gh), lh, self._stream_ptr(stream))
        self._check(rc, "atomo_payload_read_headers")
        return gh, list(lh)

    def payload_status(self, payload: Payload, stream: Optional[torch.cuda.Stream] = None):
        worst, first = ctypes.c_int32(0), ctypes.c_int32(-1)
        rc = self.lib.atomo_payload_status(self._h, ctypes.c_void_p(payload.buf.data_ptr()), payload.n_layers,
                                           ctypes.byref(worst), ctypes.byref(first), self._stream_ptr(stream))
        self._check(rc, "atomo_payload_status")
        return int(worst.value), int(first.value)

    def set_profiling(self, on: bool):
        self._check(self.lib.atomo_set_profiling(self._h, 1 if on else 0), "atomo_set_profiling")

    def stage_times(self):
        ms = (ctypes.c_float * len(STAGES))()
        ln = (ctypes.c_int64 * len(STAGES))()
        self._check(self.lib.atomo_get_stage_times(self._h, ms, ln), "atomo_get_stage_times")
        return {k: float(ms[i]) for i, k in enumerate(STAGES)}, {k: int(ln[i]) for i, k in enumerate(STAGES)}

    def stage_totals(self):
        """(ms per stage, launches per stage, calls) summed over all encode / decode calls since profiling was switched
        on; the calls themselves do not wait for their events, this does."""
        ms = (ctypes.c_double * len(STAGES))()
        ln = (ctypes.c_int64 * len(STAGES))()
        calls = ctypes.c_int64(0)
        self._check(self.lib.atomo_get_stage_totals(self._h, ms, ln, ctypes.byref(calls)), "atomo_get_stage_totals")
        return ({k: float(ms[i]) for i, k in enumerate(STAGES)}, {k: int(ln[i]) for i, k in enumerate(STAGES)},
                int(calls.value))

    def set_persistent_eig(self, enabled):
        """Eigen-solver scheme.  0 / False: Jacobi, one launch per step; 1 / True: persistent cooperative launches;
        2: Jacobi in thread-block clusters first; 3 (default): the tridiagonal routes (any short side up to 4096)."""
        self._check(self.lib.atomo_set_persistent_eig(self._h, int(enabled)), "atomo_set_persistent_eig")

    def set_entrywise_format(self, fmt: int, sat_cap: int = 0):
        """EW_EXPLICIT (idx, val per kept atom) or EW_COMPACT (16-bit entry per kept atom with p < 1, one scalar c,
        explicit values only for the atoms with p = 1, of which at most sat_cap per vector)."""
        self._check(self.lib.atomo_set_entrywise_format(self._h, int(fmt), int(sat_cap)), "atomo_set_entrywise_format")
        self._ew_format, self._ew_sat_cap = int(fmt), (int(sat_cap) if int(fmt) == EW_COMPACT else 0)

    def set_entrywise_launch(self, two_kernels):
        """0 / False (default): one cooperative kernel per vector that fits one wave of resident CTAs, the keep decisions
        taken on the candidate list of its first pass where that holds every kept atom; 1 / True: always the solve kernel
        followed by the sample / pack kernel; 2: the one-kernel form without the list.  Same payloads in every form."""
        self._check(self.lib.atomo_set_entrywise_launch(self._h, int(two_kernels)), "atomo_set_entrywise_launch")

    def entrywise_list_chunks(self, vec: int = 0):
        """(chunks of the last entry-wise encode of vector `vec` that decided on their candidate list, chunks of the
        one-kernel form: 0 if the two-kernel form ran).  Synchronises."""
        a, b = ctypes.c_uint32(0), ctypes.c_uint32(0)
        self._check(self.lib.atomo_get_entrywise_list_chunks(self._h, int(vec), ctypes.byref(a), ctypes.byref(b)),
                    "atomo_get_entrywise_list_chunks")
        return int(a.value), int(b.value)

    def table_uploads(self):
        """(calls that uploaded their descriptor tables, calls that found them on the device) since the context was made."""
        up, re = ctypes.c_int64(0), ctypes.c_int64(0)
        self._check(self.lib.atomo_get_table_uploads(self._h, ctypes.byref(up), ctypes.byref(re)), "atomo_get_table_uploads")
        return int(up.value), int(re.value)

    def set_tridiag_ctas(self, ctas_per_layer: int):
        """CTAs per layer of the band reduction (short sides above 512): 0 = chosen per batch, else 1,
        2, 4, 8 or 16.  The payload does not depend on it."""
        self._check(self.lib.atomo_set_tridiag_ctas(self._h, int(ctas_per_layer)), "atomo_set_tridiag_ctas")

    def limit_tridiag_route(self, band_ctas: int = -1, chase_clusters: int = -1):
        """Test hook: what the occupancy queries of the two-stage reduction count as at most (-1: as they are)."""
        self._check(self.lib.atomo_limit_tridiag_route(self._h, int(band_ctas), int(chase_clusters)), "atomo_limit_tridiag_route")

    def limit_workspace(self, n_bytes: int = -1):
        """Most that the context's workspace may grow to (-1: no limit); a spectral encode that needs more does without integer digits."""
        self._check(self.lib.atomo_limit_workspace(self._h, int(n_bytes)), "atomo_limit_workspace")

    def last_eig_scheme(self) -> int:
        return int(self.lib.atomo_last_eig_scheme(self._h))

    def set_gram_path(self, tensor_cores: bool):
        self._check(self.lib.atomo_set_gram_path(self._h, 1 if tensor_cores else 0), "atomo_set_gram_path")

    def set_sigma_refinement(self, min_short_side: int):
        self._check(self.lib.atomo_set_sigma_refinement(self._h, int(min_short_side)), "atomo_set_sigma_refinement")

    def set_eig_mode(self, mode: int):
        self._check(self.lib.atomo_set_eig_mode(self._h, int(mode)), "atomo_set_eig_mode")

    def set_eig_params(self, max_sweeps: int, tol: float):
        self._check(self.lib.atomo_set_eig_params(self._h, int(max_sweeps), float(tol)), "atomo_set_eig_params")
