"""ctypes binding of libarchead.so (argument marshalling only).

Every step of the forward runs in the library's HIP kernels; this module only
turns torch tensors into pointers, sizes and the caller's stream.  It fails
loudly when the library has not been built: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libarchead.so")
HOST_LIB_PATH = os.path.join(_PKG, "libarchead_host.so")

ABI_VERSION = 3
OK, E_INVALID_ARG, E_MISALIGNED, E_UNSUPPORTED, E_WORKSPACE, E_HIP = range(6)
F32, BF16, F16, I32, I64, I8, U8, I5 = range(8)
INT4_V1 = 1
OP_LOGITS, OP_LOGITS_CE, OP_ARGMAX, OP_TOPK, OP_FIDELITY, OP_BEAM = 0, 1, 2, 3, 4, 5
TOPK_MAX = 64
BEAM_MAX = 32
(LAUNCH_GEMV_BLOCKS_PER_CU, LAUNCH_GEMV_GRID, LAUNCH_DEC_BLOCKS, LAUNCH_MID_BLOCKS,
 LAUNCH_TILE_WAVES, LAUNCH_TILE_ROWS, LAUNCH_T_SPIN_LIMIT) = range(7)
NOALLOC_SCRATCH_BYTES = 4 << 20   # ARCHEAD_NOALLOC_SCRATCH_BYTES of include/archead.h


class ArcheadError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"archead status {status}: {msg}")
        self.status = status


class Desc(ctypes.Structure):
    _fields_ = [("abi_version", ctypes.c_uint32), ("V", ctypes.c_int64),
                ("d", ctypes.c_int64), ("g", ctypes.c_int64),
                ("r_c", ctypes.c_int64), ("r_r", ctypes.c_int64),
                ("g_v", ctypes.c_int64), ("g_b", ctypes.c_int64),
                ("int4_encoding", ctypes.c_int32), ("scale_dtype", ctypes.c_int32),
                ("factor_dtype", ctypes.c_int32), ("core_u_dtype", ctypes.c_int32)]

    @classmethod
    def make(cls, V, d, g, rc, rr, gV=None, gB=None, abi=ABI_VERSION,
             enc=INT4_V1, scale_dtype=F16, factor_dtype=I8, core_u_dtype=I8):
        return cls(abi, V, d, g, rc, rr, d if gV is None else gV,
                   d if gB is None else gB, enc, scale_dtype, factor_dtype, core_u_dtype)


class BuildDesc(ctypes.Structure):
    """archead_build_desc: shape and parameters of a head construction."""
    _fields_ = [("abi_version", ctypes.c_uint32), ("V", ctypes.c_int64), ("d", ctypes.c_int64),
                ("N", ctypes.c_int64), ("g", ctypes.c_int64), ("r_c", ctypes.c_int64),
                ("r_r", ctypes.c_int64), ("g_b", ctypes.c_int64), ("p", ctypes.c_double),
                ("lam", ctypes.c_double), ("oversample", ctypes.c_int64),
                ("power_iters", ctypes.c_int64)]


class Ptrs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "res_codes", "res_scales", "core_u", "core_u_scale", "core_v",
        "core_v_scale", "corr_a", "corr_a_scale", "corr_b", "corr_b_scale",
        "res_row_scales")]


class StateLayout(ctypes.Structure):
    """archead_state_layout: a row of a state, sizes and strides in bytes."""
    _fields_ = [(n, ctypes.c_int64) for n in (
        "n_outer", "positions", "pos_bytes", "src_row", "src_outer", "src_pos",
        "dst_row", "dst_outer", "dst_pos")]


class AdaptersDesc(ctypes.Structure):
    """archead_adapters: the low-rank pairs of many requests."""
    _fields_ = ([(n, ctypes.c_void_p) for n in ("a", "b", "scales", "ranks")] +
                [(n, ctypes.c_int64) for n in ("n", "R", "a_adapter", "a_row", "b_adapter", "b_row")])


_SIGS = {
    "archead_validate_desc": (ctypes.c_int, [ctypes.POINTER(Desc)]),
    "archead_create": (ctypes.c_int, [ctypes.POINTER(Desc), ctypes.POINTER(Ptrs),
                                      ctypes.POINTER(ctypes.c_void_p)]),
    "archead_destroy": (None, [ctypes.c_void_p]),
    "archead_workspace_bytes": (ctypes.c_size_t, [ctypes.c_void_p, ctypes.c_int64,
                                                  ctypes.c_int]),
    "archead_logits": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
                                      ctypes.c_int64, ctypes.c_void_p, ctypes.c_int,
                                      ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t,
                                      ctypes.c_void_p]),
    "archead_logits_ce": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
                                         ctypes.c_int64, ctypes.c_void_p, ctypes.c_int,
                                         ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                         ctypes.c_size_t, ctypes.c_void_p]),
    "archead_logits_argmax": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
                                             ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p,
                                             ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "archead_logit_fidelity_head": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p,
                                                   ctypes.c_int64, ctypes.c_int64,
                                                   ctypes.c_void_p, ctypes.c_int64,
                                                   ctypes.c_void_p, ctypes.c_void_p,
                                                   ctypes.c_void_p, ctypes.c_void_p,
                                                   ctypes.c_void_p, ctypes.c_size_t,
                                                   ctypes.c_void_p]),
    "archead_logits_topk": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
                                           ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p,
                                           ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                           ctypes.c_size_t, ctypes.c_void_p]),
    "archead_logits_noalloc": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
                                              ctypes.c_int64, ctypes.c_void_p, ctypes.c_int,
                                              ctypes.c_int64, ctypes.c_void_p]),
    "archead_fidelity_workspace_bytes": (ctypes.c_size_t, [ctypes.c_int64, ctypes.c_int64]),
    "archead_logit_fidelity": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                              ctypes.c_int64, ctypes.c_int64, ctypes.c_int64,
                                              ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                              ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                              ctypes.c_void_p]),
    "archead_build_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(BuildDesc)]),
    "archead_build_head": (ctypes.c_int, [ctypes.POINTER(BuildDesc), ctypes.c_void_p,
                                          ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64,
                                          ctypes.c_void_p, ctypes.POINTER(Ptrs), ctypes.c_void_p,
                                          ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                          ctypes.c_void_p]),
    "archead_quantize_i8": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int64,
                                           ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p,
                                           ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p]),
    "archead_matmul_i8": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                         ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                         ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
                                         ctypes.c_int64, ctypes.c_void_p, ctypes.c_int,
                                         ctypes.c_int64, ctypes.c_void_p]),
    "archead_rms_norm": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_int64,
                                        ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                        ctypes.c_int, ctypes.c_float, ctypes.c_double, ctypes.c_void_p,
                                        ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                        ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p]),
    "archead_adapters_workspace_bytes": (ctypes.c_size_t, [ctypes.c_int64, ctypes.c_int64, ctypes.c_int64,
                                                           ctypes.c_int64]),
    "archead_adapters_add": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_void_p,
                                            ctypes.c_int, ctypes.c_int64, ctypes.POINTER(AdaptersDesc),
                                            ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_int64,
                                            ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                            ctypes.c_size_t, ctypes.c_void_p]),
    "archead_head_loss_workspace_bytes": (ctypes.c_size_t, [ctypes.c_int64, ctypes.c_int64, ctypes.c_int64,
                                                            ctypes.c_void_p, ctypes.c_int64, ctypes.c_int]),
    "archead_head_loss": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64,
                                         ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_int64,
                                         ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                         ctypes.c_size_t, ctypes.c_void_p]),
    "archead_head_loss_grad": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64,
                                              ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                              ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p,
                                              ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                              ctypes.c_size_t, ctypes.c_void_p]),
    "archead_beam_workspace_bytes": (ctypes.c_size_t, [ctypes.c_int64, ctypes.c_int64]),
    "archead_beam_select": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int64,
                                           ctypes.c_int64, ctypes.c_int64, ctypes.c_int64,
                                           ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
                                           ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                           ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                           ctypes.c_size_t, ctypes.c_void_p]),
    "archead_logits_beam": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
                                           ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p,
                                           ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32,
                                           ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                           ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                           ctypes.c_void_p]),
    "archead_beam_reorder": (ctypes.c_int, [ctypes.POINTER(StateLayout), ctypes.c_int64,
                                            ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
                                            ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p,
                                            ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]),
    "archead_set_gemv_max_m": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64]),
    "archead_get_gemv_max_m": (ctypes.c_int64, [ctypes.c_void_p]),
    "archead_set_dec_range": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64]),
    "archead_get_dec_range": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int64),
                                             ctypes.POINTER(ctypes.c_int64)]),
    "archead_set_mid_range": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64]),
    "archead_get_mid_range": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int64),
                                             ctypes.POINTER(ctypes.c_int64)]),
    "archead_set_timing_events": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p,
                                                 ctypes.c_void_p]),
    "archead_set_launch": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int64]),
    "archead_get_launch": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int,
                                          ctypes.POINTER(ctypes.c_int64)]),
    "archead_prepared_bytes": (ctypes.c_size_t, [ctypes.c_void_p]),
    "archead_prepare": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                       ctypes.c_void_p]),
    "archead_packed_bytes": (ctypes.c_uint64, [ctypes.POINTER(Desc)]),
    "archead_pack_int4": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
                                         ctypes.c_void_p]),
    "archead_pack_int5": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
                                         ctypes.c_void_p]),
    "archead_unpack_int5": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
                                           ctypes.c_void_p]),
    "archead_unpack_int4": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
                                           ctypes.c_void_p]),
    "archead_status_str": (ctypes.c_char_p, [ctypes.c_int]),
    "archead_last_error": (ctypes.c_char_p, []),
}

HOST_SYMBOLS = ("archead_validate_desc", "archead_set_gemv_max_m", "archead_set_timing_events",
                "archead_get_gemv_max_m", "archead_set_dec_range", "archead_get_dec_range",
                "archead_set_mid_range", "archead_get_mid_range",
                "archead_set_launch", "archead_get_launch",
                "archead_packed_bytes", "archead_pack_int4", "archead_pack_int5",
                "archead_unpack_int5",
                "archead_unpack_int4", "archead_status_str", "archead_last_error")

_libs = {}


def _load(path: str, names) -> ctypes.CDLL:
    if path in _libs:
        return _libs[path]
    if not os.path.exists(path):
        raise RuntimeError(
            f"{os.path.basename(path)} is not built; run "
            "`python -m paper_2608_02703_amd.build` (or __graft_entry__.build())")
    h = ctypes.CDLL(path)
    for n in names:
        res, args = _SIGS[n]
        f = getattr(h, n)
        f.restype = res
        f.argtypes = args
    _libs[path] = h
    return h


def lib() -> ctypes.CDLL:
    """The HIP library (all entry points).  ARCHEAD_LIB may name another
    build of it (tuning experiments)."""
    path = os.environ.get("ARCHEAD_LIB", LIB_PATH)
    return _libs.get(path) or _load(path, _SIGS)


def host_lib(path: Optional[str] = None) -> ctypes.CDLL:
    """A host-only build of the argument checks and packers (g++)."""
    return _load(path or HOST_LIB_PATH, HOST_SYMBOLS)


def _check(st: int, L=None):
    if st != OK:
        L = L or lib()
        raise ArcheadError(st, L.archead_last_error().decode())


def validate_desc(desc: Desc, L=None) -> int:
    L = L or lib()
    return L.archead_validate_desc(ctypes.byref(desc))


def packed_bytes(desc: Desc, L=None) -> int:
    L = L or lib()
    return int(L.archead_packed_bytes(ctypes.byref(desc)))


def pack_int4(codes: np.ndarray, L=None) -> np.ndarray:
    L = L or lib()
    c = np.ascontiguousarray(codes, dtype=np.int8)
    rows, d = c.shape
    out = np.empty((rows, d // 2), dtype=np.uint8)
    _check(L.archead_pack_int4(c.ctypes.data, rows, d, out.ctypes.data), L)
    return out


def pack_int5(codes: np.ndarray, L=None) -> np.ndarray:
    """int codes [rows, r] in [-16, 15] -> ARCHEAD_I5 words uint32 [rows, ceil(r/6)]."""
    L = L or lib()
    c = np.ascontiguousarray(codes, dtype=np.int8)
    rows, r = c.shape
    out = np.empty((rows, (r + 5) // 6), dtype=np.uint32)
    _check(L.archead_pack_int5(c.ctypes.data, rows, r, out.ctypes.data), L)
    return out


def unpack_int5(words: np.ndarray, r: int, L=None) -> np.ndarray:
    L = L or lib()
    w = np.ascontiguousarray(words, dtype=np.uint32)
    if w.shape[1] != (r + 5) // 6:
        raise ValueError("ARCHEAD_I5 rows must hold ceil(r / 6) words")
    out = np.empty((w.shape[0], r), dtype=np.int8)
    _check(L.archead_unpack_int5(w.ctypes.data, w.shape[0], r, out.ctypes.data), L)
    return out


def unpack_int4(packed: np.ndarray, d: int, L=None) -> np.ndarray:
    L = L or lib()
    p = np.ascontiguousarray(packed, dtype=np.uint8)
    rows = p.shape[0]
    if p.shape[1] * 2 != d:
        raise ValueError("packed row length must be d/2")
    out = np.empty((rows, d), dtype=np.int8)
    _check(L.archead_unpack_int4(p.ctypes.data, rows, d, out.ctypes.data), L)
    return out


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


def logit_fidelity(ref, test):
    """Per-position fidelity of `test` logits to reference logits `ref`, both
    fp32 [M, V] CUDA tensors with unit column stride (archead_logit_fidelity):
    returns (kl fp32 [M], sq fp32 [M], ref_idx int64 [M], rank int64 [M]) on
    the same device, computed on the current stream."""
    import torch
    if ref.dtype != torch.float32 or test.dtype != torch.float32:
        raise TypeError("logits must be float32")
    if ref.dim() != 2 or ref.shape != test.shape:
        raise ValueError("ref and test must both be [M, V]")
    if ref.stride(1) != 1 or test.stride(1) != 1:
        raise ValueError("logit rows must be contiguous")
    M, V = ref.shape
    dev = ref.device
    kl = torch.empty(M, dtype=torch.float32, device=dev)
    sq = torch.empty(M, dtype=torch.float32, device=dev)
    idx = torch.empty(M, dtype=torch.int64, device=dev)
    rank = torch.empty(M, dtype=torch.int64, device=dev)
    L = lib()
    if M == 0:
        return kl, sq, idx, rank
    ws = torch.empty(int(L.archead_fidelity_workspace_bytes(M, V)), dtype=torch.uint8, device=dev)
    stream = ctypes.c_void_p(torch.cuda.current_stream(dev).cuda_stream)
    _check(L.archead_logit_fidelity(_ptr(ref), ref.stride(0), _ptr(test), test.stride(0), M, V,
                                    _ptr(kl), _ptr(sq), _ptr(idx), _ptr(rank), _ptr(ws),
                                    ws.numel(), stream), L)
    return kl, sq, idx, rank


_FLOAT_CODES = {}   # torch dtype -> dtype code, filled when torch is there


def _float_code(dtype, what):
    if not _FLOAT_CODES:
        import torch
        _FLOAT_CODES.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
    code = _FLOAT_CODES.get(dtype)
    if code is None:
        raise TypeError(f"{what} must be float32, bfloat16 or float16")
    return code


def _gpu_of(t, what):
    """Index of the GPU a tensor is on."""
    if not t.is_cuda:
        raise ValueError(f"{what} must be on a GPU")
    return t.get_device()


def _matrix(t, what, gpu, dtype=None, shape=None):
    """The leading dimension of a 2-D tensor on a GPU with unit column stride
    (of a single row, one that holds the row)."""
    if t.get_device() != gpu or not t.is_cuda:
        raise ValueError(f"{what} must be on GPU {gpu}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}")
    if t.dim() != 2 or (shape is not None and t.shape != shape):
        raise ValueError(f"{what} must be 2-D" if shape is None else f"{what} must have shape {list(shape)}")
    (rows, cols), (ld, step) = t.shape, t.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{what} must have unit column stride")
    return ld if rows > 1 else max(ld, cols)


def _dense(t, what, gpu, dtypes, shape):
    """Checks a contiguous tensor of a shape and one of some dtypes on a GPU."""
    if t.get_device() != gpu or not t.is_cuda:
        raise ValueError(f"{what} must be on GPU {gpu}")
    if t.dtype not in dtypes:
        raise TypeError(f"{what} must be {' or '.join(str(d) for d in dtypes)}")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous with shape {list(shape)}")


def _launch(gpu, fn, *args):
    """fn(*args, stream) with `gpu` the current one, on its current stream (its
    handle without a Stream object: these calls take a few microseconds)."""
    import torch
    if torch.cuda.current_device() == gpu:
        st = fn(*args, torch._C._cuda_getCurrentRawStream(gpu))
    else:
        with torch.cuda.device(gpu):
            st = fn(*args, torch._C._cuda_getCurrentRawStream(gpu))
    if st != OK:
        _check(st)


def quantize_i8(x, codes=None, scales=None):
    """Rows of x (float32, bfloat16 or float16 [M, d] on the GPU) rounded to
    8 bits: returns (codes int8 [M, d], scales float32 [M]) with x about codes *
    scales[:, None] (archead_quantize_i8).  Rows are tokens, or the output
    channels of a weight."""
    import torch
    gpu = _gpu_of(x, "x")
    ldx = _matrix(x, "x", gpu)
    code = _float_code(x.dtype, "x")
    M, d = x.shape
    ldc = d
    if codes is None:
        codes = torch.empty((M, d), dtype=torch.int8, device=x.device)
    else:
        ldc = _matrix(codes, "codes", gpu, torch.int8, (M, d))
    if scales is None:
        scales = torch.empty(M, dtype=torch.float32, device=x.device)
    else:
        _dense(scales, "scales", gpu, (torch.float32,), (M,))
    _launch(gpu, lib().archead_quantize_i8, x.data_ptr(), code, M, d, ldx, codes.data_ptr(), ldc,
            scales.data_ptr())
    return codes, scales


def matmul_i8(a, a_scales, b, b_scales, bias=None, out=None, out_dtype=None):
    """a int8 [M, K] x b int8 [N, K] -> out [M, N] = (a @ b.T) * a_scales[:,
    None] * b_scales (+ bias), the sums in exact integers (archead_matmul_i8).
    Scales and bias are float32; out is float32 (the default), bfloat16 or
    float16."""
    import torch
    gpu = _gpu_of(a, "a")
    lda = _matrix(a, "a", gpu, torch.int8)
    ldb = _matrix(b, "b", gpu, torch.int8)
    M, K = a.shape
    N, Kb = b.shape
    if Kb != K:
        raise ValueError("a and b must have the same number of columns")
    f32 = (torch.float32,)
    _dense(a_scales, "a_scales", gpu, f32, (M,))
    _dense(b_scales, "b_scales", gpu, f32, (N,))
    if bias is not None:
        _dense(bias, "bias", gpu, f32, (N,))
    if out is None:
        out_dtype = out_dtype or torch.float32
        code = _float_code(out_dtype, "out_dtype")
        out, ldo = torch.empty((M, N), dtype=out_dtype, device=a.device), N
    else:
        if out_dtype is not None and out.dtype != out_dtype:
            raise TypeError("out and out_dtype disagree")
        code = _float_code(out.dtype, "out")
        ldo = _matrix(out, "out", gpu, None, (M, N))
    _launch(gpu, lib().archead_matmul_i8, a.data_ptr(), lda, a_scales.data_ptr(), b.data_ptr(), ldb,
            b_scales.data_ptr(), None if bias is None else bias.data_ptr(), M, N, K, out.data_ptr(), code, ldo)
    return out


def _norm_call(x, weight, eps, residual, offset, total, out, codes, scales):
    """archead_rms_norm around its checks; returns the sums' tensor, or None."""
    import torch
    gpu = _gpu_of(x, "x")
    ldx = _matrix(x, "x", gpu)
    code = _float_code(x.dtype, "x")
    M, d = x.shape
    _dense(weight, "weight", gpu, (x.dtype, torch.float32), (d,))
    ldr = ldt = ldo = ldc = d
    if residual is not None:
        ldr = _matrix(residual, "residual", gpu, x.dtype, (M, d))
        if total is None:
            total = x.new_empty((M, d))
        else:
            ldt = _matrix(total, "total", gpu, x.dtype, (M, d))
    elif total is not None:
        raise ValueError("total needs a residual")
    if out is not None:
        ldo = _matrix(out, "out", gpu, x.dtype, (M, d))
    if codes is not None:
        ldc = _matrix(codes, "codes", gpu, torch.int8, (M, d))
        _dense(scales, "scales", gpu, (torch.float32,), (M,))
    _launch(gpu, lib().archead_rms_norm, x.data_ptr(), code, M, d, ldx, _ptr(residual), ldr, weight.data_ptr(),
            _float_code(weight.dtype, "weight"), offset, eps, _ptr(total), ldt, _ptr(out), ldo, _ptr(codes), ldc,
            _ptr(scales))
    return total


def rms_norm(x, weight, eps=1e-6, residual=None, offset=0.0, out=None, total=None):
    """Root-mean-square norm of the rows of x (float32, bfloat16 or float16
    [M, d] on the GPU, d <= 16384), of x + residual where one is given, times
    offset + weight (archead_rms_norm).  Returns the normed rows, and with a
    residual (normed rows, x + residual).  total (where the sum goes) and out may
    each be residual or x, but not both the same."""
    if out is None:
        out = x.new_empty(x.shape)
    total = _norm_call(x, weight, eps, residual, offset, total, out, None, None)
    return out if residual is None else (out, total)


def rms_norm_i8(x, weight, eps=1e-6, residual=None, offset=0.0, normed=False, codes=None, scales=None, total=None):
    """rms_norm with its rows rounded to 8 bits, for matmul_i8: returns (codes
    int8 [M, d], scales float32 [M]), then x + residual where a residual is
    given, then the rows in x's type where normed is True or a tensor for them
    (archead_rms_norm)."""
    import torch
    if codes is None:
        codes = x.new_empty(x.shape, dtype=torch.int8)
    if scales is None:
        scales = x.new_empty(x.shape[0], dtype=torch.float32)
    out = x.new_empty(x.shape) if normed is True else None if normed is False else normed
    total = _norm_call(x, weight, eps, residual, offset, total, out, codes, scales)
    return (codes, scales) + (() if residual is None else (total,)) + (() if out is None else (out,))


def _factors(t, what, gpu, dtype):
    """Steps of the adapters and of the rows of a [n, rows, columns] tensor."""
    if t.get_device() != gpu or not t.is_cuda:
        raise ValueError(f"{what} must be on GPU {gpu}")
    if t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}")
    if t.dim() != 3 or (t.stride(2) != 1 and t.shape[2] > 1):
        raise ValueError(f"{what} must be 3-D with unit column stride")
    return (t.stride(0) if t.shape[0] > 1 else 0), (t.stride(1) if t.shape[1] > 1 else t.shape[2])


def adapters_add(y, x, a, b, ids, scales=None, ranks=None, out=None, ws=None):
    """y + scales[i] * (x @ a[i].T) @ b[i].T with i = ids[m] for each token m,
    and y where ids[m] lies outside [0, n): low-rank adapters of many requests
    beside a shared projection (archead_adapters_add).  y: float32, bfloat16 or
    float16 [M, N]; x: bfloat16 or float16 [M, K]; a [n, R, K] and b [n, N, R] of
    x's type, R <= 256; ids: int32 or int64 [M]; scales: float32 [n] or None;
    ranks: int32 [n], adapters of fewer than R, or None.  out may be y."""
    import torch
    gpu = _gpu_of(y, "y")
    ldy = _matrix(y, "y", gpu)
    ldx = _matrix(x, "x", gpu)
    code, xcode = _float_code(y.dtype, "y"), _float_code(x.dtype, "x")
    (M, N), K = y.shape, x.shape[1]
    a_ad, a_row = _factors(a, "a", gpu, x.dtype)
    b_ad, b_row = _factors(b, "b", gpu, x.dtype)
    n, R = a.shape[:2]
    if x.shape[0] != M or a.shape[2] != K or b.shape != (n, N, R):
        raise ValueError("x must be [M, K], a [n, R, K] and b [n, N, R] with y [M, N]")
    _dense(ids, "ids", gpu, (torch.int64, torch.int32), (M,))
    if scales is not None:
        _dense(scales, "scales", gpu, (torch.float32,), (n,))
    if ranks is not None:
        _dense(ranks, "ranks", gpu, (torch.int32,), (n,))
    if out is None:
        out, ldo = torch.empty((M, N), dtype=y.dtype, device=y.device), N
    else:
        ldo = ldy if out is y else _matrix(out, "out", gpu, y.dtype, (M, N))
    L = lib()
    if ws is None:
        ws = torch.empty(max(L.archead_adapters_workspace_bytes(M, K, R, n), 256), dtype=torch.uint8, device=y.device)
    elif ws.get_device() != gpu or not ws.is_cuda or ws.dtype != torch.uint8 or not ws.is_contiguous():
        raise ValueError("ws must be a contiguous uint8 tensor on the same GPU")
    desc = AdaptersDesc(a.data_ptr(), b.data_ptr(), _ptr(scales), _ptr(ranks), n, R, a_ad, a_row, b_ad, b_row)
    _launch(gpu, L.archead_adapters_add, y.data_ptr(), code, ldy, x.data_ptr(), xcode, ldx, desc, ids.data_ptr(),
            I64 if ids.dtype == torch.int64 else I32, M, N, K, out.data_ptr(), ldo, ws.data_ptr(), ws.numel())
    return out


def _loss_call(x, w, targets, ws, grad):
    """Checks of a head loss's inputs: (gpu, leading arguments, M, V, d, ws)."""
    import torch
    gpu = _gpu_of(x, "x")
    ldx = _matrix(x, "x", gpu, torch.bfloat16)
    ldw = _matrix(w, "w", gpu, torch.bfloat16)
    (M, d), V = x.shape, w.shape[0]
    if w.shape[1] != d:
        raise ValueError("x and w must have the same number of columns")
    _dense(targets, "targets", gpu, (torch.int64, torch.int32), (M,))
    code = I64 if targets.dtype == torch.int64 else I32
    if ws is None:
        need = lib().archead_head_loss_workspace_bytes(M, V, d, w.data_ptr(), ldw, grad)
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=x.device)
    elif ws.get_device() != gpu or not ws.is_cuda or ws.dtype != torch.uint8 or not ws.is_contiguous():
        raise ValueError("ws must be a contiguous uint8 tensor on the same GPU")
    return gpu, (x.data_ptr(), ldx, w.data_ptr(), ldw, targets.data_ptr(), code), M, V, d, ws


def head_loss(x, w, targets, loss=None, lse=None, ws=None):
    """Softmax cross entropy of the dense head w (bfloat16 [V, d]) on the hidden
    states x (bfloat16 [M, d]) without an [M, V] array of logits
    (archead_head_loss): returns (loss float32 [M], lse float32 [M]), both 0 where
    targets (int32 or int64 [M]) lie outside [0, V).  The results carry no autograd
    graph, also where x or w require gradients: head_loss_grad forms those."""
    import torch
    gpu, args, M, V, d, ws = _loss_call(x, w, targets, ws, 0)
    loss = torch.empty(M, dtype=torch.float32, device=x.device) if loss is None else loss
    lse = torch.empty(M, dtype=torch.float32, device=x.device) if lse is None else lse
    _dense(loss, "loss", gpu, (torch.float32,), (M,))
    _dense(lse, "lse", gpu, (torch.float32,), (M,))
    _launch(gpu, lib().archead_head_loss, *args, M, V, d, loss.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.numel())
    return loss, lse


def head_loss_grad(x, w, targets, lse, grad, dx=True, dw=True, ws=None):
    """The gradients of sum(grad * loss) of head_loss, lse its second result and
    grad float32 [M] (archead_head_loss_grad): returns (dx bfloat16 [M, d], dw
    bfloat16 [V, d]).  dx and dw are True, a tensor for the result, or False where it is
    not wanted (then None is returned).  A training step goes on with
    x.backward(dx) and w.grad = dw."""
    import torch
    gpu, args, M, V, d, ws = _loss_call(x, w, targets, ws, 1)
    _dense(lse, "lse", gpu, (torch.float32,), (M,))
    _dense(grad, "grad", gpu, (torch.float32,), (M,))

    def result(t, what, rows):
        if t is None or t is False:
            return None, d
        if t is True:
            return torch.empty((rows, d), dtype=torch.bfloat16, device=x.device), d
        return t, _matrix(t, what, gpu, torch.bfloat16, (rows, d))
    (dx, lddx), (dw, lddw) = result(dx, "dx", M), result(dw, "dw", V)
    if dx is None and dw is None:
        raise ValueError("dx or dw must be wanted")
    _launch(gpu, lib().archead_head_loss_grad, *args, lse.data_ptr(), grad.data_ptr(), M, V, d, _ptr(dx), lddx, _ptr(dw), lddw,
            ws.data_ptr(), ws.numel())
    return dx, dw


def _beam_call(gpu, device, scores, n, finished, end_token, ws, ws_bytes, call):
    """Outputs and workspace of a beam selection, around call(...)."""
    import torch
    if scores.dim() != 2:
        raise ValueError("scores must be [B, K]")
    B, K = scores.shape
    _dense(scores, "scores", gpu, (torch.float32,), (B, K))
    if finished is not None:
        _dense(finished, "finished", gpu, (torch.bool, torch.uint8), (B, K))
    n = int(n)
    if not 1 <= n <= TOPK_MAX:
        raise ValueError(f"n must be in 1 .. {TOPK_MAX}")
    out = torch.empty((B, n), dtype=torch.float32, device=device)
    parents = torch.empty((B, n), dtype=torch.int64, device=device)
    tokens = torch.empty((B, n), dtype=torch.int64, device=device)
    ended = torch.empty((B, n), dtype=torch.bool, device=device) if end_token >= 0 else None
    if ws is None:
        ws = torch.empty(max(ws_bytes(B * K), 256), dtype=torch.uint8, device=device)
    elif ws.get_device() != gpu or not ws.is_cuda or ws.dtype != torch.uint8 or not ws.is_contiguous():
        raise ValueError("ws must be a contiguous uint8 tensor on the same GPU")
    call(B, K, scores.data_ptr(), _ptr(finished), int(end_token), n, out.data_ptr(), parents.data_ptr(),
         tokens.data_ptr(), _ptr(ended), ws.data_ptr(), ws.numel())
    return (out, parents, tokens) if ended is None else (out, parents, tokens, ended)


def beam_select(logits, scores, n, finished=None, end_token=-1, ws=None):
    """The n best continuations of each sequence of a beam search
    (archead_beam_select).  logits: float32, bfloat16 or float16 [B * K, V],
    row b * K + k for beam k of sequence b; scores: float32 [B, K], the beams'
    summed log-probabilities (-inf: a beam not in use); finished: bool [B, K] or
    None, beams that ended (they offer end_token with their score unchanged).
    Returns (scores float32 [B, n], parents int64 [B, n], tokens int64 [B,
    n]), best first, and with an end_token also which of them have ended, bool
    [B, n].  Empty places hold (-inf, -1, -1)."""
    gpu = _gpu_of(logits, "logits")
    ldl = _matrix(logits, "logits", gpu)
    code = _float_code(logits.dtype, "logits")
    R, V = logits.shape
    if scores.numel() != R:
        raise ValueError("logits must have a row for every beam of scores")
    L = lib()

    def call(B, K, *rest):
        _launch(gpu, L.archead_beam_select, logits.data_ptr(), code, B, K, V, ldl, *rest)
    return _beam_call(gpu, logits.device, scores, n, finished, end_token, ws,
                      lambda rows: L.archead_beam_workspace_bytes(rows, V), call)


def _extent(t):
    """[(bytes of a step, steps)] of a tensor, largest step first, and the
    contiguous bytes that are stepped."""
    width, steps = t.element_size(), []
    for st, n in sorted((st * t.element_size(), n) for n, st in zip(t.shape, t.stride()) if n > 1 and st):
        if not steps and st <= width:
            width += st * (n - 1)
        else:
            steps.insert(0, (st, n))
    return steps, width


def _share_memory(a, b):
    """Whether two tensors (of a GPU, without negative strides) hold a byte in
    common: of their steps the largest first, those that bring the rest of both
    together."""
    seen = set()

    def reach(steps, width):
        return sum(st * (n - 1) for st, n in steps) + width

    def meet(sa, sb, off):   # off: the first byte of b's rest from that of a's
        if off >= reach(sa, wa) or -off >= reach(sb, wb) or (len(sa), len(sb), off) in seen:
            return False
        if not sa and not sb:
            return True
        seen.add((len(sa), len(sb), off))
        st = max(sa[:1] + sb[:1])[0]
        na = nb = 1
        if sa and sa[0][0] == st:
            na, sa = sa[0][1], sa[1:]
        if sb and sb[0][0] == st:
            nb, sb = sb[0][1], sb[1:]
        # steps i of b less those of a with  -reach(b's rest) < off + i st < reach(a's rest)
        lo, hi = -((off + reach(sb, wb) - 1) // st), (reach(sa, wa) - 1 - off) // st
        return any(meet(sa, sb, off + i * st) for i in range(max(lo, 1 - na), min(hi, nb - 1) + 1))
    (sa, wa), (sb, wb) = _extent(a), _extent(b)
    return meet(sa, sb, b.data_ptr() - a.data_ptr())


class BeamStates:
    """The states of a beam search's rows (caches of every layer, recurrent
    states, token histories), described once and reordered after every step
    (archead_beam_reorder).

    states: tensors on one GPU of beams * B rows along `row_dim`.  out: tensors
    for the reordered states, of out_beams * B rows (default: beams) and
    otherwise alike, sharing no memory with states; or None to reorder the
    states where they are.  No two destinations share memory.  pos_dim: the
    dimension of the positions, where reorder() is to move the leading ones
    alone.  Of the remaining dimensions, those that do not lie back to back have
    to step as one."""

    def __init__(self, states, beams, out=None, out_beams=None, row_dim=0, pos_dim=None):
        states = list(states)
        self.states, self.beams = states, int(beams)
        self.in_place = out is None
        self.out = states if out is None else list(out)
        self.out_beams = self.beams if out_beams is None else int(out_beams)
        if len(self.out) != len(states):
            raise ValueError("as many out tensors as states are needed")
        if not 1 <= self.beams <= BEAM_MAX or not 1 <= self.out_beams <= TOPK_MAX:
            raise ValueError(f"beams must be in 1 .. {BEAM_MAX} and out_beams in 1 .. {TOPK_MAX}")
        if self.in_place and self.out_beams != self.beams:
            raise ValueError("reordering in place keeps the number of beams")
        self.has_pos = pos_dim is not None
        self.batch = self.device = None
        groups = {}
        for i, (s, d) in enumerate(zip(states, self.out)):
            if not s.is_cuda or d.device != s.device or (self.device or s.device) != s.device:
                raise ValueError("states and out must be on one GPU")
            self.device, self._gpu = s.device, s.get_device()
            if s.dim() == 0 or not -s.dim() <= row_dim < s.dim():
                raise ValueError("states must have a dimension row_dim")
            r = row_dim % s.dim()
            p = None if pos_dim is None else pos_dim % s.dim()
            if pos_dim is not None and (not -s.dim() <= pos_dim < s.dim() or p == r):
                raise ValueError("pos_dim must be a dimension of the states other than row_dim")
            if s.dtype != d.dtype or s.dim() != d.dim() or any(
                    s.shape[k] != d.shape[k] for k in range(s.dim()) if k != r):
                raise ValueError("out must have the states' dtype and, but for rows, their shape")
            B = s.shape[r] // self.beams
            if s.shape[r] != B * self.beams or d.shape[r] != B * self.out_beams or B != (self.batch or B):
                raise ValueError("states must have beams * B rows, out must have out_beams * B")
            self.batch = B
            key = self._layout(s, d, r, p)
            if d.numel():
                groups.setdefault(key, []).append(i)
        # by first byte, with those before that reach it: two destinations, or one
        # and a state, share no memory
        all_ = [(t, True) for t in self.out] + ([] if self.in_place else [(t, False) for t in states])
        open_ = []
        for t, written in sorted(((t, w) for t, w in all_ if t.numel()), key=lambda e: e[0].data_ptr()):
            lo, hi = self._span(t)
            open_ = [e for e in open_ if e[0] > lo]
            for _, u, w in open_:
                if (written or w) and _share_memory(u, t):
                    raise ValueError("two of the destinations share memory" if written and w
                                     else "out shares memory with states")
            open_.append((hi, t, written))
        self._groups = []
        for key, members in groups.items():
            arr = ctypes.c_void_p * len(members)
            self._groups.append((StateLayout(*key), len(members), arr(*[states[i].data_ptr() for i in members]),
                                 arr(*[self.out[i].data_ptr() for i in members])))

    @staticmethod
    def _span(t):
        lo = t.data_ptr()
        return lo, lo + (sum((n - 1) * st for n, st in zip(t.shape, t.stride())) + 1) * t.element_size()

    @staticmethod
    def _layout(s, d, r, p):
        """archead_state_layout of a state and its destination, as a tuple."""
        es = s.element_size()
        # (size, stride of s, stride of d) of the dimensions, smallest steps first
        dims = [(s.shape[k], s.stride(k) * es, d.stride(k) * es) for k in range(s.dim())
                if k not in (r, p) and s.shape[k] != 1]
        dims.sort(key=lambda t: (t[2], t[1]))
        inner, outer = es, (1, 0, 0)
        for n, a, b in dims:
            if outer[0] == 1 and a == inner and b == inner:
                inner *= n
            elif outer[0] == 1:
                outer = (n, a, b)
            elif a == outer[0] * outer[1] and b == outer[0] * outer[2]:
                outer = (outer[0] * n, outer[1], outer[2])
            else:
                raise ValueError("the dimensions of a state that do not lie back to back must step as one")
        rows = (d.shape[r], s.stride(r) * es, d.stride(r) * es)
        pos = (1, 0, 0) if p is None else (s.shape[p], s.stride(p) * es, d.stride(p) * es)
        # a destination's elements are its own: each step passes all smaller ones
        end = inner
        for n, _, b in sorted((outer, pos, rows), key=lambda t: t[2]):
            if n > 1:
                if b < end:
                    raise ValueError("elements of a destination share memory")
                end = b * (n - 1) + end
        return (outer[0], pos[0], inner, rows[1], outer[1], pos[1], rows[2], outer[2], pos[2])

    def reorder(self, parents, lengths=None):
        """Row b * out_beams + j becomes row b * beams + parents[b, j] of the
        states; parents outside [0, beams) leave it as it is.  parents: int64 or
        int32 [B, out_beams].  lengths: int32 [B] or None; positions from
        lengths[b] on stay as they are.  Returns the destinations, on the
        current stream."""
        import torch
        if not self._groups:
            return self.out
        B, n = self.batch, self.out_beams
        _dense(parents, "parents", self._gpu, (torch.int64, torch.int32), (B, n))
        if lengths is not None:
            if not self.has_pos:
                raise ValueError("lengths need pos_dim")
            _dense(lengths, "lengths", self._gpu, (torch.int32,), (B,))
        idx = I64 if parents.dtype == torch.int64 else I32
        fn = lib().archead_beam_reorder
        for layout, count, src, dst in self._groups:
            _launch(self._gpu, fn, layout, count, src, dst, B, self.beams, n, parents.data_ptr(), idx,
                    _ptr(lengths))
        return self.out


def build_head(W, H, rc: int, rr: int, g: int, p: float = 0.75, lam: float = 1e-3, gB=None,
               oversample: int = 8, power_iters: int = 4, seed: int = 0,
               return_factors: bool = False):
    """archead_build_head: construct a packed head on the GPU from a dense
    head W (fp32 [V, d] CUDA tensor) and calibration hidden states H (fp32
    [N, d] CUDA tensor), with the randomized SVD's Gaussian sketch drawn here
    from a seeded torch generator.  Returns a PackedHead over the written
    buffers (and the unquantized A_w, B_w as fp64 tensors when
    return_factors)."""
    import torch
    if W.dtype != torch.float32 or H.dtype != torch.float32 or W.dim() != 2 or H.dim() != 2:
        raise TypeError("W and H must be 2-D float32 tensors")
    if W.stride(1) != 1 or H.stride(1) != 1 or W.shape[1] != H.shape[1]:
        raise ValueError("W and H need unit column stride and the same width d")
    V, d = W.shape
    N = H.shape[0]
    gB = d if gB is None else gB
    dev = W.device
    desc = BuildDesc(ABI_VERSION, V, d, N, g, rc, rr, gB, p, lam, oversample, power_iters)
    L = lib()
    need = int(L.archead_build_workspace_bytes(ctypes.byref(desc)))
    if need == 0:
        raise ArcheadError(E_INVALID_ARG, "invalid construction descriptor")

    def buf(shape, dtype):
        n = int(np.prod(shape))
        return torch.zeros(shape, dtype=dtype, device=dev) if n else None
    bufs = {"res_codes": buf((V, d // 2), torch.uint8), "res_scales": buf((V, d // g), torch.float16),
            "core_u": buf((V, rc), torch.int8), "core_u_scale": buf((V,), torch.float16) if rc else None,
            "core_v": buf((rc, d), torch.int8), "core_v_scale": buf((rc, 1), torch.float16) if rc else None,
            "corr_a": buf((V, rr), torch.int8), "corr_a_scale": buf((V,), torch.float16) if rr else None,
            "corr_b": buf((rr, d), torch.int8),
            "corr_b_scale": buf((rr, d // gB), torch.float16) if rr else None,
            "res_row_scales": None}
    k = rr + oversample if rr else 0
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    omega = torch.randn((max(k, 1), d), dtype=torch.float64, device=dev, generator=gen)
    a_w = torch.empty((V, rr), dtype=torch.float64, device=dev) if (return_factors and rr) else None
    b_w = torch.empty((rr, d), dtype=torch.float64, device=dev) if (return_factors and rr) else None
    ws = torch.empty(need, dtype=torch.uint8, device=dev)
    ptrs = Ptrs(*[_ptr(bufs.get(n)) for n in PackedHead.BUFFERS])
    stream = ctypes.c_void_p(torch.cuda.current_stream(dev).cuda_stream)
    _check(L.archead_build_head(ctypes.byref(desc), _ptr(W), W.stride(0), _ptr(H), H.stride(0),
                                _ptr(omega), ctypes.byref(ptrs), _ptr(a_w), _ptr(b_w), _ptr(ws),
                                ws.numel(), stream), L)
    del ws
    ph = PackedHead(V, d, g, rc, rr, bufs, d, gB)
    return (ph, a_w, b_w) if return_factors else ph


class PackedHead:
    """A packed head resident on the current GPU plus its library handle.

    ``buffers`` maps the buffer names to torch tensors on the device (the
    caller keeps ownership; the handle only borrows them).  A uint8
    ``res_scales`` selects 8-bit group scale codes, with ``res_row_scales``
    (fp16 [V]) the per-row scale; an int32 ``core_u`` of ceil(rc/6) columns
    holds ARCHEAD_I5 words (5-bit codes)."""

    BUFFERS = ("res_codes", "res_scales", "core_u", "core_u_scale", "core_v",
               "core_v_scale", "corr_a", "corr_a_scale", "corr_b", "corr_b_scale",
               "res_row_scales")

    def __init__(self, V, d, g, rc, rr, buffers: dict, gV=None, gB=None):
        import torch  # noqa: F401  (device memory only)
        self.V, self.d, self.g, self.rc, self.rr = V, d, g, rc, rr
        self.gV = d if gV is None else gV
        self.gB = d if gB is None else gB
        self.buffers = buffers
        sc = buffers.get("res_scales")
        u8 = sc is not None and str(sc.dtype) == "torch.uint8"
        cu = buffers.get("core_u")
        i5 = cu is not None and str(cu.dtype) == "torch.int32"
        self.desc = Desc.make(V, d, g, rc, rr, self.gV, self.gB, scale_dtype=U8 if u8 else F16,
                              core_u_dtype=I5 if i5 else I8)
        self.ptrs = Ptrs(*[_ptr(buffers.get(n)) for n in self.BUFFERS])
        self._lib = lib()
        h = ctypes.c_void_p()
        _check(self._lib.archead_create(ctypes.byref(self.desc), ctypes.byref(self.ptrs),
                                        ctypes.byref(h)), self._lib)
        self.handle = h
        self._ws = {}
        self._prep = None

    @classmethod
    def from_arrays(cls, h, device="cuda"):
        """Upload a head given as numpy arrays (the attributes of
        synth.HeadArrays) to ``device``."""
        import torch
        bufs = {}
        for n in cls.BUFFERS:
            a = getattr(h, n, None)
            if a is None:
                bufs[n] = None
                continue
            a = np.ascontiguousarray(a)
            if a.size == 0:
                bufs[n] = None
                continue
            if a.dtype == np.float16:
                t = torch.from_numpy(a.view(np.int16)).view(torch.float16)
            elif a.dtype == np.uint32:               # ARCHEAD_I5 words
                t = torch.from_numpy(a.view(np.int32))
            elif a.dtype == np.uint8:
                t = torch.from_numpy(a)
            else:
                t = torch.from_numpy(a.astype(np.int8, copy=False))
            bufs[n] = t.to(device)
        return cls(h.V, h.d, h.g, h.rc, h.rr, bufs, getattr(h, "gV", None),
                   getattr(h, "gB", None))

    def close(self):
        if getattr(self, "handle", None):
            self._lib.archead_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ------------------------------------------------------------------
    def set_gemv_max_m(self, m: int):
        _check(self._lib.archead_set_gemv_max_m(self.handle, m), self._lib)

    def set_dec_range(self, min_m: int, max_m: int):
        _check(self._lib.archead_set_dec_range(self.handle, min_m, max_m), self._lib)

    def set_mid_range(self, min_m: int, max_m: int):
        _check(self._lib.archead_set_mid_range(self.handle, min_m, max_m), self._lib)

    def set_launch(self, knob: int, value: int):
        """archead_set_launch: one of the LAUNCH_* settings (0, or -1 for
        LAUNCH_T_SPIN_LIMIT, restores the built-in choice)."""
        _check(self._lib.archead_set_launch(self.handle, knob, value), self._lib)

    def get_launch(self, knob: int) -> int:
        v = ctypes.c_int64()
        _check(self._lib.archead_get_launch(self.handle, knob, ctypes.byref(v)), self._lib)
        return v.value

    def force_path(self, path: str):
        """Route every M to one kernel: "dec" (MFMA decode), "mid" (several
        tokens per pass over the head), "gemv" (decode GEMV), "tiled"
        (many-token MFMA) or "auto" (the built-in choice).  Shapes a kernel
        does not support still take another one."""
        off, every = (1, 0), (1, 10 ** 9)
        dec, mid, gemv = {"dec": (every, off, -1), "mid": (off, every, -1),
                          "gemv": (off, off, 10 ** 9), "tiled": (off, off, 0),
                          "auto": ((-1, -1), (-1, -1), -1)}[path]
        self.set_dec_range(*dec)
        self.set_mid_range(*mid)
        self.set_gemv_max_m(gemv)

    def set_timing_events(self, start, stop):
        """start / stop: torch.cuda.Event objects already recorded once (so
        their HIP events exist), or None to switch timing off."""
        p0 = ctypes.c_void_p(start.cuda_event) if start is not None else None
        p1 = ctypes.c_void_p(stop.cuda_event) if stop is not None else None
        _check(self._lib.archead_set_timing_events(self.handle, p0, p1), self._lib)

    def prepare(self, enable: bool = True):
        """Keep the many-token kernel's head-derived tables in a buffer owned
        by this object (built once, on the current stream), or drop it."""
        import torch
        if not enable:
            _check(self._lib.archead_prepare(self.handle, None, 0, None), self._lib)
            self._prep = None
            return
        n = int(self._lib.archead_prepared_bytes(self.handle))
        if n == 0:
            raise ValueError("this head shape has no many-token kernel")
        dev = torch.device("cuda", torch.cuda.current_device())
        buf = torch.empty(n, dtype=torch.uint8, device=dev)
        _check(self._lib.archead_prepare(self.handle, _ptr(buf), n, self._stream(dev)),
               self._lib)
        self._prep = buf

    def prepared_bytes(self) -> int:
        """archead_prepared_bytes: size of the many-token kernel's head-derived
        tables kept by prepare() (0 where the head has no such kernel)."""
        return int(self._lib.archead_prepared_bytes(self.handle))

    def workspace_bytes(self, M: int, op: int = OP_LOGITS) -> int:
        return int(self._lib.archead_workspace_bytes(self.handle, M, op))

    def workspace(self, M: int, op: int, device):
        import torch
        n = self.workspace_bytes(M, op)
        key = (str(device), n)
        ws = self._ws.get(key)
        if ws is None:
            ws = torch.empty(max(n, 256), dtype=torch.uint8, device=device)
            self._ws = {key: ws}
        return ws

    @staticmethod
    def _stream(device):
        import torch
        return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)

    def logits(self, x, out=None, out_dtype=None, ws=None):
        """x: torch.bfloat16 [M, d] (row stride may exceed d) on the GPU."""
        import torch
        if x.dtype != torch.bfloat16 or x.dim() != 2 or x.stride(1) != 1:
            raise ValueError("x must be a 2-D bf16 tensor with unit column stride")
        M = x.shape[0]
        if out is None:
            out = torch.empty((M, self.V), dtype=out_dtype or torch.float32,
                              device=x.device)
        code = {torch.float32: F32, torch.bfloat16: BF16}[out.dtype]
        ws = self.workspace(M, OP_LOGITS, x.device) if ws is None else ws
        _check(self._lib.archead_logits(
            self.handle, _ptr(x), M, x.stride(0), _ptr(out), code, out.stride(0),
            _ptr(ws), ws.numel(), self._stream(x.device)), self._lib)
        return out

    def logits_noalloc(self, x, out=None, out_dtype=None):
        """archead_logits_noalloc: the logits with the library's static
        workspace (no workspace tensor).  x: torch.bfloat16 [M, d] on the GPU."""
        import torch
        if x.dtype != torch.bfloat16 or x.dim() != 2 or x.stride(1) != 1:
            raise ValueError("x must be a 2-D bf16 tensor with unit column stride")
        M = x.shape[0]
        if out is None:
            out = torch.empty((M, self.V), dtype=out_dtype or torch.float32,
                              device=x.device)
        code = {torch.float32: F32, torch.bfloat16: BF16}[out.dtype]
        _check(self._lib.archead_logits_noalloc(
            self.handle, _ptr(x), M, x.stride(0), _ptr(out), code, out.stride(0),
            self._stream(x.device)), self._lib)
        return out

    def logits_argmax(self, x, idx=None, max_logit=None, ws=None):
        """Greedy next token: returns (idx int64 [M], max_logit fp32 [M]), the
        smallest vocabulary index of each token's largest logit."""
        import torch
        if x.dtype != torch.bfloat16 or x.dim() != 2 or x.stride(1) != 1:
            raise ValueError("x must be a 2-D bf16 tensor with unit column stride")
        M = x.shape[0]
        idx = torch.empty(M, dtype=torch.int64, device=x.device) if idx is None else idx
        if max_logit is None:
            max_logit = torch.empty(M, dtype=torch.float32, device=x.device)
        ws = self.workspace(M, OP_ARGMAX, x.device) if ws is None else ws
        _check(self._lib.archead_logits_argmax(
            self.handle, _ptr(x), M, x.stride(0), _ptr(idx), _ptr(max_logit), _ptr(ws),
            ws.numel(), self._stream(x.device)), self._lib)
        return idx, max_logit

    def logits_topk(self, x, k, vals=None, idx=None, ws=None):
        """Top-k selection: returns (vals fp32 [M, k], idx int64 [M, k]), each
        token's k largest logits in decreasing order, equal logits by
        increasing index (archead_logits_topk)."""
        import torch
        if x.dtype != torch.bfloat16 or x.dim() != 2 or x.stride(1) != 1:
            raise ValueError("x must be a 2-D bf16 tensor with unit column stride")
        M = x.shape[0]
        if vals is None:
            vals = torch.empty((M, k), dtype=torch.float32, device=x.device)
        if idx is None:
            idx = torch.empty((M, k), dtype=torch.int64, device=x.device)
        if idx.dim() != 2 or idx.stride(1) != 1 or vals.dim() != 2 or vals.stride(1) != 1 or \
                vals.stride(0) != idx.stride(0):
            raise ValueError("vals and idx must be 2-D with unit column stride and one row stride")
        ws = self.workspace(M, OP_TOPK, x.device) if ws is None else ws
        _check(self._lib.archead_logits_topk(
            self.handle, _ptr(x), M, x.stride(0), int(k), _ptr(vals), _ptr(idx), idx.stride(0),
            _ptr(ws), ws.numel(), self._stream(x.device)), self._lib)
        return vals, idx

    def logits_beam(self, x, scores, n, finished=None, end_token=-1, ws=None):
        """beam_select over this head's logits of the beams' hidden states x,
        bf16 [B * K, d] (archead_logits_beam)."""
        import torch
        gpu = _gpu_of(x, "x")
        ldx = _matrix(x, "x", gpu, torch.bfloat16)
        if x.shape[1] != self.d or scores.numel() != x.shape[0]:
            raise ValueError("x must have d columns and a row for every beam of scores")

        def call(B, K, *rest):
            _launch(gpu, self._lib.archead_logits_beam, self.handle, x.data_ptr(), B, K, ldx, *rest)
        return _beam_call(gpu, x.device, scores, n, finished, end_token, ws,
                          lambda rows: self.workspace_bytes(rows, OP_BEAM), call)

    def logit_fidelity_head(self, x, dense, ws=None):
        """Fidelity of this head to a dense bf16 head [V, d] on the tokens x,
        in the head's tile pass (archead_logit_fidelity_head): returns (kl
        fp32 [M], sq fp32 [M], ref_idx int64 [M], rank int64 [M])."""
        import torch
        if x.dtype != torch.bfloat16 or x.dim() != 2 or x.stride(1) != 1:
            raise ValueError("x must be a 2-D bf16 tensor with unit column stride")
        if dense.dtype != torch.bfloat16 or dense.dim() != 2 or dense.stride(1) != 1:
            raise ValueError("dense must be a 2-D bf16 tensor with unit column stride")
        M = x.shape[0]
        kl = torch.empty(M, dtype=torch.float32, device=x.device)
        sq = torch.empty(M, dtype=torch.float32, device=x.device)
        ref_idx = torch.empty(M, dtype=torch.int64, device=x.device)
        rank = torch.empty(M, dtype=torch.int64, device=x.device)
        ws = self.workspace(M, OP_FIDELITY, x.device) if ws is None else ws
        _check(self._lib.archead_logit_fidelity_head(
            self.handle, _ptr(x), M, x.stride(0), _ptr(dense), dense.stride(0), _ptr(kl),
            _ptr(sq), _ptr(ref_idx), _ptr(rank), _ptr(ws), ws.numel(), self._stream(x.device)),
            self._lib)
        return kl, sq, ref_idx, rank

    def logits_ce(self, x, targets, ce=None, mean=None, ws=None):
        """Fused log-softmax + cross-entropy; returns (ce [M], mean [1])."""
        import torch
        if x.dtype != torch.bfloat16 or x.dim() != 2 or x.stride(1) != 1:
            raise ValueError("x must be a 2-D bf16 tensor with unit column stride")
        M = x.shape[0]
        code = {torch.int32: I32, torch.int64: I64}[targets.dtype]
        ce = torch.empty(M, dtype=torch.float32, device=x.device) if ce is None else ce
        mean = torch.empty(1, dtype=torch.float32, device=x.device) if mean is None else mean
        ws = self.workspace(M, OP_LOGITS_CE, x.device) if ws is None else ws
        _check(self._lib.archead_logits_ce(
            self.handle, _ptr(x), M, x.stride(0), _ptr(targets), code, _ptr(ce),
            _ptr(mean), _ptr(ws), ws.numel(), self._stream(x.device)), self._lib)
        return ce, mean
