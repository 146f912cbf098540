"""ctypes binding of libcsketch.so: same names as include/csketch.h, argument marshalling only.

Tensors must live on a HIP device ("cuda" in torch), be contiguous and have the dtype the C
signature states; the binding checks that and the shapes, passes `tensor.data_ptr()` and the
current torch stream, and raises CsError on a non-zero status.  Nothing is computed here.
"""
from __future__ import annotations

import ctypes
import os

import torch

CS_MAX_R = 16
_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libcsketch.so")
_lib = None


class CsError(RuntimeError):
    pass


class CsRowPlan(ctypes.Structure):
    _fields_ = [("D", ctypes.c_uint64), ("AD", ctypes.c_uint64), ("ADs", ctypes.c_uint64),
                ("Dw", ctypes.c_uint64), ("ADw", ctypes.c_uint64), ("ADws", ctypes.c_uint64),
                ("lanes", ctypes.c_int32), ("scan_steps", ctypes.c_int32)]


CS_MAX_VISITS = 512
CS_FLAG_NO_VISIT_LIST = 1
CS_FLAG_NO_LDS_TABLE = 2


class CsVisitPlan(ctypes.Structure):
    _fields_ = [("K", ctypes.c_uint32), ("ncell", ctypes.c_uint32),
                ("cover", ctypes.c_uint64), ("gmax", ctypes.c_uint64),
                ("cost", ctypes.c_uint64), ("cost_walk", ctypes.c_uint64),
                ("gap", ctypes.c_uint64 * 4),
                ("A", ctypes.c_uint64 * 4), ("As", ctypes.c_uint64 * 4),
                ("code", ctypes.c_uint32 * (CS_MAX_VISITS // 16))]

    def gaps(self):
        """Gap of every visit, in order (decoded from the 2-bit codes)."""
        return [int(self.gap[(self.code[k // 16] >> (2 * (k % 16))) & 3]) for k in range(self.K)]


CS_ANYC_MAX_VISITS = 144


class CsAnycPlan(ctypes.Structure):
    _fields_ = [("K", ctypes.c_uint32), ("omega", ctypes.c_uint32),
                ("cover", ctypes.c_uint64), ("gmax", ctypes.c_uint64),
                ("cost", ctypes.c_uint64), ("cost_direct", ctypes.c_uint64),
                ("gap", ctypes.c_uint32 * CS_ANYC_MAX_VISITS)]

    def gaps(self):
        return [int(self.gap[k]) for k in range(self.K)]


CS_VECTOR_CELLS = 8


class CsVectorPlan(ctypes.Structure):
    _fields_ = [("none", ctypes.c_uint64), ("list", CsVisitPlan),
                ("pad", ctypes.c_uint8 * (ctypes.sizeof(CsAnycPlan) - 8 - ctypes.sizeof(CsVisitPlan)))]


class _CsLists(ctypes.Union):
    _fields_ = [("anyc", CsAnycPlan * CS_MAX_R), ("vector", CsVectorPlan * CS_MAX_R)]


class CsParams(ctypes.Structure):
    _anonymous_ = ("lists",)
    _fields_ = [("r", ctypes.c_uint32), ("c", ctypes.c_uint32),
                ("c_pow2", ctypes.c_uint32), ("flags", ctypes.c_uint32),
                ("seed", ctypes.c_uint64),
                ("a", ctypes.c_uint64 * CS_MAX_R), ("b", ctypes.c_uint64 * CS_MAX_R),
                ("as_", ctypes.c_uint64 * CS_MAX_R), ("bs", ctypes.c_uint64 * CS_MAX_R),
                ("plan", CsRowPlan * CS_MAX_R),
                ("visit", CsVisitPlan * CS_MAX_R),
                ("lists", _CsLists)]


class CsTensorList(ctypes.Structure):
    _fields_ = [("memory", ctypes.c_void_p), ("chunks", ctypes.c_int64), ("count", ctypes.c_int32),
                ("p_fmt", ctypes.c_int32), ("g_fmt", ctypes.c_int32), ("bits", ctypes.c_int32), ("values", ctypes.c_int64)]


class CsAdamw(ctypes.Structure):
    _fields_ = [*((name, ctypes.c_double) for name in ("lr", "beta1", "beta2", "eps", "weight_decay")), ("seed", ctypes.c_uint64)]


class CsPolicy(ctypes.Structure):
    _fields_ = [(name, ctypes.c_float) for name in ("clip_low", "clip_high", "kl", "entropy")]


CS_PREFERENCE_LOGISTIC, CS_PREFERENCE_HINGE, CS_PREFERENCE_SQUARE = 0, 1, 2


class CsPreference(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("mean", ctypes.c_int32), *((name, ctypes.c_float) for name in ("beta", "smoothing", "margin"))]


CS_MUON_MAX_STEPS = 16
CS_MUON_SCALE_SHAPE, CS_MUON_SCALE_RMS, CS_MUON_SCALE_ONE = 0, 1, 2


class CsMatrix(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("g", ctypes.c_void_p), ("m", ctypes.c_void_p),
                *((name, ctypes.c_int64) for name in ("count", "rows", "cols", "p_stride", "p_step", "g_stride", "g_step"))]


class CsMatrixList(ctypes.Structure):
    _fields_ = [("memory", ctypes.c_void_p),
                *((name, ctypes.c_int64) for name in ("matrices", "littles", "thins", "slabs", "pieces", "halves", "tails", "fulls", "work")),
                *((name, ctypes.c_int32) for name in ("p_fmt", "g_fmt", "terms", "moments", "half_kind", "full_kind", "gram_slices",
                                                      "square_slices", "little_cols", "most_pieces"))]


class CsMuon(ctypes.Structure):
    _fields_ = [*((name, ctypes.c_double) for name in ("lr", "momentum", "weight_decay", "eps")),
                *((name, ctypes.c_int32) for name in ("nesterov", "scale", "steps", "reserved")),
                ("coefs", ctypes.c_double * 3 * CS_MUON_MAX_STEPS)]


def library_path() -> str:
    return _LIB_PATH


_SIGNATURES = {
    "cs_params_init": [ctypes.POINTER(CsParams), ctypes.c_uint32, ctypes.c_uint32,
                       ctypes.c_uint64, ctypes.c_int64],
    "cs_hash_debug": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_int64,
                      ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p],
    "cs_hash_debug_range": [ctypes.POINTER(CsParams), ctypes.c_int64, ctypes.c_int64,
                            ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p],
    "cs_sketch_zero": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_void_p],
    "cs_sketch_accumulate": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_void_p,
                             ctypes.c_int64, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p],
    "cs_sketch_accumulate_batch": [ctypes.POINTER(CsParams), ctypes.POINTER(ctypes.c_void_p),
                                   ctypes.POINTER(ctypes.c_void_p), ctypes.c_int32,
                                   ctypes.c_int64, ctypes.c_int64, ctypes.c_float,
                                   ctypes.c_void_p],
    "cs_bundle_floats": [ctypes.POINTER(CsParams), ctypes.c_int32, ctypes.POINTER(ctypes.c_int64)],
    "cs_bundle_zero": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p],
    "cs_sketch_accumulate_bundle": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_int32,
                                    ctypes.POINTER(ctypes.c_void_p), ctypes.c_int64,
                                    ctypes.c_int64, ctypes.c_float, ctypes.c_void_p],
    "cs_sketch_accumulate_sum": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_int32,
                                 ctypes.POINTER(ctypes.c_void_p), ctypes.c_int64,
                                 ctypes.c_int64, ctypes.c_float, ctypes.c_void_p],
    "cs_bundle_merge": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_float,
                        ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_void_p],
    "cs_update_index_bytes": [ctypes.POINTER(CsParams), ctypes.c_int32, ctypes.c_int64,
                              ctypes.POINTER(ctypes.c_size_t)],
    "cs_update_index_build": [ctypes.POINTER(CsParams), ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t,
                              ctypes.c_void_p],
    "cs_update_workspace_bytes": [ctypes.POINTER(CsParams), ctypes.c_int32, ctypes.c_int64,
                                  ctypes.POINTER(ctypes.c_size_t)],
    "cs_bundle_sketch": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_int32,
                         ctypes.POINTER(ctypes.c_void_p), ctypes.c_int64, ctypes.c_float,
                         ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_size_t,
                         ctypes.c_void_p, ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p,
                         ctypes.c_float, ctypes.c_void_p],
    "cs_cell_lists_bytes": [ctypes.POINTER(CsParams), ctypes.c_int32, ctypes.c_int64,
                            ctypes.POINTER(ctypes.c_size_t)],
    "cs_cell_lists_build": [ctypes.POINTER(CsParams), ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t,
                            ctypes.c_void_p],
    "cs_bundle_sketch_lists": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_int32,
                               ctypes.POINTER(ctypes.c_void_p), ctypes.c_int64, ctypes.c_float,
                               ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_float,
                               ctypes.c_void_p, ctypes.c_void_p, ctypes.c_float, ctypes.c_void_p],
    "cs_sketch_accumulate_sparse": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_void_p,
                                    ctypes.c_void_p, ctypes.c_int64, ctypes.c_float,
                                    ctypes.c_void_p],
    "cs_sketch_merge": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_float,
                        ctypes.POINTER(ctypes.c_void_p), ctypes.c_int32, ctypes.c_float,
                        ctypes.c_void_p],
    "cs_sketch_count_nonfinite": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_void_p,
                                  ctypes.c_void_p],
    "cs_fixed_accumulate": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_void_p,
                            ctypes.c_int64, ctypes.c_int64, ctypes.c_float, ctypes.c_int32,
                            ctypes.c_void_p, ctypes.c_void_p],
    "cs_fixed_accumulate_sparse": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_void_p,
                                   ctypes.c_void_p, ctypes.c_int64, ctypes.c_float,
                                   ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p],
    "cs_fixed_to_float": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_int32,
                          ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p],
    "cs_sketch_axpby": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_float,
                        ctypes.c_void_p, ctypes.c_float, ctypes.c_void_p],
    "cs_sketch_momentum": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_void_p,
                           ctypes.c_void_p, ctypes.c_float, ctypes.c_void_p],
    "cs_estimate_workspace_bytes": [ctypes.POINTER(CsParams), ctypes.c_int64,
                                    ctypes.POINTER(ctypes.c_size_t)],
    "cs_estimate_scratch_bytes": [ctypes.POINTER(CsParams), ctypes.c_int64,
                                  ctypes.POINTER(ctypes.c_size_t)],
    "cs_sketch_estimate": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_int64,
                           ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                           ctypes.c_size_t, ctypes.c_void_p],
    "cs_sketch_estimate_sparse": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_void_p,
                                  ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p],
    "cs_topk_workspace_bytes": [ctypes.c_int64, ctypes.c_int64, ctypes.POINTER(ctypes.c_size_t)],
    "cs_heavy_hitters_topk": [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p,
                              ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                              ctypes.c_void_p],
    "cs_topk_workspace_clear": [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p],
    "cs_heavy_hitters_topk_kept": [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p,
                                   ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                   ctypes.c_void_p],
    "cs_heavy_hitters_topk_static": [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
                                     ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p],
    "cs_select_exact_topk": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64,
                             ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                             ctypes.c_void_p],
    "cs_bundle_update_launches": [ctypes.POINTER(CsParams), ctypes.c_int32, ctypes.c_int64,
                                  ctypes.POINTER(ctypes.c_int32)],
    "cs_bundle_merge_momentum": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                 ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_float,
                                 ctypes.c_void_p],
    "cs_gather_feedback": [ctypes.POINTER(CsParams), ctypes.POINTER(ctypes.c_void_p), ctypes.c_int32, ctypes.c_void_p,
                           ctypes.c_int64, ctypes.c_float, *[ctypes.c_void_p] * 6],
    "cs_sketch_estimate_topk": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int64,
                                *[ctypes.c_void_p] * 3],
    "cs_sketch_feedback_pair": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p],
    "cs_quantize16": [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p],
    "cs_dequantize16": [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p],
    "cs_bundle_merge16": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_float, ctypes.c_void_p,
                          ctypes.c_int32, ctypes.c_float, ctypes.c_int32, ctypes.c_void_p],
    "cs_sketch_l2sq": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p],
    "cs_heavymix_select": [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_void_p,
                           ctypes.c_uint64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                           ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p],
    "cs_gather_exact": [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int32, ctypes.c_void_p,
                        ctypes.c_int64, ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p],
    "cs_vectors_sum": [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int32, ctypes.c_int64,
                       ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p],
    "cs_dense_momentum": [ctypes.POINTER(ctypes.c_void_p), ctypes.POINTER(ctypes.c_void_p),
                          ctypes.POINTER(ctypes.c_void_p), ctypes.c_int32, ctypes.c_int64,
                          ctypes.c_float, ctypes.c_void_p],
    "cs_probe_stream_read": [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int32, ctypes.c_int64,
                             ctypes.c_void_p, ctypes.c_void_p],
    "cs_dense_mask": [ctypes.POINTER(ctypes.c_void_p), ctypes.POINTER(ctypes.c_void_p),
                      ctypes.c_int32, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p],
    "cs_layer_norm": [ctypes.c_void_p, *[ctypes.c_int64] * 3, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                      ctypes.c_int32, ctypes.c_float, ctypes.c_void_p, ctypes.c_int64, *[ctypes.c_void_p] * 3],
    "cs_layer_norm_grad_workspace_bytes": [ctypes.c_int64, ctypes.c_int64, ctypes.POINTER(ctypes.c_size_t)],
    "cs_layer_norm_grad": [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, *[ctypes.c_int64] * 3, ctypes.c_int32,
                           ctypes.c_void_p, ctypes.c_int32, *[ctypes.c_void_p] * 3, ctypes.c_int64,
                           *[ctypes.c_void_p] * 3, ctypes.c_size_t, ctypes.c_void_p],
    "cs_token_workspace_bytes": [ctypes.c_int64, ctypes.c_int64, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)],
    "cs_token_logprobs": [ctypes.c_void_p, *[ctypes.c_int64] * 3, ctypes.c_int32, ctypes.c_float,
                          *[ctypes.c_void_p] * 4, ctypes.c_int32, *[ctypes.c_void_p] * 3, ctypes.c_size_t, ctypes.c_void_p],
    "cs_token_logprobs_grad": [ctypes.c_void_p, *[ctypes.c_int64] * 3, ctypes.c_int32, ctypes.c_float,
                               *[ctypes.c_void_p] * 6, ctypes.c_int64, ctypes.c_void_p],
    "cs_token_loss": [ctypes.c_void_p, *[ctypes.c_int64] * 3, ctypes.c_int32, ctypes.c_float, *[ctypes.c_void_p] * 7,
                      ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p],
    "cs_tensor_list_bytes": [ctypes.POINTER(ctypes.c_int64), ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)],
    "cs_tensor_list_build": [ctypes.POINTER(ctypes.c_int64), ctypes.c_int32, ctypes.POINTER(ctypes.c_void_p), ctypes.c_int32,
                             ctypes.POINTER(ctypes.c_void_p), ctypes.c_int32, ctypes.POINTER(ctypes.c_void_p),
                             ctypes.POINTER(ctypes.c_void_p), ctypes.c_int32, ctypes.POINTER(ctypes.c_void_p),
                             ctypes.POINTER(ctypes.c_void_p), ctypes.c_void_p, ctypes.c_size_t,
                             ctypes.POINTER(CsTensorList), ctypes.c_void_p],
    "cs_grad_norm_workspace_bytes": [ctypes.POINTER(CsTensorList), ctypes.POINTER(ctypes.c_size_t)],
    "cs_grad_norm": [ctypes.POINTER(CsTensorList), ctypes.c_double, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                     ctypes.c_void_p],
    "cs_adamw_advance": [ctypes.POINTER(CsAdamw), *[ctypes.c_void_p] * 4],
    "cs_adamw_advance_scaled": [ctypes.POINTER(CsAdamw), *[ctypes.c_void_p] * 5],
    "cs_grad_norm_advance": [ctypes.POINTER(CsTensorList), ctypes.c_double, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                             ctypes.POINTER(CsAdamw), *[ctypes.c_void_p] * 4],
    "cs_policy_workspace_bytes": [ctypes.c_int64, ctypes.POINTER(ctypes.c_size_t)],
    "cs_policy_loss": [ctypes.POINTER(CsPolicy), ctypes.c_int64, *[ctypes.c_void_p] * 11, ctypes.c_size_t, ctypes.c_void_p],
    "cs_token_policy_workspace_bytes": [ctypes.c_int64, ctypes.c_int64, ctypes.POINTER(ctypes.c_size_t)],
    "cs_token_policy_loss": [ctypes.POINTER(CsPolicy), ctypes.c_void_p, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int32,
                             ctypes.c_float, *[ctypes.c_void_p] * 11, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p],
    "cs_preference_workspace_bytes": [ctypes.c_int64, ctypes.c_int64, ctypes.POINTER(ctypes.c_size_t)],
    "cs_preference_loss": [ctypes.POINTER(CsPreference), ctypes.c_int64, ctypes.c_int64, *[ctypes.c_void_p] * 10, ctypes.c_size_t,
                           ctypes.c_void_p],
    "cs_matrix_list_bytes": [ctypes.POINTER(CsMatrix), ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)],
    "cs_matrix_list_build": [ctypes.POINTER(CsMatrix), ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
                             ctypes.c_size_t, ctypes.POINTER(CsMatrixList), ctypes.c_void_p],
    "cs_muon_workspace_bytes": [ctypes.POINTER(CsMatrixList), ctypes.POINTER(ctypes.c_size_t)],
    "cs_muon_step": [ctypes.POINTER(CsMuon), ctypes.POINTER(CsMatrixList), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                     ctypes.c_size_t, ctypes.c_void_p],
    "cs_orthogonalize": [ctypes.POINTER(CsMuon), ctypes.POINTER(CsMatrixList), ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p],
    "cs_adamw_step": [ctypes.POINTER(CsAdamw), ctypes.c_int64, ctypes.POINTER(CsTensorList), *[ctypes.c_void_p] * 3],
    "cs_moments_read": [ctypes.POINTER(CsTensorList), ctypes.c_void_p],
    "cs_moments_write": [ctypes.POINTER(CsTensorList), ctypes.c_void_p],
    "cs_sketch_feedback": [ctypes.POINTER(CsParams), ctypes.c_void_p, ctypes.c_void_p,
                           ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p],
}


def load_library():
    """Loads libcsketch.so built by paper_1903_04488_amd/build.py; fails loudly if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise CsError(f"{_LIB_PATH} is not built: run `python -c 'import __graft_entry__ as g; "
                      "g.build()'` (there is no fallback path)")
    lib = ctypes.CDLL(_LIB_PATH)
    for name, argtypes in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.argtypes = argtypes
        fn.restype = ctypes.c_int
    lib.cs_status_string.argtypes = [ctypes.c_int]
    lib.cs_status_string.restype = ctypes.c_char_p
    _lib = lib
    return lib


def exported_symbols():
    return list(_SIGNATURES) + ["cs_status_string"]


def cs_status_string(status: int) -> str:
    return load_library().cs_status_string(int(status)).decode()


def _check(status: int, what: str):
    if status != 0:
        raise CsError(f"{what}: {cs_status_string(status)} ({status})")


def _address(t: torch.Tensor, dtype, name: str, numel: int | None = None) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise CsError(f"{name} must be a tensor on the GPU")
    if t.dtype != dtype:
        raise CsError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise CsError(f"{name} must be contiguous")
    if numel is not None and t.numel() != numel:
        raise CsError(f"{name} must have {numel} elements, got {t.numel()}")
    return t.data_ptr()


def _dev(t: torch.Tensor, dtype, name: str, numel: int | None = None) -> int:
    # A step of a short vector waits for the host, and its calls check twenty tensors: one expression for those that are fine,
    # the address as it is (a ctypes object for it is as dear as two of the checks).  d = 784, W = 4: 27 us of host work a step,
    # 22.5 with this, _bundle_floats and the loop in _ptr_array.
    if (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.is_contiguous()
            and (numel is None or t.numel() == numel)):
        return t.data_ptr()
    return _address(t, dtype, name, numel)


def _stream(t: torch.Tensor) -> int:
    # the raw handle: building a torch.cuda.Stream object for it costs ten times as much
    return torch._C._cuda_getCurrentRawStream(t.get_device())


class DeviceVectors(tuple):
    """W vectors of the same length on the GPU, checked once and handed to several calls in place of
    the list: with hundreds of workers the checks are most of a small step's host time."""

    def __new__(cls, tensors, dtype=torch.float32, name: str = "vectors"):
        self = super().__new__(cls, tensors)
        if not self:
            raise CsError(f"{name} must be a non-empty list")
        self.d = self[0].numel()
        self.dtype = dtype
        self.ptrs = _ptr_array(tuple(self), dtype, name, self.d)
        return self


def _ptr_array(tensors, dtype, name, numel=None):
    if isinstance(tensors, DeviceVectors):
        if tensors.dtype != dtype or (numel is not None and tensors.d != numel):
            raise CsError(f"{name} must hold vectors of {numel} elements of {dtype}")
        return tensors.ptrs
    try:
        for t in tensors:
            if not (t.is_cuda and t.dtype is dtype and t.is_contiguous() and (numel is None or t.numel() == numel)):
                break
        else:
            return (ctypes.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])
    except AttributeError:
        pass
    for w, t in enumerate(tensors):                  # names the one that is not
        _address(t, dtype, f"{name}[{w}]", numel)
    return (ctypes.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])


def _cells(p: CsParams) -> int:
    return p.r * p.c


def _bundle_floats(p: CsParams, W: int) -> int:
    """what cs_bundle_floats says (W >= 1)"""
    return -(-W // CS_BUNDLE_GROUP) * CS_BUNDLE_GROUP * p.r * p.c


# ------------------------------------------------------------------------------------------
def cs_params_init(r: int, c: int, seed: int, d_hint: int = 0) -> CsParams:
    p = CsParams()
    _check(load_library().cs_params_init(ctypes.byref(p), r, c, seed, d_hint), "cs_params_init")
    return p


def cs_hash_debug(p, idx, bucket, sign):
    n = idx.numel()
    _check(load_library().cs_hash_debug(
        ctypes.byref(p), _dev(idx, torch.int64, "idx"), n,
        _dev(bucket, torch.int32, "bucket", p.r * n), _dev(sign, torch.int8, "sign", p.r * n),
        _stream(idx)), "cs_hash_debug")


def cs_hash_debug_range(p, i0, n, bucket, sign):
    _check(load_library().cs_hash_debug_range(
        ctypes.byref(p), i0, n,
        _dev(bucket, torch.int32, "bucket", p.r * n), _dev(sign, torch.int8, "sign", p.r * n),
        _stream(bucket)), "cs_hash_debug_range")


def cs_sketch_zero(p, S):
    _check(load_library().cs_sketch_zero(
        ctypes.byref(p), _dev(S, torch.float32, "S", _cells(p)), _stream(S)), "cs_sketch_zero")


def cs_sketch_accumulate(p, S, g, i0: int = 0, scale: float = 1.0):
    _check(load_library().cs_sketch_accumulate(
        ctypes.byref(p), _dev(S, torch.float32, "S", _cells(p)), _dev(g, torch.float32, "g"),
        g.numel(), i0, scale, _stream(S)), "cs_sketch_accumulate")


def cs_sketch_accumulate_batch(p, S_w, g_w, i0: int = 0, scale: float = 1.0):
    if len(S_w) != len(g_w) or len(S_w) == 0:
        raise CsError("S_w and g_w must be non-empty lists of equal length")
    d = g_w[0].numel()
    _check(load_library().cs_sketch_accumulate_batch(
        ctypes.byref(p), _ptr_array(S_w, torch.float32, "S_w", _cells(p)),
        _ptr_array(g_w, torch.float32, "g_w", d), len(S_w), d, i0, scale, _stream(S_w[0])),
        "cs_sketch_accumulate_batch")


CS_BUNDLE_GROUP = 8


def cs_bundle_floats(p, W: int) -> int:
    out = ctypes.c_int64(0)
    _check(load_library().cs_bundle_floats(ctypes.byref(p), W, ctypes.byref(out)),
           "cs_bundle_floats")
    return int(out.value)


def cs_bundle_zero(p, T, W: int):
    _check(load_library().cs_bundle_zero(
        ctypes.byref(p), _dev(T, torch.float32, "T", cs_bundle_floats(p, W)), W, _stream(T)),
        "cs_bundle_zero")


def cs_sketch_accumulate_bundle(p, T, g_w, i0: int = 0, scale: float = 1.0):
    W = len(g_w)
    if W == 0:
        raise CsError("g_w must be a non-empty list")
    d = g_w[0].numel()
    _check(load_library().cs_sketch_accumulate_bundle(
        ctypes.byref(p), _dev(T, torch.float32, "T", cs_bundle_floats(p, W)), W,
        _ptr_array(g_w, torch.float32, "g_w", d), d, i0, scale, _stream(T)),
        "cs_sketch_accumulate_bundle")


def cs_sketch_accumulate_sum(p, S, g_w, i0: int = 0, scale: float = 1.0):
    W = len(g_w)
    if W == 0:
        raise CsError("g_w must be a non-empty list")
    d = g_w[0].numel()
    _check(load_library().cs_sketch_accumulate_sum(
        ctypes.byref(p), _dev(S, torch.float32, "S", _cells(p)), W,
        _ptr_array(g_w, torch.float32, "g_w", d), d, i0, scale, _stream(S)),
        "cs_sketch_accumulate_sum")


def cs_bundle_update_launches(p, W: int, d: int) -> int:
    n = ctypes.c_int32(0)
    _check(load_library().cs_bundle_update_launches(ctypes.byref(p), W, d, ctypes.byref(n)),
           "cs_bundle_update_launches")
    return int(n.value)


def cs_bundle_merge(p, dst, T, W: int, alpha: float = 1.0, beta: float = 0.0):
    _check(load_library().cs_bundle_merge(
        ctypes.byref(p), _dev(dst, torch.float32, "dst", _cells(p)), beta,
        _dev(T, torch.float32, "T", cs_bundle_floats(p, W)), W, alpha, _stream(dst)),
        "cs_bundle_merge")


def cs_sketch_accumulate_sparse(p, S, idx, val, scale: float = 1.0):
    n = idx.numel()
    _check(load_library().cs_sketch_accumulate_sparse(
        ctypes.byref(p), _dev(S, torch.float32, "S", _cells(p)),
        _dev(idx, torch.int64, "idx"), _dev(val, torch.float32, "val", n), n, scale,
        _stream(S)), "cs_sketch_accumulate_sparse")


def cs_sketch_merge(p, dst, src, alpha: float = 1.0, beta: float = 0.0):
    _check(load_library().cs_sketch_merge(
        ctypes.byref(p), _dev(dst, torch.float32, "dst", _cells(p)), beta,
        _ptr_array(src, torch.float32, "src", _cells(p)), len(src), alpha, _stream(dst)),
        "cs_sketch_merge")


def cs_sketch_axpby(p, y, a: float, x, b: float):
    _check(load_library().cs_sketch_axpby(
        ctypes.byref(p), _dev(y, torch.float32, "y", _cells(p)), a,
        _dev(x, torch.float32, "x", _cells(p)), b, _stream(y)), "cs_sketch_axpby")


def cs_sketch_momentum(p, S_u, S_v, S_t, rho: float):
    _check(load_library().cs_sketch_momentum(
        ctypes.byref(p), _dev(S_u, torch.float32, "S_u", _cells(p)),
        _dev(S_v, torch.float32, "S_v", _cells(p)), _dev(S_t, torch.float32, "S_t", _cells(p)),
        rho, _stream(S_u)), "cs_sketch_momentum")


def cs_sketch_count_nonfinite(p, S, count):
    _check(load_library().cs_sketch_count_nonfinite(
        ctypes.byref(p), _dev(S, torch.float32, "S", _cells(p)), _dev(count, torch.int64, "count", 1),
        _stream(S)), "cs_sketch_count_nonfinite")


CS_FIXED_MAX_FRAC_BITS = 62


def _dropped(dropped):
    if dropped is None:
        return ctypes.c_void_p(0)
    return _dev(dropped, torch.int64, "dropped", 1)


def cs_fixed_accumulate(p, acc, g, frac_bits: int, i0: int = 0, scale: float = 1.0, dropped=None):
    _check(load_library().cs_fixed_accumulate(
        ctypes.byref(p), _dev(acc, torch.int64, "acc", _cells(p)), _dev(g, torch.float32, "g"),
        g.numel(), i0, scale, frac_bits, _dropped(dropped), _stream(acc)), "cs_fixed_accumulate")


def cs_fixed_accumulate_sparse(p, acc, idx, val, frac_bits: int, scale: float = 1.0, dropped=None):
    n = idx.numel()
    _check(load_library().cs_fixed_accumulate_sparse(
        ctypes.byref(p), _dev(acc, torch.int64, "acc", _cells(p)), _dev(idx, torch.int64, "idx"),
        _dev(val, torch.float32, "val", n), n, scale, frac_bits, _dropped(dropped),
        _stream(acc)), "cs_fixed_accumulate_sparse")


def cs_fixed_to_float(p, acc, frac_bits: int, S, alpha: float = 1.0):
    _check(load_library().cs_fixed_to_float(
        ctypes.byref(p), _dev(acc, torch.int64, "acc", _cells(p)), frac_bits, alpha,
        _dev(S, torch.float32, "S", _cells(p)), _stream(acc)), "cs_fixed_to_float")


def cs_estimate_workspace_bytes(p, d: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load_library().cs_estimate_workspace_bytes(ctypes.byref(p), d, ctypes.byref(out)),
           "cs_estimate_workspace_bytes")
    return int(out.value)


CS_TOPK_HIST_BINS = 2048
CS_TOPK_SMALL_D = 32768
CS_QUERY_CHOOSE_CELLS = 6144


def _hist(hist):
    if hist is None:
        return ctypes.c_void_p(0)
    return _dev(hist, torch.int64, "hist", CS_TOPK_HIST_BINS)


def cs_estimate_scratch_bytes(p, d: int) -> int:
    n = ctypes.c_size_t()
    _check(load_library().cs_estimate_scratch_bytes(ctypes.byref(p), d, ctypes.byref(n)), "cs_estimate_scratch_bytes")
    return n.value


def cs_sketch_estimate(p, S, est, i0: int = 0, workspace=None, hist=None):
    d = est.numel()
    ws_ptr, ws_bytes = ctypes.c_void_p(0), 0
    if workspace is not None:
        ws_ptr = _dev(workspace, torch.uint8, "workspace")
        ws_bytes = workspace.numel()
    _check(load_library().cs_sketch_estimate(
        ctypes.byref(p), _dev(S, torch.float32, "S", _cells(p)), d, i0,
        _dev(est, torch.float32, "est"), _hist(hist), ws_ptr, ws_bytes, _stream(S)),
        "cs_sketch_estimate")


def cs_sketch_estimate_sparse(p, S, idx, out):
    n = idx.numel()
    _check(load_library().cs_sketch_estimate_sparse(
        ctypes.byref(p), _dev(S, torch.float32, "S", _cells(p)), _dev(idx, torch.int64, "idx"),
        n, _dev(out, torch.float32, "out", n), _stream(S)), "cs_sketch_estimate_sparse")


def cs_topk_workspace_bytes(d: int, k: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load_library().cs_topk_workspace_bytes(d, k, ctypes.byref(out)),
           "cs_topk_workspace_bytes")
    return int(out.value)


def cs_heavy_hitters_topk(est, k: int, idx_out, val_out, workspace, hist=None):
    d = est.numel()
    _check(load_library().cs_heavy_hitters_topk(
        _dev(est, torch.float32, "est"), d, k, _hist(hist), _dev(idx_out, torch.int64, "idx_out", k),
        _dev(val_out, torch.float32, "val_out", k) if val_out is not None else ctypes.c_void_p(0),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(est)),
        "cs_heavy_hitters_topk")


def cs_topk_workspace_clear(workspace):
    _check(load_library().cs_topk_workspace_clear(
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(workspace)), "cs_topk_workspace_clear")


def cs_heavy_hitters_topk_kept(est, k: int, idx_out, val_out, workspace, hist=None):
    d = est.numel()
    _check(load_library().cs_heavy_hitters_topk_kept(
        _dev(est, torch.float32, "est"), d, k, _hist(hist), _dev(idx_out, torch.int64, "idx_out", k),
        _dev(val_out, torch.float32, "val_out", k) if val_out is not None else ctypes.c_void_p(0),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(est)),
        "cs_heavy_hitters_topk_kept")


def cs_bundle_merge_momentum(p, S_t, S_u, S_v, T, W: int, alpha: float, rho: float):
    n = _cells(p)
    _check(load_library().cs_bundle_merge_momentum(
        ctypes.byref(p), _dev(S_t, torch.float32, "S_t", n), _dev(S_u, torch.float32, "S_u", n),
        _dev(S_v, torch.float32, "S_v", n), _dev(T, torch.float32, "T", cs_bundle_floats(p, W)), W, alpha, rho,
        _stream(S_t)), "cs_bundle_merge_momentum")


def cs_update_index_bytes(p, W: int, d: int) -> int:
    n = ctypes.c_size_t()
    _check(load_library().cs_update_index_bytes(ctypes.byref(p), W, d, ctypes.byref(n)), "cs_update_index_bytes")
    return n.value


def cs_update_index_build(p, d: int, index):
    _check(load_library().cs_update_index_build(ctypes.byref(p), d, _dev(index, torch.uint8, "index"), index.numel(),
                                                _stream(index)), "cs_update_index_build")


def cs_update_workspace_bytes(p, W: int, d: int) -> int:
    n = ctypes.c_size_t()
    _check(load_library().cs_update_workspace_bytes(ctypes.byref(p), W, d, ctypes.byref(n)),
           "cs_update_workspace_bytes")
    return n.value


def cs_bundle_sketch(p, T, g_w, index, workspace, scale: float = 1.0, S_t=None, alpha: float = 1.0, S_u=None, S_v=None,
                     rho: float = 0.0):
    """T (or None, for up to 8 workers with S_t): the bundle, written whole; S_t, S_u, S_v: merge and momentum with it"""
    W, n = len(g_w), _cells(p)
    if W == 0:
        raise CsError("g_w must be a non-empty list")
    d = g_w[0].numel()

    def table(S, name):
        return None if S is None else _dev(S, torch.float32, name, n)

    _check(load_library().cs_bundle_sketch(
        ctypes.byref(p), None if T is None else _dev(T, torch.float32, "T", cs_bundle_floats(p, W)), W,
        _ptr_array(g_w, torch.float32, "g_w", d), d, scale, _dev(index, torch.uint8, "index"), index.numel(),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), table(S_t, "S_t"), alpha, table(S_u, "S_u"),
        table(S_v, "S_v"), rho, _stream(index)), "cs_bundle_sketch")


def cs_cell_lists_bytes(p, W: int, d: int) -> int:
    n = ctypes.c_size_t()
    _check(load_library().cs_cell_lists_bytes(ctypes.byref(p), W, d, ctypes.byref(n)), "cs_cell_lists_bytes")
    return n.value


def cs_cell_lists_build(p, d: int, lists):
    _check(load_library().cs_cell_lists_build(ctypes.byref(p), d, _dev(lists, torch.uint8, "lists"), lists.numel(),
                                              _stream(lists)), "cs_cell_lists_build")


def cs_bundle_sketch_lists(p, T, g_w, lists, scale: float = 1.0, S_t=None, alpha: float = 1.0, S_u=None, S_v=None,
                           rho: float = 0.0):
    W = len(g_w)
    if W == 0:
        raise CsError("g_w must be a non-empty list")
    d, n = g_w[0].numel(), _cells(p)
    table = lambda t, name: None if t is None else _dev(t, torch.float32, name, n)              # noqa: E731
    _check(load_library().cs_bundle_sketch_lists(
        ctypes.byref(p), None if T is None else _dev(T, torch.float32, "T", _bundle_floats(p, W)), W,
        _ptr_array(g_w, torch.float32, "g_w", d), d, scale, _dev(lists, torch.uint8, "lists"), lists.numel(),
        table(S_t, "S_t"), alpha, table(S_u, "S_u"), table(S_v, "S_v"), rho, _stream(lists)), "cs_bundle_sketch_lists")


def cs_sketch_feedback_pair(p, S_v, S_u, idx, val_v, val_u):
    k, n = idx.numel(), _cells(p)
    _check(load_library().cs_sketch_feedback_pair(
        ctypes.byref(p), _dev(S_v, torch.float32, "S_v", n), _dev(S_u, torch.float32, "S_u", n),
        _dev(idx, torch.int64, "idx"), k, _dev(val_v, torch.float32, "val_v", k),
        _dev(val_u, torch.float32, "val_u", k), _stream(S_v)), "cs_sketch_feedback_pair")


def cs_gather_feedback(p, vec, idx, out, S_v, S_u, val_v, val_u, alpha: float = 1.0):
    k, n = idx.numel(), _cells(p)
    _check(load_library().cs_gather_feedback(
        ctypes.byref(p), _ptr_array(vec, torch.float32, "vec", vec[0].numel()), len(vec), _dev(idx, torch.int64, "idx"), k,
        alpha, _dev(out, torch.float32, "out", k), _dev(S_v, torch.float32, "S_v", n), _dev(S_u, torch.float32, "S_u", n),
        _dev(val_v, torch.float32, "val_v", k), _dev(val_u, torch.float32, "val_u", k), _stream(S_v)), "cs_gather_feedback")


def cs_sketch_estimate_topk(p, S, est, k: int, idx_out, val_out):
    _check(load_library().cs_sketch_estimate_topk(
        ctypes.byref(p), _dev(S, torch.float32, "S", _cells(p)), est.numel(), _dev(est, torch.float32, "est"), k,
        _dev(idx_out, torch.int64, "idx_out", k),
        _dev(val_out, torch.float32, "val_out", k) if val_out is not None else ctypes.c_void_p(0), _stream(S)),
        "cs_sketch_estimate_topk")


def cs_heavy_hitters_topk_static(est, k: int, idx_out, val_out):
    d = est.numel()
    _check(load_library().cs_heavy_hitters_topk_static(
        _dev(est, torch.float32, "est"), d, k, _dev(idx_out, torch.int64, "idx_out", k),
        _dev(val_out, torch.float32, "val_out", k) if val_out is not None else ctypes.c_void_p(0),
        _stream(est)), "cs_heavy_hitters_topk_static")


def cs_select_exact_topk(cand, x, k: int, idx_out, val_out, workspace):
    n = cand.numel()
    _check(load_library().cs_select_exact_topk(
        _dev(cand, torch.int64, "cand"), _dev(x, torch.float32, "x", n), n, k,
        _dev(idx_out, torch.int64, "idx_out", k),
        _dev(val_out, torch.float32, "val_out", k) if val_out is not None else ctypes.c_void_p(0),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(x)),
        "cs_select_exact_topk")


CS_FMT_BF16, CS_FMT_F16, CS_FMT_F32 = 0, 1, 2


def cs_quantize16(x, out, fmt: int):
    """out: int16 tensor (torch has no uint16 arithmetic; the bit patterns are what matters)"""
    n = x.numel()
    _check(load_library().cs_quantize16(_dev(x, torch.float32, "x"), n,
                                        _dev(out, torch.int16, "out", n), fmt, _stream(x)),
           "cs_quantize16")


def cs_dequantize16(q, out, fmt: int):
    n = q.numel()
    _check(load_library().cs_dequantize16(_dev(q, torch.int16, "q"), n,
                                          _dev(out, torch.float32, "out", n), fmt, _stream(q)),
           "cs_dequantize16")


def cs_bundle_merge16(p, dst, T16, W: int, fmt: int, alpha: float = 1.0, beta: float = 0.0):
    _check(load_library().cs_bundle_merge16(
        ctypes.byref(p), _dev(dst, torch.float32, "dst", _cells(p)), beta,
        _dev(T16, torch.int16, "T16", cs_bundle_floats(p, W)), W, alpha, fmt, _stream(dst)),
        "cs_bundle_merge16")


def cs_sketch_l2sq(p, S, out):
    _check(load_library().cs_sketch_l2sq(
        ctypes.byref(p), _dev(S, torch.float32, "S", _cells(p)),
        _dev(out, torch.float64, "out", 1 + p.r), _stream(S)), "cs_sketch_l2sq")


def cs_heavymix_select(est, k: int, l2sq, rng_seed: int, idx_out, val_out, n_heavy, workspace):
    d = est.numel()
    null = ctypes.c_void_p(0)
    _check(load_library().cs_heavymix_select(
        _dev(est, torch.float32, "est"), d, k, _dev(l2sq, torch.float64, "l2sq"),
        rng_seed & 0xFFFFFFFFFFFFFFFF, _dev(idx_out, torch.int64, "idx_out", k),
        _dev(val_out, torch.float32, "val_out", k) if val_out is not None else null,
        _dev(n_heavy, torch.int64, "n_heavy", 1) if n_heavy is not None else null,
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(est)),
        "cs_heavymix_select")


def cs_gather_exact(vec, idx, out, alpha: float = 1.0):
    k = idx.numel()
    d = vec[0].numel()
    _check(load_library().cs_gather_exact(
        _ptr_array(vec, torch.float32, "vec", d), len(vec), _dev(idx, torch.int64, "idx"), k,
        alpha, _dev(out, torch.float32, "out", k), _stream(out)), "cs_gather_exact")


def cs_vectors_sum(x_w, out, alpha: float = 1.0):
    W = len(x_w)
    if W == 0:
        raise CsError("x_w must be a non-empty list")
    d = x_w[0].numel()
    _check(load_library().cs_vectors_sum(
        _ptr_array(x_w, torch.float32, "x_w", d), W, d, alpha, _dev(out, torch.float32, "out", d),
        _stream(out)), "cs_vectors_sum")


def cs_dense_momentum(u_w, v_w, g_w, rho: float):
    W, d = len(g_w), g_w[0].numel()
    if len(u_w) != W or len(v_w) != W:
        raise CsError("u_w, v_w and g_w must have one tensor per worker")
    _check(load_library().cs_dense_momentum(
        _ptr_array(u_w, torch.float32, "u_w", d), _ptr_array(v_w, torch.float32, "v_w", d),
        _ptr_array(g_w, torch.float32, "g_w", d), W, d, rho, _stream(g_w[0])), "cs_dense_momentum")


def cs_dense_mask(u_w, v_w, idx):
    W = len(u_w)
    if len(v_w) != W:
        raise CsError("u_w and v_w must have one tensor per worker")
    d = u_w[0].numel()
    _check(load_library().cs_dense_mask(
        _ptr_array(u_w, torch.float32, "u_w", d), _ptr_array(v_w, torch.float32, "v_w", d), W,
        _dev(idx, torch.int64, "idx"), idx.numel(), _stream(idx)), "cs_dense_mask")


def cs_probe_stream_read(x_w, out):
    d = x_w[0].numel()
    _check(load_library().cs_probe_stream_read(
        _ptr_array(x_w, torch.float32, "x_w", d), len(x_w), d, _dev(out, torch.float32, "out", 1),
        _stream(out)), "cs_probe_stream_read")


def cs_sketch_feedback(p, S, idx, val):
    k = idx.numel()
    _check(load_library().cs_sketch_feedback(
        ctypes.byref(p), _dev(S, torch.float32, "S", _cells(p)), _dev(idx, torch.int64, "idx"),
        k, _dev(val, torch.float32, "val", k), _stream(S)), "cs_sketch_feedback")


# ------------------------------------------------------------------------------------------
# layer norm, token log probabilities, AdamW
CS_TOKEN_MAX_TOP = 64
CS_ADAMW_BLOCK = 256
CS_ADAMW_COEFS = 10
_FMT = {torch.bfloat16: CS_FMT_BF16, torch.float16: CS_FMT_F16, torch.float32: CS_FMT_F32}


# Small calls wait for the host, and a call for rows checks up to nine tensors.  Those below see in one expression that all of them
# are as they should be (on the GPU, of the sizes and types that are wanted, rows contiguous at any distance) and take the addresses
# as they are; anything else goes the longer way, which names what is wrong (norm of 1 x 512: 3.3 us of checks in a call, 2.2 with this;
# forward and backward of strided rows 31 x 20: 20.2 us a pass when strides went the longer way, 15 now).
def _rows(t, name: str, like=None):
    """(address, row stride) of a 2-d tensor whose rows are contiguous; of the shape and type of `like`"""
    # (a call for one token waits for the host: what is fine is seen first)
    if (isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 2 and t.dtype in _FMT and t.is_contiguous()
            and (like is None or (t.dtype is like.dtype and t.shape == like.shape))):
        cols = t.size(1)
        if cols:
            return t.data_ptr(), cols
    return _rows_address(t, name, like)


def _rows_address(t, name: str, like):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise CsError(f"{name} must be a tensor on the GPU")
    if t.dtype not in _FMT:
        raise CsError(f"{name} must have dtype bfloat16, float16 or float32, got {t.dtype}")
    shape = t.shape
    if len(shape) != 2 or shape[1] == 0:
        raise CsError(f"{name} must have two dimensions, rows of at least one value, got {tuple(shape)}")
    if like is not None and (shape != like.shape or t.dtype is not like.dtype):
        raise CsError(f"{name} must have shape {tuple(like.shape)} and dtype {like.dtype}, got {tuple(shape)}, {t.dtype}")
    cols = shape[1]
    step, one = t.stride()
    if one != 1 and cols > 1:
        raise CsError(f"{name} must have contiguous rows")
    if shape[0] <= 1:
        step = cols
    if step < cols:
        raise CsError(f"{name} must have rows that do not overlap")
    return t.data_ptr(), step


def _maybe(t, dtype, name: str, numel: int):
    if t is None:
        return None
    if (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.is_contiguous()
            and (numel is None or t.numel() == numel)):
        return t.data_ptr()
    return _address(t, dtype, name, numel)


def _weights_dtype(x, *given):
    """the type of a norm's weights: that of the rows, or float32"""
    dtype = torch.float32
    for w in reversed([w for w in given if w is not None]):
        if not isinstance(w, torch.Tensor):
            raise CsError("weight and bias must be tensors on the GPU")
        dtype = w.dtype
    if dtype is not x.dtype and dtype is not torch.float32:
        raise CsError(f"weight and bias must have dtype {x.dtype} or float32, got {dtype}")
    return dtype


def cs_layer_norm(x, weight, bias, y, mean=None, rstd=None, eps: float = 1e-5):
    """x, y: [rows, cols], contiguous rows; weight, bias: [cols] or None; mean, rstd: [rows] float32 or both None"""
    f32 = torch.float32
    try:
        rows, cols = x.shape
        (step, one), (out_step, out_one) = x.stride(), y.stride()
        dt, wt = x.dtype, weight.dtype
        if (one == out_one == 1 and step >= cols <= out_step and x.is_cuda and dt in _FMT and cols and y.dtype is dt and y.is_cuda
                and y.shape == x.shape and (wt is dt or wt is f32) and weight.is_contiguous() and weight.is_cuda
                and weight.numel() == cols
                and (bias is None or (bias.dtype is wt and bias.is_contiguous() and bias.is_cuda and bias.numel() == cols))
                and (mean is None if rstd is None else
                     mean.dtype is f32 and mean.is_contiguous() and mean.is_cuda and mean.numel() == rows
                     and rstd.dtype is f32 and rstd.is_contiguous() and rstd.is_cuda and rstd.numel() == rows)):
            status = (_lib or load_library()).cs_layer_norm(
                x.data_ptr(), rows, cols, step, _FMT[dt], weight.data_ptr(), None if bias is None else bias.data_ptr(), _FMT[wt], eps,
                y.data_ptr(), out_step,
                None if mean is None else mean.data_ptr(), None if rstd is None else rstd.data_ptr(), _stream(x))
            if status:
                _check(status, "cs_layer_norm")
            return
    except (AttributeError, ValueError, TypeError):
        pass
    at, step = _rows(x, "x")
    out, out_step = _rows(y, "y", x)
    rows, cols = x.shape
    dtype = _weights_dtype(x, weight, bias)
    _check(load_library().cs_layer_norm(
        at, rows, cols, step, _FMT[x.dtype], _maybe(weight, dtype, "weight", cols), _maybe(bias, dtype, "bias", cols), _FMT[dtype],
        eps, out, out_step, _maybe(mean, torch.float32, "mean", rows),
        _maybe(rstd, torch.float32, "rstd", rows), _stream(x)), "cs_layer_norm")


def cs_layer_norm_grad_workspace_bytes(rows: int, cols: int) -> int:
    n = ctypes.c_size_t()
    _check(load_library().cs_layer_norm_grad_workspace_bytes(rows, cols, ctypes.byref(n)), "cs_layer_norm_grad_workspace_bytes")
    return n.value


def cs_layer_norm_grad(dy, x, weight, mean, rstd, dx, dweight, dbias, workspace):
    """dx, dweight, dbias: each may be None (workspace too, without the last two)"""
    f32 = torch.float32
    try:
        rows, cols = x.shape
        (step, one), (d_step, d_one), (out_step, out_one) = x.stride(), dy.stride(), dx.stride()
        dt, wt = x.dtype, weight.dtype
        if (one == d_one == out_one == 1 and step >= cols and d_step >= cols <= out_step
                and x.is_cuda and dt in _FMT and cols and (wt is dt or wt is f32)
                and dy.dtype is dt and dy.is_cuda and dy.shape == x.shape
                and dx.dtype is dt and dx.is_cuda and dx.shape == x.shape
                and weight.is_contiguous() and weight.is_cuda and weight.numel() == cols
                and dweight.dtype is wt and dweight.is_contiguous() and dweight.is_cuda and dweight.numel() == cols
                and (dbias is None or (dbias.dtype is wt and dbias.is_contiguous() and dbias.is_cuda and dbias.numel() == cols))
                and mean.dtype is f32 and mean.is_contiguous() and mean.is_cuda and mean.numel() == rows
                and rstd.dtype is f32 and rstd.is_contiguous() and rstd.is_cuda and rstd.numel() == rows
                and workspace.dtype is torch.uint8 and workspace.is_contiguous() and workspace.is_cuda):
            status = (_lib or load_library()).cs_layer_norm_grad(
                dy.data_ptr(), d_step, x.data_ptr(), step, rows, cols, _FMT[dt], weight.data_ptr(), _FMT[wt], mean.data_ptr(),
                rstd.data_ptr(), dx.data_ptr(), out_step, dweight.data_ptr(), None if dbias is None else dbias.data_ptr(),
                workspace.data_ptr(), workspace.numel(), _stream(x))
            if status:
                _check(status, "cs_layer_norm_grad")
            return
    except (AttributeError, ValueError, TypeError):
        pass
    at, step = _rows(x, "x")
    d, d_step = _rows(dy, "dy", x)
    out, out_step = _rows(dx, "dx", x) if dx is not None else (None, 0)
    rows, cols = x.shape
    dtype = _weights_dtype(x, weight, dweight, dbias)
    _check(load_library().cs_layer_norm_grad(
        d, d_step, at, step, rows, cols, _FMT[x.dtype], _maybe(weight, dtype, "weight", cols), _FMT[dtype],
        _dev(mean, torch.float32, "mean", rows), _dev(rstd, torch.float32, "rstd", rows), out, out_step,
        _maybe(dweight, dtype, "dweight", cols), _maybe(dbias, dtype, "dbias", cols),
        _maybe(workspace, torch.uint8, "workspace", None), workspace.numel() if workspace is not None else 0, _stream(x)),
        "cs_layer_norm_grad")


def cs_token_workspace_bytes(rows: int, vocab: int, top: int = 0) -> int:
    n = ctypes.c_size_t()
    _check(load_library().cs_token_workspace_bytes(rows, vocab, top, ctypes.byref(n)), "cs_token_workspace_bytes")
    return n.value


def cs_token_logprobs(logits, target, logp, entropy, lse, top_idx, top_logp, workspace, scale: float = 1.0):
    """logits: [rows, vocab]; target: [rows] int64; logp, entropy, lse: [rows] float32; top_idx, top_logp: [rows, top] int64
    and float32.  None where it is not wanted."""
    f32, i64 = torch.float32, torch.int64
    try:
        rows, vocab = logits.shape
        step, one = logits.stride()
        dt = logits.dtype
        top = 0 if top_idx is None and top_logp is None else top_idx.shape[1]
        if (one == 1 and step >= vocab and logits.is_cuda and dt in _FMT and vocab
                and target.dtype is i64 and target.is_contiguous() and target.is_cuda and target.numel() == rows
                and logp.dtype is f32 and logp.is_contiguous() and logp.is_cuda and logp.numel() == rows
                and entropy.dtype is f32 and entropy.is_contiguous() and entropy.is_cuda and entropy.numel() == rows
                and lse.dtype is f32 and lse.is_contiguous() and lse.is_cuda and lse.numel() == rows
                and (not top or (top_idx.dtype is i64 and top_idx.is_contiguous() and top_idx.is_cuda
                                 and top_logp.dtype is f32 and top_logp.is_contiguous() and top_logp.is_cuda
                                 and top_idx.shape == top_logp.shape == (rows, top)))
                and workspace.dtype is torch.uint8 and workspace.is_contiguous() and workspace.is_cuda):
            status = (_lib or load_library()).cs_token_logprobs(
                logits.data_ptr(), rows, vocab, step, _FMT[dt], scale, target.data_ptr(), logp.data_ptr(), entropy.data_ptr(),
                lse.data_ptr(), top, top_idx.data_ptr() if top else None, top_logp.data_ptr() if top else None,
                workspace.data_ptr(), workspace.numel(), _stream(logits))
            if status:
                _check(status, "cs_token_logprobs")
            return
    except (AttributeError, ValueError, IndexError, TypeError):
        pass
    at, step = _rows(logits, "logits")
    rows, vocab = logits.shape
    top = 0
    if top_idx is not None or top_logp is not None:
        if not isinstance(top_idx, torch.Tensor) or not isinstance(top_logp, torch.Tensor) or top_idx.shape != top_logp.shape or top_idx.dim() != 2 or len(top_idx) != rows:
            raise CsError(f"top_idx and top_logp must be [{rows}, top] both")
        top = top_idx.shape[1]
    f32 = torch.float32
    _check(load_library().cs_token_logprobs(
        at, rows, vocab, step, _FMT[logits.dtype], scale, _maybe(target, torch.int64, "target", rows),
        _maybe(logp, f32, "logp", rows), _maybe(entropy, f32, "entropy", rows), _maybe(lse, f32, "lse", rows), top,
        _maybe(top_idx, torch.int64, "top_idx", None), _maybe(top_logp, f32, "top_logp", None),
        _maybe(workspace, torch.uint8, "workspace", None), workspace.numel() if workspace is not None else 0,
        _stream(logits)), "cs_token_logprobs")


def cs_token_logprobs_grad(logits, target, lse, entropy, g_logp, g_entropy, dlogits, scale: float = 1.0):
    f32 = torch.float32
    try:
        rows, vocab = logits.shape
        (step, one), (out_step, out_one) = logits.stride(), dlogits.stride()
        dt = logits.dtype
        if (one == out_one == 1 and step >= vocab <= out_step and logits.is_cuda and dt in _FMT and vocab
                and dlogits.dtype is dt and dlogits.is_cuda and dlogits.shape == logits.shape
                and target.dtype is torch.int64 and target.is_contiguous() and target.is_cuda and target.numel() == rows
                and lse.dtype is f32 and lse.is_contiguous() and lse.is_cuda and lse.numel() == rows
                and entropy.dtype is f32 and entropy.is_contiguous() and entropy.is_cuda and entropy.numel() == rows
                and g_logp.dtype is f32 and g_logp.is_contiguous() and g_logp.is_cuda and g_logp.numel() == rows
                and (g_entropy is None or (g_entropy.dtype is f32 and g_entropy.is_contiguous() and g_entropy.is_cuda
                                           and g_entropy.numel() == rows))):
            status = (_lib or load_library()).cs_token_logprobs_grad(
                logits.data_ptr(), rows, vocab, step, _FMT[dt], scale, target.data_ptr(), lse.data_ptr(), entropy.data_ptr(),
                g_logp.data_ptr(), None if g_entropy is None else g_entropy.data_ptr(), dlogits.data_ptr(), out_step, _stream(logits))
            if status:
                _check(status, "cs_token_logprobs_grad")
            return
    except (AttributeError, ValueError, TypeError):
        pass
    at, step = _rows(logits, "logits")
    out, out_step = _rows(dlogits, "dlogits", logits)
    rows, vocab = logits.shape
    f32 = torch.float32
    _check(load_library().cs_token_logprobs_grad(
        at, rows, vocab, step, _FMT[logits.dtype], scale, _maybe(target, torch.int64, "target", rows),
        _dev(lse, f32, "lse", rows), _maybe(entropy, f32, "entropy", rows), _maybe(g_logp, f32, "g_logp", rows),
        _maybe(g_entropy, f32, "g_entropy", rows), out, out_step, _stream(logits)), "cs_token_logprobs_grad")


def cs_token_loss(logits, target, g_logp, g_entropy, logp, entropy, lse, dlogits, workspace, scale: float = 1.0):
    f32 = torch.float32
    try:
        rows, vocab = logits.shape
        (step, one), (out_step, out_one) = logits.stride(), dlogits.stride()
        dt = logits.dtype
        if (one == out_one == 1 and step >= vocab <= out_step and logits.is_cuda and dt in _FMT and vocab
                and dlogits.dtype is dt and dlogits.is_cuda and dlogits.shape == logits.shape
                and target.dtype is torch.int64 and target.is_contiguous() and target.is_cuda and target.numel() == rows
                and logp.dtype is f32 and logp.is_contiguous() and logp.is_cuda and logp.numel() == rows
                and lse.dtype is f32 and lse.is_contiguous() and lse.is_cuda and lse.numel() == rows
                and entropy.dtype is f32 and entropy.is_contiguous() and entropy.is_cuda and entropy.numel() == rows
                and g_logp.dtype is f32 and g_logp.is_contiguous() and g_logp.is_cuda and g_logp.numel() == rows
                and (g_entropy is None or (g_entropy.dtype is f32 and g_entropy.is_contiguous() and g_entropy.is_cuda
                                           and g_entropy.numel() == rows))
                and workspace.dtype is torch.uint8 and workspace.is_contiguous() and workspace.is_cuda):
            status = (_lib or load_library()).cs_token_loss(
                logits.data_ptr(), rows, vocab, step, _FMT[dt], scale, target.data_ptr(), g_logp.data_ptr(),
                None if g_entropy is None else g_entropy.data_ptr(), logp.data_ptr(), entropy.data_ptr(), lse.data_ptr(),
                dlogits.data_ptr(), out_step, workspace.data_ptr(), workspace.numel(), _stream(logits))
            if status:
                _check(status, "cs_token_loss")
            return
    except (AttributeError, ValueError, TypeError):
        pass
    at, step = _rows(logits, "logits")
    out, out_step = _rows(dlogits, "dlogits", logits)
    rows, vocab = logits.shape
    f32 = torch.float32
    _check(load_library().cs_token_loss(
        at, rows, vocab, step, _FMT[logits.dtype], scale, _dev(target, torch.int64, "target", rows),
        _dev(g_logp, f32, "g_logp", rows), _maybe(g_entropy, f32, "g_entropy", rows), _dev(logp, f32, "logp", rows),
        _dev(entropy, f32, "entropy", rows), _dev(lse, f32, "lse", rows), out, out_step,
        _maybe(workspace, torch.uint8, "workspace", None), workspace.numel() if workspace is not None else 0,
        _stream(logits)), "cs_token_loss")


def _same_dtype(tensors, name):
    dtype = tensors[0].dtype if tensors else torch.float32
    if dtype not in _FMT:
        raise CsError(f"{name} must have dtype bfloat16, float16 or float32, got {dtype}")
    return dtype


class TensorList:
    """Many tensors checked once and laid out on the GPU for one launch over all of them (cs_tensor_list_build).  Holds the
    tensors; `refresh` where some have moved.  m_exp and v_exp say that the moments are in 8 bits."""

    def __init__(self, p, g, m, v, m_exp=None, v_exp=None):
        self.memory = None
        self.c = CsTensorList()
        self.refresh(p, g, m, v, m_exp, v_exp)

    def refresh(self, p, g, m, v, m_exp=None, v_exp=None):
        bits = 32 if m_exp is None and v_exp is None else 8
        n = [x.numel() for x in p]
        each = {"p": (p, _same_dtype(p, "p")), "g": (g, _same_dtype(g, "g")),
                "m": (m, torch.uint8 if bits == 8 else torch.float32), "v": (v, torch.uint8 if bits == 8 else torch.float32)}
        if bits == 8:
            each |= {"m_exp": (m_exp, torch.uint8), "v_exp": (v_exp, torch.uint8)}
        ptrs = {}
        for name, (tensors, dtype) in each.items():
            if tensors is None or len(tensors) != len(n):
                raise CsError(f"{name} must have {len(n)} tensors")
            size = [-(-x // CS_ADAMW_BLOCK) for x in n] if name.endswith("_exp") else n
            ptrs[name] = (ctypes.c_void_p * len(n))(*[_dev(t, dtype, f"{name}[{i}]", k)
                                                      for i, (t, k) in enumerate(zip(tensors, size))])
        sizes, need = (ctypes.c_int64 * len(n))(*n), ctypes.c_size_t()
        _check(load_library().cs_tensor_list_bytes(sizes, len(n), ctypes.byref(need)), "cs_tensor_list_bytes")
        device = p[0].device if p else torch.device("cuda", torch.cuda.current_device())
        index = p[0].get_device() if p else 0
        if any(t.get_device() != index for tensors, _ in each.values() for t in tensors):
            raise CsError("the tensors of a list must be on one GPU")
        memory, c = self.memory, CsTensorList()
        if memory is None or memory.numel() < need.value or memory.device != device:
            memory = torch.empty(need.value, dtype=torch.uint8, device=device)
        _check(load_library().cs_tensor_list_build(
            sizes, len(n), ptrs["p"], _FMT[each["p"][1]], ptrs["g"], _FMT[each["g"][1]], ptrs["m"], ptrs["v"], bits,
            ptrs.get("m_exp"), ptrs.get("v_exp"), memory.data_ptr(), memory.numel(), ctypes.byref(c), _stream(memory)),
            "cs_tensor_list_build")
        # (only now: a list that could not be built anew is the one that it was, its memory and its tensors held)
        self.device, self.memory, self.c = device, memory, c
        self.tensors = {name: list(tensors) for name, (tensors, _) in each.items()}


def cs_grad_norm_workspace_bytes(tensors: TensorList) -> int:
    n = ctypes.c_size_t()
    _check(load_library().cs_grad_norm_workspace_bytes(ctypes.byref(tensors.c), ctypes.byref(n)), "cs_grad_norm_workspace_bytes")
    return n.value


def cs_grad_norm(tensors: TensorList, max_norm: float, out, workspace):
    _check(load_library().cs_grad_norm(
        ctypes.byref(tensors.c), max_norm, _dev(out, torch.float32, "out", 2), _dev(workspace, torch.uint8, "workspace"),
        workspace.numel(), _stream(tensors.memory)), "cs_grad_norm")


def cs_adamw_advance(h: CsAdamw, step, coefs, lr=None, grad_scale=None):
    """step: int64 tensor of one value, counted up; lr: float64 tensor of one value, or None for h.lr; grad_scale: float32 tensor of one
    value, nothing is done where it is not finite (cs_adamw_advance_scaled)"""
    _check(load_library().cs_adamw_advance_scaled(
        ctypes.byref(h), _dev(step, torch.int64, "step", 1), _maybe(lr, torch.float64, "lr", 1),
        _maybe(grad_scale, torch.float32, "grad_scale", 1), _dev(coefs, torch.float32, "coefs", CS_ADAMW_COEFS), _stream(step)),
        "cs_adamw_advance")


def cs_grad_norm_advance(tensors: TensorList, max_norm: float, out, workspace, h: CsAdamw, step, coefs, lr=None):
    """cs_grad_norm, and cs_adamw_advance where the norm is finite"""
    f32, lib = torch.float32, _lib or load_library()
    try:
        if (out.dtype is f32 and out.is_cuda and out.is_contiguous() and out.numel() == 2
                and workspace.dtype is torch.uint8 and workspace.is_cuda and workspace.is_contiguous()
                and step.dtype is torch.int64 and step.is_cuda and step.numel() == 1
                and coefs.dtype is f32 and coefs.is_cuda and coefs.is_contiguous() and coefs.numel() == CS_ADAMW_COEFS
                and (lr is None or lr.dtype is torch.float64 and lr.is_cuda and lr.numel() == 1)):
            status = lib.cs_grad_norm_advance(
                tensors.c, max_norm, out.data_ptr(), workspace.data_ptr(), workspace.numel(), h, step.data_ptr(),
                None if lr is None else lr.data_ptr(), coefs.data_ptr(), _stream(tensors.memory))
            if status:
                _check(status, "cs_grad_norm_advance")
            return
    except (AttributeError, TypeError):
        pass
    _check(load_library().cs_grad_norm_advance(
        ctypes.byref(tensors.c), max_norm, _dev(out, torch.float32, "out", 2), _dev(workspace, torch.uint8, "workspace"),
        workspace.numel(), ctypes.byref(h), _dev(step, torch.int64, "step", 1), _maybe(lr, torch.float64, "lr", 1),
        _dev(coefs, torch.float32, "coefs", CS_ADAMW_COEFS), _stream(tensors.memory)), "cs_grad_norm_advance")


def cs_adamw_step(h: CsAdamw, step: int, tensors: TensorList, coefs=None, grad_scale=None):
    f32 = torch.float32
    try:
        if ((coefs is None or coefs.dtype is f32 and coefs.is_cuda and coefs.is_contiguous() and coefs.numel() == CS_ADAMW_COEFS)
                and (grad_scale is None or grad_scale.dtype is f32 and grad_scale.is_cuda and grad_scale.numel() == 1)):
            status = (_lib or load_library()).cs_adamw_step(
                h, step, tensors.c, None if coefs is None else coefs.data_ptr(), None if grad_scale is None else grad_scale.data_ptr(),
                _stream(tensors.memory))
            if status:
                _check(status, "cs_adamw_step")
            return
    except (AttributeError, TypeError):
        pass
    _check(load_library().cs_adamw_step(
        ctypes.byref(h), step, ctypes.byref(tensors.c), _maybe(coefs, torch.float32, "coefs", CS_ADAMW_COEFS),
        _maybe(grad_scale, torch.float32, "grad_scale", 1), _stream(tensors.memory)), "cs_adamw_step")


def cs_moments_read(tensors: TensorList):
    _check(load_library().cs_moments_read(ctypes.byref(tensors.c), _stream(tensors.memory)), "cs_moments_read")


def cs_moments_write(tensors: TensorList):
    _check(load_library().cs_moments_write(ctypes.byref(tensors.c), _stream(tensors.memory)), "cs_moments_write")


# ------------------------------------------------------------------------------------------
# losses of answers, orthogonalised momentum
def _same_gpu(like, **tensors):
    """the address of every tensor (None: no address): (tensor, dtype, length or None) each, on the GPU of `like`"""
    index = like.get_device()
    out = []
    for name, (t, dtype, numel) in tensors.items():
        if t is None:
            out.append(None)
            continue
        out.append(_dev(t, dtype, name, numel))
        if t.get_device() != index:
            raise CsError(f"{name} must be on the same GPU as the others")
    return out


def _somewhere(t):
    """an address in place of a workspace of no bytes: of none at all a batch of nothing would leave its sums as they are"""
    return None if t is None else t.data_ptr()


def cs_policy_workspace_bytes(rows: int) -> int:
    n = ctypes.c_size_t()
    _check(load_library().cs_policy_workspace_bytes(rows, ctypes.byref(n)), "cs_policy_workspace_bytes")
    return n.value


def _needed(**tensors):
    for name, t in tensors.items():
        if t is None:
            raise CsError(f"{name} must be given")


def cs_policy_loss(h: CsPolicy, logp, entropy, old_logp, ref_logp, advantage, weight, loss, g_logp, g_entropy, sums, workspace):
    """all [rows] float32 but sums [4]; entropy may be None where h.entropy is 0, ref_logp where h.kl is 0, an output where it is not
    wanted"""
    f32 = torch.float32
    try:
        n, gpu = logp.numel(), logp.get_device()
        given = [t for t in (logp, entropy, old_logp, ref_logp, advantage, weight, loss, g_logp, g_entropy) if t is not None]
        if (gpu >= 0 and old_logp is not None and advantage is not None and weight is not None
                and all([t.dtype is f32 and t.numel() == n and t.get_device() == gpu and t.is_contiguous() for t in given])
                and (sums is None or sums.dtype is f32 and sums.numel() == 4 and sums.get_device() == gpu and sums.is_contiguous())
                and workspace.dtype is torch.uint8 and workspace.get_device() == gpu and workspace.is_contiguous()):
            status = (_lib or load_library()).cs_policy_loss(
                h, n, logp.data_ptr(), None if entropy is None else entropy.data_ptr(), old_logp.data_ptr(),
                None if ref_logp is None else ref_logp.data_ptr(), advantage.data_ptr(), weight.data_ptr(), None if loss is None else loss.data_ptr(),
                None if g_logp is None else g_logp.data_ptr(), None if g_entropy is None else g_entropy.data_ptr(),
                None if sums is None else sums.data_ptr(), workspace.data_ptr() or _somewhere(sums), workspace.numel(), _stream(logp))
            if status:
                _check(status, "cs_policy_loss")
            return
    except (AttributeError, TypeError):
        pass
    _dev(logp, f32, "logp")
    _needed(old_logp=old_logp, advantage=advantage, weight=weight, workspace=workspace)
    n = logp.numel()
    at = _same_gpu(logp, logp=(logp, f32, n), entropy=(entropy, f32, n), old_logp=(old_logp, f32, n), ref_logp=(ref_logp, f32, n),
                   advantage=(advantage, f32, n), weight=(weight, f32, n), loss=(loss, f32, n), g_logp=(g_logp, f32, n),
                   g_entropy=(g_entropy, f32, n), sums=(sums, f32, 4), workspace=(workspace, torch.uint8, None))
    at[-1] = at[-1] or _somewhere(sums)
    _check(load_library().cs_policy_loss(h, n, *at, workspace.numel(), _stream(logp)), "cs_policy_loss")


def cs_token_policy_workspace_bytes(rows: int, vocab: int) -> int:
    n = ctypes.c_size_t()
    _check(load_library().cs_token_policy_workspace_bytes(rows, vocab, ctypes.byref(n)), "cs_token_policy_workspace_bytes")
    return n.value


def cs_token_policy_loss(h: CsPolicy, logits, target, old_logp, ref_logp, advantage, weight, logp, entropy, lse, loss, sums, dlogits,
                         workspace, scale: float = 1.0):
    """logits, dlogits: [rows, vocab]; the rest as for cs_token_loss and cs_policy_loss; loss and sums may be None"""
    f32 = torch.float32
    try:
        rows, vocab = logits.shape
        (step, one), (out_step, out_one) = logits.stride(), dlogits.stride()
        dt, gpu = logits.dtype, logits.get_device()
        given = [t for t in (ref_logp, loss) if t is not None]
        if (one == out_one == 1 and step >= vocab <= out_step and gpu >= 0 and dt in _FMT and vocab
                and dlogits.dtype is dt and dlogits.get_device() == gpu and dlogits.shape == logits.shape
                and target.dtype is torch.int64 and target.is_contiguous() and target.get_device() == gpu and target.numel() == rows
                and all([t.dtype is f32 and t.numel() == rows and t.get_device() == gpu and t.is_contiguous()
                         for t in [old_logp, advantage, weight, logp, entropy, lse, *given]])
                and (sums is None or sums.dtype is f32 and sums.numel() == 4 and sums.get_device() == gpu and sums.is_contiguous())
                and workspace.dtype is torch.uint8 and workspace.is_contiguous() and workspace.get_device() == gpu):
            status = (_lib or load_library()).cs_token_policy_loss(
                h, logits.data_ptr(), rows, vocab, step, _FMT[dt], scale, target.data_ptr(), old_logp.data_ptr(),
                None if ref_logp is None else ref_logp.data_ptr(), advantage.data_ptr(), weight.data_ptr(), logp.data_ptr(),
                entropy.data_ptr(), lse.data_ptr(), None if loss is None else loss.data_ptr(), None if sums is None else sums.data_ptr(),
                dlogits.data_ptr(), out_step, workspace.data_ptr() or _somewhere(sums), workspace.numel(), _stream(logits))
            if status:
                _check(status, "cs_token_policy_loss")
            return
    except (AttributeError, ValueError, TypeError):
        pass
    at, step = _rows(logits, "logits")
    out, out_step = _rows(dlogits, "dlogits", logits)
    rows, vocab = logits.shape
    _needed(target=target, old_logp=old_logp, advantage=advantage, weight=weight, logp=logp, entropy=entropy, lse=lse,
            workspace=workspace)
    if dlogits.get_device() != logits.get_device():
        raise CsError("dlogits must be on the same GPU as the others")
    t, old, ref, a, w, lp, ent, ls, lo, su, ws = _same_gpu(
        logits, target=(target, torch.int64, rows), old_logp=(old_logp, f32, rows), ref_logp=(ref_logp, f32, rows),
        advantage=(advantage, f32, rows), weight=(weight, f32, rows), logp=(logp, f32, rows), entropy=(entropy, f32, rows),
        lse=(lse, f32, rows), loss=(loss, f32, rows), sums=(sums, f32, 4), workspace=(workspace, torch.uint8, None))
    _check(load_library().cs_token_policy_loss(
        h, at, rows, vocab, step, _FMT[logits.dtype], scale, t, old, ref, a, w, lp, ent, ls, lo, su, out, out_step, ws or _somewhere(sums),
        workspace.numel(), _stream(logits)), "cs_token_policy_loss")


def cs_preference_workspace_bytes(tokens: int, pairs: int) -> int:
    n = ctypes.c_size_t()
    _check(load_library().cs_preference_workspace_bytes(tokens, pairs, ctypes.byref(n)), "cs_preference_workspace_bytes")
    return n.value


def cs_preference_loss(h: CsPreference, logp, ref_logp, counts, begin, weight, loss, reward, g_logp, sums, workspace):
    """logp, ref_logp (or None), g_logp (or None): [tokens] float32; counts: [tokens] bool or uint8, or None; begin: [2 pairs + 1] int64;
    weight (or None), loss: [pairs] float32; reward: [2 pairs], sums: [3] float32"""
    f32 = torch.float32
    try:
        n, gpu, ends = logp.numel(), logp.get_device(), begin.numel()
        pairs = ends // 2
        given = [(t, k) for t, k in ((ref_logp, n), (g_logp, n), (weight, pairs)) if t is not None]
        if (gpu >= 0 and ends % 2 and logp.dtype is f32 and logp.is_contiguous()
                and all([t.dtype is f32 and t.numel() == k and t.get_device() == gpu and t.is_contiguous()
                         for t, k in [(loss, pairs), (reward, 2 * pairs), (sums, 3), *given]])
                and begin.dtype is torch.int64 and begin.get_device() == gpu and begin.is_contiguous()
                and (counts is None or (counts.dtype is torch.bool or counts.dtype is torch.uint8) and counts.numel() == n
                     and counts.get_device() == gpu and counts.is_contiguous())
                and workspace.dtype is torch.uint8 and workspace.get_device() == gpu and workspace.is_contiguous()):
            status = (_lib or load_library()).cs_preference_loss(
                h, n, pairs, logp.data_ptr(), None if ref_logp is None else ref_logp.data_ptr(), None if counts is None else counts.data_ptr(),
                begin.data_ptr(), None if weight is None else weight.data_ptr(), loss.data_ptr(), reward.data_ptr(),
                None if g_logp is None else g_logp.data_ptr(), sums.data_ptr(), workspace.data_ptr() or _somewhere(sums), workspace.numel(), _stream(logp))
            if status:
                _check(status, "cs_preference_loss")
            return
    except (AttributeError, TypeError):
        pass
    _dev(logp, f32, "logp")
    _dev(begin, torch.int64, "begin")
    _needed(loss=loss, reward=reward, sums=sums, workspace=workspace)
    if begin.numel() % 2 == 0:
        raise CsError(f"begin must have 2 pairs + 1 values, got {begin.numel()}")
    n, pairs = logp.numel(), begin.numel() // 2
    kind = torch.bool if isinstance(counts, torch.Tensor) and counts.dtype is torch.bool else torch.uint8
    at = _same_gpu(logp, logp=(logp, f32, n), ref_logp=(ref_logp, f32, n), counts=(counts, kind, n), begin=(begin, torch.int64, None),
                   weight=(weight, f32, pairs), loss=(loss, f32, pairs), reward=(reward, f32, 2 * pairs), g_logp=(g_logp, f32, n),
                   sums=(sums, f32, 3), workspace=(workspace, torch.uint8, None))
    at[-1] = at[-1] or _somewhere(sums)
    _check(load_library().cs_preference_loss(h, n, pairs, *at, workspace.numel(), _stream(logp)), "cs_preference_loss")


def _stack(t, name: str, dtype, shape=None):
    """(address, count, rows, cols, row stride, matrix step) of a matrix or a stack of matrices whose rows are contiguous"""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise CsError(f"{name} must be a tensor on the GPU")
    if t.dtype is not dtype:
        raise CsError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if t.dim() not in (2, 3) or (shape is not None and t.shape != shape):
        raise CsError(f"{name} must have " + ("two or three dimensions" if shape is None else f"shape {tuple(shape)}") + f", got {tuple(t.shape)}")
    count, rows, cols = (1, *t.shape) if t.dim() == 2 else t.shape
    step, (stride, one) = (0 if t.dim() == 2 else t.stride(0)), t.stride()[-2:]
    if t.numel() == 0:
        return t.data_ptr(), count, rows, cols, cols, rows * cols
    if one != 1 and cols > 1:
        raise CsError(f"{name} must have contiguous rows")
    stride, step = stride if rows > 1 else cols, step if count > 1 else 0
    if stride < cols or (count > 1 and step < (rows - 1) * stride + cols):
        raise CsError(f"{name} must have rows and matrices that do not overlap, one matrix after the other")
    return t.data_ptr(), count, rows, cols, stride, step


class _Place:
    """where a stack lies: rows of `length` bytes, `pitch` bytes apart in a matrix, matrices `step` bytes apart"""

    __slots__ = ("name", "written", "index", "begin", "end", "count", "rows", "length", "pitch", "step", "one")

    def __init__(self, name, written, index, at, size, count, rows, cols, stride, step):
        self.name, self.written, self.index, self.begin, self.count, self.rows = name, written, index, at, count, rows
        self.length, self.pitch, self.step = cols * size, stride * size, step * size
        self.one = (rows - 1) * self.pitch + self.length
        self.end = at + (count - 1) * self.step + self.one

    def row_begins(self):
        return (self.begin + self.step * torch.arange(self.count)[:, None] + self.pitch * torch.arange(self.rows)).flatten()


def _apart(a: _Place, b: _Place) -> bool:
    """whether two stacks share no byte: their spans do not meet, or they are columns of the same rows or matrices of the same stack, or else by
    looking at every row"""
    if a.end <= b.begin or b.end <= a.begin:
        return True
    off = b.begin - a.begin
    if a.pitch == b.pitch and all(x.count == 1 or x.step % a.pitch == 0 for x in (a, b)):
        if off % a.pitch >= a.length and -off % a.pitch >= b.length:
            return True
    if a.count > 1 and a.step == b.step and b.count > 1 and off % a.step >= a.one and -off % a.step >= b.one:
        return True
    begins = torch.cat([a.row_begins(), b.row_begins()])
    ends = torch.cat([a.row_begins() + a.length, b.row_begins() + b.length])
    order = begins.argsort()
    return bool((ends[order][:-1] <= begins[order][1:]).all())


def _all_apart(places):
    """no matrix that is written shares memory with another one's (places: the arguments of _Place)"""
    spans = sorted([(at, at + size * ((count - 1) * step + (rows - 1) * stride + cols))
                    for _, _, _, at, size, count, rows, cols, stride, step in places])
    if all([spans[i][1] <= spans[i + 1][0] for i in range(len(spans) - 1)]):
        return
    places = sorted([_Place(*x) for x in places], key=lambda x: x.begin)
    for i, a in enumerate(places):
        for b in places[i + 1:]:
            if b.begin >= a.end:
                break
            # (the arrays of one stack are looked at by the library)
            if a.index != b.index and (a.written or b.written) and not _apart(a, b):
                raise CsError(f"{a.name}[{a.index}] and {b.name}[{b.index}] overlap")


class MatrixList:
    """Matrices, or stacks of them ([count, rows, cols]), checked once and laid out on the GPU for the same launches over all of them
    (cs_matrix_list_build).  p: what is written; g: gradients, or what is orthogonalised; m: moments (float32, contiguous) or None.  terms: 1 or
    2, how much of their factors the products take.  What is written may share no memory with another matrix's.  Holds the tensors; `refresh`
    where some have moved."""

    def __init__(self, p, g, m=None, terms: int = 1):
        self.memory, self.terms = None, terms
        self.c = CsMatrixList()
        self.refresh(p, g, m)

    def refresh(self, p, g, m=None):
        p, g, m = list(p), list(g), None if m is None else list(m)
        if len(g) != len(p) or (m is not None and len(m) != len(p)):
            raise CsError(f"p, g and m must have {len(p)} tensors each")
        p_type, g_type = _same_dtype(p, "p"), _same_dtype(g, "g")
        stacks, places, p_size, g_size = (CsMatrix * len(p))(), [], p_type.itemsize, g_type.itemsize
        for i in range(len(p)):
            at, count, rows, cols, p_stride, p_step = _stack(p[i], f"p[{i}]", p_type)
            g_at, *_, g_stride, g_step = _stack(g[i], f"g[{i}]", g_type, p[i].shape)
            moment = None
            if m is not None:
                moment = _dev(m[i], torch.float32, f"m[{i}]", p[i].numel())
                if m[i].shape != p[i].shape:
                    raise CsError(f"m[{i}] must have shape {tuple(p[i].shape)}, got {tuple(m[i].shape)}")
            if count and rows and cols:
                places.append(("p", True, i, at, p_size, count, rows, cols, p_stride, p_step))
                places.append(("g", False, i, g_at, g_size, count, rows, cols, g_stride, g_step))
                if moment:
                    places.append(("m", True, i, moment, 4, count, rows, cols, cols, rows * cols))
            stacks[i] = CsMatrix(at, g_at, moment, count, rows, cols, p_stride, p_step, g_stride, g_step)
        for name, written in (("p", p), ("m", m or [])):
            begins = [t.data_ptr() for t in written if t.numel()]
            if len(set(begins)) != len(begins):
                raise CsError(f"{name} has a tensor twice")
        _all_apart(places)
        device = p[0].device if p else torch.device("cuda", torch.cuda.current_device())
        if any(t.device != device for t in p + g + (m or [])):
            raise CsError("the tensors of a list must be on one GPU")
        need, c = ctypes.c_size_t(), CsMatrixList()
        _check(load_library().cs_matrix_list_bytes(stacks, len(p), self.terms, ctypes.byref(need)), "cs_matrix_list_bytes")
        memory = self.memory
        if memory is None or memory.numel() < need.value or memory.device != device:
            memory = torch.empty(need.value, dtype=torch.uint8, device=device)
        _check(load_library().cs_matrix_list_build(stacks, len(p), _FMT[p_type], _FMT[g_type], self.terms, memory.data_ptr(), memory.numel(),
                                                   ctypes.byref(c), _stream(memory)), "cs_matrix_list_build")
        # (only now: a list that could not be built anew is the one that it was)
        self.device, self.memory, self.c, self.tensors = device, memory, c, (p, g, m)


def cs_muon_workspace_bytes(matrices: MatrixList) -> int:
    n = ctypes.c_size_t()
    _check(load_library().cs_muon_workspace_bytes(matrices.c, ctypes.byref(n)), "cs_muon_workspace_bytes")
    return n.value


def cs_muon_step(h: CsMuon, matrices: MatrixList, workspace, lr=None, grad_scale=None):
    """lr: float64 tensor of one value in place of h.lr; grad_scale: float32 tensor of one value"""
    lr_at, scale_at, ws = _same_gpu(matrices.memory, lr=(lr, torch.float64, 1), grad_scale=(grad_scale, torch.float32, 1),
                                    workspace=(workspace, torch.uint8, None))
    _check(load_library().cs_muon_step(h, matrices.c, lr_at, scale_at, ws, workspace.numel(), _stream(matrices.memory)), "cs_muon_step")


def cs_orthogonalize(h: CsMuon, matrices: MatrixList, workspace):
    ws, = _same_gpu(matrices.memory, workspace=(workspace, torch.uint8, None))
    _check(load_library().cs_orthogonalize(h, matrices.c, ws, workspace.numel(), _stream(matrices.memory)), "cs_orthogonalize")
