"""Python binding of libmmee (include/mmee.h): argument marshalling only.

Every number comes out of the HIP kernels behind the C ABI.  There is no CPU
fallback: importing this package without a built libmmee.so raises, and calls
on a machine without a GPU return MMEE_EDEVICE (raised as MmeeError).

With torch in the same process import torch first: the library then uses the HIP runtime
that torch brings, and streams and device memory are shared.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("MMEE_LIB") or os.path.join(_HERE, "libmmee.so")

OBJ_ENERGY, OBJ_LATENCY, OBJ_LATENCY_THEN_ENERGY, OBJ_EDP = 0, 1, 2, 3
SEARCH_PRUNED, SEARCH_EXHAUSTIVE, SEARCH_ORDERED_SUM = 0, 1, 2
OK, EINVAL, ERANGE, ENOFEASIBLE, EDEVICE, EOVERFLOW, ETOOBIG, EWORKSPACE = 0, -1, -2, -3, -4, -5, -6, -7
F16, BF16 = 0, 1
PAIRS = {"halves": 0, "neighbours": 1}
ACTS = {"silu": 0, "gelu": 1, "gelu_tanh": 2, "relu": 3, "sigmoid": 4}


class MmeeError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {_strerror(code)} (code {code})")


class Workload(C.Structure):
    _fields_ = [("B", C.c_uint32), ("H", C.c_uint32), ("N", C.c_uint32), ("d", C.c_uint32),
                ("word_bytes", C.c_uint32), ("tiling_mode", C.c_uint32),
                ("c_softmax", C.c_uint32), ("reserved", C.c_uint32)]


class Chain(C.Structure):
    _fields_ = [("batch", C.c_uint32), ("I", C.c_uint32), ("K", C.c_uint32), ("L", C.c_uint32),
                ("J", C.c_uint32), ("word_bytes", C.c_uint32), ("tiling_mode", C.c_uint32),
                ("c_softmax", C.c_uint32)]


class Hw(C.Structure):
    _fields_ = [("pe_rows", C.c_uint32), ("pe_cols", C.c_uint32), ("n_arrays", C.c_uint32),
                ("rf_bytes", C.c_uint32), ("gb_bytes", C.c_uint64),
                ("e_dram", C.c_double), ("e_gb", C.c_double), ("e_rf", C.c_double),
                ("e_mac", C.c_double), ("dram_bw", C.c_double), ("gb_bw", C.c_double)]


class Mapping(C.Structure):
    _fields_ = [("idx", C.c_uint64), ("xG", C.c_uint32 * 4), ("xD", C.c_uint32 * 4),
                ("order", C.c_uint8 * 4), ("level", C.c_uint8 * 4),
                ("recompute", C.c_uint8), ("stat1", C.c_uint8), ("stat2", C.c_uint8),
                ("fused", C.c_uint8)]


class Cost(C.Structure):
    _fields_ = [("bs_words", C.c_uint64), ("da_words", C.c_uint64), ("br_words", C.c_uint64),
                ("mac_total", C.c_uint64), ("comp_cycles", C.c_uint64),
                ("energy_pj", C.c_double), ("latency_cycles", C.c_double),
                ("valid", C.c_uint32), ("reason", C.c_uint32)]


class Result(C.Structure):
    _fields_ = [("best", Mapping), ("cost", Cost), ("space", C.c_uint64), ("evaluated", C.c_uint64),
                ("seconds", C.c_double), ("kernel_seconds", C.c_double)]


class RowStats(C.Structure):
    _fields_ = [("rows_total", C.c_uint32 * 4), ("rows_valid", C.c_uint32 * 4),
                ("rows_kept", C.c_uint32 * 4)]


class _Call(C.Structure):
    """Arguments of a call on device buffers, marshalled once for repeated calls; holds on to the tensors it was made from."""

    def use_workspace(self, tensor):
        """Give the call a contiguous device buffer as its workspace."""
        _on_device("use_workspace", "the workspace", tensor)
        if not tensor.is_contiguous():
            raise _invalid("use_workspace", "the workspace has to be contiguous")
        self.workspace, self.workspace_bytes = tensor.data_ptr(), tensor.numel() * tensor.element_size()
        self._workspace = tensor
        return self


_Strides = C.c_int64 * 3


class Attn(_Call):
    _fields_ = [("dtype", C.c_uint32), ("batch", C.c_uint32), ("heads", C.c_uint32), ("kv_heads", C.c_uint32),
                ("head_dim", C.c_uint32), ("q_len", C.c_uint32), ("kv_len", C.c_uint32), ("scale", C.c_float),
                ("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("o", C.c_void_p),
                ("q_stride", _Strides), ("k_stride", _Strides), ("v_stride", _Strides), ("o_stride", _Strides),
                ("lse", C.c_void_p), ("kv_lens", C.c_void_p), ("key_mask", C.c_void_p), ("mask_stride", C.c_int64),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64), ("reserved", C.c_uint64)]


class AttnGrads(_Call):
    _fields_ = [("d_o", C.c_void_p), ("dq", C.c_void_p), ("dk", C.c_void_p), ("dv", C.c_void_p),
                ("do_stride", _Strides), ("dq_stride", _Strides), ("dk_stride", _Strides), ("dv_stride", _Strides)]


class TreeAttn(_Call):
    _fields_ = [("dtype", C.c_uint32), ("batch", C.c_uint32), ("heads", C.c_uint32), ("kv_heads", C.c_uint32),
                ("head_dim", C.c_uint32), ("nodes", C.c_uint32), ("page_tokens", C.c_uint32), ("pages_per_seq", C.c_uint32),
                ("n_pages", C.c_uint32), ("scale", C.c_float),
                ("q", C.c_void_p), ("k_pages", C.c_void_p), ("v_pages", C.c_void_p), ("o", C.c_void_p),
                ("q_stride", _Strides), ("k_stride", _Strides), ("v_stride", _Strides), ("o_stride", _Strides),
                ("page_table", C.c_void_p), ("table_stride", C.c_int64), ("cache_lens", C.c_void_p), ("node_counts", C.c_void_p),
                ("ancestors", C.c_void_p), ("lse", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64), ("reserved", C.c_uint64)]


class Ffn(_Call):
    _fields_ = [("dtype", C.c_uint32), ("act", C.c_uint32), ("rows", C.c_uint32), ("in_dim", C.c_uint32), ("hidden_dim", C.c_uint32),
                ("out_dim", C.c_uint32), ("x", C.c_void_p), ("w_gate", C.c_void_p), ("w_up", C.c_void_p), ("w_down", C.c_void_p),
                ("y", C.c_void_p), ("hidden", C.c_void_p), ("gate", C.c_void_p), ("up", C.c_void_p),
                ("x_stride", C.c_int64), ("gate_stride", C.c_int64), ("up_stride", C.c_int64), ("down_stride", C.c_int64),
                ("y_stride", C.c_int64), ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64), ("reserved", C.c_uint64)]


class FfnGrads(_Call):
    _fields_ = [("dy", C.c_void_p), ("dx", C.c_void_p), ("dw_gate", C.c_void_p), ("dw_up", C.c_void_p), ("dw_down", C.c_void_p),
                ("dy_stride", C.c_int64), ("dx_stride", C.c_int64)]


_Two = C.c_int64 * 2


class QkRotate(_Call):
    _fields_ = [("dtype", C.c_uint32), ("pairs", C.c_uint32), ("tokens", C.c_uint32), ("heads", C.c_uint32), ("kv_heads", C.c_uint32),
                ("head_dim", C.c_uint32), ("rot_dim", C.c_uint32), ("axes", C.c_uint32), ("eps", C.c_float),
                ("q", C.c_void_p), ("k", C.c_void_p), ("q_out", C.c_void_p), ("k_out", C.c_void_p),
                ("q_stride", _Two), ("k_stride", _Two), ("q_out_stride", _Two), ("k_out_stride", _Two),
                ("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("freqs", C.c_void_p), ("positions", C.c_void_p), ("axis_stride", C.c_int64),
                ("axis_of", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64), ("reserved", C.c_uint64)]


class QkRotateGrads(_Call):
    _fields_ = [("dq_out", C.c_void_p), ("dk_out", C.c_void_p), ("dq", C.c_void_p), ("dk", C.c_void_p), ("dq_weight", C.c_void_p),
                ("dk_weight", C.c_void_p), ("dq_out_stride", _Two), ("dk_out_stride", _Two), ("dq_stride", _Two), ("dk_stride", _Two)]


class CacheAppend(_Call):
    _fields_ = [("dtype", C.c_uint32), ("pairs", C.c_uint32), ("tokens", C.c_uint32), ("seqs", C.c_uint32), ("heads", C.c_uint32),
                ("kv_heads", C.c_uint32), ("head_dim", C.c_uint32), ("rot_dim", C.c_uint32), ("axes", C.c_uint32), ("page_tokens", C.c_uint32),
                ("pages_per_seq", C.c_uint32), ("n_pages", C.c_uint32), ("eps", C.c_float),
                ("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("q_out", C.c_void_p), ("k_pages", C.c_void_p), ("v_pages", C.c_void_p),
                ("q_stride", _Two), ("k_stride", _Two), ("v_stride", _Two), ("q_out_stride", _Two), ("k_pages_stride", _Strides),
                ("v_pages_stride", _Strides), ("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("freqs", C.c_void_p), ("positions", C.c_void_p),
                ("axis_stride", C.c_int64), ("axis_of", C.c_void_p), ("starts", C.c_void_p), ("counts", C.c_void_p), ("cache_lens", C.c_void_p),
                ("page_table", C.c_void_p), ("table_stride", C.c_int64), ("reserved", C.c_uint64)]


class PromptAttn(_Call):
    _fields_ = [("dtype", C.c_uint32), ("causal", C.c_uint32), ("seqs", C.c_uint32), ("heads", C.c_uint32), ("kv_heads", C.c_uint32),
                ("head_dim", C.c_uint32), ("q_tokens", C.c_uint32), ("kv_tokens", C.c_uint32), ("scale", C.c_float),
                ("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("o", C.c_void_p),
                ("q_stride", _Two), ("k_stride", _Two), ("v_stride", _Two), ("o_stride", _Two), ("q_starts", C.c_void_p), ("kv_starts", C.c_void_p),
                ("lse", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64), ("reserved", C.c_uint64)]


class PromptAttnGrads(_Call):
    _fields_ = [("d_o", C.c_void_p), ("dq", C.c_void_p), ("dk", C.c_void_p), ("dv", C.c_void_p),
                ("do_stride", _Two), ("dq_stride", _Two), ("dk_stride", _Two), ("dv_stride", _Two)]


COST_DTYPE = np.dtype([("bs_words", "<u8"), ("da_words", "<u8"), ("br_words", "<u8"),
                       ("mac_total", "<u8"), ("comp_cycles", "<u8"),
                       ("energy_pj", "<f8"), ("latency_cycles", "<f8"),
                       ("valid", "<u4"), ("reason", "<u4")])
assert COST_DTYPE.itemsize == C.sizeof(Cost) == 64


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()'). "
            "There is no CPU fallback for the MMEE kernels.")
    L = C.CDLL(LIB_PATH)
    P = C.POINTER
    L.mmee_space_size.argtypes = [P(Workload), P(Hw), P(C.c_uint64)]
    L.mmee_decode.argtypes = [P(Workload), P(Hw), P(C.c_uint64), C.c_uint64, P(Mapping)]
    L.mmee_eval_batch.argtypes = [P(Workload), P(Hw), C.c_uint64, C.c_uint64, C.c_void_p]
    L.mmee_search.argtypes = [P(Workload), P(Hw), C.c_int, P(Result)]
    L.mmee_search_ex.argtypes = [P(Workload), P(Hw), C.c_int, C.c_uint32, P(Result)]
    L.mmee_search_multi.argtypes = [P(Workload), P(Hw), P(C.c_int), C.c_uint32, C.c_uint32, P(Result)]
    L.mmee_search_many.argtypes = [P(Workload), P(Hw), P(C.c_int), C.c_uint32, C.c_uint32, P(Result),
                                   P(C.c_int)]
    L.mmee_chain_space_size.argtypes = [P(Chain), P(Hw), P(C.c_uint64)]
    L.mmee_energy_regrouped.argtypes = [P(Workload), P(Hw), C.c_uint32, P(C.c_int)]
    L.mmee_chain_energy_regrouped.argtypes = [P(Chain), P(Hw), C.c_uint32, P(C.c_int)]
    L.mmee_chain_decode.argtypes = [P(Chain), P(Hw), P(C.c_uint64), C.c_uint64, P(Mapping)]
    L.mmee_chain_eval_batch.argtypes = [P(Chain), P(Hw), C.c_uint64, C.c_uint64, C.c_void_p]
    L.mmee_chain_search_multi.argtypes = [P(Chain), P(Hw), P(C.c_int), C.c_uint32, C.c_uint32, P(Result)]
    L.mmee_chain_search_many.argtypes = [P(Chain), P(Hw), P(C.c_int), C.c_uint32, C.c_uint32, P(Result),
                                         P(C.c_int)]
    L.mmee_pareto.argtypes = [P(Workload), P(Hw), C.c_uint32, P(Result), C.c_uint32, P(C.c_uint32)]
    L.mmee_chain_pareto.argtypes = [P(Chain), P(Hw), C.c_uint32, P(Result), C.c_uint32, P(C.c_uint32)]
    L.mmee_front_bs_da.argtypes = [P(Workload), P(Hw), C.c_uint32, P(Result), C.c_uint32, P(C.c_uint32)]
    L.mmee_chain_front_bs_da.argtypes = [P(Chain), P(Hw), C.c_uint32, P(Result), C.c_uint32, P(C.c_uint32)]
    L.mmee_search_noalloc.argtypes = [P(Workload), P(Hw), C.c_int, C.c_uint32, C.c_void_p]
    L.mmee_offline_stats.argtypes = [P(RowStats)]
    L.mmee_offline_rows.argtypes = [C.c_uint32, C.c_uint32, P(C.c_uint32), C.c_uint32, P(C.c_uint32)]
    L.mmee_attn_workspace.argtypes = [P(Attn), C.c_int, P(C.c_uint64)]
    L.mmee_attn_forward.argtypes = [P(Attn)]
    L.mmee_attn_backward.argtypes = [P(Attn), P(AttnGrads)]
    L.mmee_tree_attn_workspace.argtypes = [P(TreeAttn), P(C.c_uint64)]
    L.mmee_tree_attn_forward.argtypes = [P(TreeAttn)]
    L.mmee_ffn_workspace.argtypes = [P(Ffn), C.c_int, P(C.c_uint64)]
    L.mmee_ffn_forward.argtypes = [P(Ffn)]
    L.mmee_ffn_backward.argtypes = [P(Ffn), P(FfnGrads)]
    L.mmee_qk_rotate_workspace.argtypes = [P(QkRotate), P(C.c_uint64)]
    L.mmee_qk_rotate_forward.argtypes = [P(QkRotate)]
    L.mmee_qk_rotate_backward.argtypes = [P(QkRotate), P(QkRotateGrads)]
    L.mmee_cache_append_forward.argtypes = [P(CacheAppend)]
    L.mmee_prompt_attn_workspace.argtypes = [P(PromptAttn), C.c_int, P(C.c_uint64)]
    L.mmee_prompt_attn_forward.argtypes = [P(PromptAttn)]
    L.mmee_prompt_attn_backward.argtypes = [P(PromptAttn), P(PromptAttnGrads)]
    L.mmee_set_stream.argtypes = [C.c_void_p]
    L.mmee_shutdown.argtypes = []
    L.mmee_shutdown.restype = None
    L.mmee_strerror.argtypes = [C.c_int]
    L.mmee_strerror.restype = C.c_char_p
    for name in ("mmee_space_size", "mmee_decode", "mmee_eval_batch", "mmee_search", "mmee_search_ex",
                 "mmee_search_multi", "mmee_search_many", "mmee_search_noalloc", "mmee_offline_stats", "mmee_offline_rows", "mmee_set_stream",
                 "mmee_chain_space_size", "mmee_chain_decode", "mmee_chain_eval_batch",
                 "mmee_chain_search_multi", "mmee_chain_search_many", "mmee_pareto", "mmee_chain_pareto",
                 "mmee_front_bs_da", "mmee_chain_front_bs_da",
                 "mmee_attn_workspace", "mmee_attn_forward", "mmee_attn_backward", "mmee_tree_attn_workspace", "mmee_tree_attn_forward",
                 "mmee_ffn_workspace", "mmee_ffn_forward", "mmee_ffn_backward",
                 "mmee_qk_rotate_workspace", "mmee_qk_rotate_forward", "mmee_qk_rotate_backward", "mmee_cache_append_forward",
                 "mmee_prompt_attn_workspace", "mmee_prompt_attn_forward", "mmee_prompt_attn_backward"):
        getattr(L, name).restype = C.c_int
    return L


_lib = _load()


def _strerror(code: int) -> str:
    return _lib.mmee_strerror(code).decode()


def _check(code: int, where: str, allow=()):
    if code != OK and code not in allow:
        raise MmeeError(code, where)
    return code


def workload(cfg) -> Workload:
    if isinstance(cfg, Workload):
        return cfg
    return Workload(cfg["B"], cfg["H"], cfg["N"], cfg["d"], cfg["word_bytes"],
                    cfg["tiling_mode"], cfg["c_softmax"], 0)


def chain(cfg) -> Chain:
    if isinstance(cfg, Chain):
        return cfg
    return Chain(cfg["batch"], cfg["I"], cfg["K"], cfg["L"], cfg["J"], cfg["word_bytes"],
                 cfg["tiling_mode"], cfg["c_softmax"])


def hw(cfg) -> Hw:
    if isinstance(cfg, Hw):
        return cfg
    return Hw(cfg["pe_rows"], cfg["pe_cols"], cfg["n_arrays"], cfg["rf_bytes"], cfg["gb_bytes"],
              cfg["e_dram"], cfg["e_gb"], cfg["e_rf"], cfg["e_mac"], cfg["dram_bw"], cfg["gb_bw"])


def mmee_space_size(w, h) -> int:
    out = C.c_uint64()
    _check(_lib.mmee_space_size(C.byref(workload(w)), C.byref(hw(h)), C.byref(out)), "mmee_space_size")
    return out.value


def mmee_energy_regrouped(w, h, flags: int = SEARCH_PRUNED) -> bool:
    out = C.c_int()
    _check(_lib.mmee_energy_regrouped(C.byref(workload(w)), C.byref(hw(h)), flags, C.byref(out)),
           "mmee_energy_regrouped")
    return bool(out.value)


def mmee_chain_energy_regrouped(c, h, flags: int = SEARCH_PRUNED) -> bool:
    out = C.c_int()
    _check(_lib.mmee_chain_energy_regrouped(C.byref(chain(c)), C.byref(hw(h)), flags, C.byref(out)),
           "mmee_chain_energy_regrouped")
    return bool(out.value)


def mmee_decode(w, h, indices):
    idx = np.ascontiguousarray(indices, dtype=np.uint64)
    out = (Mapping * len(idx))()
    _check(_lib.mmee_decode(C.byref(workload(w)), C.byref(hw(h)),
                            idx.ctypes.data_as(C.POINTER(C.c_uint64)), len(idx), out), "mmee_decode")
    return list(out)


def mmee_eval_batch(w, h, first_idx: int, n: int, out=None):
    """Costs of n consecutive candidates.  out=None: returns a numpy record array (host);
    out=<int>: a device pointer to n 64-byte records, filled in place (nothing is copied back)."""
    if out is None:
        host = np.zeros(n, dtype=COST_DTYPE)
        _check(_lib.mmee_eval_batch(C.byref(workload(w)), C.byref(hw(h)), first_idx, n,
                                    host.ctypes.data), "mmee_eval_batch")
        return host
    _check(_lib.mmee_eval_batch(C.byref(workload(w)), C.byref(hw(h)), first_idx, n, C.c_void_p(int(out))),
           "mmee_eval_batch")
    return None


def mmee_search(w, h, objective: int) -> Result:
    r = Result()
    _check(_lib.mmee_search(C.byref(workload(w)), C.byref(hw(h)), objective, C.byref(r)), "mmee_search")
    return r


def mmee_search_ex(w, h, objective: int, flags: int = SEARCH_PRUNED, allow_infeasible: bool = False):
    r = Result()
    code = _check(_lib.mmee_search_ex(C.byref(workload(w)), C.byref(hw(h)), objective, flags, C.byref(r)),
                  "mmee_search_ex", allow=(ENOFEASIBLE,) if allow_infeasible else ())
    return (code, r) if allow_infeasible else r


def mmee_search_noalloc(w, h, objective: int, flags: int, out_dev: int) -> None:
    """Enqueue one search that allocates nothing; out_dev is a device pointer to one Result record,
    valid after the caller has synchronised the library's stream."""
    _check(_lib.mmee_search_noalloc(C.byref(workload(w)), C.byref(hw(h)), objective, flags,
                                    C.c_void_p(int(out_dev))), "mmee_search_noalloc")


def mmee_search_multi(w, h, objectives, flags: int = SEARCH_PRUNED):
    n = len(objectives)
    objs = (C.c_int * n)(*objectives)
    out = (Result * n)()
    _check(_lib.mmee_search_multi(C.byref(workload(w)), C.byref(hw(h)), objs, n, flags, out), "mmee_search_multi")
    return list(out)


class ManyPoints:
    """The argument arrays of mmee_search_many, marshalled once for repeated calls."""

    def __init__(self, points):
        n = self.n = len(points)
        self.ws = (Workload * n)(*[workload(p[0]) for p in points])
        self.hs = (Hw * n)(*[hw(p[1]) for p in points])
        self.objs = (C.c_int * n)(*[p[2] for p in points])
        self.out = (Result * n)()
        self.codes = (C.c_int * n)()


def mmee_search_many(points, flags: int = SEARCH_PRUNED):
    """points: sequence of (workload, hw, objective), or a ManyPoints made from one (its result
    arrays are then reused by the next call).  Returns (results, codes)."""
    m = points if isinstance(points, ManyPoints) else ManyPoints(points)
    _check(_lib.mmee_search_many(m.ws, m.hs, m.objs, m.n, flags, m.out, m.codes), "mmee_search_many", allow=(ENOFEASIBLE,))
    if m is points:
        return m.out, m.codes                   # the arrays themselves: valid until the next call with this ManyPoints
    return list(m.out), list(m.codes)


def mmee_chain_space_size(c, h) -> int:
    out = C.c_uint64()
    _check(_lib.mmee_chain_space_size(C.byref(chain(c)), C.byref(hw(h)), C.byref(out)), "mmee_chain_space_size")
    return out.value


def mmee_chain_decode(c, h, indices):
    idx = np.ascontiguousarray(indices, dtype=np.uint64)
    out = (Mapping * len(idx))()
    _check(_lib.mmee_chain_decode(C.byref(chain(c)), C.byref(hw(h)),
                                  idx.ctypes.data_as(C.POINTER(C.c_uint64)), len(idx), out), "mmee_chain_decode")
    return list(out)


def mmee_chain_eval_batch(c, h, first_idx: int, n: int, out=None):
    if out is None:
        host = np.zeros(n, dtype=COST_DTYPE)
        _check(_lib.mmee_chain_eval_batch(C.byref(chain(c)), C.byref(hw(h)), first_idx, n,
                                          host.ctypes.data), "mmee_chain_eval_batch")
        return host
    _check(_lib.mmee_chain_eval_batch(C.byref(chain(c)), C.byref(hw(h)), first_idx, n, C.c_void_p(int(out))),
           "mmee_chain_eval_batch")
    return None


def mmee_chain_search_multi(c, h, objectives, flags: int = SEARCH_PRUNED):
    n = len(objectives)
    objs = (C.c_int * n)(*objectives)
    out = (Result * n)()
    _check(_lib.mmee_chain_search_multi(C.byref(chain(c)), C.byref(hw(h)), objs, n, flags, out),
           "mmee_chain_search_multi")
    return list(out)


def mmee_chain_search_many(points, flags: int = SEARCH_PRUNED):
    """points: sequence of (chain, hw, objective).  Returns (results, codes)."""
    n = len(points)
    cs = (Chain * n)(*[chain(p[0]) for p in points])
    hs = (Hw * n)(*[hw(p[1]) for p in points])
    objs = (C.c_int * n)(*[p[2] for p in points])
    out = (Result * n)()
    codes = (C.c_int * n)()
    _check(_lib.mmee_chain_search_many(cs, hs, objs, n, flags, out, codes), "mmee_chain_search_many",
           allow=(ENOFEASIBLE,))
    return list(out), list(codes)


def _pareto(fn, name, problem, h, flags, capacity):
    out = (Result * capacity)()
    n = C.c_uint32()
    code = _check(fn(C.byref(problem), C.byref(hw(h)), flags, out, capacity, C.byref(n)), name,
                  allow=(ENOFEASIBLE, EOVERFLOW))
    return code, list(out[:n.value])


def mmee_pareto(w, h, flags: int = SEARCH_PRUNED, capacity: int = 256):
    """Energy-latency Pareto front by ascending latency.  Returns (code, [Result])."""
    return _pareto(_lib.mmee_pareto, "mmee_pareto", workload(w), h, flags, capacity)


def mmee_chain_pareto(c, h, flags: int = SEARCH_PRUNED, capacity: int = 256):
    return _pareto(_lib.mmee_chain_pareto, "mmee_chain_pareto", chain(c), h, flags, capacity)


def mmee_front_bs_da(w, h, flags: int = SEARCH_PRUNED, capacity: int = 1024):
    """DRAM access versus buffer size front by ascending buffer size.  Returns (code, [Result])."""
    return _pareto(_lib.mmee_front_bs_da, "mmee_front_bs_da", workload(w), h, flags, capacity)


def mmee_chain_front_bs_da(c, h, flags: int = SEARCH_PRUNED, capacity: int = 1024):
    return _pareto(_lib.mmee_chain_front_bs_da, "mmee_chain_front_bs_da", chain(c), h, flags, capacity)


def mmee_offline_stats() -> RowStats:
    s = RowStats()
    _check(_lib.mmee_offline_stats(C.byref(s)), "mmee_offline_stats")
    return s


def mmee_offline_rows(group: int, which: int = 1):
    """Row numbers (inside group g = r + 2 f) that denote a dataflow (which=0) or survive pruning (which=1)."""
    out = (C.c_uint32 * 15000)()
    n = C.c_uint32()
    _check(_lib.mmee_offline_rows(group, which, out, 15000, C.byref(n)), "mmee_offline_rows")
    return list(out[:n.value])


# ---- running the chains: tensors of any library that have data_ptr(), shape, stride(), dtype, element_size() and numel() ----

_FLOATS = {"torch.float16": F16, "torch.bfloat16": BF16}


def _invalid(where: str, why: str):
    e = MmeeError(EINVAL, where)
    e.args = (f"{e.args[0]}: {why}",)
    return e


def _float_type(where, tensors):
    """The common dtype of 16-bit device tensors whose last dimension is contiguous."""
    kinds = {str(t.dtype) for t in tensors.values()}
    if len(kinds) != 1 or not kinds <= set(_FLOATS):
        raise _invalid(where, f"float16 or bfloat16 throughout is wanted, got {', '.join(sorted(kinds))}")
    for name, t in tensors.items():
        _on_device(where, name, t)
        if t.shape[-1] > 1 and t.stride()[-1] != 1:
            raise _invalid(where, f"{name}: the last dimension has to be contiguous")
    return _FLOATS[kinds.pop()]


def _on_device(where, name, t):
    if not t.is_cuda:
        raise _invalid(where, f"{name} is not on the GPU")


def _shaped(where, name, t, *shape):
    if tuple(t.shape) != shape:
        raise _invalid(where, f"{name} has shape {tuple(t.shape)}, {shape} is wanted")


def _whole(where, name, t, shape, kinds, contiguous=True):
    """A device pointer to whole numbers or 32-bit floats of that shape, or None."""
    if t is None:
        return None
    _shaped(where, name, t, *shape)
    _on_device(where, name, t)
    if str(t.dtype) not in kinds:
        raise _invalid(where, f"{name} is {t.dtype}, {' or '.join(kinds)} is wanted")
    if contiguous and not t.is_contiguous():
        raise _invalid(where, f"{name} has to be contiguous")
    return t.data_ptr()


def _scale(where, head_dim, given):
    if head_dim == 0:
        raise _invalid(where, "the head size is 0")
    return head_dim ** -0.5 if given is None else given


def _three(t):
    return _Strides(*t.stride()[:3])


def attn(q, k, v, o, lse=None, scale: float | None = None, kv_lens=None, key_mask=None) -> Attn:
    """Arguments of mmee_attn_forward and mmee_attn_backward.  q, o [batch, q_len, heads, head_dim]; k, v [batch, kv_len, kv_heads,
    head_dim], any strides but of the last dimension; lse float32 [batch, heads, q_len] (wanted for the backward call); kv_lens int32 [batch]; key_mask
    uint8 or bool [batch, kv_len], 0: the key does not count.  scale: 1 / sqrt(head_dim) unless given."""
    where = "attn"
    dtype = _float_type(where, {"q": q, "k": k, "v": v, "o": o})
    if len(q.shape) != 4 or len(k.shape) != 4:
        raise _invalid(where, "q and k have four dimensions")
    B, Lq, H, d = q.shape
    Lk, Hkv = k.shape[1:3]
    _shaped(where, "k", k, B, Lk, Hkv, d)
    _shaped(where, "v", v, B, Lk, Hkv, d)
    _shaped(where, "o", o, B, Lq, H, d)
    mask = _whole(where, "key_mask", key_mask, (B, Lk), ("torch.uint8", "torch.bool"), contiguous=False)
    if mask and Lk > 1 and key_mask.stride()[1] != 1:
        raise _invalid(where, "key_mask: the last dimension has to be contiguous")
    a = Attn(dtype, B, H, Hkv, d, Lq, Lk, _scale(where, d, scale), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
             _three(q), _three(k), _three(v), _three(o), _whole(where, "lse", lse, (B, H, Lq), ("torch.float32",)),
             _whole(where, "kv_lens", kv_lens, (B,), ("torch.int32",)), mask, key_mask.stride()[0] if mask else 0)
    a._tensors = (q, k, v, o, lse, kv_lens, key_mask)
    return a


def attn_grads(do, dq, dk, dv) -> AttnGrads:
    """Output gradient and gradients of mmee_attn_backward, shaped as o, q, k and v."""
    _float_type("attn_grads", {"do": do, "dq": dq, "dk": dk, "dv": dv})
    _shaped("attn_grads", "dq", dq, *do.shape)
    _shaped("attn_grads", "dv", dv, *dk.shape)
    g = AttnGrads(do.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), _three(do), _three(dq), _three(dk), _three(dv))
    g._tensors = (do, dq, dk, dv)
    return g


def mmee_attn_workspace(a: Attn, backward: bool = False) -> int:
    out = C.c_uint64()
    _check(_lib.mmee_attn_workspace(C.byref(a), int(backward), C.byref(out)), "mmee_attn_workspace")
    return out.value


def mmee_attn_forward(a: Attn) -> None:
    _check(_lib.mmee_attn_forward(C.byref(a)), "mmee_attn_forward")


def mmee_attn_backward(a: Attn, g: AttnGrads) -> None:
    do, dq, dk, dv = g._tensors
    q, k = a._tensors[:2]
    for name, t, like in (("do", do, q), ("dk", dk, k)):
        _shaped("mmee_attn_backward", name, t, *like.shape)
        if t.dtype != like.dtype:
            raise _invalid("mmee_attn_backward", f"{name} is {t.dtype}, {like.dtype} is wanted")
    _check(_lib.mmee_attn_backward(C.byref(a), C.byref(g)), "mmee_attn_backward")


def tree_attn(q, k_pages, v_pages, page_table, cache_lens, ancestors, o, node_counts=None, lse=None, scale: float | None = None) -> TreeAttn:
    """Arguments of mmee_tree_attn_forward.  q, o [batch, nodes, heads, head_dim]; k_pages, v_pages [n_pages, page_tokens, kv_heads, head_dim];
    page_table int32 [batch, pages_per_seq]; cache_lens, node_counts int32 [batch]; ancestors int64 (bit patterns) [batch, nodes,
    ceil(nodes / 64)]; lse float32 [batch, heads, nodes]."""
    where = "tree_attn"
    dtype = _float_type(where, {"q": q, "k_pages": k_pages, "v_pages": v_pages, "o": o})
    if len(q.shape) != 4 or len(k_pages.shape) != 4 or len(page_table.shape) != 2:
        raise _invalid(where, "q and k_pages have four dimensions, page_table two")
    B, n, H, d = q.shape
    P, page, Hkv = k_pages.shape[:3]
    _shaped(where, "k_pages", k_pages, P, page, Hkv, d)
    _shaped(where, "v_pages", v_pages, P, page, Hkv, d)
    _shaped(where, "o", o, B, n, H, d)
    width = page_table.shape[1]
    table = _whole(where, "page_table", page_table, (B, width), ("torch.int32",), contiguous=False)
    if width > 1 and page_table.stride()[1] != 1:
        raise _invalid(where, "page_table: the last dimension has to be contiguous")
    t = TreeAttn(dtype, B, H, Hkv, d, n, page, width, P, _scale(where, d, scale),
                 q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), o.data_ptr(), _three(q), _three(k_pages), _three(v_pages), _three(o),
                 table, page_table.stride()[0], _whole(where, "cache_lens", cache_lens, (B,), ("torch.int32",)),
                 _whole(where, "node_counts", node_counts, (B,), ("torch.int32",)),
                 _whole(where, "ancestors", ancestors, (B, n, (n + 63) // 64), ("torch.int64", "torch.uint64")),
                 _whole(where, "lse", lse, (B, H, n), ("torch.float32",)))
    t._tensors = (q, k_pages, v_pages, page_table, cache_lens, ancestors, o, node_counts, lse)
    return t


def mmee_tree_attn_workspace(t: TreeAttn) -> int:
    out = C.c_uint64()
    _check(_lib.mmee_tree_attn_workspace(C.byref(t), C.byref(out)), "mmee_tree_attn_workspace")
    return out.value


def mmee_tree_attn_forward(t: TreeAttn) -> None:
    _check(_lib.mmee_tree_attn_forward(C.byref(t)), "mmee_tree_attn_forward")


def ffn(x, w_gate, w_up, w_down, y, hidden, act: str = "silu", gate=None, up=None) -> Ffn:
    """Arguments of mmee_ffn_forward and mmee_ffn_backward.  x [rows, in_dim], w_gate and w_up [hidden_dim, in_dim], w_down [out_dim,
    hidden_dim], y [rows, out_dim]; hidden, and gate and up (wanted for the backward call), [rows, hidden_dim] contiguous."""
    where = "ffn"
    if hidden is None:
        raise _invalid(where, "hidden is wanted")
    kept = {name: t for name, t in (("hidden", hidden), ("gate", gate), ("up", up)) if t is not None}
    dtype = _float_type(where, {"x": x, "w_gate": w_gate, "w_up": w_up, "w_down": w_down, "y": y, **kept})
    if act not in ACTS:
        raise _invalid(where, f"act is one of {', '.join(ACTS)}")
    if len(x.shape) != 2 or len(w_gate.shape) != 2 or len(w_down.shape) != 2:
        raise _invalid(where, "x and the weights have two dimensions")
    (M, K), F, J = x.shape, w_gate.shape[0], w_down.shape[0]
    _shaped(where, "w_gate", w_gate, F, K)
    _shaped(where, "w_up", w_up, F, K)
    _shaped(where, "w_down", w_down, J, F)
    _shaped(where, "y", y, M, J)
    for name, t in kept.items():
        _shaped(where, name, t, M, F)
        if not t.is_contiguous():
            raise _invalid(where, f"{name} has to be contiguous")
    f = Ffn(dtype, ACTS[act], M, K, F, J, x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(), y.data_ptr(), hidden.data_ptr(),
            None if gate is None else gate.data_ptr(), None if up is None else up.data_ptr(),
            x.stride()[0], w_gate.stride()[0], w_up.stride()[0], w_down.stride()[0], y.stride()[0])
    f._tensors = (x, w_gate, w_up, w_down, y, hidden, gate, up)
    return f


def ffn_grads(dy, dx, dw_gate, dw_up, dw_down) -> FfnGrads:
    """Output gradient and gradients of mmee_ffn_backward, shaped as y, x and the weights; the weights' gradients contiguous."""
    where = "ffn_grads"
    _float_type(where, {"dy": dy, "dx": dx, "dw_gate": dw_gate, "dw_up": dw_up, "dw_down": dw_down})
    for name, t in (("dw_gate", dw_gate), ("dw_up", dw_up), ("dw_down", dw_down)):
        if not t.is_contiguous():
            raise _invalid(where, f"{name} has to be contiguous")
    g = FfnGrads(dy.data_ptr(), dx.data_ptr(), dw_gate.data_ptr(), dw_up.data_ptr(), dw_down.data_ptr(), dy.stride()[0], dx.stride()[0])
    g._tensors = (dy, dx, dw_gate, dw_up, dw_down)
    return g


def mmee_ffn_workspace(f: Ffn, backward: bool = False) -> int:
    out = C.c_uint64()
    _check(_lib.mmee_ffn_workspace(C.byref(f), int(backward), C.byref(out)), "mmee_ffn_workspace")
    return out.value


def mmee_ffn_forward(f: Ffn) -> None:
    _check(_lib.mmee_ffn_forward(C.byref(f)), "mmee_ffn_forward")


def mmee_ffn_backward(f: Ffn, g: FfnGrads) -> None:
    x, w_gate, w_up, w_down, y = f._tensors[:5]
    for (name, t), like in zip((("dy", g._tensors[0]), ("dx", g._tensors[1]), ("dw_gate", g._tensors[2]), ("dw_up", g._tensors[3]), ("dw_down", g._tensors[4])),
                               (y, x, w_gate, w_up, w_down)):
        _shaped("mmee_ffn_backward", name, t, *like.shape)
        if t.dtype != like.dtype:
            raise _invalid("mmee_ffn_backward", f"{name} is {t.dtype}, {like.dtype} is wanted")
    _check(_lib.mmee_ffn_backward(C.byref(f), C.byref(g)), "mmee_ffn_backward")


def _two(t):
    return _Two(*t.stride()[:2])


def _rotation(where, tokens, head_dim, freqs, positions, axis_of, pairs):
    """rot_dim, axes, and freqs, positions, axis stride and axis_of as pointers, of a rotation (none without freqs)."""
    if pairs not in PAIRS:
        raise _invalid(where, f"pairs is one of {', '.join(PAIRS)}")
    if freqs is None:
        if positions is not None or axis_of is not None:
            raise _invalid(where, "positions without freqs")
        return 0, 1, None, None, 0, None
    if len(freqs.shape) != 1 or 2 * freqs.shape[0] > head_dim:
        raise _invalid(where, f"freqs has shape {tuple(freqs.shape)}, (rot_dim / 2,) is wanted")
    rot = 2 * freqs.shape[0]
    axes, stride = 1, 0
    if positions is not None:
        if len(positions.shape) == 2:
            axes, stride = positions.shape[0], positions.stride()[0]
        _whole(where, "positions", positions, (axes, tokens) if len(positions.shape) == 2 else (tokens,), ("torch.int32",), contiguous=False)
        if tokens > 1 and positions.stride()[-1] != 1:
            raise _invalid(where, "positions: the last dimension has to be contiguous")
    return (rot, axes, _whole(where, "freqs", freqs, (rot // 2,), ("torch.float64",)), None if positions is None else positions.data_ptr(), stride,
            _whole(where, "axis_of", axis_of, (rot // 2,), ("torch.uint8",)))


def _norm_weights(where, head_dim, given):
    """Norm weights by name -> pointers, of the tensors' type (which _float_type has seen to)."""
    for name, t in given.items():
        if t is not None:
            _shaped(where, name, t, head_dim)
    return [None if t is None else t.data_ptr() for t in given.values()]


def qk_rotate(q, k, q_out, k_out, freqs, positions, axis_of=None, q_weight=None, k_weight=None, eps: float = 1e-6, pairs: str = "halves") -> QkRotate:
    """Arguments of mmee_qk_rotate_forward and mmee_qk_rotate_backward.  q, q_out [tokens, heads, head_dim]; k, k_out [tokens, kv_heads,
    head_dim], any strides but of the last dimension; freqs float64 [rot_dim / 2] in radians a position, or None: no rotation; positions int32
    [tokens] or [axes, tokens], with axis_of uint8 [rot_dim / 2]; q_weight, k_weight [head_dim]: the norms' weights, or None: no norms."""
    where = "qk_rotate"
    kept = {name: t for name, t in (("q_weight", q_weight), ("k_weight", k_weight)) if t is not None}
    dtype = _float_type(where, {"q": q, "k": k, "q_out": q_out, "k_out": k_out, **kept})
    if len(q.shape) != 3 or len(k.shape) != 3:
        raise _invalid(where, "q and k have three dimensions")
    T, H, d = q.shape
    Hkv = k.shape[1]
    _shaped(where, "k", k, T, Hkv, d)
    _shaped(where, "q_out", q_out, T, H, d)
    _shaped(where, "k_out", k_out, T, Hkv, d)
    if (q_weight is None) != (k_weight is None):
        raise _invalid(where, "q_weight and k_weight come together")
    if freqs is not None and positions is None:
        raise _invalid(where, "positions are wanted")
    rot, axes, freq_at, positions_at, axis_stride, axis_at = _rotation(where, T, d, freqs, positions, axis_of, pairs)
    r = QkRotate(dtype, PAIRS[pairs], T, H, Hkv, d, rot, axes, eps, q.data_ptr(), k.data_ptr(), q_out.data_ptr(), k_out.data_ptr(), _two(q), _two(k), _two(q_out),
                 _two(k_out), *_norm_weights(where, d, {"q_weight": q_weight, "k_weight": k_weight}), freq_at, positions_at, axis_stride, axis_at)
    r._tensors = (q, k, q_weight, k_weight, q_out, k_out, freqs, positions, axis_of)
    return r


def qk_rotate_grads(dq_out, dk_out, dq, dk, dq_weight=None, dk_weight=None) -> QkRotateGrads:
    """Output gradients and gradients of mmee_qk_rotate_backward, shaped as q_out, k_out, q, k and the weights."""
    where = "qk_rotate_grads"
    kept = {name: t for name, t in (("dq_weight", dq_weight), ("dk_weight", dk_weight)) if t is not None}
    _float_type(where, {"dq_out": dq_out, "dk_out": dk_out, "dq": dq, "dk": dk, **kept})
    if len(dq_out.shape) != 3 or len(dk_out.shape) != 3:
        raise _invalid(where, "dq_out and dk_out have three dimensions")
    _shaped(where, "dq", dq, *dq_out.shape)
    _shaped(where, "dk", dk, *dk_out.shape)
    g = QkRotateGrads(dq_out.data_ptr(), dk_out.data_ptr(), dq.data_ptr(), dk.data_ptr(),
                      *_norm_weights(where, dq_out.shape[2], {"dq_weight": dq_weight, "dk_weight": dk_weight}), _two(dq_out), _two(dk_out), _two(dq), _two(dk))
    g._tensors = (dq_out, dk_out, dq, dk, dq_weight, dk_weight)
    return g


def mmee_qk_rotate_workspace(r: QkRotate) -> int:
    out = C.c_uint64()
    _check(_lib.mmee_qk_rotate_workspace(C.byref(r), C.byref(out)), "mmee_qk_rotate_workspace")
    return out.value


def mmee_qk_rotate_forward(r: QkRotate) -> None:
    _check(_lib.mmee_qk_rotate_forward(C.byref(r)), "mmee_qk_rotate_forward")


def mmee_qk_rotate_backward(r: QkRotate, g: QkRotateGrads) -> None:
    where = "mmee_qk_rotate_backward"
    for name, t, like in zip(("dq", "dk", "dq_weight", "dk_weight"), g._tensors[2:], r._tensors):
        if (t is None) != (like is None):
            raise _invalid(where, f"{name} is {'wanted' if t is None else 'not wanted'}")
        if t is not None:
            _shaped(where, name, t, *like.shape)
            if t.dtype != like.dtype:
                raise _invalid(where, f"{name} is {t.dtype}, {like.dtype} is wanted")
    _check(_lib.mmee_qk_rotate_backward(C.byref(r), C.byref(g)), where)


def cache_append(k, v, k_pages, v_pages, page_table, cache_lens, starts=None, counts=None, q=None, q_out=None, freqs=None, positions=None, axis_of=None,
                 q_weight=None, k_weight=None, eps: float = 1e-6, pairs: str = "halves") -> CacheAppend:
    """Arguments of mmee_cache_append_forward.  k, v [tokens, kv_heads, head_dim]; k_pages, v_pages [n_pages, page_tokens, kv_heads, head_dim];
    page_table int32 [seqs, pages_per_seq]; cache_lens, counts int32 [seqs]; starts int32 [seqs + 1], or None: as many tokens of every
    sequence; q, q_out [tokens, heads, head_dim] or None; the rest as for qk_rotate, positions None: those in the cache."""
    where = "cache_append"
    if (q is None) != (q_out is None):
        raise _invalid(where, "q and q_out come together")
    kept = {name: t for name, t in (("q", q), ("q_out", q_out), ("q_weight", q_weight), ("k_weight", k_weight)) if t is not None}
    dtype = _float_type(where, {"k": k, "v": v, "k_pages": k_pages, "v_pages": v_pages, **kept})
    if len(k.shape) != 3 or len(k_pages.shape) != 4 or len(page_table.shape) != 2:
        raise _invalid(where, "k has three dimensions, k_pages four, page_table two")
    T, Hkv, d = k.shape
    P, page = k_pages.shape[:2]
    B, width = page_table.shape
    _shaped(where, "v", v, T, Hkv, d)
    _shaped(where, "k_pages", k_pages, P, page, Hkv, d)
    _shaped(where, "v_pages", v_pages, P, page, Hkv, d)
    H = 0
    if q is not None:
        if len(q.shape) != 3:
            raise _invalid(where, "q has three dimensions")
        H = q.shape[1]
        _shaped(where, "q", q, T, H, d)
        _shaped(where, "q_out", q_out, T, H, d)
    if (q_weight is None) != (k_weight is None or q is None):
        raise _invalid(where, "q_weight and k_weight come together, q_weight with q alone")
    table = _whole(where, "page_table", page_table, (B, width), ("torch.int32",), contiguous=False)
    if width > 1 and page_table.stride()[1] != 1:
        raise _invalid(where, "page_table: the last dimension has to be contiguous")
    rot, axes, freq_at, positions_at, axis_stride, axis_at = _rotation(where, T, d, freqs, positions, axis_of, pairs)
    none = _Two(0, 0)
    c = CacheAppend(dtype, PAIRS[pairs], T, B, H, Hkv, d, rot, axes, page, width, P, eps, None if q is None else q.data_ptr(), k.data_ptr(), v.data_ptr(),
                    None if q is None else q_out.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), none if q is None else _two(q), _two(k), _two(v),
                    none if q is None else _two(q_out), _three(k_pages), _three(v_pages), *_norm_weights(where, d, {"q_weight": q_weight, "k_weight": k_weight}),
                    freq_at, positions_at, axis_stride, axis_at, _whole(where, "starts", starts, (B + 1,), ("torch.int32",)),
                    _whole(where, "counts", counts, (B,), ("torch.int32",)), _whole(where, "cache_lens", cache_lens, (B,), ("torch.int32",)),
                    table, page_table.stride()[0])
    c._tensors = (k, v, k_pages, v_pages, page_table, cache_lens, starts, counts, q, q_out, freqs, positions, axis_of, q_weight, k_weight)
    return c


def mmee_cache_append_forward(c: CacheAppend) -> None:
    _check(_lib.mmee_cache_append_forward(C.byref(c)), "mmee_cache_append_forward")


def prompt_attn(q, k, v, o, q_starts, kv_starts=None, lse=None, scale: float | None = None, causal: bool = True) -> PromptAttn:
    """Arguments of mmee_prompt_attn_forward and mmee_prompt_attn_backward.  q, o [q_tokens, heads, head_dim]; k, v [kv_tokens, kv_heads,
    head_dim], any strides but of the last dimension; q_starts, kv_starts int32 [seqs + 1], kv_starts None: q_starts; lse float32 [heads,
    q_tokens] (wanted for the backward call).  scale: 1 / sqrt(head_dim) unless given."""
    where = "prompt_attn"
    dtype = _float_type(where, {"q": q, "k": k, "v": v, "o": o})
    if len(q.shape) != 3 or len(k.shape) != 3 or len(q_starts.shape) != 1:
        raise _invalid(where, "q and k have three dimensions, q_starts one")
    Tq, H, d = q.shape
    Tk, Hkv = k.shape[:2]
    _shaped(where, "k", k, Tk, Hkv, d)
    _shaped(where, "v", v, Tk, Hkv, d)
    _shaped(where, "o", o, Tq, H, d)
    if kv_starts is None and Tk != Tq:
        raise _invalid(where, "kv_starts are wanted where there are not as many keys as rows")
    seqs = q_starts.shape[0] - 1
    if seqs < 1:
        raise _invalid(where, "q_starts has a start and an end at least")
    a = PromptAttn(dtype, bool(causal), seqs, H, Hkv, d, Tq, Tk, _scale(where, d, scale), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), _two(q), _two(k),
                   _two(v), _two(o), _whole(where, "q_starts", q_starts, (seqs + 1,), ("torch.int32",)), _whole(where, "kv_starts", kv_starts, (seqs + 1,), ("torch.int32",)),
                   _whole(where, "lse", lse, (H, Tq), ("torch.float32",)))
    a._tensors = (q, k, v, o, q_starts, kv_starts, lse)
    return a


def prompt_attn_grads(do, dq, dk, dv) -> PromptAttnGrads:
    """Output gradient and gradients of mmee_prompt_attn_backward, shaped as o, q, k and v."""
    where = "prompt_attn_grads"
    _float_type(where, {"do": do, "dq": dq, "dk": dk, "dv": dv})
    if len(do.shape) != 3 or len(dk.shape) != 3:
        raise _invalid(where, "do and dk have three dimensions")
    _shaped(where, "dq", dq, *do.shape)
    _shaped(where, "dv", dv, *dk.shape)
    g = PromptAttnGrads(do.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), _two(do), _two(dq), _two(dk), _two(dv))
    g._tensors = (do, dq, dk, dv)
    return g


def mmee_prompt_attn_workspace(a: PromptAttn, backward: bool = False) -> int:
    out = C.c_uint64()
    _check(_lib.mmee_prompt_attn_workspace(C.byref(a), int(backward), C.byref(out)), "mmee_prompt_attn_workspace")
    return out.value


def mmee_prompt_attn_forward(a: PromptAttn) -> None:
    _check(_lib.mmee_prompt_attn_forward(C.byref(a)), "mmee_prompt_attn_forward")


def mmee_prompt_attn_backward(a: PromptAttn, g: PromptAttnGrads) -> None:
    do, dq, dk, dv = g._tensors
    q, k = a._tensors[:2]
    for name, t, like in (("do", do, q), ("dk", dk, k)):
        _shaped("mmee_prompt_attn_backward", name, t, *like.shape)
        if t.dtype != like.dtype:
            raise _invalid("mmee_prompt_attn_backward", f"{name} is {t.dtype}, {like.dtype} is wanted")
    _check(_lib.mmee_prompt_attn_backward(C.byref(a), C.byref(g)), "mmee_prompt_attn_backward")


def mmee_set_stream(stream_ptr: int | None):
    _check(_lib.mmee_set_stream(C.c_void_p(stream_ptr or 0)), "mmee_set_stream")


def mmee_shutdown():
    _lib.mmee_shutdown()
