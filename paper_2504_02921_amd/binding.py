"""ctypes binding of libhyperrerank.so: the same entry points as include/hyperrerank.h.

Only argument marshalling happens here.  PyTorch provides device memory and
streams; every step of the scoring pass runs inside the library's HIP kernels.
There is no fallback: if the shared library is missing, importing this module
raises.
"""

from __future__ import annotations

import ctypes as C
import operator
import os
from typing import Dict, List, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhyperrerank.so")

HR_F32, HR_BF16, HR_FP8_E4M3 = 0, 1, 2
DTYPE_CODE = {"f32": HR_F32, "bf16": HR_BF16, "fp8": HR_FP8_E4M3}
PAGE_TOKENS = 16

STATUS = {
    0: "HR_OK", -1: "HR_ERR_INVALID_ARG", -2: "HR_ERR_POOL_TOO_SMALL", -3: "HR_ERR_PAGE_RANGE",
    -4: "HR_ERR_PAGE_IN_USE", -5: "HR_ERR_PAGE_DUP", -6: "HR_ERR_LEN_RANGE", -7: "HR_ERR_TABLE_SHORT",
    -8: "HR_ERR_TOKEN_RANGE", -9: "HR_ERR_WORKSPACE_SMALL", -10: "HR_ERR_UNSUPPORTED_SHAPE",
    -11: "HR_ERR_DEVICE", -12: "HR_ERR_POOL_FULL", -13: "HR_ERR_MISMATCH",
}
HR_OK = 0
for _code, _name in STATUS.items():
    globals()[_name] = _code


class hr_pool_cfg(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("page_tokens", C.c_int32), ("num_pages", C.c_int32), ("kv_dtype", C.c_int32)]


class hr_model_cfg(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("hidden", C.c_int32), ("n_q_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("ffn", C.c_int32), ("vocab", C.c_int32),
                ("yes_id", C.c_int32), ("no_id", C.c_int32), ("dtype", C.c_int32),
                ("rope_base", C.c_float), ("rms_eps", C.c_float)]


class hr_range_report(C.Structure):
    _fields_ = [("overflow", C.c_int64), ("underflow", C.c_int64), ("nonfinite_inputs", C.c_int64),
                ("fp8_nan_codes", C.c_int64), ("fp8_bad_scales", C.c_int64), ("reserved", C.c_int64 * 3)]

    def as_dict(self):
        return {k: int(getattr(self, k)) for k in ("overflow", "underflow", "nonfinite_inputs", "fp8_nan_codes", "fp8_bad_scales")}


class hr_rope_cfg(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rotary_dim", C.c_int32), ("layout", C.c_int32), ("scaling", C.c_int32),
                ("amplitude", C.c_float), ("base", C.c_float), ("factor", C.c_float), ("original_len", C.c_float),
                ("low", C.c_float), ("high", C.c_float)]


class hr_rope_tensor(C.Structure):
    _fields_ = [("in_", C.c_void_p), ("out", C.c_void_p), ("n_heads", C.c_int32), ("in_token_stride", C.c_int64),
                ("in_head_stride", C.c_int64), ("out_token_stride", C.c_int64), ("out_head_stride", C.c_int64)]


class hr_doc_list(C.Structure):
    _fields_ = [("n_docs", C.c_int32), ("n_pages", C.c_int32), ("doc_lens", C.c_void_p), ("page_cu", C.c_void_p), ("pages", C.c_void_p)]


class hr_pair_tables(C.Structure):
    _fields_ = [("n_pairs", C.c_int32), ("max_tokens", C.c_int32), ("pt_stride", C.c_int32), ("n_q_heads", C.c_int32),
                ("q_cu", C.c_void_p), ("doc_lens", C.c_void_p), ("page_table", C.c_void_p), ("tok_pos", C.c_void_p),
                ("tok_pair", C.c_void_p), ("order", C.c_void_p), ("report", C.c_void_p), ("sched", C.c_void_p), ("sched_bytes", C.c_size_t)]


class hr_attention_args(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("layer", C.c_int32), ("scale", C.c_float), ("cap", C.c_float), ("window", C.c_int32),
                ("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p),
                ("slopes", C.c_void_p), ("prefix_lens", C.c_void_p)] + \
               [(t + s, C.c_int64) for t in ("q", "k", "v", "out") for s in ("_token_stride", "_head_stride")]


_PP = C.POINTER(C.c_void_p)


class hr_weight_ptrs(C.Structure):
    _fields_ = [("embedding", C.c_void_p), ("final_norm", C.c_void_p),
                ("wq", _PP), ("wk", _PP), ("wv", _PP), ("wo", _PP), ("wg", _PP), ("wu", _PP), ("wd", _PP),
                ("norm1", _PP), ("norm2", _PP)]


EXPORTS = [
    "hr_status_str", "hr_last_error", "hr_kv_pool_bytes", "hr_kv_pool_create", "hr_kv_pool_destroy", "hr_kv_pool_free_pages",
    "hr_kv_pool_alloc_pages", "hr_doc_kv_write", "hr_doc_kv_read", "hr_doc_kv_free", "hr_kv_page_record_bytes", "hr_kv_pages_out",
    "hr_kv_pages_in", "hr_kv_page_record4_bytes", "hr_kv_pages_out4", "hr_kv_pages_in4", "hr_weights_pack_bytes", "hr_weights_load",
    "hr_model_destroy", "hr_rerank_workspace_bytes", "hr_rerank_score", "hr_rerank_static_scratch_bytes",
    "hr_rerank_score_static", "hr_rerank_plan_create", "hr_rerank_plan_set_inputs", "hr_rerank_plan_run",
    "hr_rerank_plan_destroy", "hr_model_set_precise_layers", "hr_model_precise_layers", "hr_rerank_set_streams", "hr_rerank_parts", "hr_rerank_validate",
    "hr_rerank_full_workspace_bytes", "hr_rerank_score_full", "hr_doc_prefill_workspace_bytes", "hr_doc_prefill", "hr_attention_path", "hr_gemm_path",
    "hr_rerank_topk", "hr_rerank_topk_host", "hr_model_range_report", "hr_kv_pool_range_report", "hr_probe_read_bandwidth", "hr_profile_enable", "hr_profile_select", "hr_profile_count", "hr_profile_name", "hr_profile_read",
    "hr_rope_frequencies", "hr_rope_apply", "hr_pair_tables_sched_bytes", "hr_pair_tables_build", "hr_pair_attention_workspace_bytes", "hr_pair_attention",
]


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it first (python -m paper_2504_02921_amd.build "
                          "or __graft_entry__.build()); there is no CPU fallback")
    # PyTorch ships its own HIP runtime; it must be the one this library binds to, or streams and
    # allocations made by torch would belong to a different runtime instance.  Loading torch first
    # puts its libamdhip64 (same soname) in the process before ours is resolved.
    import torch  # noqa: F401
    bundled = os.path.join(os.path.dirname(torch.__file__), "lib", "libamdhip64.so")
    if os.path.exists(bundled):
        C.CDLL(bundled, mode=C.RTLD_GLOBAL)
    lib = C.CDLL(LIB_PATH)
    i32p = C.c_void_p                  # int32 arrays of the host: an address, or anything ctypes takes as a pointer
    sig = {
        "hr_status_str": (C.c_char_p, [C.c_int]),
        "hr_last_error": (C.c_char_p, []),
        "hr_kv_pool_bytes": (C.c_size_t, [C.POINTER(hr_pool_cfg)]),
        "hr_kv_pool_create": (C.c_int, [C.POINTER(hr_pool_cfg), C.c_void_p, C.c_size_t, C.POINTER(C.c_void_p)]),
        "hr_kv_pool_destroy": (None, [C.c_void_p]),
        "hr_kv_pool_free_pages": (C.c_int64, [C.c_void_p]),
        "hr_kv_pool_alloc_pages": (C.c_int, [C.c_void_p, C.c_int32, i32p]),
        "hr_doc_kv_write": (C.c_int, [C.c_void_p, C.c_int32, i32p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
        "hr_doc_kv_read": (C.c_int, [C.c_void_p, C.c_int32, i32p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
        "hr_doc_kv_free": (C.c_int, [C.c_void_p, i32p, C.c_int32]),
        "hr_kv_page_record_bytes": (C.c_size_t, [C.c_void_p]),
        "hr_kv_pages_out": (C.c_int, [C.c_void_p, C.c_int32, i32p, C.c_void_p, C.c_void_p]),
        "hr_kv_pages_in": (C.c_int, [C.c_void_p, C.c_int32, i32p, C.c_void_p, C.c_void_p]),
        "hr_kv_page_record4_bytes": (C.c_size_t, [C.c_void_p]),
        "hr_kv_pages_out4": (C.c_int, [C.c_void_p, C.c_int32, i32p, C.c_void_p, C.c_void_p]),
        "hr_kv_pages_in4": (C.c_int, [C.c_void_p, C.c_int32, i32p, C.c_void_p, C.c_void_p]),
        "hr_weights_pack_bytes": (C.c_size_t, [C.POINTER(hr_model_cfg)]),
        "hr_weights_load": (C.c_int, [C.POINTER(hr_model_cfg), C.POINTER(hr_weight_ptrs), C.c_void_p, C.c_size_t,
                                      C.c_void_p, C.POINTER(C.c_void_p)]),
        "hr_model_destroy": (None, [C.c_void_p]),
        "hr_rerank_workspace_bytes": (C.c_size_t, [C.c_void_p, C.c_int32, C.c_int64, C.c_int32]),
        "hr_rerank_score": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, i32p, C.c_int32, i32p, i32p, i32p,
                                      C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]),
        "hr_rerank_static_scratch_bytes": (C.c_size_t, []),
        "hr_rerank_score_static": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, i32p, C.c_int32, i32p, i32p, i32p,
                                             C.c_void_p, C.c_void_p]),
        "hr_rerank_plan_create": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, i32p, i32p, C.c_int32, C.c_void_p, C.c_size_t,
                                            C.POINTER(C.c_void_p)]),
        "hr_rerank_plan_set_inputs": (C.c_int, [C.c_void_p, i32p, i32p]),
        "hr_rerank_plan_run": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
        "hr_rerank_plan_destroy": (None, [C.c_void_p]),
        "hr_model_set_precise_layers": (C.c_int, [C.c_void_p, C.c_int]),
        "hr_model_precise_layers": (C.c_int, [C.c_void_p]),
        "hr_rerank_set_streams": (C.c_int, [C.c_void_p, C.c_int]),
        "hr_rerank_parts": (C.c_int, [C.c_void_p, C.c_int64]),
        "hr_rerank_validate": (C.c_int, [C.POINTER(hr_model_cfg), C.c_void_p, C.c_int32, i32p, C.c_int32, i32p, i32p, i32p]),
        "hr_rerank_full_workspace_bytes": (C.c_size_t, [C.c_void_p, C.c_int32, C.c_int64]),
        "hr_rerank_score_full": (C.c_int, [C.c_void_p, C.c_int32, i32p, i32p, i32p, i32p, C.c_void_p, C.c_size_t,
                                           C.c_void_p, C.c_void_p]),
        "hr_doc_prefill_workspace_bytes": (C.c_size_t, [C.c_void_p, C.c_int32, C.c_int64]),
        "hr_doc_prefill": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, i32p, i32p, i32p, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]),
        "hr_attention_path": (C.c_char_p, [C.c_void_p, C.c_void_p]),
        "hr_gemm_path": (C.c_char_p, [C.c_void_p]),
        "hr_rerank_topk_host": (C.c_int, [C.c_void_p, i32p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]),
        "hr_rerank_topk": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]),
        "hr_model_range_report": (C.c_int, [C.c_void_p, C.POINTER(hr_range_report)]),
        "hr_kv_pool_range_report": (C.c_int, [C.c_void_p, C.POINTER(hr_range_report)]),
        "hr_probe_read_bandwidth": (C.c_int, [C.c_void_p, C.c_size_t, C.c_void_p, C.c_size_t, C.c_int, C.c_void_p]),
        "hr_profile_enable": (C.c_int, [C.c_void_p, C.c_int]),
        "hr_profile_select": (C.c_int, [C.c_void_p, C.c_uint32]),
        "hr_profile_count": (C.c_int, []),
        "hr_profile_name": (C.c_char_p, [C.c_int]),
        "hr_profile_read": (C.c_int, [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_int64)]),
        "hr_rope_frequencies": (C.c_int, [C.POINTER(hr_rope_cfg), C.c_void_p]),
        "hr_rope_apply": (C.c_int, [C.POINTER(hr_rope_cfg), C.c_void_p, C.c_int, C.c_int64, C.c_void_p, C.c_int32, C.c_int32,
                                    C.POINTER(hr_rope_tensor), C.c_int32, C.c_int, C.c_void_p]),
        "hr_pair_tables_sched_bytes": (C.c_size_t, [C.c_void_p, C.c_int32, C.c_int32, C.c_int32]),
        "hr_pair_tables_build": (C.c_int, [C.c_void_p, C.POINTER(hr_doc_list), C.c_void_p, C.c_void_p, C.POINTER(hr_pair_tables), C.c_void_p]),
        "hr_pair_attention_workspace_bytes": (C.c_size_t, [C.c_void_p, C.POINTER(hr_pair_tables)]),
        "hr_pair_attention": (C.c_int, [C.c_void_p, C.POINTER(hr_pair_tables), C.POINTER(hr_attention_args), C.c_void_p, C.c_size_t, C.c_void_p]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


lib = _load()


class HrError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        detail = lib.hr_last_error().decode() if status == -11 else ""
        super().__init__(f"{where}: {STATUS.get(status, status)} ({lib.hr_status_str(status).decode()}) {detail}")


def check(status: int, where: str) -> None:
    if status != HR_OK:
        raise HrError(status, where)


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(a, np.int32)


def _i32p(a: Optional[np.ndarray]):
    """Address of an int32 array (a plain integer: a typed ctypes pointer costs 3 us, as much as a launch)."""
    return None if a is None else a.ctypes.data


def _stream_ptr(stream=None) -> int:
    if stream is not None:
        return stream.cuda_stream
    import torch
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


# ----------------------------------------------------------------------------------------------
# thin, same-named wrappers (raw pointers in, status out)
# ----------------------------------------------------------------------------------------------
def make_pool_cfg(n_layers, n_kv_heads, head_dim, num_pages, kv_dtype) -> hr_pool_cfg:
    return hr_pool_cfg(n_layers, n_kv_heads, head_dim, PAGE_TOKENS, num_pages, DTYPE_CODE.get(kv_dtype, kv_dtype))


def make_model_cfg(m) -> hr_model_cfg:
    """m: any object with the ModelCfg fields of the workload generators."""
    return hr_model_cfg(m.n_layers, m.hidden, m.n_q_heads, m.n_kv_heads, m.head_dim, m.ffn, m.vocab,
                        m.yes_id, m.no_id, DTYPE_CODE[m.dtype], float(m.rope_base), float(m.rms_eps))


def hr_kv_pool_bytes(cfg: hr_pool_cfg) -> int:
    return int(lib.hr_kv_pool_bytes(C.byref(cfg)))


def hr_kv_pool_create(cfg: hr_pool_cfg, dev_ptr: int, nbytes: int):
    out = C.c_void_p()
    st = lib.hr_kv_pool_create(C.byref(cfg), C.c_void_p(dev_ptr), nbytes, C.byref(out))
    return st, out


def hr_weights_pack_bytes(cfg: hr_model_cfg) -> int:
    return int(lib.hr_weights_pack_bytes(C.byref(cfg)))


# ----------------------------------------------------------------------------------------------
# convenience holders: own the torch tensors behind the handles
# ----------------------------------------------------------------------------------------------
# Up to this many queries the offsets travel as kernel arguments, 256 a launch; beyond, one upload and one launch are less.
# Offsets as arguments / uploaded, whole calls: 1 query 11.9 / 25.2 us, 256 10.9 / 26.4, 512 13.7 / 27.5, 1024 20.9 / 27.4, 4096
# 79.5 / 39.9, 16384 181 / 42.
_TOPK_HOST_QUERIES = 1024


def rerank_topk(scores, seg_offsets, k: int, with_scores: bool = False, stream=None):
    """Per-query top-k of device scores: seg_offsets (host ints, [n_queries + 1]) delimits each query's pairs.
    Returns an int32 device tensor [n_queries][k] of candidate indices inside each segment (-1 padded), and the
    matching scores when asked."""
    import torch
    seg = _i32(seg_offsets)
    n_q = len(seg) - 1
    max_c = max(int((seg[1:] - seg[:-1]).max()) if n_q > 0 else 1, k, 1)      # an upper bound is all the library needs
    idx = torch.empty((max(n_q, 0), k), dtype=torch.int32, device=scores.device)
    sc = torch.empty((max(n_q, 0), k), dtype=torch.float32, device=scores.device) if with_scores else None
    out = (idx.data_ptr(), sc.data_ptr() if with_scores else None, _stream_ptr(stream))
    if n_q > _TOPK_HOST_QUERIES:
        with torch.cuda.stream(stream):              # the offsets belong to the stream that reads them (None: the current one)
            if not torch.cuda.is_current_stream_capturing():      # a blocking upload cannot be captured
                seg_dev = torch.from_numpy(seg).to(scores.device)
                check(lib.hr_rerank_topk(scores.data_ptr(), seg_dev.data_ptr(), n_q, max_c, k, *out), "hr_rerank_topk")
                return (idx, sc) if with_scores else idx
    check(lib.hr_rerank_topk_host(scores.data_ptr(), _i32p(seg), n_q, max_c, k, *out), "hr_rerank_topk")
    return (idx, sc) if with_scores else idx


def probe_read_bandwidth(src, sink, to_lds: bool = False, stream=None) -> None:
    """One read-only pass of the library's streaming yardstick kernel over the device tensor `src`."""
    check(lib.hr_probe_read_bandwidth(src.data_ptr(), src.numel() * src.element_size(), sink.data_ptr(),
                                      sink.numel() * sink.element_size(), 1 if to_lds else 0, _stream_ptr(stream)),
          "hr_probe_read_bandwidth")


class KVPool:
    """Device buffer + library handle of one paged document-KV pool."""

    def __init__(self, n_layers: int, n_kv_heads: int, head_dim: int, num_pages: int, kv_dtype: str, device="cuda:0"):
        import torch
        self.cfg = make_pool_cfg(n_layers, n_kv_heads, head_dim, num_pages, kv_dtype)
        self.kv_dtype = kv_dtype
        nbytes = hr_kv_pool_bytes(self.cfg)
        if nbytes == 0:
            raise HrError(HR_ERR_INVALID_ARG, "hr_kv_pool_bytes")
        self.mem = torch.zeros(nbytes, dtype=torch.uint8, device=device)
        self._dims = (n_layers, n_kv_heads, head_dim)
        self.kv_fp8 = self.cfg.kv_dtype == HR_FP8_E4M3
        self._read_dtype = {HR_F32: torch.float32, HR_BF16: torch.float16, HR_FP8_E4M3: torch.uint8}[self.cfg.kv_dtype]
        st, self.handle = hr_kv_pool_create(self.cfg, self.mem.data_ptr(), nbytes)
        check(st, "hr_kv_pool_create")

    def write(self, doc_len: int, page_ids, k, v, k_scale=None, v_scale=None, stream=None) -> None:
        """k, v: device tensors [L][doc_len][n_kv][d] in the pool dtype (uint8 codes for fp8)."""
        ids = _i32(page_ids)
        assert k.is_contiguous() and v.is_contiguous() and k.is_cuda and v.is_cuda
        ks = k_scale.data_ptr() if k_scale is not None else None
        vs = v_scale.data_ptr() if v_scale is not None else None
        st = lib.hr_doc_kv_write(self.handle, int(doc_len), _i32p(ids), k.data_ptr(), v.data_ptr(),
                                 ks, vs, _stream_ptr(stream))
        check(st, "hr_doc_kv_write")

    def read(self, doc_len: int, page_ids, stream=None):
        """The document's K/V back from its pages: device tensors [L][doc_len][n_kv][d] in the pool's element type
        (float32, float16 for 16-bit pools, uint8 codes for fp8), plus K / V scales [L][n_pages][n_kv] for fp8."""
        import torch
        ids = _i32(page_ids)
        L, n_kv, d = self._dims
        k = self.mem.new_empty((L, int(doc_len), n_kv, d), dtype=self._read_dtype)
        v = torch.empty_like(k)
        if self.kv_fp8:
            ks = self.mem.new_empty((L, len(ids), n_kv), dtype=torch.float32)
            vs = torch.empty_like(ks)
            check(lib.hr_doc_kv_read(self.handle, int(doc_len), _i32p(ids), k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(),
                                     _stream_ptr(stream)), "hr_doc_kv_read")
            return k, v, ks, vs
        check(lib.hr_doc_kv_read(self.handle, int(doc_len), _i32p(ids), k.data_ptr(), v.data_ptr(), None, None, _stream_ptr(stream)),
              "hr_doc_kv_read")
        return k, v

    def free(self, page_ids) -> None:
        ids = _i32(page_ids)
        check(lib.hr_doc_kv_free(self.handle, _i32p(ids), len(ids)), "hr_doc_kv_free")

    def range_report(self) -> dict:
        r = hr_range_report()
        check(lib.hr_kv_pool_range_report(self.handle, C.byref(r)), "hr_kv_pool_range_report")
        return r.as_dict()

    @property
    def page_record_bytes(self) -> int:
        return int(lib.hr_kv_page_record_bytes(self.handle))

    @property
    def page_record4_bytes(self) -> int:
        return int(lib.hr_kv_page_record4_bytes(self.handle))

    def pages_out4(self, page_ids, records, stream=None) -> None:
        """4-bit records (16-bit pools): quantised as the pages leave."""
        ids = _i32(page_ids)
        assert records.numel() * records.element_size() >= len(ids) * self.page_record4_bytes
        check(lib.hr_kv_pages_out4(self.handle, len(ids), _i32p(ids), records.data_ptr(), _stream_ptr(stream)),
              "hr_kv_pages_out4")

    def pages_in4(self, page_ids, records, stream=None) -> None:
        ids = _i32(page_ids)
        assert records.numel() * records.element_size() >= len(ids) * self.page_record4_bytes
        check(lib.hr_kv_pages_in4(self.handle, len(ids), _i32p(ids), records.data_ptr(), _stream_ptr(stream)),
              "hr_kv_pages_in4")

    def pages_out(self, page_ids, records, stream=None) -> None:
        """records: uint8 tensor of len(page_ids) * page_record_bytes, on the device or in pinned host memory."""
        ids = _i32(page_ids)
        assert records.numel() * records.element_size() >= len(ids) * self.page_record_bytes
        check(lib.hr_kv_pages_out(self.handle, len(ids), _i32p(ids), records.data_ptr(), _stream_ptr(stream)),
              "hr_kv_pages_out")

    def pages_in(self, page_ids, records, stream=None) -> None:
        ids = _i32(page_ids)
        assert records.numel() * records.element_size() >= len(ids) * self.page_record_bytes
        check(lib.hr_kv_pages_in(self.handle, len(ids), _i32p(ids), records.data_ptr(), _stream_ptr(stream)),
              "hr_kv_pages_in")

    def alloc(self, n: int) -> np.ndarray:
        out = np.zeros(n, np.int32)
        check(lib.hr_kv_pool_alloc_pages(self.handle, n, _i32p(out)), "hr_kv_pool_alloc_pages")
        return out

    @property
    def free_pages(self) -> int:
        return int(lib.hr_kv_pool_free_pages(self.handle))

    def close(self):
        if getattr(self, "handle", None):
            lib.hr_kv_pool_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ----------------------------------------------------------------------------------------------
# operators for models whose layers the caller runs
# ----------------------------------------------------------------------------------------------
ROPE_LAYOUT = {"half": 0, "interleaved": 1}
ROPE_SCALING = {"none": 0, "linear": 1, "base": 2, "bands": 3, "ramp": 4}
TABLES_BAD_DOC, TABLES_BAD_LENGTH, TABLES_CUT, TABLES_BAD_PAGE = 1, 2, 4, 8
_ACT_CODE: Dict = {}      # torch.dtype -> hr_dtype of activations


def _act_code(dtype) -> Optional[int]:
    if not _ACT_CODE:
        import torch
        _ACT_CODE.update({torch.float32: HR_F32, torch.bfloat16: HR_BF16})
    return _ACT_CODE.get(dtype)


def _refuse(what: str):
    raise HrError(HR_ERR_INVALID_ARG, what)


def _strides(t, rows: int, heads: Optional[int], d: int, like, what: str):
    """(heads, token stride, head stride) of a tensor [rows or more][heads][d] of the type and on the device of `like`, channels adjacent."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or shape[2] != d or shape[0] < rows or (heads is not None and shape[1] != heads) or (d > 1 and shape[0] and stride[2] != 1) \
            or t.dtype != like.dtype or t.device != like.device:
        _refuse(f"{what}: [{rows}][{heads if heads is not None else 'heads'}][{d}] with adjacent channels, {like.dtype} on {like.device} expected; "
                f"got {tuple(shape)}, strides {tuple(stride)}, {t.dtype} on {t.device}")
    return shape[1], stride[0], stride[1]


def _used_on(stream, *tensors) -> None:
    """Tells the allocator that `stream`, if it is not the current one, works with these tensors: their memory is not given out again before it is done,
    though the caller lets go of them."""
    if stream is not None and stream.cuda_stream != _stream_ptr():
        for t in tensors:
            if t is not None and t.numel():
                t.record_stream(stream)


def _no_gradients(tensors, what: str) -> None:
    """These calls have no backward pass: results of tensors that ask for one would look like constants to autograd."""
    for t in tensors:
        if t is not None and t.requires_grad:
            import torch
            if torch.is_grad_enabled():
                _refuse(f"{what}: no gradients are computed; call it under torch.no_grad(), or with detached tensors")


def _ints(t, n: int, device, what: str):
    import torch
    if t.dtype != torch.int32 or t.device != device or t.numel() < n or not t.is_contiguous():
        _refuse(f"{what}: {n} contiguous int32 on {device} expected, got {tuple(t.shape)} {t.dtype} on {t.device}")
    return t.data_ptr()


def _int32(x, what: str) -> int:
    """A number that the C side takes as int32 (ctypes would wrap it around)."""
    x = operator.index(x)
    if not 0 <= x < 1 << 31:
        _refuse(f"{what}: 0 .. 2^31 - 1 expected, got {x}")
    return x


def _elsewhere(device) -> bool:
    """Whether another device than `device` is the current one."""
    import torch
    if device.type != "cuda":
        _refuse(f"device tensors expected, got {device}")
    return torch._C._cuda_getDevice() != device.index


def _new(like, stream, shape=None, dtype=None):
    """A contiguous tensor like `like`, of the shape and type given, that belongs to the stream that will write it (None: the current one)."""
    import torch
    if stream is None:
        if shape is None:
            return torch.empty_like(like, memory_format=torch.contiguous_format)
        return torch.empty(shape, dtype=dtype, device=like.device)
    with torch.cuda.stream(stream):
        return _new(like, None, shape, dtype)


class Rope:
    """Rotary positions (hr_rope_apply).  rotary_dim: leading channels that are turned (None: all); scaling, factor, original_len,
    low, high: see hr_rope_cfg; amplitude None: 1, and for "ramp" 0.1 ln(factor) + 1.  freqs: rotary_dim / 2 frequencies of the
    caller's own, in radians per position, instead of those."""

    def __init__(self, head_dim: int, base: float = 10000.0, rotary_dim: Optional[int] = None, layout: str = "half", scaling: str = "none",
                 factor: float = 1.0, original_len: float = 0.0, low: float = 1.0, high: float = 4.0, amplitude: Optional[float] = None, freqs=None):
        if layout not in ROPE_LAYOUT or scaling not in ROPE_SCALING:
            _refuse(f"Rope: layout one of {sorted(ROPE_LAYOUT)}, scaling one of {sorted(ROPE_SCALING)}")
        if amplitude is None:
            amplitude = 0.1 * float(np.log(factor)) + 1.0 if scaling == "ramp" and factor >= 1.0 else 1.0
        r = _int32(head_dim if rotary_dim is None else rotary_dim, "Rope: rotary_dim")
        head_dim = _int32(head_dim, "Rope: head_dim")
        self.cfg = hr_rope_cfg(head_dim, r, ROPE_LAYOUT[layout], ROPE_SCALING[scaling], amplitude, base, factor, original_len, low, high)
        if freqs is None:
            self.freqs = np.zeros(max(r // 2, 1), np.float64)
            check(lib.hr_rope_frequencies(C.byref(self.cfg), self.freqs.ctypes.data), "hr_rope_frequencies")
        else:
            self.freqs = np.ascontiguousarray(freqs, np.float64)
            if self.freqs.shape != (r // 2,):
                _refuse(f"Rope: {r // 2} frequencies expected, got {self.freqs.shape}")
        self._freqs = self.freqs.ctypes.data

    def apply(self, positions, *tensors, out=None, period: int = 0, inverse: bool = False, stream=None):
        """Turns one or two tensors [tokens][heads][head_dim] (bf16 or fp32; views with any token and head stride).  positions: int32
        tensor [tokens] (tokens with a negative one are left out), or an int: token t is at positions + t % period (period 0: + t).
        out: as many tensors, which may be `tensors` themselves (None: new ones).  Returns the list of outputs.  No gradients: tensors that
        require them are refused outside torch.no_grad()."""
        d = self.cfg.head_dim
        if not 1 <= len(tensors) <= 2:
            _refuse("Rope.apply: one or two tensors")
        x0 = tensors[0]
        code, dev = _act_code(x0.dtype), x0.device
        if code is None or x0.dim() != 3:
            _refuse(f"Rope.apply: [tokens][heads][{d}] in float32 or bfloat16, got {tuple(x0.shape)} {x0.dtype}")
        if _elsewhere(dev):
            import torch
            with torch.cuda.device(dev):
                return self.apply(positions, *tensors, out=out, period=period, inverse=inverse, stream=stream)
        _no_gradients(tensors if out is None else (*tensors, *out), "Rope.apply")
        T = x0.shape[0]
        ptr = given = None
        if hasattr(positions, "data_ptr"):
            ptr, given, positions = _ints(positions, T, dev, "Rope.apply: positions"), positions, 0
        else:
            positions, period = _int32(positions, "Rope.apply: positions"), _int32(period, "Rope.apply: period")
        sides = (hr_rope_tensor * len(tensors))()
        if out is not None and len(out) != len(tensors):
            _refuse("Rope.apply: as many outputs as tensors")
        outs = []
        for i, x in enumerate(tensors):
            heads, xt, xh = _strides(x, T, None, d, x0, "Rope.apply: input")
            if out is None:
                y, yt, yh = _new(x, stream), heads * d, d
            else:
                y = out[i]
                _, yt, yh = _strides(y, T, heads, d, x0, "Rope.apply: output")
            if x.shape[0] != T or y.shape[0] != T:
                _refuse("Rope.apply: as many tokens everywhere")
            outs.append(y)
            sides[i].__init__(x.data_ptr(), y.data_ptr(), heads, xt, xh, yt, yh)
        if T > 0:
            check(lib.hr_rope_apply(C.byref(self.cfg), self._freqs, code, T, ptr, positions, period, sides, len(sides),
                                    1 if inverse else 0, _stream_ptr(stream)), "hr_rope_apply")
            _used_on(stream, given, *tensors, *outs)
        return outs


class DocList:
    """The documents a batch may ask for: int32 device tensors doc_lens [n], page_cu [n + 1] and the page ids it points into."""

    def __init__(self, doc_lens, page_cu, pages):
        dev = doc_lens.device
        n = doc_lens.numel()
        self.tensors = (doc_lens, page_cu, pages)
        self.device = dev
        self.c = hr_doc_list(n, pages.numel(), _ints(doc_lens, n, dev, "DocList: doc_lens"), _ints(page_cu, n + 1, dev, "DocList: page_cu"),
                             _ints(pages, 0, dev, "DocList: pages"))


class PairTables:
    """Device tables of a batch of n_pairs pairs with room for max_tokens query tokens and pt_stride pages a document (hr_pair_tables).
    build() fills q_cu, doc_lens, page_table, tok_pos, tok_pair, order and report, and comes before an attention; n_q_heads is that of the
    attention that will read them."""

    def __init__(self, pool: KVPool, n_pairs: int, max_tokens: int, pt_stride: int, n_q_heads: int):
        import torch
        self.pool, self.n_pairs, self.max_tokens, self.n_q_heads = pool, n_pairs, max_tokens, n_q_heads
        self.device = pool.mem.device
        for what, x in (("n_pairs", n_pairs), ("max_tokens", max_tokens), ("pt_stride", pt_stride), ("n_q_heads", n_q_heads)):
            _int32(x, f"PairTables: {what}")
        nbytes = int(lib.hr_pair_tables_sched_bytes(pool.handle, n_pairs, max_tokens, n_q_heads))
        if nbytes == 0:
            raise HrError(HR_ERR_INVALID_ARG, "hr_pair_tables_sched_bytes")
        new = lambda *shape: torch.empty(shape, dtype=torch.int32, device=self.device)      # noqa: E731
        self.q_cu, self.doc_lens, self.page_table = new(n_pairs + 1), new(n_pairs), new(n_pairs, pt_stride)
        self.tok_pos, self.tok_pair, self.order, self.report = new(max_tokens), new(max_tokens), new(n_pairs), new(4)
        self.sched = new(nbytes // 4)
        self.built = False
        self.tensors = (self.q_cu, self.doc_lens, self.page_table, self.tok_pos, self.tok_pair, self.order, self.report, self.sched)
        self.c = hr_pair_tables(n_pairs, max_tokens, pt_stride, n_q_heads, *[t.data_ptr() for t in self.tensors], nbytes)
        self.workspace_bytes = int(lib.hr_pair_attention_workspace_bytes(pool.handle, C.byref(self.c)))

    def build(self, docs: DocList, pair_doc, query_lens, stream=None) -> "PairTables":
        """pair_doc, query_lens: int32 device tensors [n_pairs]; a pair without a document has -1."""
        n, dev = self.n_pairs, self.device
        if docs.device != dev:
            _refuse(f"PairTables.build: documents on {dev} expected, got {docs.device}")
        if _elsewhere(dev):
            import torch
            with torch.cuda.device(dev):
                return self.build(docs, pair_doc, query_lens, stream)
        check(lib.hr_pair_tables_build(self.pool.handle, C.byref(docs.c), _ints(pair_doc, n, dev, "PairTables.build: pair_doc"),
                                       _ints(query_lens, n, dev, "PairTables.build: query_lens"), C.byref(self.c), _stream_ptr(stream)),
              "hr_pair_tables_build")
        self.built = True
        _used_on(stream, pair_doc, query_lens, *docs.tensors, *self.tensors)
        return self


def pair_attention(pool: KVPool, layer: int, tables: PairTables, q, k=None, v=None, out=None, scale: Optional[float] = None, cap: float = 0.0,
                   slopes=None, window: int = 0, prefix_lens=None, with_lse: bool = False, stream=None):
    """Attention of the pairs' query tokens over their documents' pages and, with k and v, their own keys (hr_pair_attention).
    q [max_tokens][n_q_heads][d], k and v [max_tokens][n_kv_heads][d]: bf16 (16-bit and fp8 pools) or fp32 (fp32 pools), views with any
    token and head stride; slopes: fp32 [n_q_heads]; prefix_lens: int32 [n_pairs].  Returns out (rows behind the last token are left as they
    are, in a new tensor unset), with_lse: and the rows' log-sums [max_tokens][n_q_heads].  No gradients: tensors that require them are refused
    outside torch.no_grad()."""
    import torch
    dev, n_q, T = tables.device, tables.n_q_heads, tables.max_tokens
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return pair_attention(pool, layer, tables, q, k, v, out, scale, cap, slopes, window, prefix_lens, with_lse, stream)
    _, n_kv, d = pool._dims
    code = _act_code(q.dtype)
    if pool is not tables.pool or q.device != dev:
        _refuse(f"pair_attention: the tables' own pool and tensors on {dev} expected, got {q.device}")
    _no_gradients((q, k, v, out, slopes), "pair_attention")
    if not tables.built:
        _refuse("pair_attention: tables that build() has not filled")
    if scale == 0.0:
        _refuse("pair_attention: scale: None (1 / sqrt(head_dim)) or a number that is not 0")
    layer, window = _int32(layer, "pair_attention: layer"), _int32(window, "pair_attention: window")
    if code is None or (k is None) != (v is None):
        _refuse("pair_attention: float32 or bfloat16, and both of k and v or neither")
    _, q_t, q_h = _strides(q, T, n_q, d, q, "pair_attention: q")
    k_p = v_p = None
    k_t = k_h = v_t = v_h = 0
    if k is not None:
        _, k_t, k_h = _strides(k, T, n_kv, d, q, "pair_attention: k")
        _, v_t, v_h = _strides(v, T, n_kv, d, q, "pair_attention: v")
        k_p, v_p = k.data_ptr(), v.data_ptr()
    if slopes is not None and (slopes.dtype != torch.float32 or slopes.device != dev or slopes.numel() != n_q or not slopes.is_contiguous()):
        _refuse(f"pair_attention: slopes: {n_q} contiguous float32 on {dev} expected")
    prefix = None if prefix_lens is None else _ints(prefix_lens, tables.n_pairs, dev, "pair_attention: prefix_lens")
    if out is None:
        out = _new(q, stream)
    _, o_t, o_h = _strides(out, T, n_q, d, q, "pair_attention: out")
    lse = _new(q, stream, (T, n_q), torch.float32) if with_lse else None
    ws = _new(q, stream, (tables.workspace_bytes,), torch.uint8) if tables.workspace_bytes else None
    args = hr_attention_args(code, layer, 0.0 if scale is None else scale, cap, window, q.data_ptr(), k_p, v_p, out.data_ptr(),
                             None if lse is None else lse.data_ptr(), None if slopes is None else slopes.data_ptr(), prefix,
                             q_t, q_h, k_t, k_h, v_t, v_h, o_t, o_h)
    if T > 0:
        check(lib.hr_pair_attention(pool.handle, C.byref(tables.c), C.byref(args), None if ws is None else ws.data_ptr(),
                                    tables.workspace_bytes, _stream_ptr(stream)), "hr_pair_attention")
        _used_on(stream, q, k, v, out, slopes, prefix_lens, pool.mem, *tables.tensors)
    return (out, lse) if with_lse else out


_LAYER_KINDS = ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "norm1", "norm2")


class Plan:
    """A fixed-shape scoring plan (hr_rerank_plan_*): owns its workspace tensor; run() is stream work only."""

    def __init__(self, model: "Model", pool: KVPool, doc_lens, query_lens, pt_stride: int):
        import torch
        self.model, self.pool = model, pool
        dl, ql = _i32(doc_lens), _i32(query_lens)
        self.n_pairs, self.pt_stride = len(dl), int(pt_stride)
        nbytes = int(lib.hr_rerank_workspace_bytes(model.handle, self.n_pairs, int(ql.sum()), self.pt_stride))
        self.ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=model.device)
        out = C.c_void_p()
        check(lib.hr_rerank_plan_create(model.handle, pool.handle, self.n_pairs, _i32p(dl), _i32p(ql), self.pt_stride,
                                        self.ws.data_ptr(), self.ws.numel(), C.byref(out)), "hr_rerank_plan_create")
        self.handle = out

    def set_inputs(self, page_table, query_tokens) -> None:
        pt, qt = _i32(page_table), _i32(query_tokens)
        check(lib.hr_rerank_plan_set_inputs(self.handle, _i32p(pt), _i32p(qt)), "hr_rerank_plan_set_inputs")

    def run(self, out, stream=None):
        check(lib.hr_rerank_plan_run(self.handle, out.data_ptr(), _stream_ptr(stream)), "hr_rerank_plan_run")
        return out[:self.n_pairs]

    def close(self):
        if getattr(self, "handle", None):
            lib.hr_rerank_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Model:
    """Uploads weights (numpy fp32 arrays holding values of the model dtype), packs them, keeps the handle."""

    def __init__(self, model_cfg, weights, device="cuda:0"):
        import torch
        self.m = model_cfg
        self.device = device
        self.cfg = make_model_cfg(model_cfg)
        tdt = torch.float32 if model_cfg.dtype == "f32" else torch.bfloat16

        def up(a, dt):
            return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(device=device, dtype=dt)

        self.embedding = up(weights.get("embedding", -1), tdt)
        self.final_norm = up(weights.get("final_norm", -1), torch.float32)
        L = model_cfg.n_layers
        per_layer: Dict[str, List] = {k: [] for k in _LAYER_KINDS}
        for l in range(L):
            for k in _LAYER_KINDS:
                per_layer[k].append(up(weights.get(k, l), torch.float32 if k.startswith("norm") else tdt))
        self.norm1, self.norm2 = per_layer["norm1"], per_layer["norm2"]
        arrays = {k: (C.c_void_p * L)(*[t.data_ptr() for t in per_layer[k]]) for k in _LAYER_KINDS}
        ptrs = hr_weight_ptrs(self.embedding.data_ptr(), self.final_norm.data_ptr(),
                              *[C.cast(arrays[k], _PP) for k in _LAYER_KINDS])
        nbytes = hr_weights_pack_bytes(self.cfg)
        if nbytes == 0:
            raise HrError(HR_ERR_INVALID_ARG, "hr_weights_pack_bytes")
        self.pack = torch.empty(nbytes, dtype=torch.uint8, device=device)
        out = C.c_void_p()
        st = lib.hr_weights_load(C.byref(self.cfg), C.byref(ptrs), self.pack.data_ptr(), nbytes,
                                 _stream_ptr(), C.byref(out))
        check(st, "hr_weights_load")
        self.handle = out
        torch.cuda.synchronize()
        del per_layer, arrays          # the matrices now live in the packed copy
        self._ws = None

    def _workspace(self, nbytes: int):
        import torch
        if self._ws is None or self._ws.numel() < nbytes:
            self._ws = None
            self._ws = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        return self._ws

    def range_report(self) -> dict:
        r = hr_range_report()
        check(lib.hr_model_range_report(self.handle, C.byref(r)), "hr_model_range_report")
        return r.as_dict()

    def gemm_path(self) -> str:
        return lib.hr_gemm_path(self.handle).decode()

    def attention_path(self, pool: KVPool) -> str:
        return lib.hr_attention_path(self.handle, pool.handle).decode()

    def profile_enable(self, on: bool) -> None:
        check(lib.hr_profile_enable(self.handle, 1 if on else 0), "hr_profile_enable")

    def profile_select(self, names=None) -> None:
        """Time only the named kernel classes (None: all)."""
        n = lib.hr_profile_count()
        all_names = [lib.hr_profile_name(i).decode() for i in range(n)]
        mask = 0xFFFFFFFF if names is None else sum(1 << all_names.index(x) for x in names)
        check(lib.hr_profile_select(self.handle, mask), "hr_profile_select")

    def profile_read(self) -> Dict[str, Dict[str, float]]:
        n = lib.hr_profile_count()
        ms = (C.c_double * n)()
        cnt = (C.c_int64 * n)()
        check(lib.hr_profile_read(self.handle, ms, cnt), "hr_profile_read")
        return {lib.hr_profile_name(i).decode(): {"ms": float(ms[i]), "launches": int(cnt[i])} for i in range(n)}

    def score(self, pool: KVPool, page_table, doc_lens, query_tokens, query_lens, out=None, stream=None):
        import torch
        pt = _i32(page_table)
        if pt.ndim == 1:
            pt = pt.reshape(len(doc_lens), -1)
        dl, qt, ql = _i32(doc_lens), _i32(query_tokens), _i32(query_lens)
        P = len(dl)
        stride = pt.shape[1] if pt.ndim == 2 else 0
        nbytes = int(lib.hr_rerank_workspace_bytes(self.handle, P, int(ql.sum()), stride))
        ws = self._workspace(max(nbytes, 256))
        scores = out if out is not None else torch.empty(max(P, 1), dtype=torch.float32, device=self.device)
        st = lib.hr_rerank_score(self.handle, pool.handle, P, _i32p(pt), stride, _i32p(dl), _i32p(qt), _i32p(ql),
                                 ws.data_ptr(), ws.numel(), scores.data_ptr(), _stream_ptr(stream))
        check(st, "hr_rerank_score")
        return scores[:P]

    def score_static(self, pool: KVPool, page_table, doc_lens, query_tokens, query_lens, out, stream=None):
        """hr_rerank_score_static: the workspace is the library's own static device array; `out` is the caller's
        fp32 device tensor of at least len(doc_lens) scores (nothing is allocated here either)."""
        pt = _i32(page_table)
        if pt.ndim == 1:
            pt = pt.reshape(len(doc_lens), -1)
        dl, qt, ql = _i32(doc_lens), _i32(query_tokens), _i32(query_lens)
        P = len(dl)
        stride = pt.shape[1] if pt.ndim == 2 else 0
        st = lib.hr_rerank_score_static(self.handle, pool.handle, P, _i32p(pt), stride, _i32p(dl), _i32p(qt), _i32p(ql),
                                        out.data_ptr(), _stream_ptr(stream))
        check(st, "hr_rerank_score_static")
        return out[:P]

    def parts(self, total_q_tokens: int) -> int:
        return int(lib.hr_rerank_parts(self.handle, int(total_q_tokens)))

    def set_precise_layers(self, n: int) -> None:
        check(lib.hr_model_set_precise_layers(self.handle, int(n)), "hr_model_set_precise_layers")

    def precise_layers(self) -> int:
        return int(lib.hr_model_precise_layers(self.handle))

    def set_streams(self, n: int) -> None:
        check(lib.hr_rerank_set_streams(self.handle, int(n)), "hr_rerank_set_streams")

    def score_full(self, doc_tokens: Sequence[np.ndarray], query_tokens: Sequence[np.ndarray], out=None, stream=None):
        import torch
        P = len(doc_tokens)
        dl = _i32([len(d) for d in doc_tokens])
        ql = _i32([len(q) for q in query_tokens])
        dt = _i32(np.concatenate(doc_tokens)) if P and dl.sum() else np.zeros(1, np.int32)
        qt = _i32(np.concatenate(query_tokens)) if P else np.zeros(1, np.int32)
        total = int(dl.sum() + ql.sum())
        nbytes = int(lib.hr_rerank_full_workspace_bytes(self.handle, P, total))
        ws = self._workspace(max(nbytes, 256))
        scores = out if out is not None else torch.empty(max(P, 1), dtype=torch.float32, device=self.device)
        st = lib.hr_rerank_score_full(self.handle, P, _i32p(dt), _i32p(dl), _i32p(qt), _i32p(ql),
                                      ws.data_ptr(), ws.numel(), scores.data_ptr(), _stream_ptr(stream))
        check(st, "hr_rerank_score_full")
        return scores[:P]

    def doc_prefill(self, pool: KVPool, doc_tokens: Sequence[np.ndarray], page_lists: Sequence[np.ndarray], stream=None) -> None:
        """Compute and store the documents' K/V on the device (stage one)."""
        n = len(doc_tokens)
        dl = _i32([len(d) for d in doc_tokens])
        stride = max(len(p) for p in page_lists)
        pt = np.full((n, stride), -1, np.int32)
        for i, pg in enumerate(page_lists):
            pt[i, :len(pg)] = pg
        toks = _i32(np.concatenate(doc_tokens))
        nbytes = int(lib.hr_doc_prefill_workspace_bytes(self.handle, n, int(dl.sum())))
        if nbytes == 0:
            raise HrError(HR_ERR_UNSUPPORTED_SHAPE, "hr_doc_prefill_workspace_bytes")
        ws = self._workspace(nbytes)
        st = lib.hr_doc_prefill(self.handle, pool.handle, n, _i32p(toks), _i32p(dl), _i32p(pt), stride,
                                ws.data_ptr(), ws.numel(), _stream_ptr(stream))
        check(st, "hr_doc_prefill")

    def close(self):
        if getattr(self, "handle", None):
            lib.hr_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
