"""Thin ctypes binding of ``libdresd.so`` (see ``include/dresd.h``).

Argument marshalling only: every step of the retrieval path runs in the CUDA
kernels behind the C ABI.  There is no CPU fallback -- if the library is
missing or a call fails, a :class:`DresdError` is raised.

Functions carry the C names (``dresd_store_create`` ...); :class:`Store` wraps
them for torch tensors (used for device memory and streams only).
"""
from __future__ import annotations

import contextlib
import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdresd.so")
LIB_DEBUG_PATH = os.path.join(_HERE, "libdresd_debug.so")    # loaded instead when DRESD_DEBUG=1 (bounds-checked build)

DRESD_F32, DRESD_F16, DRESD_BF16 = 0, 1, 2
DTYPE_CODE = {"f32": DRESD_F32, "f16": DRESD_F16, "bf16": DRESD_BF16}
DRESD_OK = 0
STATUS_NAME = {0: "DRESD_OK", -1: "DRESD_ERR_INVALID", -2: "DRESD_ERR_UNSUPPORTED",
               -3: "DRESD_ERR_ALLOC", -4: "DRESD_ERR_CUDA", -5: "DRESD_ERR_TIMEOUT",
               -6: "DRESD_ERR_INTERNAL"}
MAX_BATCH, MAX_TOP_N, MAX_DIM = 64, 32, 4096

EXPORTS = (
    "dresd_store_create", "dresd_store_set_preprocess", "dresd_retrieve", "dresd_retrieve_host",
    "dresd_preprocess", "dresd_store_status", "dresd_store_set_option",
    "dresd_store_profile_read", "dresd_store_last_launches", "dresd_store_last_key_passes",
    "dresd_last_error",
    "dresd_store_destroy", "dresd_retrieve_noalloc", "dresd_store_enable_first_token_filter",
    "dresd_retrieve_filtered", "dresd_drafts_prepare", "dresd_drafts_accept",
    "dresd_merge_shards", "dresd_build_keys", "dresd_fit_zscore", "dresd_set_global_option", "dresd_quantise_keys", "dresd_store_attach_quantised",
    "dresd_retrieve_quantised", "dresd_store_index_first_tokens", "dresd_merge_shards_packed",
    "dresd_noalloc_status", "dresd_debug_build", "dresd_store_debug_selftest",
    "dresd_kv_create", "dresd_kv_destroy", "dresd_kv_append", "dresd_kv_read", "dresd_kv_attend",
    "dresd_kv_keep_draft", "dresd_kv_status", "dresd_kv_set_option", "dresd_kv_last_launches", "dresd_kv_debug_selftest",
)


class dresd_kv_batch(ctypes.Structure):
    """The C struct: device addresses of a batch of chunks, and its sizes."""
    _fields_ = [("page_table", ctypes.c_void_p), ("ctx", ctypes.c_void_p), ("start", ctypes.c_void_p),
                ("B", ctypes.c_int32), ("table_width", ctypes.c_int32), ("rows", ctypes.c_int32),
                ("max_chunk", ctypes.c_int32)]


class DresdError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAME.get(status, status)}: {message}")
        self.status = status
        self.message = message


_lib = None


def load(path: str | None = None) -> ctypes.CDLL:
    """Load the CUDA library; raises if it has not been built."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or (LIB_DEBUG_PATH if os.environ.get("DRESD_DEBUG") == "1" else LIB_PATH)
    if not os.path.exists(p):
        raise DresdError(-4, f"{p} not found: build it with `python -m paper_2502_15572_b200.build` "
                             "(there is no CPU fallback)")
    lib = ctypes.CDLL(p)
    c = ctypes
    vp, i32, i64, f32 = c.c_void_p, c.c_int, c.c_int64, c.c_float
    lib.dresd_store_create.restype = i32
    lib.dresd_store_create.argtypes = [vp, vp, i64, i32, i32, i32, c.POINTER(vp)]
    lib.dresd_store_set_preprocess.restype = i32
    lib.dresd_store_set_preprocess.argtypes = [vp, i32, vp, vp, f32, vp, vp]
    lib.dresd_retrieve.restype = i32
    lib.dresd_retrieve.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp, vp]
    lib.dresd_retrieve_host.restype = i32
    lib.dresd_retrieve_host.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp, vp]
    lib.dresd_preprocess.restype = i32
    lib.dresd_preprocess.argtypes = [vp, vp, i32, vp, vp]
    lib.dresd_store_status.restype = i32
    lib.dresd_store_status.argtypes = [vp]
    lib.dresd_store_set_option.restype = i32
    lib.dresd_store_set_option.argtypes = [vp, c.c_char_p, i32]
    lib.dresd_store_profile_read.restype = i32
    lib.dresd_store_profile_read.argtypes = [vp, c.POINTER(c.c_double), c.POINTER(c.c_int)]
    lib.dresd_store_last_launches.restype = i32
    lib.dresd_store_last_launches.argtypes = [vp]
    lib.dresd_store_last_key_passes.restype = c.c_double
    lib.dresd_store_last_key_passes.argtypes = [vp]
    lib.dresd_last_error.restype = c.c_char_p
    lib.dresd_last_error.argtypes = []
    lib.dresd_store_destroy.restype = None
    lib.dresd_store_destroy.argtypes = [vp]
    lib.dresd_store_enable_first_token_filter.restype = i32
    lib.dresd_store_enable_first_token_filter.argtypes = [vp, vp]
    lib.dresd_store_index_first_tokens.restype = i32
    lib.dresd_store_index_first_tokens.argtypes = [vp, vp]
    lib.dresd_retrieve_filtered.restype = i32
    lib.dresd_retrieve_filtered.argtypes = [vp, vp, vp, i32, i32, i32, vp, vp, vp, vp]
    lib.dresd_drafts_prepare.restype = i32
    lib.dresd_drafts_prepare.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, vp]
    lib.dresd_drafts_accept.restype = i32
    lib.dresd_drafts_accept.argtypes = [vp, vp, vp, i32, i32, i32, vp, vp, vp, vp]
    lib.dresd_merge_shards.restype = i32
    lib.dresd_merge_shards.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp]
    lib.dresd_merge_shards_packed.restype = i32
    lib.dresd_merge_shards_packed.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, vp, vp]
    lib.dresd_build_keys.restype = i32
    lib.dresd_build_keys.argtypes = [vp, i64, i32, i32, vp, vp, f32, vp, i32, vp, vp, vp]
    lib.dresd_quantise_keys.restype = i32
    lib.dresd_quantise_keys.argtypes = [vp, i64, i32, i32, vp, vp]
    lib.dresd_store_attach_quantised.restype = i32
    lib.dresd_store_attach_quantised.argtypes = [vp, vp]
    lib.dresd_retrieve_quantised.restype = i32
    lib.dresd_retrieve_quantised.argtypes = [vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp]
    lib.dresd_set_global_option.restype = i32
    lib.dresd_set_global_option.argtypes = [ctypes.c_char_p, i32]
    lib.dresd_fit_zscore.restype = i32
    lib.dresd_fit_zscore.argtypes = [vp, i64, i32, i32, vp, vp, vp]
    lib.dresd_retrieve_noalloc.restype = i32
    lib.dresd_retrieve_noalloc.argtypes = [vp, vp, i64, i32, i32, i32, vp, i32, i32, i32, vp, vp, vp, vp]
    lib.dresd_noalloc_status.restype = i32
    lib.dresd_noalloc_status.argtypes = [vp]
    lib.dresd_debug_build.restype = i32
    lib.dresd_debug_build.argtypes = []
    lib.dresd_store_debug_selftest.restype = i32
    lib.dresd_store_debug_selftest.argtypes = [vp, vp]
    batch = c.POINTER(dresd_kv_batch)
    lib.dresd_kv_create.restype = i32
    lib.dresd_kv_create.argtypes = [vp, vp, vp, vp, i32, i64, i32, i32, i32, i32, c.POINTER(vp)]
    lib.dresd_kv_destroy.restype = None
    lib.dresd_kv_destroy.argtypes = [vp]
    lib.dresd_kv_append.restype = i32
    lib.dresd_kv_append.argtypes = [vp, i32, batch, vp, i64, i64, vp, i64, i64, vp]
    lib.dresd_kv_read.restype = i32
    lib.dresd_kv_read.argtypes = [vp, i32, batch, vp, vp, vp]
    lib.dresd_kv_attend.restype = i32
    lib.dresd_kv_attend.argtypes = [vp, i32, batch, vp, i64, i64, i32, f32, vp, i32, vp, vp, vp]
    lib.dresd_kv_keep_draft.restype = i32
    lib.dresd_kv_keep_draft.argtypes = [vp, batch, vp, vp, i32, i32, vp]
    lib.dresd_kv_status.restype = i32
    lib.dresd_kv_status.argtypes = [vp]
    lib.dresd_kv_set_option.restype = i32
    lib.dresd_kv_set_option.argtypes = [vp, c.c_char_p, i32]
    lib.dresd_kv_debug_selftest.restype = i32
    lib.dresd_kv_debug_selftest.argtypes = [vp, vp]
    lib.dresd_kv_last_launches.restype = i32
    lib.dresd_kv_last_launches.argtypes = [vp]
    if path is None:
        _lib = lib
    return lib


def dresd_last_error() -> str:
    return load().dresd_last_error().decode()


def _check(status: int) -> None:
    if status != DRESD_OK:
        raise DresdError(status, dresd_last_error())


# ---- the C calls, by name, on raw addresses -----------------------------------
def dresd_store_create(keys_ptr: int, next_tokens_ptr: int, N: int, d: int, dtype: int,
                       stored_len: int) -> int:
    h = ctypes.c_void_p()
    _check(load().dresd_store_create(keys_ptr, next_tokens_ptr, N, d, dtype, stored_len, ctypes.byref(h)))
    return h.value


def dresd_store_set_preprocess(store: int, d_in: int, mean_ptr, var_ptr, eps_z: float, W_ptr,
                               pca_mean_ptr) -> None:
    _check(load().dresd_store_set_preprocess(store, d_in, mean_ptr, var_ptr, eps_z, W_ptr, pca_mean_ptr))


def dresd_retrieve(store: int, queries_ptr: int, B: int, top_n: int, draft_len: int, out_ids_ptr: int,
                   out_scores_ptr: int, out_tokens_ptr: int, stream: int = 0) -> None:
    _check(load().dresd_retrieve(store, queries_ptr, B, top_n, draft_len, out_ids_ptr, out_scores_ptr,
                                 out_tokens_ptr, stream))


def dresd_store_enable_first_token_filter(store: int, stream: int = 0) -> None:
    _check(load().dresd_store_enable_first_token_filter(store, stream))


def dresd_store_index_first_tokens(store: int, stream: int = 0) -> None:
    _check(load().dresd_store_index_first_tokens(store, stream))


def dresd_retrieve_filtered(store: int, queries_ptr: int, first_tokens_ptr, B: int, top_n: int, draft_len: int,
                            out_ids_ptr: int, out_scores_ptr: int, out_tokens_ptr: int, stream: int = 0) -> None:
    _check(load().dresd_retrieve_filtered(store, queries_ptr, first_tokens_ptr, B, top_n, draft_len,
                                          out_ids_ptr, out_scores_ptr, out_tokens_ptr, stream))


def dresd_drafts_prepare(tokens_ptr: int, ids_ptr: int, B: int, n: int, L: int, eos_id: int,
                         out_drafts_ptr: int, out_valid_ptr: int, stream: int = 0) -> None:
    _check(load().dresd_drafts_prepare(tokens_ptr, ids_ptr, B, n, L, eos_id, out_drafts_ptr, out_valid_ptr, stream))


def dresd_drafts_accept(drafts_ptr: int, valid_ptr: int, llm_ptr: int, B: int, n: int, L: int,
                        out_best_ptr: int, out_len_ptr: int, out_tokens_ptr: int, stream: int = 0) -> None:
    _check(load().dresd_drafts_accept(drafts_ptr, valid_ptr, llm_ptr, B, n, L, out_best_ptr, out_len_ptr,
                                      out_tokens_ptr, stream))


def dresd_merge_shards_packed(packed_ptr: int, offsets_ptr: int, P: int, B: int, top_n: int, draft_len: int,
                              out_ids_ptr: int, out_scores_ptr: int, out_tokens_ptr: int, stream: int = 0) -> None:
    _check(load().dresd_merge_shards_packed(packed_ptr, offsets_ptr, P, B, top_n, draft_len, out_ids_ptr,
                                            out_scores_ptr, out_tokens_ptr, stream))


def dresd_merge_shards(ids_ptr: int, scores_ptr: int, tokens_ptr: int, offsets_ptr: int, P: int, B: int,
                       top_n: int, draft_len: int, out_ids_ptr: int, out_scores_ptr: int, out_tokens_ptr: int,
                       stream: int = 0) -> None:
    _check(load().dresd_merge_shards(ids_ptr, scores_ptr, tokens_ptr, offsets_ptr, P, B, top_n, draft_len,
                                     out_ids_ptr, out_scores_ptr, out_tokens_ptr, stream))


def dresd_build_keys(hidden_ptr: int, N: int, d_in: int, dtype: int, mean_ptr, var_ptr, eps_z: float, W_ptr: int,
                     d: int, pca_mean_ptr, out_keys_ptr: int, stream: int = 0) -> None:
    """Eq. 1 -> v W -> Eq. 2 over N rows of hidden states: builds the datastore's key matrix."""
    _check(load().dresd_build_keys(hidden_ptr, N, d_in, dtype, mean_ptr, var_ptr, eps_z, W_ptr, d, pca_mean_ptr,
                                   out_keys_ptr, stream))


def dresd_quantise_keys(keys_ptr: int, N: int, d: int, dtype: int, out_q8_ptr: int, stream: int = 0) -> None:
    _check(load().dresd_quantise_keys(keys_ptr, N, d, dtype, out_q8_ptr, stream))


def dresd_store_attach_quantised(store: int, keys_q8_ptr: int) -> None:
    _check(load().dresd_store_attach_quantised(store, keys_q8_ptr))


def dresd_retrieve_quantised(store: int, queries_ptr: int, first_tokens_ptr, B: int, top_n: int, draft_len: int,
                             candidates: int, out_ids_ptr: int, out_scores_ptr: int, out_tokens_ptr: int,
                             stream: int = 0) -> None:
    _check(load().dresd_retrieve_quantised(store, queries_ptr, first_tokens_ptr, B, top_n, draft_len, candidates,
                                           out_ids_ptr, out_scores_ptr, out_tokens_ptr, stream))


def dresd_set_global_option(name: str, value: int) -> None:
    _check(load().dresd_set_global_option(name.encode(), int(value)))


def dresd_fit_zscore(sample_ptr: int, N: int, d_in: int, dtype: int, out_mean_ptr: int, out_var_ptr: int,
                     stream: int = 0) -> None:
    """E[V] and population Var[V] of Eq. 1 from a sample of N stored embeddings."""
    _check(load().dresd_fit_zscore(sample_ptr, N, d_in, dtype, out_mean_ptr, out_var_ptr, stream))


def dresd_retrieve_host(store: int, queries_ptr: int, B: int, top_n: int, draft_len: int,
                        out_ids_ptr: int, out_scores_ptr: int, out_tokens_ptr: int, stream: int = 0) -> None:
    _check(load().dresd_retrieve_host(store, queries_ptr, B, top_n, draft_len, out_ids_ptr,
                                      out_scores_ptr, out_tokens_ptr, stream))


def dresd_preprocess(store: int, queries_ptr: int, B: int, out_qhat_ptr: int, stream: int = 0) -> None:
    _check(load().dresd_preprocess(store, queries_ptr, B, out_qhat_ptr, stream))


def dresd_store_status(store: int) -> None:
    _check(load().dresd_store_status(store))


def dresd_store_set_option(store: int, name: str, value: int) -> None:
    _check(load().dresd_store_set_option(store, name.encode(), value))


def dresd_store_profile_read(store: int):
    """Returns ``(scan_ms_total, calls)``."""
    ms, n = ctypes.c_double(0.0), ctypes.c_int(0)
    _check(load().dresd_store_profile_read(store, ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


def dresd_store_last_launches(store: int) -> int:
    return int(load().dresd_store_last_launches(store))


def dresd_store_last_key_passes(store: int) -> float:
    return float(load().dresd_store_last_key_passes(store))


def dresd_store_destroy(store: int) -> None:
    load().dresd_store_destroy(store)


def dresd_retrieve_noalloc(keys_ptr: int, next_tokens_ptr: int, N: int, d: int, dtype: int,
                           stored_len: int, queries_ptr: int, B: int, top_n: int, draft_len: int,
                           out_ids_ptr: int, out_scores_ptr: int, out_tokens_ptr: int, stream: int = 0) -> None:
    """Retrieval without any device allocation (static in-library workspace, B <= 8).

    For hosts that may not call cudaMalloc when a draft is needed; see the
    header for the limits and the rule that calls must not overlap on the GPU.
    """
    _check(load().dresd_retrieve_noalloc(keys_ptr, next_tokens_ptr, N, d, dtype, stored_len, queries_ptr,
                                         B, top_n, draft_len, out_ids_ptr, out_scores_ptr, out_tokens_ptr,
                                         stream))


def dresd_debug_build() -> int:
    """1 when the loaded library is the bounds-checked debug build."""
    return int(load().dresd_debug_build())


def dresd_store_debug_selftest(store: int, stream: int = 0) -> None:
    _check(load().dresd_store_debug_selftest(store, stream))


def dresd_noalloc_status(stream: int = 0) -> None:
    """Waits for `stream`; raises DRESD_ERR_TIMEOUT if a device-side wait of the last
    dresd_retrieve_noalloc() call expired."""
    _check(load().dresd_noalloc_status(stream))


def dresd_kv_create(k_pages_ptr: int, v_pages_ptr: int, k_exps_ptr, v_exps_ptr, layers: int, num_pages: int,
                    kv_heads: int, page_size: int, head_dim: int, dtype: int) -> int:
    h = ctypes.c_void_p()
    _check(load().dresd_kv_create(k_pages_ptr, v_pages_ptr, k_exps_ptr, v_exps_ptr, layers, num_pages, kv_heads,
                                  page_size, head_dim, dtype, ctypes.byref(h)))
    return h.value


def dresd_kv_append(kv: int, layer: int, batch: dresd_kv_batch, k_ptr: int, k_row: int, k_head: int, v_ptr: int,
                    v_row: int, v_head: int, stream: int = 0) -> None:
    _check(load().dresd_kv_append(kv, layer, batch, k_ptr, k_row, k_head, v_ptr, v_row, v_head, stream))


def dresd_kv_read(kv: int, layer: int, batch: dresd_kv_batch, out_k_ptr: int, out_v_ptr: int, stream: int = 0) -> None:
    _check(load().dresd_kv_read(kv, layer, batch, out_k_ptr, out_v_ptr, stream))


def dresd_kv_attend(kv: int, layer: int, batch: dresd_kv_batch, q_ptr: int, q_row: int, q_head: int, heads: int,
                    scale: float, mask_ptr, mask_words: int, out_ptr: int, out_lse_ptr, stream: int = 0) -> None:
    _check(load().dresd_kv_attend(kv, layer, batch, q_ptr, q_row, q_head, heads, scale, mask_ptr, mask_words, out_ptr,
                                  out_lse_ptr, stream))


def dresd_kv_keep_draft(kv: int, batch: dresd_kv_batch, best_ptr: int, length_ptr: int, n: int, L: int,
                        stream: int = 0) -> None:
    _check(load().dresd_kv_keep_draft(kv, batch, best_ptr, length_ptr, n, L, stream))


def dresd_kv_status(kv: int) -> None:
    _check(load().dresd_kv_status(kv))


def dresd_kv_set_option(kv: int, name: str, value: int) -> None:
    _check(load().dresd_kv_set_option(kv, name.encode(), value))


def dresd_kv_debug_selftest(kv: int, stream: int = 0) -> None:
    _check(load().dresd_kv_debug_selftest(kv, stream))


def dresd_kv_last_launches(kv: int) -> int:
    return int(load().dresd_kv_last_launches(kv))


def dresd_kv_destroy(kv: int) -> None:
    load().dresd_kv_destroy(kv)


# ---- torch convenience ----------------------------------------------------------
_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _allocated_on(stream):
    """Results are allocated on the stream that writes them: memory of the current stream's pool may still be in use by
    what is queued there, and is given out there again while `stream` writes it."""
    return contextlib.nullcontext() if stream is None else _torch().cuda.stream(stream)


def to_device(array, dtype: str, device="cuda"):
    """Upload a numpy array holding store-dtype values (bit patterns for 16-bit)."""
    import numpy as np
    torch = _torch()
    a = np.ascontiguousarray(array)
    if dtype == "bf16":
        return torch.from_numpy(a.view(np.int16)).to(device).view(torch.bfloat16)
    if dtype == "f16":
        return torch.from_numpy(a.view(np.float16)).to(device)
    return torch.from_numpy(a.astype(np.float32, copy=False)).to(device)


class Store:
    """A datastore on the current CUDA device; tensors passed in are borrowed."""

    def __init__(self, keys, next_tokens, dtype: str):
        torch = _torch()
        want = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
        if not keys.is_cuda or not next_tokens.is_cuda:
            raise DresdError(-1, "keys and next_tokens must be CUDA tensors (there is no CPU path)")
        if keys.dtype != want or next_tokens.dtype != torch.int32:
            raise DresdError(-1, f"keys must be {want}, next_tokens int32")
        if not keys.is_contiguous() or not next_tokens.is_contiguous():
            raise DresdError(-1, "keys and next_tokens must be contiguous")
        self.dtype = dtype
        self.torch_dtype = want
        self.keys, self.next_tokens = keys, next_tokens       # keep alive
        self.N, self.d = keys.shape
        self.stored_len = next_tokens.shape[1]
        self.d_in = self.d
        self._pre = None
        self.handle = dresd_store_create(keys.data_ptr(), next_tokens.data_ptr(), self.N, self.d,
                                         DTYPE_CODE[dtype], self.stored_len)

    def set_preprocess(self, d_in, mean=None, var=None, eps_z=1e-5, W=None, pca_mean=None):
        self._pre = (mean, var, W, pca_mean)                  # keep alive
        ptr = lambda t: None if t is None else t.data_ptr()
        dresd_store_set_preprocess(self.handle, d_in, ptr(mean), ptr(var), eps_z, ptr(W), ptr(pca_mean))
        self.d_in = d_in

    def set_option(self, name: str, value: int):
        dresd_store_set_option(self.handle, name, value)

    def retrieve(self, queries, top_n: int, draft_len: int, out=None, stream=None):
        """Returns ``(ids [B][n] int32, scores [B][n] f32, tokens [B][n][L] int32)`` on the device."""
        torch = _torch()
        B = queries.shape[0]
        if out is None:
            dev = queries.device
            with _allocated_on(stream):
                out = (torch.empty((B, top_n), dtype=torch.int32, device=dev),
                       torch.empty((B, top_n), dtype=torch.float32, device=dev),
                       torch.empty((B, top_n, draft_len), dtype=torch.int32, device=dev))
        ids, scores, tokens = out
        s = (stream or torch.cuda.current_stream()).cuda_stream
        dresd_retrieve(self.handle, queries.data_ptr(), B, top_n, draft_len, ids.data_ptr(),
                       scores.data_ptr(), tokens.data_ptr(), s)
        return ids, scores, tokens

    def enable_first_token_filter(self, stream=None):
        s = (stream or _torch().cuda.current_stream()).cuda_stream
        dresd_store_enable_first_token_filter(self.handle, s)

    def index_first_tokens(self, stream=None):
        """For a store whose rows are sorted by first stored token: filtered calls then scan only
        the rows of the queries' tokens."""
        s = (stream or _torch().cuda.current_stream()).cuda_stream
        dresd_store_index_first_tokens(self.handle, s)

    def retrieve_filtered(self, queries, first_tokens, top_n: int, draft_len: int, out=None, stream=None):
        """Like retrieve(), restricted per query to keys whose first stored token is first_tokens[b]."""
        torch = _torch()
        B = queries.shape[0]
        if out is None:
            dev = queries.device
            with _allocated_on(stream):
                out = (torch.empty((B, top_n), dtype=torch.int32, device=dev),
                       torch.empty((B, top_n), dtype=torch.float32, device=dev),
                       torch.empty((B, top_n, draft_len), dtype=torch.int32, device=dev))
        ids, scores, tokens = out
        s = (stream or torch.cuda.current_stream()).cuda_stream
        dresd_retrieve_filtered(self.handle, queries.data_ptr(),
                                None if first_tokens is None else first_tokens.data_ptr(), B, top_n, draft_len,
                                ids.data_ptr(), scores.data_ptr(), tokens.data_ptr(), s)
        return ids, scores, tokens

    def attach_quantised(self, stream=None):
        """Build the 8-bit (E4M3) copy of the keys on the device and attach it; returns the copy."""
        torch = _torch()
        s = (stream or torch.cuda.current_stream()).cuda_stream
        with _allocated_on(stream):
            q8 = torch.empty((self.N, self.d), dtype=torch.uint8, device=self.keys.device)
        dresd_quantise_keys(self.keys.data_ptr(), self.N, self.d, DTYPE_CODE[self.dtype], q8.data_ptr(), s)
        dresd_store_attach_quantised(self.handle, q8.data_ptr())
        self.keys_q8 = q8                                # keep the borrowed buffer alive
        return q8

    def retrieve_quantised(self, queries, top_n: int, draft_len: int, candidates: int, out=None, stream=None,
                           first_tokens=None):
        """Candidates by 8-bit approximate score, exact re-ranking of `candidates` rows per query;
        first_tokens (int32 device tensor [B], -1 = any) restricts the candidates per query."""
        torch = _torch()
        B = queries.shape[0]
        if out is None:
            dev = queries.device
            with _allocated_on(stream):
                out = (torch.empty((B, top_n), dtype=torch.int32, device=dev),
                       torch.empty((B, top_n), dtype=torch.float32, device=dev),
                       torch.empty((B, top_n, draft_len), dtype=torch.int32, device=dev))
        ids, scores, tokens = out
        s = (stream or torch.cuda.current_stream()).cuda_stream
        dresd_retrieve_quantised(self.handle, queries.data_ptr(),
                                 None if first_tokens is None else first_tokens.data_ptr(), B, top_n, draft_len,
                                 candidates, ids.data_ptr(), scores.data_ptr(), tokens.data_ptr(), s)
        return ids, scores, tokens

    def retrieve_host(self, queries, top_n: int, draft_len: int, out, stream=None):
        """Host (pinned) tensors in and out; blocks until the results are on the host."""
        torch = _torch()
        ids, scores, tokens = out
        s = (stream or torch.cuda.current_stream()).cuda_stream
        dresd_retrieve_host(self.handle, queries.data_ptr(), queries.shape[0], top_n, draft_len,
                            ids.data_ptr(), scores.data_ptr(), tokens.data_ptr(), s)
        return ids, scores, tokens

    def preprocess(self, queries, stream=None):
        torch = _torch()
        B = queries.shape[0]
        with _allocated_on(stream):
            out = torch.empty((B, self.d), dtype=torch.float32, device=queries.device)
        s = (stream or torch.cuda.current_stream()).cuda_stream
        dresd_preprocess(self.handle, queries.data_ptr(), B, out.data_ptr(), s)
        return out

    def status(self):
        dresd_store_status(self.handle)

    def profile_read(self):
        return dresd_store_profile_read(self.handle)

    def last_key_passes(self) -> float:
        return dresd_store_last_key_passes(self.handle)

    def last_launches(self) -> int:
        return dresd_store_last_launches(self.handle)

    def close(self):
        if getattr(self, "handle", None):
            dresd_store_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _raw_stream(device_index: int, stream) -> int:
    """cudaStream_t of `stream`, or of the device's current stream."""
    if stream is not None:
        return stream.cuda_stream
    return _torch()._C._cuda_getCurrentRawStream(device_index)


def draft_mask(n: int, L: int, device="cuda"):
    """Visibility bits of a chunk that is a sequence's last token and its n drafts of L tokens, int32
    [1 + n L][words]: every token sees the first one and its own draft up to itself."""
    import numpy as np
    size = 1 + n * L
    seen = np.zeros((size, (size + 31) // 32 * 32), dtype=np.uint8)
    seen[:, 0] = 1
    for r in range(n):
        at = 1 + r * L
        seen[at:at + L, at:at + L] = np.tri(L, dtype=np.uint8)
    words = np.packbits(seen, axis=1, bitorder="little").view("<i4")
    return _torch().from_numpy(np.ascontiguousarray(words)).to(device)


class KvBatch:
    """A batch of chunks (``dresd_kv_batch``): int32 CUDA tensors of one device, borrowed; their contents are read when a
    call runs."""

    def __init__(self, page_table, ctx, start, rows: int, max_chunk: int = 0):
        torch = _torch()
        self.device_index = page_table.get_device()           # -1: not a CUDA tensor
        for name, t, dims in (("page_table", page_table, 2), ("ctx", ctx, 1), ("start", start, 1)):
            if t.get_device() != self.device_index:
                raise DresdError(-1, f"{name} is on another device than page_table")
            if not t.is_cuda or t.dtype != torch.int32 or t.dim() != dims or not t.is_contiguous():
                raise DresdError(-1, f"{name} must be a contiguous int32 CUDA tensor with {dims} dimension(s)")
        B, width = page_table.shape
        if ctx.shape[0] != B or start.shape[0] != B + 1:
            raise DresdError(-1, f"ctx has {ctx.shape[0]} and start {start.shape[0]} entries for {B} sequences")
        self.page_table, self.ctx, self.start = page_table, ctx, start          # keep alive
        self.B, self.rows, self.max_chunk = B, rows, max_chunk
        self.c = dresd_kv_batch(page_table.data_ptr(), ctx.data_ptr(), start.data_ptr(), B, width, rows, max_chunk)


class KvCache:
    """A paged key/value cache on the current CUDA device; tensors passed in are borrowed.  All tensors, the batches' too, are
    of that device, which has to be the current one in every call.

    k_pages, v_pages: [layers][num_pages][kv_heads][page_size][head_dim] in `dtype`, or uint8 with
    k_exps, v_exps: uint8 [layers][num_pages][kv_heads][page_size] (8-bit rows)."""

    def __init__(self, k_pages, v_pages, dtype: str, k_exps=None, v_exps=None):
        torch = _torch()
        if dtype not in ("f16", "bf16"):
            raise DresdError(-2, f"the cache holds f16, bf16 or 8-bit rows, not {dtype}")
        self.torch_dtype = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
        if (k_exps is None) != (v_exps is None):
            raise DresdError(-1, "k_exps and v_exps go together")
        held = self.torch_dtype if k_exps is None else torch.uint8
        for name, t in (("k_pages", k_pages), ("v_pages", v_pages)):
            if not t.is_cuda or t.dtype != held or t.dim() != 5 or not t.is_contiguous():
                raise DresdError(-1, f"{name} must be a contiguous {held} CUDA tensor with 5 dimensions")
        if v_pages.shape != k_pages.shape:
            raise DresdError(-1, "k_pages and v_pages must have the same shape")
        for name, t in (("k_exps", k_exps), ("v_exps", v_exps)):
            if t is not None and (not t.is_cuda or t.dtype != torch.uint8 or t.shape != k_pages.shape[:4] or
                                  not t.is_contiguous()):
                raise DresdError(-1, f"{name} must be a contiguous uint8 CUDA tensor of shape {tuple(k_pages.shape[:4])}")
        self.device_index = k_pages.get_device()
        for name, t in (("v_pages", v_pages), ("k_exps", k_exps), ("v_exps", v_exps)):
            if t is not None and t.get_device() != self.device_index:
                raise DresdError(-1, f"{name} is on another device than k_pages")
        self.dtype = dtype
        self.k_pages, self.v_pages, self.k_exps, self.v_exps = k_pages, v_pages, k_exps, v_exps   # keep alive
        self.layers, self.num_pages, self.kv_heads, self.page_size, self.head_dim = k_pages.shape
        ptr = lambda t: None if t is None else t.data_ptr()
        self.handle = dresd_kv_create(k_pages.data_ptr(), v_pages.data_ptr(), ptr(k_exps), ptr(v_exps), self.layers,
                                      self.num_pages, self.kv_heads, self.page_size, self.head_dim, DTYPE_CODE[dtype])

    def _batch(self, batch):
        if batch.device_index != self.device_index:
            raise DresdError(-1, f"the batch is on cuda:{batch.device_index}, the cache on cuda:{self.device_index}")

    def _rows(self, name, t, batch, heads=None):
        """Distances of rows and heads of a [rows][heads][head_dim] tensor."""
        self._batch(batch)
        shape = t.shape
        if t.dtype != self.torch_dtype or t.get_device() != self.device_index or len(shape) != 3:
            raise DresdError(-1, f"{name} must be a {self.torch_dtype} tensor with 3 dimensions on cuda:{self.device_index}")
        if shape[0] != batch.rows or shape[2] != self.head_dim or (heads is not None and shape[1] != heads):
            raise DresdError(-1, f"{name} has shape {tuple(shape)}")
        row, head, last = t.stride()
        if last != 1:
            raise DresdError(-1, f"{name}: the elements of a head must be adjacent")
        return row, head

    def append(self, layer: int, k, v, batch: KvBatch, stream=None):
        """Writes the chunks' keys and values, [rows][kv_heads][head_dim] (slices of a joint projection are fine)."""
        k_row, k_head = self._rows("k", k, batch, self.kv_heads)
        v_row, v_head = self._rows("v", v, batch, self.kv_heads)
        dresd_kv_append(self.handle, layer, batch.c, k.data_ptr(), k_row, k_head, v.data_ptr(), v_row, v_head,
                        _raw_stream(self.device_index, stream))

    def read(self, layer: int, batch: KvBatch, out=None, stream=None):
        """Returns ``(k, v)``, dense [rows][kv_heads][head_dim], of the positions ctx[b] .. of every sequence."""
        torch = _torch()
        self._batch(batch)
        shape = (batch.rows, self.kv_heads, self.head_dim)
        if out is None:
            with _allocated_on(stream):
                k, v = torch.empty((2, *shape), dtype=self.torch_dtype, device=self.k_pages.device).unbind(0)
        else:
            k, v = out
            for name, t in (("out k", k), ("out v", v)):
                if t.shape != shape or t.dtype != self.torch_dtype or t.get_device() != self.device_index or not t.is_contiguous():
                    raise DresdError(-1, f"{name} must be a contiguous {self.torch_dtype} tensor of shape {shape} on cuda:{self.device_index}")
        dresd_kv_read(self.handle, layer, batch.c, k.data_ptr(), v.data_ptr(), _raw_stream(self.device_index, stream))
        return k, v

    def attend(self, layer: int, q, batch: KvBatch, scale: float | None = None, mask=None, out=None, lse=None, stream=None):
        """Attention of the chunks' tokens, q [rows][heads][head_dim], over the cache; returns `out`, dense like q.
        scale: 1 / sqrt(head_dim) if not given.  mask: int32 [rows][words], None = causal (see draft_mask).
        lse: fp32 [rows][heads] to be filled, optional."""
        torch = _torch()
        q_row, q_head = self._rows("q", q, batch)
        rows, heads, d = q.shape
        if out is None:
            with _allocated_on(stream):
                out = torch.empty((rows, heads, d), dtype=self.torch_dtype, device=self.k_pages.device)
        elif out.shape != q.shape or out.dtype != q.dtype or out.get_device() != self.device_index or not out.is_contiguous():
            raise DresdError(-1, f"out must be a contiguous {q.dtype} tensor of shape {tuple(q.shape)} on cuda:{self.device_index}")
        if lse is not None and (lse.shape != (rows, heads) or lse.dtype != torch.float32 or lse.get_device() != self.device_index or
                                not lse.is_contiguous()):
            raise DresdError(-1, f"lse must be a contiguous float32 tensor of shape {(rows, heads)} on cuda:{self.device_index}")
        mask_ptr, words = None, 0
        if mask is not None:
            if mask.dtype != torch.int32 or mask.get_device() != self.device_index or mask.dim() != 2 or mask.shape[0] != rows or \
                    not mask.is_contiguous():
                raise DresdError(-1, f"mask must be a contiguous int32 tensor of {rows} rows on cuda:{self.device_index}")
            mask_ptr, words = mask.data_ptr(), mask.shape[1]
        dresd_kv_attend(self.handle, layer, batch.c, q.data_ptr(), q_row, q_head, heads,
                        d ** -0.5 if scale is None else scale, mask_ptr, words, out.data_ptr(),
                        None if lse is None else lse.data_ptr(), _raw_stream(self.device_index, stream))
        return out

    def keep_draft(self, batch: KvBatch, best, length, n: int, L: int, stream=None):
        """Moves the accepted drafts' tokens into place in every layer (best, length: of dresd_drafts_accept)."""
        int32 = _torch().int32
        self._batch(batch)
        for name, t in (("best", best), ("length", length)):
            if t.dtype != int32 or t.get_device() != self.device_index or t.shape != (batch.B,) or not t.is_contiguous():
                raise DresdError(-1, f"{name} must be a contiguous int32 tensor of {batch.B} entries on cuda:{self.device_index}")
        dresd_kv_keep_draft(self.handle, batch.c, best.data_ptr(), length.data_ptr(), n, L,
                            _raw_stream(self.device_index, stream))

    def set_option(self, name: str, value: int):
        dresd_kv_set_option(self.handle, name, value)

    def status(self):
        dresd_kv_status(self.handle)

    def last_launches(self) -> int:
        return dresd_kv_last_launches(self.handle)

    def close(self):
        if getattr(self, "handle", None):
            dresd_kv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
