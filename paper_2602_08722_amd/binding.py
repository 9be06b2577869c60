"""ctypes binding of libquoka's C ABI (see include/quoka.h).

Argument marshalling only: every function takes torch tensors that already live on the GPU, passes
their device pointers and the current HIP stream to the C entry point of the same name, and raises
QuokaError on a non-zero status.  No arithmetic of the method happens in Python, and there is no
fallback: if the shared library has not been built the import of a symbol fails loudly.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

QUOKA_F32 = 0
QUOKA_BF16 = 1
QUOKA_PAGES_RAW = 0
QUOKA_PAGES_FP8 = 1

_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)

_LIB_NAME = "libquoka.so"
_lib: Optional[ctypes.CDLL] = None

EXPORTS = (
    "quoka_workspace_bytes", "quoka_select_queries", "quoka_score_keys", "quoka_topk_keys", "quoka_select_keys",
    "quoka_sparse_attn", "quoka_dense_attn", "quoka_chunk_attn", "quoka_prefill_workspace_bytes", "quoka_prefill_attn",
    "quoka_topk_keys_noalloc", "quoka_cache_write", "quoka_cache_read", "quoka_paged_workspace_bytes", "quoka_paged_attn",
    "quoka_probe_mfma", "quoka_probe_read", "quoka_probe_attn_mix", "quoka_probe_attn_plan", "quoka_status_string", "quoka_version",
)
_STATUS_EXPORTS = EXPORTS[:-2]   # everything that returns a quoka_status


class QuokaError(RuntimeError):
    def __init__(self, fn: str, status: int, msg: str):
        super().__init__(f"{fn} failed: status {status} ({msg})")
        self.status = status


class QuokaShape(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("chunk_len", ctypes.c_int32), ("max_kv_len", ctypes.c_int32),
        ("n_retain", ctypes.c_int32), ("max_budget", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("score_flags", ctypes.c_int32),
        ("q_stride", ctypes.c_int64 * 3), ("kv_stride", ctypes.c_int64 * 3),
        ("ck_stride", ctypes.c_int64 * 3), ("o_stride", ctypes.c_int64 * 3),
    ]

    @property
    def n_keep(self) -> int:
        return min(self.n_retain, self.chunk_len)


class QuokaPages(ctypes.Structure):
    _fields_ = [
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
        ("page_table", ctypes.c_void_p), ("stride", ctypes.c_int64 * 3),
        ("n_pages", ctypes.c_int32), ("page_len", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("format", ctypes.c_int32),
    ]


def library_path() -> str:
    return os.path.join(os.path.dirname(os.path.abspath(__file__)), _LIB_NAME)


def load_library() -> ctypes.CDLL:
    """Load the in-tree libquoka.so; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is not None:
        return _lib
    path = library_path()
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} not found: build it with `python -m paper_2602_08722_amd.build`")
    lib = ctypes.CDLL(path)
    P, I32P, F32P, SZ = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t
    SH = ctypes.POINTER(QuokaShape)
    lib.quoka_workspace_bytes.argtypes = [SH, ctypes.POINTER(ctypes.c_size_t)]
    lib.quoka_prefill_workspace_bytes.argtypes = [SH, ctypes.POINTER(ctypes.c_size_t)]
    lib.quoka_select_queries.argtypes = [SH, P, I32P, F32P, P, SZ, P]
    lib.quoka_score_keys.argtypes = [SH, F32P, P, I32P, F32P, P, SZ, P]
    lib.quoka_topk_keys.argtypes = [SH, F32P, I32P, I32P, I32P, I32P, P, SZ, P]
    lib.quoka_select_keys.argtypes = [SH, F32P, P, I32P, I32P, F32P, I32P, I32P, P, SZ, P]
    lib.quoka_sparse_attn.argtypes = [SH, P, P, P, I32P, I32P, P, P, P, F32P, P, SZ, P]
    lib.quoka_dense_attn.argtypes = [SH, P, P, P, I32P, P, P, P, F32P, P, SZ, P]
    lib.quoka_chunk_attn.argtypes = [SH, P, P, P, I32P, I32P, P, P, I32P, F32P, F32P, I32P, I32P, P, F32P, P, SZ, P]
    lib.quoka_prefill_attn.argtypes = [SH, ctypes.c_int, P, P, P, I32P, I32P, I32P, F32P, F32P, I32P, I32P, P, P, SZ, P]
    lib.quoka_topk_keys_noalloc.argtypes = [SH, F32P, I32P, I32P, I32P, I32P, P]
    PG = ctypes.POINTER(QuokaPages)
    lib.quoka_cache_write.argtypes = [SH, PG, P, P, I32P, I32P, P]
    lib.quoka_cache_read.argtypes = [SH, PG, I32P, P, P, P]
    lib.quoka_paged_workspace_bytes.argtypes = [SH, ctypes.POINTER(ctypes.c_size_t)]
    lib.quoka_paged_attn.argtypes = [SH, PG, P, I32P, I32P, I32P, I32P, P, F32P, P, SZ, P]
    lib.quoka_probe_mfma.argtypes = [ctypes.c_int, ctypes.c_int, F32P, P]
    lib.quoka_probe_read.argtypes = [P, SZ, F32P, P]
    lib.quoka_probe_attn_mix.argtypes = [ctypes.c_int, ctypes.c_int, F32P, P]
    for name in _STATUS_EXPORTS:
        getattr(lib, name).restype = ctypes.c_int
    lib.quoka_status_string.argtypes = [ctypes.c_int]
    lib.quoka_status_string.restype = ctypes.c_char_p
    lib.quoka_version.argtypes = []
    lib.quoka_version.restype = ctypes.c_int
    _lib = lib
    return lib


def _check(fn: str, status: int) -> None:
    if status != 0:
        raise QuokaError(fn, status, load_library().quoka_status_string(status).decode())


# A call marshals up to 17 arguments, which is a third of what enqueuing four launches takes: plain integers (the entry points'
# argtypes turn them into pointers) and the current stream's handle without a Stream object around it.
def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _strides3(t: torch.Tensor):
    assert t.dim() == 4 and t.stride(3) == 1, "expected [batch, heads, tokens, head_dim] with head_dim contiguous"
    return (ctypes.c_int64 * 3)(t.stride(0), t.stride(1), t.stride(2))


def _ints(x, dev) -> torch.Tensor:
    """Lengths or budgets as kernels read them: int32, on `dev`, dense (a tensor that is so already stays the caller's own)."""
    return torch.as_tensor(x, dtype=torch.int32).to(dev).contiguous()


QUOKA_SCORE_DOT, QUOKA_SCORE_MEAN, QUOKA_SELECT_UNIFORM, QUOKA_SCORE_QBAR_BF16, QUOKA_ATTN_SCALE_F32 = 1, 2, 4, 8, 16   # quoka.h


def make_shape(q: torch.Tensor, k_cache: torch.Tensor, k_chunk: torch.Tensor, out: torch.Tensor,
               n_retain: int, max_budget: int, score_flags: int = 0) -> QuokaShape:
    """Describe the problem from the tensors' own shapes and strides (no copies)."""
    b, n_q, C, d = q.shape
    n_kv, t_max = k_cache.shape[1], k_cache.shape[2]
    if q.dtype == torch.bfloat16:
        dt = QUOKA_BF16
    elif q.dtype == torch.float32:
        dt = QUOKA_F32
    else:
        raise TypeError(f"unsupported dtype {q.dtype}")
    s = QuokaShape()
    s.batch, s.n_q_heads, s.n_kv_heads, s.head_dim = b, n_q, n_kv, d
    s.chunk_len, s.max_kv_len, s.n_retain, s.max_budget = C, t_max, n_retain, max_budget
    s.dtype, s.score_flags = dt, int(score_flags)
    s.q_stride = _strides3(q)
    if t_max > 0:
        s.kv_stride = _strides3(k_cache)
    else:
        s.kv_stride = (ctypes.c_int64 * 3)(0, 0, d)
    s.ck_stride = _strides3(k_chunk)
    s.o_stride = _strides3(out)
    return s


def make_pages(k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
               v_scale: Optional[torch.Tensor] = None) -> QuokaPages:
    """Describe a pool of pages [n_pages, n_KV, page_len, d] and its page table [b, max_pages] from the tensors' own shapes and
    strides (no copies; the caller keeps the tensors).  torch.float8_e4m3fn pages need k_scale and v_scale [n_pages, n_KV, page_len]
    uint8; other pages are rows in the dtype of the calls that use them."""
    fp8 = k_pages.dtype == torch.float8_e4m3fn
    if not fp8 and k_pages.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"unsupported dtype of pages {k_pages.dtype}")
    if v_pages.dtype != k_pages.dtype or v_pages.shape != k_pages.shape or v_pages.stride() != k_pages.stride():
        raise ValueError("K and V pages share shape, strides and dtype")
    if page_table.dtype != torch.int32 or page_table.dim() != 2 or not page_table.is_contiguous():
        raise ValueError("page_table is a dense int32 tensor [batch, max_pages]")
    if fp8:
        for t in (k_scale, v_scale):
            if t is None or t.dtype != torch.uint8 or t.shape != k_pages.shape[:3] or not t.is_contiguous():
                raise ValueError("8-bit pages need dense uint8 scales [n_pages, n_KV, page_len]")
    if any(t.device != k_pages.device for t in (v_pages, page_table) + ((k_scale, v_scale) if fp8 else ())):
        raise ValueError("pages, scales and page table are on one device")
    p = QuokaPages()
    p.stride = _strides3(k_pages)
    p.n_pages, _, p.page_len, _ = k_pages.shape
    p.max_pages = page_table.shape[1]
    p.format = QUOKA_PAGES_FP8 if fp8 else QUOKA_PAGES_RAW
    p.k, p.v, p.page_table = k_pages.data_ptr(), v_pages.data_ptr(), page_table.data_ptr()
    if fp8:
        p.k_scale, p.v_scale = k_scale.data_ptr(), v_scale.data_ptr()
    return p


def quoka_version() -> int:
    return load_library().quoka_version()


def quoka_workspace_bytes(shape: QuokaShape) -> int:
    n = ctypes.c_size_t(0)
    _check("quoka_workspace_bytes", load_library().quoka_workspace_bytes(ctypes.byref(shape), ctypes.byref(n)))
    return int(n.value)


def quoka_prefill_workspace_bytes(shape: QuokaShape) -> int:
    n = ctypes.c_size_t(0)
    _check("quoka_prefill_workspace_bytes",
           load_library().quoka_prefill_workspace_bytes(ctypes.byref(shape), ctypes.byref(n)))
    return int(n.value)


def quoka_select_queries(shape, q, q_idx, qbar, workspace, stream=None) -> None:
    _check("quoka_select_queries", load_library().quoka_select_queries(
        ctypes.byref(shape), _ptr(q), _ptr(q_idx), _ptr(qbar), _ptr(workspace), workspace.numel(), _stream(stream)))


def quoka_score_keys(shape, qbar, k_cache, kv_lens, scores, workspace, stream=None) -> None:
    _check("quoka_score_keys", load_library().quoka_score_keys(
        ctypes.byref(shape), _ptr(qbar), _ptr(k_cache), _ptr(kv_lens), _ptr(scores), _ptr(workspace),
        workspace.numel(), _stream(stream)))


def quoka_topk_keys(shape, scores, kv_lens, budgets, k_idx, k_cnt, workspace, stream=None) -> None:
    _check("quoka_topk_keys", load_library().quoka_topk_keys(
        ctypes.byref(shape), _ptr(scores), _ptr(kv_lens), _ptr(budgets), _ptr(k_idx), _ptr(k_cnt), _ptr(workspace),
        workspace.numel(), _stream(stream)))


def quoka_select_keys(shape, qbar, k_cache, kv_lens, budgets, scores, k_idx, k_cnt, workspace, stream=None) -> None:
    _check("quoka_select_keys", load_library().quoka_select_keys(
        ctypes.byref(shape), _ptr(qbar), _ptr(k_cache), _ptr(kv_lens), _ptr(budgets), _ptr(scores), _ptr(k_idx),
        _ptr(k_cnt), _ptr(workspace), workspace.numel(), _stream(stream)))


def quoka_topk_keys_noalloc(shape, scores, kv_lens, budgets, k_idx, k_cnt, stream=None) -> None:
    _check("quoka_topk_keys_noalloc", load_library().quoka_topk_keys_noalloc(
        ctypes.byref(shape), _ptr(scores), _ptr(kv_lens), _ptr(budgets), _ptr(k_idx), _ptr(k_cnt), _stream(stream)))


def quoka_probe_mfma(blocks: int, iters: int, sink, stream=None) -> None:
    _check("quoka_probe_mfma", load_library().quoka_probe_mfma(int(blocks), int(iters), _ptr(sink), _stream(stream)))


def quoka_probe_attn_mix(blocks: int, steps: int, sink, stream=None) -> None:
    _check("quoka_probe_attn_mix", load_library().quoka_probe_attn_mix(int(blocks), int(steps), _ptr(sink),
                                                                       _stream(stream)))


def quoka_probe_attn_plan(shape: QuokaShape, sparse: bool):
    """(row blocks per block, blocks that share a key list) of the bf16 attention kernel for this shape; (0, 0) where another takes it."""
    rows, splits = ctypes.c_int32(0), ctypes.c_int32(0)
    _check("quoka_probe_attn_plan", load_library().quoka_probe_attn_plan(
        ctypes.byref(shape), int(bool(sparse)), ctypes.byref(rows), ctypes.byref(splits)))
    return rows.value, splits.value


def quoka_probe_read(src, nbytes: int, sink, stream=None) -> None:
    _check("quoka_probe_read", load_library().quoka_probe_read(_ptr(src), int(nbytes), _ptr(sink), _stream(stream)))


def quoka_sparse_attn(shape, q, k_cache, v_cache, k_idx, k_cnt, k_chunk, v_chunk, out, lse, workspace,
                      stream=None) -> None:
    _check("quoka_sparse_attn", load_library().quoka_sparse_attn(
        ctypes.byref(shape), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(k_idx), _ptr(k_cnt), _ptr(k_chunk),
        _ptr(v_chunk), _ptr(out), _ptr(lse), _ptr(workspace), workspace.numel(), _stream(stream)))


def quoka_dense_attn(shape, q, k_cache, v_cache, kv_lens, k_chunk, v_chunk, out, lse, workspace, stream=None) -> None:
    _check("quoka_dense_attn", load_library().quoka_dense_attn(
        ctypes.byref(shape), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(kv_lens), _ptr(k_chunk), _ptr(v_chunk),
        _ptr(out), _ptr(lse), _ptr(workspace), workspace.numel(), _stream(stream)))


def quoka_chunk_attn(shape, q, k_cache, v_cache, kv_lens, budgets, k_chunk, v_chunk, q_idx, qbar, scores, k_idx,
                     k_cnt, out, lse, workspace, stream=None) -> None:
    _check("quoka_chunk_attn", load_library().quoka_chunk_attn(
        ctypes.byref(shape), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(kv_lens), _ptr(budgets), _ptr(k_chunk),
        _ptr(v_chunk), _ptr(q_idx), _ptr(qbar), _ptr(scores), _ptr(k_idx), _ptr(k_cnt), _ptr(out), _ptr(lse),
        _ptr(workspace), workspace.numel(), _stream(stream)))


def quoka_prefill_attn(shape, sparse, q, k, v, kv_lens_all, budgets_all, q_idx, qbar, scores, k_idx, k_cnt, out,
                       workspace, stream=None) -> None:
    _check("quoka_prefill_attn", load_library().quoka_prefill_attn(
        ctypes.byref(shape), int(bool(sparse)), _ptr(q), _ptr(k), _ptr(v), _ptr(kv_lens_all), _ptr(budgets_all),
        _ptr(q_idx), _ptr(qbar), _ptr(scores), _ptr(k_idx), _ptr(k_cnt), _ptr(out), _ptr(workspace),
        workspace.numel(), _stream(stream)))


def quoka_cache_write(shape, pages, k_chunk, v_chunk, kv_lens, chunk_lens=None, stream=None) -> None:
    _check("quoka_cache_write", load_library().quoka_cache_write(
        ctypes.byref(shape), ctypes.byref(pages), _ptr(k_chunk), _ptr(v_chunk), _ptr(kv_lens), _ptr(chunk_lens), _stream(stream)))


def quoka_cache_read(shape, pages, kv_lens, k_out, v_out, stream=None) -> None:
    _check("quoka_cache_read", load_library().quoka_cache_read(
        ctypes.byref(shape), ctypes.byref(pages), _ptr(kv_lens), _ptr(k_out), _ptr(v_out), _stream(stream)))


def quoka_paged_workspace_bytes(shape: QuokaShape) -> int:
    n = ctypes.c_size_t(0)
    _check("quoka_paged_workspace_bytes",
           load_library().quoka_paged_workspace_bytes(ctypes.byref(shape), ctypes.byref(n)))
    return int(n.value)


def quoka_paged_attn(shape, pages, q, kv_lens, chunk_lens, k_idx, k_cnt, out, lse, workspace, stream=None) -> None:
    _check("quoka_paged_attn", load_library().quoka_paged_attn(
        ctypes.byref(shape), ctypes.byref(pages), _ptr(q), _ptr(kv_lens), _ptr(chunk_lens), _ptr(k_idx), _ptr(k_cnt), _ptr(out),
        _ptr(lse), _ptr(workspace), workspace.numel(), _stream(stream)))


class PrefillBuffers:
    """Device buffers for chunked prefill of a whole prompt (allocation only; torch owns the memory).

    q [b, n_Q, L, d], k / v [b, n_KV, L, d]; `budget` is B_SA per chunk: an int, or a callable of the cache length.
    """

    def __init__(self, q, k, v, chunk, n_retain, budget, score_flags=0):
        dev = q.device
        b, n_q, L, d = q.shape
        n_kv = k.shape[1]
        self.q, self.k, self.v = q, k, v
        n_chunks = -(-L // chunk)
        lens = [[i * chunk] * b for i in range(n_chunks)]
        bud = [[int(budget(i * chunk)) if callable(budget) else int(budget)] * b for i in range(n_chunks)]
        max_budget = max(0, min(max(x[0] for x in bud), L))
        self.kv_lens_all = torch.tensor(lens, dtype=torch.int32, device=dev)
        self.budgets_all = torch.tensor(bud, dtype=torch.int32, device=dev)
        self.out = torch.empty_like(q)
        # the shape describes one chunk of `chunk` rows taken from the prompt tensors (their strides, no copies)
        self.shape = make_shape(q[:, :, :chunk], k, k[:, :, :chunk], self.out[:, :, :chunk], n_retain, max_budget,
                                score_flags)
        n_keep = self.shape.n_keep
        self.q_idx = torch.empty((b, n_q, n_keep), dtype=torch.int32, device=dev)
        self.qbar = torch.empty((b, n_kv, n_keep, d), dtype=torch.float32, device=dev)
        self.scores = torch.empty((b, n_kv, L), dtype=torch.float32, device=dev)
        self.k_idx = torch.empty((b, n_kv, max(max_budget, 1)), dtype=torch.int32, device=dev)
        self.k_cnt = torch.empty((b, n_kv), dtype=torch.int32, device=dev)
        self.workspace = torch.empty(quoka_prefill_workspace_bytes(self.shape), dtype=torch.uint8, device=dev)

    def run(self, sparse=True):
        quoka_prefill_attn(self.shape, sparse, self.q, self.k, self.v, self.kv_lens_all, self.budgets_all, self.q_idx,
                           self.qbar, self.scores, self.k_idx, self.k_cnt, self.out, self.workspace)
        return self.out


class ChunkBuffers:
    """Device buffers for one chunk-attention problem (allocation only; torch owns the memory)."""

    def __init__(self, q, k_cache, v_cache, k_chunk, v_chunk, kv_lens, budgets, n_retain, max_budget=None,
                 score_flags=0):
        dev = q.device
        b, n_q, C, d = q.shape
        n_kv, t_max = k_cache.shape[1], k_cache.shape[2]
        self.q, self.k_cache, self.v_cache, self.k_chunk, self.v_chunk = q, k_cache, v_cache, k_chunk, v_chunk
        self.kv_lens = _ints(kv_lens, dev)
        self.budgets = _ints(budgets, dev)
        if max_budget is None:
            max_budget = min(int(max(budgets)), t_max) if len(budgets) else 0
        self.out = torch.empty_like(q)
        self.shape = make_shape(q, k_cache, k_chunk, self.out, n_retain, max_budget, score_flags)
        n_keep = self.shape.n_keep
        self.q_idx = torch.empty((b, n_q, n_keep), dtype=torch.int32, device=dev)
        self.qbar = torch.empty((b, n_kv, n_keep, d), dtype=torch.float32, device=dev)
        self.scores = torch.empty((b, n_kv, max(t_max, 1)), dtype=torch.float32, device=dev)
        self.k_idx = torch.empty((b, n_kv, max(max_budget, 1)), dtype=torch.int32, device=dev)
        self.k_cnt = torch.empty((b, n_kv), dtype=torch.int32, device=dev)
        self.lse = torch.empty((b, n_q, C), dtype=torch.float32, device=dev)
        self.workspace = torch.empty(quoka_workspace_bytes(self.shape), dtype=torch.uint8, device=dev)

    # the five stage calls and the fused convenience call, on the current stream
    def select_queries(self):
        quoka_select_queries(self.shape, self.q, self.q_idx, self.qbar, self.workspace)

    def score_keys(self):
        quoka_score_keys(self.shape, self.qbar, self.k_cache, self.kv_lens, self.scores, self.workspace)

    def topk_keys(self):
        quoka_topk_keys(self.shape, self.scores, self.kv_lens, self.budgets, self.k_idx, self.k_cnt, self.workspace)

    def select_keys(self):
        quoka_select_keys(self.shape, self.qbar, self.k_cache, self.kv_lens, self.budgets, self.scores, self.k_idx,
                          self.k_cnt, self.workspace)

    def sparse_attn(self, out=None, lse=None):
        quoka_sparse_attn(self.shape, self.q, self.k_cache, self.v_cache, self.k_idx, self.k_cnt, self.k_chunk,
                          self.v_chunk, self.out if out is None else out, self.lse if lse is None else lse,
                          self.workspace)
        return self.out if out is None else out

    def dense_attn(self, out=None, lse=None):
        quoka_dense_attn(self.shape, self.q, self.k_cache, self.v_cache, self.kv_lens, self.k_chunk, self.v_chunk,
                         self.out if out is None else out, self.lse if lse is None else lse, self.workspace)
        return self.out if out is None else out

    def chunk_attn(self):
        quoka_chunk_attn(self.shape, self.q, self.k_cache, self.v_cache, self.kv_lens, self.budgets, self.k_chunk,
                         self.v_chunk, self.q_idx, self.qbar, self.scores, self.k_idx, self.k_cnt, self.out, self.lse,
                         self.workspace)
        return self.out


class PagedCache:
    """A pool of pages and the page table of a batch (the caller's tensors, kept alive here).

    k_pages / v_pages [n_pages, n_KV, page_len, d] (torch.float8_e4m3fn with scales, or the dtype of the queries), page_table
    [b, max_pages] int32: the page of every sequence's tokens 0 .. page_len - 1, page_len .. 2 * page_len - 1 and so on.  A longer
    (or shorter) table of the same batch may take page_table's place; another pool is another PagedCache.
    """

    def __init__(self, k_pages, v_pages, page_table, k_scale=None, v_scale=None):
        self._pool, self._page_table = (k_pages, v_pages, k_scale, v_scale), page_table
        self.pages = make_pages(k_pages, v_pages, page_table, k_scale, v_scale)   # (addresses: of the tensors that are kept here)

    k_pages = property(lambda self: self._pool[0])
    v_pages = property(lambda self: self._pool[1])
    k_scale = property(lambda self: self._pool[2])
    v_scale = property(lambda self: self._pool[3])

    @property
    def page_table(self):
        return self._page_table

    @page_table.setter
    def page_table(self, page_table):
        k_pages, v_pages, k_scale, v_scale = self._pool
        pages = make_pages(k_pages, v_pages, page_table, k_scale, v_scale)
        if page_table.shape[0] != self._page_table.shape[0]:
            raise ValueError("a page table that takes another's place is of the same batch")
        self._page_table, self.pages = page_table, pages

    @classmethod
    def allocate(cls, n_pages, page_len, n_kv, head_dim, page_table, dtype=torch.float8_e4m3fn):
        """A pool of its own, on the page table's device."""
        dev = page_table.device
        shape = (n_pages, n_kv, page_len, head_dim)
        scales = [None, None]
        if dtype == torch.float8_e4m3fn:
            scales = [torch.empty(shape[:3], dtype=torch.uint8, device=dev) for _ in range(2)]
        return cls(torch.empty(shape, dtype=dtype, device=dev), torch.empty(shape, dtype=dtype, device=dev), page_table, *scales)


class PagedBuffers:
    """Device buffers for one chunk over a cache in pages (allocation only; torch owns the memory).

    kv_lens [b]: tokens cached before the chunk, none more than max_kv_len.  q [b, n_Q, C, d] and, to be written, k_chunk / v_chunk
    [b, n_KV, C, d]; whichever is not given is not needed for the calls that are made.  chunk_lens [b]: tokens of the chunk that
    each sequence has (None: all).  Key lists k_idx [b, n_KV, B_max] and k_cnt [b, n_KV] are the caller's, or, with `budgets` [b]
    and n_retain, chosen by chunk_attn().

        buf.write()        the chunk's rows into the pages
        buf.attn()         attention over all cached rows and the chunk's       (the chunk's rows have been written)
        buf.sparse_attn()  over the listed rows and the chunk's
        buf.chunk_attn()   the method's step over pages: write, read K back, select keys, sparse_attn
        buf.read(k, v)     the cached rows as contiguous tensors; either may be None
    """

    def __init__(self, cache, kv_lens, max_kv_len, q=None, k_chunk=None, v_chunk=None, chunk_lens=None, k_idx=None, k_cnt=None,
                 budgets=None, n_retain=1, score_flags=0):
        pages = cache.k_pages
        dev = pages.device
        n_kv, d = pages.shape[1], pages.shape[3]
        self.cache, self.q, self.k_chunk, self.v_chunk = cache, q, k_chunk, v_chunk
        self.kv_lens = _ints(kv_lens, dev)
        self.chunk_lens = None if chunk_lens is None else _ints(chunk_lens, dev)
        b = self.kv_lens.numel()
        if cache.page_table.shape[0] != b or (self.chunk_lens is not None and self.chunk_lens.numel() != b):
            raise ValueError("page_table, kv_lens and chunk_lens are of one batch")
        if any(t is not None and t.device != dev for t in (q, k_chunk, v_chunk, k_idx, k_cnt)):
            raise ValueError("queries, new keys and values and key lists are on the pages' device")
        self.max_kv_len = int(max_kv_len)
        new = q if q is not None else k_chunk
        dtype = new.dtype if new is not None else (torch.bfloat16 if pages.dtype == torch.float8_e4m3fn else pages.dtype)
        if dtype not in (torch.float32, torch.bfloat16):
            raise TypeError(f"unsupported dtype {dtype}")
        if pages.dtype not in (torch.float8_e4m3fn, dtype):
            raise TypeError(f"pages of {pages.dtype} with a chunk of {dtype}")
        C = 1 if new is None else new.shape[2]
        for t, heads in ((q, None), (k_chunk, n_kv), (v_chunk, n_kv)):
            if t is not None and (t.dtype != dtype or t.dim() != 4 or (t.shape[0], t.shape[2], t.shape[3]) != (b, C, d) or
                                  (heads is not None and t.shape[1] != heads)):
                raise ValueError("q [b, n_Q, C, d], k_chunk and v_chunk [b, n_KV, C, d] share batch, chunk length, head size and dtype")
        if (k_chunk is None) != (v_chunk is None) or (k_chunk is not None and k_chunk.stride() != v_chunk.stride()):
            raise ValueError("k_chunk and v_chunk are given together and share strides")
        self.budgets = None if budgets is None else _ints(budgets, dev)
        if self.budgets is not None:
            if q is None or k_chunk is None or chunk_lens is not None or k_idx is not None:
                raise ValueError("a selection of keys needs q, k_chunk and v_chunk, whole chunks and no lists of its own")
            if self.budgets.numel() != b:
                raise ValueError("kv_lens and budgets are of one batch")
            max_budget = max(0, min(int(max(budgets)), self.max_kv_len))
            k_idx = torch.empty((b, n_kv, max(max_budget, 1)), dtype=torch.int32, device=dev)
            k_cnt = torch.empty((b, n_kv), dtype=torch.int32, device=dev)
        else:
            max_budget = 0 if k_idx is None else min(k_idx.shape[2], self.max_kv_len)
        self.k_idx, self.k_cnt = k_idx, k_cnt
        if k_idx is not None and (k_cnt is None or k_idx.dtype != torch.int32 or k_cnt.dtype != torch.int32 or k_idx.shape[:2] != (b, n_kv) or
                                  not k_idx.is_contiguous() or (k_idx.shape[2] != max_budget and self.budgets is None) or
                                  k_cnt.shape != (b, n_kv) or not k_cnt.is_contiguous()):
            raise ValueError("k_idx [b, n_KV, B_max] with B_max <= max_kv_len and k_cnt [b, n_KV] are dense int32 tensors")
        self.out = None if q is None else torch.empty_like(q)
        s = self.shape = QuokaShape()
        s.batch, s.n_q_heads, s.n_kv_heads, s.head_dim = b, n_kv if q is None else q.shape[1], n_kv, d
        s.chunk_len, s.max_kv_len, s.n_retain, s.max_budget = C, self.max_kv_len, n_retain, max_budget
        s.dtype = {torch.float32: QUOKA_F32, torch.bfloat16: QUOKA_BF16}[dtype]
        s.score_flags = int(score_flags)
        s.q_stride = (ctypes.c_int64 * 3)(0, 0, d) if q is None else _strides3(q)
        s.o_stride = (ctypes.c_int64 * 3)(0, 0, d) if q is None else _strides3(self.out)
        s.kv_stride = (ctypes.c_int64 * 3)(n_kv * self.max_kv_len * d, self.max_kv_len * d, d)
        s.ck_stride = (ctypes.c_int64 * 3)(0, 0, d) if k_chunk is None else _strides3(k_chunk)
        self._read_shape, self._read_layout = None, None
        if q is not None:
            self.lse = torch.empty((b, s.n_q_heads, C), dtype=torch.float32, device=dev)
            n = quoka_paged_workspace_bytes(s)
            if self.budgets is not None:
                n = max(n, quoka_workspace_bytes(s))
                self.q_idx = torch.empty((b, s.n_q_heads, s.n_keep), dtype=torch.int32, device=dev)
                self.qbar = torch.empty((b, n_kv, s.n_keep, d), dtype=torch.float32, device=dev)
                self.scores = torch.empty((b, n_kv, max(self.max_kv_len, 1)), dtype=torch.float32, device=dev)
                self.k_back = torch.empty((b, n_kv, max(self.max_kv_len, 1), d), dtype=dtype, device=dev)
            self.workspace = torch.empty(n, dtype=torch.uint8, device=dev)

    def write(self):
        if self.k_chunk is None:
            raise ValueError("no chunk to write")
        quoka_cache_write(self.shape, self.cache.pages, self.k_chunk, self.v_chunk, self.kv_lens, self.chunk_lens)

    def read(self, k_out, v_out=None):
        """k_out, v_out [b, n_KV, max_kv_len, d], bfloat16 or float32; rows past a sequence's length stay as they are."""
        some = k_out if k_out is not None else v_out
        if some is None:
            raise ValueError("nothing to read into")
        layout = (some.dtype, some.shape, some.stride(), some.device)
        if layout != self._read_layout:   # (the description of a layout, not of a tensor: any tensors of it may follow)
            s, pages = self.shape, self.cache.k_pages
            if pages.dtype not in (torch.float8_e4m3fn, some.dtype) or some.dtype not in (torch.float32, torch.bfloat16):
                raise TypeError(f"pages of {pages.dtype} as {some.dtype}")
            if some.shape != (s.batch, s.n_kv_heads, self.max_kv_len, s.head_dim):
                raise ValueError(f"expected [b, n_KV, max_kv_len, d], got {tuple(some.shape)}")
            if some.device != pages.device:
                raise ValueError("k_out and v_out are on the pages' device")
            r = QuokaShape.from_buffer_copy(s)
            r.dtype = QUOKA_BF16 if some.dtype == torch.bfloat16 else QUOKA_F32
            r.kv_stride = _strides3(some)
            self._read_shape, self._read_layout = r, layout
        if k_out is not None and v_out is not None and (v_out.dtype, v_out.shape, v_out.stride(), v_out.device) != layout:
            raise ValueError("k_out and v_out share shape, strides, dtype and device")
        if self.max_kv_len > 0:
            quoka_cache_read(self._read_shape, self.cache.pages, self.kv_lens, k_out, v_out)

    def _attend(self, k_idx, k_cnt):
        if self.q is None:
            raise ValueError("no queries")
        quoka_paged_attn(self.shape, self.cache.pages, self.q, self.kv_lens, self.chunk_lens, k_idx, k_cnt, self.out, self.lse,
                         self.workspace)
        return self.out

    def attn(self):
        return self._attend(None, None)

    def sparse_attn(self):
        if self.k_idx is None:
            raise ValueError("no key lists")
        return self._attend(self.k_idx, self.k_cnt)

    def chunk_attn(self):
        if self.budgets is None:
            raise ValueError("no budgets")
        self.write()
        if self.max_kv_len > 0:
            quoka_cache_read(self.shape, self.cache.pages, self.kv_lens, self.k_back, None)
        quoka_select_queries(self.shape, self.q, self.q_idx, self.qbar, self.workspace)
        quoka_select_keys(self.shape, self.qbar, self.k_back, self.kv_lens, self.budgets, self.scores, self.k_idx, self.k_cnt,
                          self.workspace)
        return self.sparse_attn()
