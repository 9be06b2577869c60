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
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)   # (of a process that has tensors on one: 0.2 us less)

_LIB_NAME = "libquoka.so"
_lib: Optional[ctypes.CDLL] = None

EXPORTS = (
    "quoka_workspace_bytes", "quoka_select_queries", "quoka_score_keys", "quoka_topk_keys", "quoka_select_keys",
    "quoka_sparse_attn", "quoka_dense_attn", "quoka_chunk_attn", "quoka_prefill_workspace_bytes", "quoka_prefill_attn",
    "quoka_topk_keys_noalloc", "quoka_cache_write", "quoka_cache_read", "quoka_paged_workspace_bytes", "quoka_paged_attn",
    "quoka_cross_attn", "quoka_cache_compact", "quoka_cache_copy", "quoka_pages_workspace_bytes", "quoka_pages_resize",
    "quoka_pages_fork", "quoka_verify_workspace_bytes", "quoka_verify_draft",
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


class QuokaPageOwners(ctypes.Structure):
    _fields_ = [
        ("ref", ctypes.c_void_p), ("page_table", ctypes.c_void_p), ("held", ctypes.c_void_p),
        ("n_pages", ctypes.c_int32), ("page_len", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("batch", ctypes.c_int32),
    ]


class QuokaDraftShape(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("n_draft", ctypes.c_int32), ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("target_stride", ctypes.c_int64 * 2), ("draft_stride", ctypes.c_int64 * 2),
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
    lib.quoka_cross_attn.argtypes = [SH, PG, P, I32P, I32P, P, F32P, P, SZ, P]
    lib.quoka_cache_compact.argtypes = [SH, PG, PG, I32P, I32P, P]
    lib.quoka_cache_copy.argtypes = [SH, PG, PG, I32P, ctypes.c_int32, I32P, I32P, ctypes.c_int32, P]
    OW, DS = ctypes.POINTER(QuokaPageOwners), ctypes.POINTER(QuokaDraftShape)
    lib.quoka_pages_workspace_bytes.argtypes = [OW, ctypes.POINTER(ctypes.c_size_t)]
    lib.quoka_pages_resize.argtypes = [OW, I32P, I32P, P, SZ, P]
    lib.quoka_pages_fork.argtypes = [OW, OW, I32P, I32P, I32P, I32P, I32P, P, SZ, P]
    lib.quoka_verify_workspace_bytes.argtypes = [DS, ctypes.POINTER(ctypes.c_size_t)]
    lib.quoka_verify_draft.argtypes = [DS, P, P, I32P, F32P, I32P, I32P, I32P, P, SZ, P]
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
    return _raw_stream(_device())


def _here(index) -> None:
    """Calls go to the current device's stream: tensors of another device (its index; None: the host's) are refused."""
    if index is None:
        if torch.cuda.is_available():
            raise ValueError("tensors of no GPU")
    elif index != _device():
        raise ValueError(f"tensors of device {index}, and the current one is {_device()}")


def _is_dense(t: torch.Tensor, n: int, device: torch.device) -> bool:
    """Whether t is [n] int32, on the device, one element behind the other."""
    return t.dtype == torch.int32 and t.dim() == 1 and t.numel() == n and t.is_contiguous() and t.device == device


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


def quoka_cross_attn(shape, pages, q, kv_lens, chunk_lens, out, lse, workspace, stream=None) -> None:
    _check("quoka_cross_attn", load_library().quoka_cross_attn(
        ctypes.byref(shape), ctypes.byref(pages), _ptr(q), _ptr(kv_lens), _ptr(chunk_lens), _ptr(out), _ptr(lse), _ptr(workspace),
        workspace.numel(), _stream(stream)))


def quoka_cache_compact(shape, src, dst, k_idx, k_cnt, stream=None) -> None:
    _check("quoka_cache_compact", load_library().quoka_cache_compact(
        ctypes.byref(shape), ctypes.byref(src), ctypes.byref(dst), _ptr(k_idx), _ptr(k_cnt), _stream(stream)))


def quoka_cache_copy(shape, src, dst, parents, n_parents, first, lens, max_rows, stream=None) -> None:
    _check("quoka_cache_copy", load_library().quoka_cache_copy(
        ctypes.byref(shape), ctypes.byref(src), ctypes.byref(dst), _ptr(parents), n_parents, _ptr(first), _ptr(lens), max_rows,
        _stream(stream)))


def quoka_pages_workspace_bytes(owners: QuokaPageOwners) -> int:
    n = ctypes.c_size_t(0)
    _check("quoka_pages_workspace_bytes",
           load_library().quoka_pages_workspace_bytes(ctypes.byref(owners), ctypes.byref(n)))
    return int(n.value)


def quoka_pages_resize(owners, lens, lacking, workspace, stream=None) -> None:
    _check("quoka_pages_resize", load_library().quoka_pages_resize(
        ctypes.byref(owners), _ptr(lens), _ptr(lacking), _ptr(workspace), workspace.numel(), _stream(stream)))


def quoka_pages_fork(source, children, parents, lens, first, child_lens, lacking, workspace, stream=None) -> None:
    _check("quoka_pages_fork", load_library().quoka_pages_fork(
        ctypes.byref(source), ctypes.byref(children), _ptr(parents), _ptr(lens), _ptr(first), _ptr(child_lens), _ptr(lacking),
        _ptr(workspace), workspace.numel(), _stream(stream)))


def quoka_verify_workspace_bytes(shape: QuokaDraftShape) -> int:
    n = ctypes.c_size_t(0)
    _check("quoka_verify_workspace_bytes",
           load_library().quoka_verify_workspace_bytes(ctypes.byref(shape), ctypes.byref(n)))
    return int(n.value)


def quoka_verify_draft(shape, target, draft, tokens, uniform, draft_lens, n_accepted, tokens_out, workspace, stream=None) -> None:
    _check("quoka_verify_draft", load_library().quoka_verify_draft(
        ctypes.byref(shape), _ptr(target), _ptr(draft), _ptr(tokens), _ptr(uniform), _ptr(draft_lens), _ptr(n_accepted),
        _ptr(tokens_out), _ptr(workspace), workspace.numel(), _stream(stream)))


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
        # what rows that move in or out have to agree in, and the description of such a call
        _, n_kv, _, d = k_pages.shape
        self._rows = (k_pages.dtype, n_kv, d, k_pages.device)
        self._batch, self._device, self._index = page_table.shape[0], k_pages.device, k_pages.device.index
        self._shapes = {}

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

    def _moves(self, source, max_kv_len=0, max_budget=0):
        """The description of a call that brings rows of `source` here."""
        if source._rows != self._rows:
            if source._rows[0] != self._rows[0]:
                raise TypeError(f"pages of {source._rows[0]} into pages of {self._rows[0]}")
            raise ValueError("caches that rows move between share KV heads, head size and device")
        _here(self._index)
        s = self._shapes.get((max_kv_len, max_budget))
        if s is None:   # (never changed once it is there: other threads may be in a call)
            s, (dtype, n_kv, d, _) = QuokaShape(), self._rows
            s.batch, s.n_q_heads, s.n_kv_heads = self._batch, n_kv, n_kv
            s.head_dim, s.chunk_len, s.n_retain = d, 1, 1
            s.dtype = QUOKA_F32 if dtype == torch.float32 else QUOKA_BF16
            s.q_stride = s.kv_stride = s.ck_stride = s.o_stride = (ctypes.c_int64 * 3)(0, 0, d)
            s.max_kv_len, s.max_budget = max_kv_len, max_budget
            if len(self._shapes) == 16:
                self._shapes.clear()
            self._shapes[max_kv_len, max_budget] = s
        return s

    def compact(self, source, k_idx, k_cnt):
        """The rows that k_idx [b, n_KV, B_max] lists, k_cnt [b, n_KV] of them, from the pages of `source`, another PagedCache of the same
        batch, one behind the other into the pages of this one.  Entries are cut to the positions of the source's table, and to as many as a
        cache that is attended may have (2^24 - 1; float32 rows of 128: 2^23 - 1)."""
        dtype, n_kv, d, _ = self._rows
        lists, b, dev = k_idx.shape, self._batch, self._device
        if (k_idx.dtype != torch.int32 or k_cnt.dtype != torch.int32 or len(lists) != 3 or lists[0] != b or lists[1] != n_kv or
                k_cnt.shape != (b, n_kv) or not k_idx.is_contiguous() or not k_cnt.is_contiguous()):
            raise ValueError("k_idx [b, n_KV, B_max] and k_cnt [b, n_KV] are dense int32 tensors")
        if k_idx.device != dev or k_cnt.device != dev:
            raise ValueError("key lists are on the pages' device")
        if source._batch != b:
            raise ValueError("caches that rows move between are of one batch")
        # (the positions that the source's table has, as far as any call may have them: quoka_shape's limits, in the dtype that _moves gives it)
        theirs = source.pages
        room = min(theirs.max_pages * theirs.page_len, (1 << 24) - 1, (1 << 32) // ((4 if dtype == torch.float32 else 2) * d) - 1)
        quoka_cache_compact(self._moves(source, room, lists[2]), theirs, self.pages, k_idx, k_cnt)

    def copy(self, source, parents=None, first=None, lens=None, max_rows=None):
        """Rows first[b] .. lens[b] - 1 of sequence parents[b] of `source`, another PagedCache, to the same positions of sequence b.  (After
        PagedSequences.fork: its parents, first and lens.)  parents None: sequence b itself; first None: 0.  No sequence has more than
        max_rows of them (None: page_len, what a fork leaves to be copied)."""
        dev, b, n_parents = self._device, self._batch, source._batch
        if lens is None:
            raise ValueError("no lengths")
        for t in (parents, first, lens):
            if t is not None and not _is_dense(t, b, dev):
                raise ValueError("parents, first and lens [b] are dense int32 tensors on the pages' device")
        if parents is None and n_parents < b:
            raise ValueError("a source of fewer sequences needs parents")
        quoka_cache_copy(self._moves(source), source.pages, self.pages, parents, n_parents, first, lens,
                         self.pages.page_len if max_rows is None else int(max_rows))


class PagedBuffers:
    """Device buffers for one chunk over a cache in pages (allocation only; torch owns the memory).

    kv_lens [b]: tokens cached before the chunk, none more than max_kv_len.  q [b, n_Q, C, d] and, to be written, k_chunk / v_chunk
    [b, n_KV, C, d]; whichever is not given is not needed for the calls that are made.  chunk_lens [b]: tokens of the chunk that
    each sequence has (None: all).  Key lists k_idx [b, n_KV, B_max] and k_cnt [b, n_KV] are the caller's, or, with `budgets` [b]
    and n_retain, chosen by chunk_attn().

        buf.write()        the chunk's rows into the pages
        buf.attn()         attention over all cached rows and the chunk's       (the chunk's rows have been written)
        buf.sparse_attn()  over the listed rows and the chunk's
        buf.cross_attn()   over all cached rows and no others: kv_lens states of an encoder that the cache holds
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

    def cross_attn(self):
        if self.q is None:
            raise ValueError("no queries")
        _here(self.cache._index)
        quoka_cross_attn(self.shape, self.cache.pages, self.q, self.kv_lens, self.chunk_lens, self.out, self.lse, self.workspace)
        return self.out

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


class PagedSequences:
    """The pages that the sequences of a batch hold (the caller's tensors, kept alive here).

    ref [n_pages] int32: holders of every page of the pool, over all batches, 0 for a free one.  page_table [b, max_pages] int32, held [b]
    int32: entries of each row that are in use.  page_table is what a PagedCache (of every layer) takes.

        seqs.resize(lens)                   pages for the first lens[b] positions of every sequence; what lies behind is given back
        children.fork(seqs, parents, lens)  children go on from sequences parents[b] of `seqs`, of which lens tokens are cached: whole pages
                                            are shared, and PagedCache.copy(.., parents, children.first, children.lens) brings the rest

    lacking [1]: how many pages the last call would have needed beyond those that were free.  first, lens [b]: of the last fork.
    A sequence that is cut back into a page that it shares goes on by a fork to that length, not by writing there.
    """

    def __init__(self, ref, page_table, held, page_len):
        for t, dims in ((ref, 1), (page_table, 2), (held, 1)):
            if t.dtype != torch.int32 or t.dim() != dims or not t.is_contiguous() or t.device != ref.device:
                raise ValueError("ref [n_pages], page_table [b, max_pages] and held [b] are dense int32 tensors on one device")
        if held.shape[0] != page_table.shape[0]:
            raise ValueError("page_table and held are of one batch")
        self._tensors, self._device, self._index = (ref, page_table, held), ref.device, ref.device.index
        o = self.owners = QuokaPageOwners()   # (addresses: of the tensors that are kept here)
        o.ref, o.page_table, o.held = ref.data_ptr(), page_table.data_ptr(), held.data_ptr()
        o.n_pages, o.page_len, o.max_pages, o.batch = ref.shape[0], int(page_len), page_table.shape[1], page_table.shape[0]
        self.workspace = torch.empty(quoka_pages_workspace_bytes(o), dtype=torch.uint8, device=ref.device)
        self.lacking = torch.zeros(1, dtype=torch.int32, device=ref.device)
        self.first, self.lens = (torch.zeros_like(held) for _ in range(2))

    ref = property(lambda self: self._tensors[0])
    page_table = property(lambda self: self._tensors[1])
    held = property(lambda self: self._tensors[2])

    @classmethod
    def allocate(cls, n_pages, page_len, batch, max_pages, device="cuda"):
        """Sequences that hold nothing, over a pool of which every page is free."""
        ref = torch.zeros(n_pages, dtype=torch.int32, device=device)
        return cls._empty(ref, page_len, batch, max_pages)

    def another(self, batch, max_pages=None):
        """Sequences of another batch that hold nothing, over the same pool."""
        o = self.owners
        return self._empty(self.ref, o.page_len, batch, o.max_pages if max_pages is None else max_pages)

    @classmethod
    def _empty(cls, ref, page_len, batch, max_pages):
        table = torch.full((batch, max_pages), -1, dtype=torch.int32, device=ref.device)
        return cls(ref, table, torch.zeros(batch, dtype=torch.int32, device=ref.device), page_len)

    def _lens(self, x, n):
        if not _is_dense(x, n, self._device):
            raise ValueError("lengths and parents are dense int32 tensors, one for each sequence, on the pages' device")
        return x

    def resize(self, lens):
        _here(self._index)
        o = self.owners
        quoka_pages_resize(o, self._lens(lens, o.batch), self.lacking, self.workspace)

    def fork(self, source, parents, lens):
        """parents [b]: sequences of `source` (others: no parent).  lens: cached tokens of the sequences of `source`, each."""
        _here(self._index)
        o, theirs = self.owners, source.owners
        quoka_pages_fork(theirs, o, self._lens(parents, o.batch), self._lens(lens, theirs.batch), self.first, self.lens, self.lacking,
                         self.workspace)


class DraftBuffers:
    """Device buffers for the verification of drafted tokens (allocation only; torch owns the memory).

    target [b, n + 1, vocab]: the target's probabilities of each of the n drafted tokens and of the one behind them, bfloat16 or float32;
    draft [b, n, vocab]: what the tokens were drawn from (None: they were looked up); tokens [b, n] int32; uniform [b, n + 1] float32:
    random numbers from [0, 1); draft_lens [b]: tokens that each sequence has drafted (None: n).

        n_accepted, tokens_out = buf.verify()   [b] and [b, n + 1] int32: accepted tokens, the one after them, and -1
    """

    def __init__(self, target, tokens, uniform, draft=None, draft_lens=None):
        dev = target.device
        if target.dtype not in (torch.float32, torch.bfloat16):
            raise TypeError(f"unsupported dtype {target.dtype}")
        if draft is not None and draft.dtype != target.dtype:
            raise TypeError(f"drafts of {draft.dtype} with a target of {target.dtype}")
        if target.dim() != 3 or target.shape[1] < 2:
            raise ValueError("target [b, n + 1, vocab], n >= 1")
        b, n, vocab = target.shape[0], target.shape[1] - 1, target.shape[2]
        if draft is not None and draft.shape != (b, n, vocab):
            raise ValueError("target [b, n + 1, vocab] and draft [b, n, vocab] share batch, tokens and vocabulary")
        if any(t is not None and t.stride(2) != 1 and vocab > 1 for t in (target, draft)):
            raise ValueError("probabilities of a token are contiguous")
        if tokens.dtype != torch.int32 or tokens.shape != (b, n) or not tokens.is_contiguous():
            raise ValueError("tokens [b, n] is a dense int32 tensor")
        if uniform.dtype != torch.float32 or uniform.shape != (b, n + 1) or not uniform.is_contiguous():
            raise ValueError("uniform [b, n + 1] is a dense float32 tensor")
        if any(t is not None and t.device != dev for t in (draft, tokens, uniform)):
            raise ValueError("probabilities, tokens and random numbers are on one device")
        self.target, self.draft, self.tokens, self.uniform = target, draft, tokens, uniform
        self._index = dev.index
        self.draft_lens = None if draft_lens is None else _ints(draft_lens, dev)
        if self.draft_lens is not None and self.draft_lens.numel() != b:
            raise ValueError("target and draft_lens are of one batch")
        s = self.shape = QuokaDraftShape()
        s.batch, s.n_draft, s.vocab = b, n, vocab
        s.dtype = QUOKA_BF16 if target.dtype == torch.bfloat16 else QUOKA_F32
        s.target_stride = (ctypes.c_int64 * 2)(target.stride(0), target.stride(1))
        s.draft_stride = (ctypes.c_int64 * 2)(*(draft.stride()[:2] if draft is not None else (0, 0)))
        self.n_accepted = torch.empty(b, dtype=torch.int32, device=dev)
        self.tokens_out = torch.empty((b, n + 1), dtype=torch.int32, device=dev)
        self.workspace = torch.empty(quoka_verify_workspace_bytes(s), dtype=torch.uint8, device=dev)

    def verify(self):
        _here(self._index)
        quoka_verify_draft(self.shape, self.target, self.draft, self.tokens, self.uniform, self.draft_lens, self.n_accepted,
                           self.tokens_out, self.workspace)
        return self.n_accepted, self.tokens_out
