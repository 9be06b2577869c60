"""What the entry points for caches in pages refuse, and what their structure looks like, without a GPU: nothing is launched."""
import ctypes

import pytest
import torch

import paper_2602_08722_amd as pk
from tests.test_abi import _shape

AT, WS, BIG = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x10000), ctypes.c_size_t(1 << 40)   # never followed


def _pages(**kw):
    p = pk.QuokaPages()
    vals = dict(k=0x1000, v=0x2000, k_scale=0x3000, v_scale=0x3001, page_table=0x4000, n_pages=100, page_len=16, max_pages=80,
                format=pk.QUOKA_PAGES_FP8)
    stride = kw.pop("stride", (2 * 16 * 128, 16 * 128, 128))
    vals.update(kw)
    for k, v in vals.items():
        setattr(p, k, v)
    p.stride = (ctypes.c_int64 * 3)(*stride)
    return p


def _calls(shape, pages):
    """Status of each entry point with otherwise valid arguments that lead to a refusal."""
    lib = pk.load_library()
    s, p = ctypes.byref(shape), None if pages is None else ctypes.byref(pages)
    return (lib.quoka_cache_write(s, p, AT, AT, AT, None, None), lib.quoka_cache_read(s, p, AT, AT, AT, None),
            lib.quoka_paged_attn(s, p, AT, AT, None, None, None, AT, None, WS, BIG, None))


def test_struct_layout():
    # five pointers, three int64, four int32
    assert ctypes.sizeof(pk.QuokaPages) == 5 * 8 + 3 * 8 + 4 * 4
    assert pk.QuokaPages.stride.offset == 40 and pk.QuokaPages.n_pages.offset == 64
    lib = pk.load_library()
    assert lib.quoka_version() >= 200


@pytest.mark.parametrize("kw,code", [
    (dict(k=0), 1), (dict(v=0), 1), (dict(page_table=0), 1), (dict(k_scale=0), 1), (dict(v_scale=0), 1),
    (dict(k=0x1008), 1), (dict(v=0x1004), 1),
    (dict(n_pages=0), 1), (dict(max_pages=0), 1), (dict(page_len=0), 1), (dict(page_len=48), 1), (dict(page_len=-16), 1),
    (dict(page_len=131072), 2), (dict(format=2), 2), (dict(format=-1), 2),
    (dict(max_pages=62), 1),                                          # 62 * 16 tokens for 1000
    (dict(stride=(4096, 2048, 64)), 1), (dict(stride=(4096, 2048, 136)), 1), (dict(stride=(4104, 2048, 128)), 1),
    (dict(stride=(4096, -2048, 128)), 1),
])
def test_bad_pages_are_refused(kw, code):
    assert _calls(_shape(pk), _pages(**kw)) == (code,) * 3


def test_no_pages_and_bad_shapes_are_refused():
    assert _calls(_shape(pk), None) == (1,) * 3
    for kw, code in ((dict(head_dim=96), 2), (dict(dtype=7), 2), (dict(batch=0), 1), (dict(n_q_heads=7), 1), (dict(chunk_len=8193), 2)):
        assert _calls(_shape(pk, **kw), _pages()) == (code,) * 3
    n = ctypes.c_size_t(0)
    assert pk.load_library().quoka_paged_workspace_bytes(ctypes.byref(_shape(pk, head_dim=32)), ctypes.byref(n)) == 2
    assert pk.load_library().quoka_paged_workspace_bytes(ctypes.byref(_shape(pk)), None) == 1


def test_bad_pointers_and_workspaces_are_refused():
    lib, p = pk.load_library(), ctypes.byref(_pages())
    odd, null = ctypes.c_void_p(0x1004), None
    s = ctypes.byref(_shape(pk))
    for args in ((null, AT, AT), (AT, null, AT), (AT, AT, null), (odd, AT, AT), (AT, odd, AT)):
        assert lib.quoka_cache_write(s, p, *args, None, None) == 1
    for args in ((null, AT, AT), (AT, null, null), (AT, odd, AT), (AT, AT, odd)):
        assert lib.quoka_cache_read(s, p, *args, None) == 1
    for q, lens, idx, cnt, out, ws, code in ((null, AT, null, null, AT, WS, 1), (AT, null, null, null, AT, WS, 1),
                                             (AT, AT, AT, null, AT, WS, 1), (AT, AT, null, null, null, WS, 1),
                                             (odd, AT, null, null, AT, WS, 1), (AT, AT, null, null, odd, WS, 1),
                                             (AT, AT, null, null, AT, null, 1), (AT, AT, null, null, AT, ctypes.c_void_p(0x10010), 3)):
        assert lib.quoka_paged_attn(s, p, q, lens, None, idx, cnt, out, None, ws, BIG, None) == code
    need = ctypes.c_size_t(0)
    assert lib.quoka_paged_workspace_bytes(s, ctypes.byref(need)) == 0 and need.value > 0 and need.value % 256 == 0
    assert lib.quoka_paged_attn(s, p, AT, AT, None, None, None, AT, None, WS, ctypes.c_size_t(need.value - 1), None) == 3


def _cache(dtype=torch.float8_e4m3fn, batch=2, n_kv=2, d=64, page_len=16, cols=4):
    return pk.PagedCache.allocate(10, page_len, n_kv, d, torch.zeros((batch, cols), dtype=torch.int32), dtype=dtype)


def test_the_binding_refuses_tensors_that_do_not_fit(monkeypatch):
    monkeypatch.setattr(pk.binding, "_stream", lambda stream: None)   # (no GPU to ask; every call below is refused ahead of it)
    pool = torch.zeros(10, 2, 16, 64, dtype=torch.bfloat16)
    table = torch.zeros(2, 4, dtype=torch.int32)
    scale = torch.zeros(10, 2, 16, dtype=torch.uint8)
    with pytest.raises(TypeError):
        pk.make_pages(pool.half(), pool.half(), table)
    for args in ((pool, pool[:5], table), (pool, pool.float(), table), (pool, pool, table.long()), (pool, pool, table[0]),
                 (pool.to(torch.float8_e4m3fn),) * 2 + (table,), (pool.to(torch.float8_e4m3fn),) * 2 + (table, scale, scale[:, :, :8])):
        with pytest.raises(ValueError):
            pk.make_pages(*args)
    cache = _cache()
    q, kc = torch.zeros(2, 4, 3, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16)
    pk.PagedBuffers(cache, [1, 2], 60, q=q, k_chunk=kc, v_chunk=kc)
    with pytest.raises(TypeError):   # 16-bit pages with a float32 chunk
        pk.PagedBuffers(_cache(torch.bfloat16), [1, 2], 60, q=q.float())
    idx, cnt = torch.zeros(2, 2, 5, dtype=torch.int32), torch.zeros(2, 2, dtype=torch.int32)
    for how in (dict(k_chunk=kc), dict(q=q[:1]), dict(q=q, k_chunk=kc[:, :, :2], v_chunk=kc[:, :, :2]), dict(q=q, k_chunk=q, v_chunk=q),
                dict(q=q, chunk_lens=[1]), dict(q=q, k_idx=idx), dict(q=q, k_idx=idx.long(), k_cnt=cnt), dict(q=q, k_idx=idx[:, :, ::2], k_cnt=cnt),
                dict(q=q, budgets=[3, 3]), dict(q=q, k_chunk=kc, v_chunk=kc, budgets=[3, 3], chunk_lens=[1, 1]),
                dict(k_chunk=kc, v_chunk=kc.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3))):
        with pytest.raises(ValueError):
            pk.PagedBuffers(cache, [1, 2], 60, **how)
    with pytest.raises(ValueError):
        pk.PagedBuffers(cache, [1, 2, 3], 60)
    with pytest.raises(pk.QuokaError):   # a table of 64 positions
        pk.PagedBuffers(cache, [1, 2], 65, k_chunk=kc, v_chunk=kc).write()
    bare = pk.PagedBuffers(cache, [1, 2], 60)
    for call in (bare.write, bare.attn, bare.sparse_attn, bare.chunk_attn):
        with pytest.raises(ValueError):
            call()
    out = torch.zeros(2, 2, 60, 64, dtype=torch.bfloat16)
    for args, error in (((out.half(),), TypeError), ((out[:, :, :59],), ValueError), ((out, out.float()), ValueError)):
        with pytest.raises(error):
            bare.read(*args)
    with pytest.raises(TypeError):
        pk.PagedBuffers(_cache(torch.float32), [1, 2], 60).read(out)


def _pages_accepted(shape, pages):
    """Whether the entry points take the pages: with a null pointer, which they look at last, the refusal is another one."""
    lib = pk.load_library()
    s, p = ctypes.byref(shape), ctypes.byref(pages)
    codes = (lib.quoka_cache_write(s, p, None, AT, AT, None, None), lib.quoka_cache_read(s, p, None, AT, AT, None),
             lib.quoka_paged_attn(s, p, None, AT, None, None, None, AT, None, WS, BIG, None))
    assert codes in ((1,) * 3, (2,) * 3)
    return codes[0] == 1


@pytest.mark.parametrize("fmt,dtype,es", [("fp8", "bf16", 1), ("fp8", "f32", 1), ("raw", "bf16", 2), ("raw", "f32", 4)])
@pytest.mark.parametrize("d,token", [(128, 144), (128, 128), (64, 80), (64, 208)])
def test_the_last_row_of_a_head_ends_within_64_gib(fmt, dtype, es, d, token):
    """Pages of 16 tokens; the page stride brings the end of the last row to 64 GiB exactly, then one step of 16 elements past it."""
    shape = _shape(pk, head_dim=d, dtype=pk.QUOKA_BF16 if dtype == "bf16" else pk.QUOKA_F32)
    limit = (64 << 30) // es
    for n_pages in (2, 5, 65):
        # (the page stride is a multiple of 16 elements: n_pages - 1 divides what is left of the limit, or the next smaller one is taken)
        room = limit - d - 15 * token
        stride = room // (n_pages - 1) // 16 * 16
        how = dict(n_pages=n_pages, max_pages=63, format=pk.QUOKA_PAGES_FP8 if fmt == "fp8" else pk.QUOKA_PAGES_RAW)
        assert _pages_accepted(shape, _pages(stride=(stride, 16 * token, token), **how))
        assert not _pages_accepted(shape, _pages(stride=(stride + 16, 16 * token, token), **how))


def test_the_number_of_scales_and_of_keys_is_limited():
    # 2^32 scales: 2 KV heads, 65536 tokens a page, 2^15 pages (and rows that lie in the same places, for a span below 64 GiB)
    flat = dict(stride=(128, 128, 128), page_len=65536, max_pages=1)
    assert _pages_accepted(_shape(pk), _pages(n_pages=1 << 15, **flat))
    assert not _pages_accepted(_shape(pk), _pages(n_pages=(1 << 15) + 1, **flat))
    # batch * (max_kv_len + chunk_len + 32) below 2^36
    lib = pk.load_library()
    pages = ctypes.byref(_pages(n_pages=100, page_len=65536, max_pages=256))
    for batch, chunk, code in ((4096, 63, 1), (4096, 64, 2), (4097, 63, 2), (4095, 64, 1)):
        shape = _shape(pk, batch=batch, max_kv_len=(1 << 24) - 96, chunk_len=chunk, max_budget=0)
        shape.kv_stride = (ctypes.c_int64 * 3)(0, 0, 128)
        assert lib.quoka_paged_attn(ctypes.byref(shape), pages, AT, AT, None, None, None, AT, None, None, BIG, None) == code


def test_a_cache_describes_the_tensors_that_it_has():
    """A page table may be replaced (sequences grow), and calls see the new one; one that does not fit is refused and changes
    nothing; pools stay what they are."""
    cache = _cache()
    first = cache.page_table
    assert cache.pages.page_table == first.data_ptr() and cache.pages.max_pages == 4
    grown = torch.zeros((2, 9), dtype=torch.int32)
    cache.page_table = grown
    assert cache.page_table is grown
    assert cache.pages.page_table == grown.data_ptr() and cache.pages.max_pages == 9
    for bad in (grown[0], grown.long(), grown[:, ::2], torch.zeros((3, 9), dtype=torch.int32), torch.zeros((1, 9), dtype=torch.int32)):
        with pytest.raises(ValueError):
            cache.page_table = bad
        assert cache.page_table is grown and cache.pages.page_table == grown.data_ptr() and cache.pages.max_pages == 9
    for name in ("k_pages", "v_pages", "k_scale", "v_scale"):
        held = getattr(cache, name)
        with pytest.raises(AttributeError):
            setattr(cache, name, held.clone())
        assert getattr(cache, name) is held and getattr(cache.pages, name[:1] if name.endswith("pages") else name) == held.data_ptr()


def test_lengths_and_budgets_may_be_views_of_any_strides():
    """Kernels read dense arrays: what lies between the entries of a strided view must not be taken for lengths."""
    cache = _cache()
    q, kc = torch.zeros(2, 4, 3, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16)
    pairs = torch.tensor([[5, 100], [6, 200]], dtype=torch.int32)
    for view in (pairs[:, 0], pairs.t()[0], pairs[:, :1], pairs[:, 0].flip(0).flip(0)):
        buf = pk.PagedBuffers(cache, view, 60, q=q, k_chunk=kc, v_chunk=kc, chunk_lens=view)
        for t in (buf.kv_lens, buf.chunk_lens):
            assert t.is_contiguous() and t.flatten().tolist() == [5, 6]
        buf = pk.PagedBuffers(cache, view, 60, q=q, k_chunk=kc, v_chunk=kc, budgets=view)
        assert buf.budgets.is_contiguous() and buf.budgets.flatten().tolist() == [5, 6] and buf.shape.max_budget == 6
    alone = torch.tensor([3], dtype=torch.int32).expand(2)   # one length for all
    buf = pk.PagedBuffers(cache, alone, 60, q=q)
    assert buf.kv_lens.is_contiguous() and buf.kv_lens.tolist() == [3, 3]
    dense = torch.tensor([5, 6], dtype=torch.int32)          # a program's own tensor stays the one that is read
    assert pk.PagedBuffers(cache, dense, 60, q=q).kv_lens.data_ptr() == dense.data_ptr()
    one = torch.zeros(2, 2, 60, 64, dtype=torch.bfloat16)
    buf = pk.ChunkBuffers(q, one, one, kc, kc, pairs[:, 0], pairs[:, 0], 1)
    assert buf.kv_lens.is_contiguous() and buf.budgets.is_contiguous() and buf.kv_lens.tolist() == buf.budgets.tolist() == [5, 6]


def test_budgets_of_another_batch_are_refused():
    q, kc = torch.zeros(2, 4, 3, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16)
    for budgets in ([3], [3, 3, 3]):
        with pytest.raises(ValueError):
            pk.PagedBuffers(_cache(), [1, 2], 60, q=q, k_chunk=kc, v_chunk=kc, budgets=budgets)


def test_tensors_on_another_device_are_refused():
    """An address is read on the GPU whatever device it is of: a list left on the host would fault there.  (Tensors without storage stand for
    those of another device.)"""
    table, scale = torch.zeros((2, 4), dtype=torch.int32), torch.zeros(10, 2, 16, dtype=torch.uint8)
    pool = torch.zeros(10, 2, 16, 64, dtype=torch.bfloat16)
    pool8 = pool.to(torch.float8_e4m3fn)
    there = lambda x: x.to("meta")  # noqa: E731
    for args in ((pool, there(pool), table), (pool, pool, there(table)), (pool8, pool8, table, scale, there(scale)),
                 (pool8, pool8, table, there(scale), scale)):
        with pytest.raises(ValueError):
            pk.make_pages(*args)
    cache = _cache()
    with pytest.raises(ValueError):
        cache.page_table = there(table)
    q, kc = torch.zeros(2, 4, 3, 64, dtype=torch.bfloat16), torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16)
    idx, cnt = torch.zeros(2, 2, 5, dtype=torch.int32), torch.zeros(2, 2, dtype=torch.int32)
    for how in (dict(q=there(q)), dict(q=q, k_chunk=there(kc), v_chunk=kc), dict(q=q, k_chunk=kc, v_chunk=there(kc)),
                dict(q=q, k_idx=there(idx), k_cnt=cnt), dict(q=q, k_idx=idx, k_cnt=there(cnt))):
        with pytest.raises(ValueError):
            pk.PagedBuffers(cache, [1, 2], 60, **how)
    out = torch.zeros(2, 2, 60, 64, dtype=torch.bfloat16)
    for args in ((there(out),), (out, there(out)), (None, there(out))):
        with pytest.raises(ValueError):
            pk.PagedBuffers(cache, [1, 2], 60).read(*args)


def test_chunks_of_other_dtypes_are_refused_as_such():
    for dtype in (torch.float16, torch.float64):
        for how in (dict(q=torch.zeros(2, 4, 3, 64, dtype=dtype)), dict(k_chunk=torch.zeros(2, 2, 3, 64, dtype=dtype), v_chunk=torch.zeros(2, 2, 3, 64, dtype=dtype))):
            with pytest.raises(TypeError):
                pk.PagedBuffers(_cache(), [1, 2], 60, **how)


def test_a_read_into_nothing_is_refused():
    with pytest.raises(ValueError):
        pk.PagedBuffers(_cache(), [1, 2], 60).read(None)
