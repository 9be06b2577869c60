"""What cross attention, the verification of drafted tokens and the upkeep of pages refuse, and what their structures look like, without a
GPU: nothing is launched."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2602_08722_amd as pk
from tests import generation_plain as G
from tests.test_abi import _shape
from tests.test_paged_abi import _cache, _pages

AT, OTHER, WS, BIG = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x2000), ctypes.c_void_p(0x10000), ctypes.c_size_t(1 << 40)   # never followed
ODD, NULL = ctypes.c_void_p(0x1002), None


@pytest.fixture(autouse=True)
def no_stream(monkeypatch):
    monkeypatch.setattr(pk.binding, "_stream", lambda stream: None)   # (no GPU to ask; every call below is refused ahead of it)


def _owners(**kw):
    o = pk.QuokaPageOwners()
    for k, v in dict(dict(ref=0x1000, page_table=0x2000, held=0x3000, n_pages=100, page_len=16, max_pages=8, batch=3), **kw).items():
        setattr(o, k, v)
    return o


def _drafts(**kw):
    s = pk.QuokaDraftShape()
    strides = {k: kw.pop(k, (4000, 1000)) for k in ("target_stride", "draft_stride")}
    for k, v in dict(dict(batch=2, n_draft=3, vocab=1000, dtype=pk.QUOKA_F32), **kw).items():
        setattr(s, k, v)
    for k, v in strides.items():
        setattr(s, k, (ctypes.c_int64 * 2)(*v))
    return s


def test_struct_layouts():
    assert ctypes.sizeof(pk.QuokaPageOwners) == 3 * 8 + 4 * 4 and pk.QuokaPageOwners.n_pages.offset == 24
    assert ctypes.sizeof(pk.QuokaDraftShape) == 4 * 4 + 4 * 8 and pk.QuokaDraftShape.target_stride.offset == 16


# ---- cross attention and moves of rows --------------------------------------------------------------------------------

def _calls(shape, pages):
    lib = pk.load_library()
    s, p = ctypes.byref(shape), None if pages is None else ctypes.byref(pages)
    good = ctypes.byref(_pages(page_table=0x5000))
    return (lib.quoka_cross_attn(s, p, AT, AT, None, AT, None, WS, BIG, None), lib.quoka_cache_compact(s, p, good, AT, AT, None),
            lib.quoka_cache_compact(s, good, p, AT, AT, None), lib.quoka_cache_copy(s, p, good, AT, 2, AT, AT, 16, None),
            lib.quoka_cache_copy(s, good, p, AT, 2, AT, AT, 16, None))


@pytest.mark.parametrize("kw,code", [
    (dict(k=0), 1), (dict(v=0), 1), (dict(page_table=0), 1), (dict(k_scale=0), 1), (dict(k=0x1008), 1), (dict(n_pages=0), 1), (dict(max_pages=0), 1),
    (dict(page_len=48), 1), (dict(page_len=131072), 2), (dict(format=2), 2), (dict(stride=(4096, 2048, 64)), 1), (dict(stride=(4104, 2048, 128)), 1),
])
def test_bad_pages_are_refused(kw, code):
    assert _calls(_shape(pk), _pages(**kw)) == (code,) * 5


def test_no_pages_and_bad_shapes_are_refused():
    assert _calls(_shape(pk), None) == (1,) * 5
    for kw, code in ((dict(head_dim=96), 2), (dict(dtype=7), 2), (dict(batch=0), 1), (dict(n_q_heads=7), 1)):
        assert _calls(_shape(pk, **kw), _pages()) == (code,) * 5


def test_tables_hold_what_is_asked_of_them():
    """max_kv_len 1000 and max_budget 100 in pages of 16: 63 pages of the states and of the source, 7 of what lists go to."""
    lib, s = pk.load_library(), ctypes.byref(_shape(pk))
    p = {n: ctypes.byref(_pages(max_pages=n, page_table=0x4000 + n)) for n in (1, 6, 62, 63)}
    assert lib.quoka_cross_attn(s, p[62], AT, AT, None, AT, None, WS, BIG, None) == 1
    assert lib.quoka_cache_compact(s, p[62], p[63], AT, AT, None) == 1
    assert lib.quoka_cache_compact(s, p[63], p[6], AT, AT, None) == 1


def test_bad_pointers_and_arguments_are_refused():
    lib, s = pk.load_library(), ctypes.byref(_shape(pk))
    a, b = ctypes.byref(_pages()), ctypes.byref(_pages(page_table=0x5000))
    for q, lens, out, ws, code in ((NULL, AT, AT, WS, 1), (AT, NULL, AT, WS, 1), (AT, AT, NULL, WS, 1), (AT, AT, AT, NULL, 1), (ODD, AT, AT, WS, 1),
                                   (AT, AT, ODD, WS, 1), (AT, AT, AT, ctypes.c_void_p(0x10010), 3)):
        assert lib.quoka_cross_attn(s, a, q, lens, None, out, None, ws, BIG, None) == code
    need = ctypes.c_size_t(0)
    assert lib.quoka_paged_workspace_bytes(s, ctypes.byref(need)) == 0
    assert lib.quoka_cross_attn(s, a, AT, AT, None, AT, None, WS, ctypes.c_size_t(need.value - 1), None) == 3
    for args in ((NULL, AT), (AT, NULL)):
        assert lib.quoka_cache_compact(s, a, b, *args, None) == 1
    assert lib.quoka_cache_compact(s, a, a, AT, AT, None) == 1                       # onto itself
    raw = ctypes.byref(_pages(format=pk.QUOKA_PAGES_RAW, page_table=0x5000))
    assert lib.quoka_cache_compact(s, a, raw, AT, AT, None) == 1                     # another format
    for parents, n, lens, rows, code in ((AT, 2, NULL, 16, 1), (AT, 0, AT, 16, 1), (AT, 2, AT, -1, 1), (NULL, 0, AT, 16, 1), (AT, 2, AT, 1 << 24, 2)):
        assert lib.quoka_cache_copy(s, a, b, parents, n, AT, lens, rows, None) == code
    assert lib.quoka_cache_copy(s, a, raw, AT, 2, AT, AT, 16, None) == 1 and lib.quoka_cache_copy(s, a, a, AT, 2, AT, AT, 16, None) == 1
    assert lib.quoka_cache_copy(s, a, b, AT, 2, AT, AT, 0, None) == 0                # no rows: nothing to launch
    assert lib.quoka_cache_compact(ctypes.byref(_shape(pk, max_budget=0)), a, b, None, AT, None) == 0


# quoka_paged_attn in float32: partials of 32 rows of d outputs and two sums each, one for every row block and eight units of 32 keys, at most 512
def _attn_bytes(s):
    blocks = s.batch * s.n_kv_heads * -(-s.chunk_len * (s.n_q_heads // s.n_kv_heads) // 32)
    shares = min(-(-(-(-s.max_kv_len // 32) + -(-s.chunk_len // 32)) // 8), 64)
    return -(-min(blocks * shares, 512) * 32 * (s.head_dim + 2) * 4 // 256) * 256


@pytest.mark.parametrize("kw,parts", [
    (dict(), 0), (dict(batch=8, chunk_len=1, max_kv_len=40000, head_dim=64), 0), (dict(n_q_heads=32, n_kv_heads=8, chunk_len=512, max_kv_len=8192), 0),
    (dict(chunk_len=540, max_kv_len=5000), 680), (dict(batch=2, chunk_len=270, max_kv_len=5000, head_dim=64), 680),
])
def test_a_float32_workspace_is_as_large_as_its_call_wants(kw, parts):
    """parts: of cross attention, where they are more than those of attention over the chunk's own rows too."""
    lib, shape, n = pk.load_library(), _shape(pk, dtype=pk.QUOKA_F32, **kw), ctypes.c_size_t(0)
    s, need = ctypes.byref(shape), max(_attn_bytes(shape), parts * 32 * (shape.head_dim + 2) * 4)
    assert lib.quoka_paged_workspace_bytes(s, ctypes.byref(n)) == 0 and n.value == need
    pages = ctypes.byref(_pages(max_pages=1 << 16))
    less = ctypes.c_size_t(_attn_bytes(shape) - 1)
    assert lib.quoka_paged_attn(s, pages, AT, AT, None, None, None, AT, None, WS, less, None) == 3
    if parts:
        assert lib.quoka_cross_attn(s, pages, AT, AT, None, AT, None, WS, ctypes.c_size_t(need - 1), None) == 3


# ---- who holds the pages ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kw,code", [
    (dict(ref=0), 1), (dict(page_table=0), 1), (dict(held=0), 1), (dict(n_pages=0), 1), (dict(max_pages=0), 1), (dict(batch=0), 1),
    (dict(page_len=0), 1), (dict(page_len=24), 1), (dict(page_len=-16), 1), (dict(page_len=1 << 17), 2), (dict(batch=65536), 2),
    (dict(n_pages=(1 << 30) + 1), 2), (dict(batch=1 << 15, max_pages=1 << 16), 2),
])
def test_bad_owners_are_refused(kw, code):
    lib, bad, good, n = pk.load_library(), ctypes.byref(_owners(**kw)), ctypes.byref(_owners(page_table=0x7000, held=0x8000)), ctypes.c_size_t(0)
    assert lib.quoka_pages_workspace_bytes(bad, ctypes.byref(n)) == code
    assert lib.quoka_pages_resize(bad, AT, AT, WS, BIG, None) == code
    for pair in ((bad, good), (good, bad)):
        assert lib.quoka_pages_fork(*pair, AT, AT, OTHER, OTHER, AT, WS, BIG, None) == code


def test_owners_that_do_not_belong_together_and_bad_pointers_are_refused():
    lib, o, n = pk.load_library(), _owners(), ctypes.c_size_t(0)
    at = ctypes.byref(o)
    assert lib.quoka_pages_workspace_bytes(None, ctypes.byref(n)) == 1 and lib.quoka_pages_workspace_bytes(at, None) == 1
    assert lib.quoka_pages_workspace_bytes(at, ctypes.byref(n)) == 0 and n.value % 256 == 0 and n.value > 0
    for args, code in (((NULL, AT, WS, BIG), 1), ((AT, NULL, WS, BIG), 1), ((AT, AT, NULL, BIG), 1), ((AT, AT, ctypes.c_void_p(0x10010), BIG), 3),
                       ((AT, AT, WS, ctypes.c_size_t(n.value - 1)), 3)):
        assert lib.quoka_pages_resize(at, *args, None) == code
    for kw in (dict(), dict(page_table=0x7000), dict(held=0x8000), dict(page_table=0x7000, held=0x8000, ref=0x9000),
               dict(page_table=0x7000, held=0x8000, page_len=32), dict(page_table=0x7000, held=0x8000, n_pages=99)):
        assert lib.quoka_pages_fork(at, ctypes.byref(_owners(**kw)), AT, AT, OTHER, OTHER, AT, WS, BIG, None) == 1
    for kw in (dict(page_table=o.page_table + 4 * (o.batch * o.max_pages - 1), held=0x8000), dict(page_table=0x70000, held=o.held + 4)):
        assert lib.quoka_pages_fork(at, ctypes.byref(_owners(**kw)), AT, AT, OTHER, OTHER, AT, WS, BIG, None) == 1   # in part
    child = ctypes.byref(_owners(page_table=0x7000, held=0x8000))
    later = ctypes.c_void_p(AT.value + 4)
    for args in ((AT, AT, later, OTHER, AT), (AT, AT, OTHER, later, AT)):   # outputs over the lengths
        assert lib.quoka_pages_fork(at, child, *args, WS, BIG, None) == 1
    for args in ((NULL, AT, OTHER, OTHER, AT), (AT, NULL, OTHER, OTHER, AT), (AT, AT, NULL, OTHER, AT), (AT, AT, OTHER, NULL, AT),
                 (AT, AT, OTHER, OTHER, NULL), (AT, AT, OTHER, AT, AT)):   # (the last: lengths in and out in one place)
        assert lib.quoka_pages_fork(at, child, *args, WS, BIG, None) == 1
    assert lib.quoka_pages_fork(at, child, AT, AT, OTHER, OTHER, AT, WS, ctypes.c_size_t(8), None) == 3


def test_outputs_of_a_fork_over_its_inputs_or_each_other_are_refused():
    """Of three children from two sequences: any of the three outputs that shares a word with the parents, the lengths, the three arrays of
    either batch, or another output.  (In batches of more than a block's, threads read some of them after others wrote.)"""
    lib, n = pk.load_library(), ctypes.c_size_t(0)
    source, kids = _owners(ref=0x100000, page_table=0x200000, held=0x300000, batch=2), _owners(ref=0x100000, page_table=0x400000, held=0x500000)
    assert lib.quoka_pages_workspace_bytes(ctypes.byref(kids), ctypes.byref(n)) == 0
    arrays = dict(parents=(0x600000, 3), lens=(0x700000, 2), first=(0x800000, 3), child_lens=(0x900000, 3), lacking=(0xA00000, 1))
    others = dict(arrays, ref=(0x100000, 100), table=(0x200000, 2 * 8), kids_table=(0x400000, 3 * 8), held=(0x300000, 2), kids_held=(0x500000, 3))
    for out in ("first", "child_lens", "lacking"):
        for name, (start, words) in others.items():
            if name == out:
                continue
            for at in (start, start + 4 * (words - 1), start - 4 * (arrays[out][1] - 1)):   # on it, over its end, over its start
                a = {k: ctypes.c_void_p(at if k == out else v[0]) for k, v in arrays.items()}
                assert lib.quoka_pages_fork(ctypes.byref(source), ctypes.byref(kids), a["parents"], a["lens"], a["first"], a["child_lens"], a["lacking"],
                                            WS, n, None) == 1, (out, name, hex(at))


# ---- verification -----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), 1), (dict(n_draft=0), 1), (dict(vocab=0), 1), (dict(target_stride=(-1, 1000)), 1), (dict(draft_stride=(4000, -8)), 1),
    (dict(dtype=2), 2), (dict(batch=65536), 2), (dict(n_draft=65536), 2), (dict(vocab=(1 << 24) + 1), 2),
])
def test_bad_drafts_are_refused(kw, code):
    lib, s, n = pk.load_library(), ctypes.byref(_drafts(**kw)), ctypes.c_size_t(0)
    assert lib.quoka_verify_workspace_bytes(s, ctypes.byref(n)) == code
    assert lib.quoka_verify_draft(s, AT, AT, AT, AT, None, AT, AT, WS, BIG, None) == code


def test_bad_pointers_of_a_verification_are_refused():
    lib, n = pk.load_library(), ctypes.c_size_t(0)
    s = ctypes.byref(_drafts())
    assert lib.quoka_verify_draft(None, AT, AT, AT, AT, None, AT, AT, WS, BIG, None) == 1
    assert lib.quoka_verify_workspace_bytes(s, None) == 1 and lib.quoka_verify_workspace_bytes(s, ctypes.byref(n)) == 0 and n.value % 256 == 0
    for i in (0, 2, 3, 5, 6):
        args = [AT, AT, AT, AT, None, AT, AT]
        args[i] = NULL
        assert lib.quoka_verify_draft(s, *args, WS, BIG, None) == 1
    assert lib.quoka_verify_draft(s, AT, AT, AT, AT, OTHER, OTHER, AT, WS, BIG, None) == 1   # lengths in, accepted tokens out
    assert lib.quoka_verify_draft(s, ODD, AT, AT, AT, None, AT, AT, WS, BIG, None) == 1
    assert lib.quoka_verify_draft(s, AT, ODD, AT, AT, None, AT, AT, WS, BIG, None) == 1
    for ws, size, code in ((NULL, BIG, 1), (ctypes.c_void_p(0x10010), BIG, 3), (WS, ctypes.c_size_t(n.value - 1), 3)):
        assert lib.quoka_verify_draft(s, AT, AT, AT, AT, None, AT, AT, ws, size, None) == code


def test_outputs_of_a_verification_over_its_inputs_or_each_other_are_refused():
    """Two sequences of three drafted tokens: counts and tokens that come out share no word with drafted tokens, random numbers, lengths or each
    other.  (Blocks of one sequence would read what those of another wrote.)"""
    lib, n, s = pk.load_library(), ctypes.c_size_t(0), ctypes.byref(_drafts())
    assert lib.quoka_verify_workspace_bytes(s, ctypes.byref(n)) == 0
    arrays = dict(tokens=(0x600000, 6), uniform=(0x700000, 8), draft_lens=(0x800000, 2), n_accepted=(0x900000, 2), tokens_out=(0xA00000, 8))
    for out in ("n_accepted", "tokens_out"):
        for name, (start, words) in arrays.items():
            if name == out:
                continue
            for at in (start, start + 4 * (words - 1), start - 4 * (arrays[out][1] - 1)):   # on it, over its end, over its start
                a = {k: ctypes.c_void_p(at if k == out else v[0]) for k, v in arrays.items()}
                assert lib.quoka_verify_draft(s, AT, AT, a["tokens"], a["uniform"], a["draft_lens"], a["n_accepted"], a["tokens_out"], WS, n, None) == 1, \
                    (out, name, hex(at))


# ---- the binding ------------------------------------------------------------------------------------------------------

def _ints(*x):
    return torch.tensor(x, dtype=torch.int32)


def test_sequences_refuse_tensors_that_do_not_fit():
    ref, table, held = torch.zeros(50, dtype=torch.int32), torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    seqs = pk.PagedSequences(ref, table, held, 16)
    assert seqs.ref is ref and seqs.page_table is table and seqs.held is held
    there = lambda x: x.to("meta")  # noqa: E731
    for args in ((ref.long(), table, held), (ref, table.long(), held), (ref, table, held.long()), (ref, table[0], held), (ref, table[:, ::2], held),
                 (ref[::2], table, held), (ref, table, held[:2]), (ref, there(table), held), (ref, table, there(held))):
        with pytest.raises(ValueError):
            pk.PagedSequences(*args, 16)
    with pytest.raises(pk.QuokaError):
        pk.PagedSequences(ref, table, held, 24)
    for lens in (_ints(1, 2), _ints(1, 2, 3).long(), _ints(1, 2, 3).view(3, 1), torch.zeros(6, dtype=torch.int32)[::2], there(_ints(1, 2, 3))):
        with pytest.raises(ValueError):
            seqs.resize(lens)
        with pytest.raises(ValueError):
            seqs.another(3).fork(seqs, lens, _ints(1, 2, 3))
        with pytest.raises(ValueError):
            seqs.another(3).fork(seqs, _ints(0, 1, 2), lens)
    with pytest.raises(pk.QuokaError):
        seqs.fork(seqs, _ints(0, 1, 2), _ints(1, 2, 3))
    with pytest.raises(pk.QuokaError):   # another pool
        pk.PagedSequences.allocate(50, 16, 3, 4, "cpu").fork(seqs, _ints(0, 1, 2), _ints(1, 2, 3))
    kid = seqs.another(5, 7)
    assert kid.page_table.shape == (5, 7) and bool((kid.page_table == -1).all()) and kid.ref is ref and not kid.held.any()


def test_moves_refuse_caches_that_do_not_fit():
    cache, other = _cache(), _cache()
    idx, cnt = torch.zeros(2, 2, 5, dtype=torch.int32), torch.zeros(2, 2, dtype=torch.int32)
    for bad in (_cache(torch.bfloat16), _cache(torch.float32)):
        with pytest.raises(TypeError):
            other.compact(bad, idx, cnt)
        with pytest.raises(TypeError):
            other.copy(bad, lens=_ints(1, 2))
    for bad in (_cache(n_kv=1), _cache(d=128), _cache(batch=3)):
        with pytest.raises(ValueError):
            other.compact(bad, idx, cnt)
    for bad in (_cache(n_kv=1), _cache(d=128), _cache(batch=1)):   # (a source of fewer sequences: without parents)
        with pytest.raises(ValueError):
            other.copy(bad, lens=_ints(1, 2))
    for lists in ((idx.long(), cnt), (idx, cnt.long()), (idx[:1], cnt), (idx, cnt[:, :1]), (idx[:, :, ::2], cnt), (idx.to("meta"), cnt), (idx, cnt.to("meta"))):
        with pytest.raises(ValueError):
            other.compact(cache, *lists)
    with pytest.raises(pk.QuokaError):   # lists longer than this cache's table has room for
        other.compact(_cache(cols=9), torch.zeros(2, 2, 65, dtype=torch.int32), cnt)
    for how in (dict(), dict(lens=_ints(1)), dict(lens=_ints(1, 2).long()), dict(lens=_ints(1, 2), first=_ints(1)), dict(lens=_ints(1, 2), parents=_ints(0, 1, 1)),
                dict(lens=_ints(1, 2).to("meta"))):
        with pytest.raises(ValueError):
            other.copy(cache, **how)
    with pytest.raises(pk.QuokaError):
        cache.copy(cache, lens=_ints(1, 2))
    with pytest.raises(ValueError):
        pk.PagedBuffers(cache, [1, 2], 60).cross_attn()


@pytest.mark.parametrize("dtype,d,most", [(torch.float8_e4m3fn, 128, 2 ** 24 - 1), (torch.bfloat16, 128, 2 ** 24 - 1), (torch.bfloat16, 64, 2 ** 24 - 1),
                                          (torch.float32, 64, 2 ** 24 - 1), (torch.float32, 128, 2 ** 23 - 1)])
def test_lists_reach_every_position_that_a_call_may_have(dtype, d, most, monkeypatch):
    """Of a table with room for more: as many as attention and selection take, which refuse one more."""
    table = torch.zeros(1, 1 << 10, dtype=torch.int32)
    there, pool = torch.zeros(1, 1, 16, d, dtype=dtype), torch.empty_strided((1, 1, 1 << 15, d), (0, 0, d, 1), dtype=dtype)
    scales = [torch.zeros(1, 1, n, dtype=torch.uint8) for n in (1 << 15, 16)] if dtype == torch.float8_e4m3fn else [None, None]
    cache, to = pk.PagedCache(pool, pool, table, *[scales[0]] * 2), pk.PagedCache(there, there, table[:, :4].contiguous(), *[scales[1]] * 2)
    shapes = []
    monkeypatch.setattr(pk.binding, "quoka_cache_compact", lambda shape, *a: shapes.append(shape))
    to.compact(cache, torch.zeros(1, 1, 5, dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32))
    s, n = shapes[0], ctypes.c_size_t(0)
    assert s.max_kv_len == most
    for t, code in ((most, 0), (most + 1, 2)):
        s.max_kv_len = t
        assert pk.load_library().quoka_paged_workspace_bytes(ctypes.byref(s), ctypes.byref(n)) == code


def test_drafts_refuse_tensors_that_do_not_fit():
    p, q = torch.zeros(2, 4, 100), torch.zeros(2, 3, 100)
    x, u = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 4)
    pk.DraftBuffers(p, x, u, draft=q, draft_lens=[1, 2])
    pk.DraftBuffers(p.bfloat16(), x, u)
    for how, error in ((dict(target=p.half()), TypeError), (dict(draft=q.bfloat16()), TypeError), (dict(target=p[0]), ValueError),
                       (dict(target=p[:, :1]), ValueError), (dict(draft=q[:, :2]), ValueError), (dict(draft=q[:, :, :99]), ValueError),
                       (dict(target=torch.zeros(2, 100, 4).transpose(1, 2)), ValueError), (dict(tokens=x.long()), ValueError),
                       (dict(tokens=x[:1]), ValueError), (dict(tokens=torch.zeros(3, 2, dtype=torch.int32).t()), ValueError),
                       (dict(uniform=u.double()), ValueError), (dict(uniform=u[:, :3]), ValueError), (dict(uniform=torch.zeros(4, 2).t()), ValueError),
                       (dict(draft_lens=[1]), ValueError), (dict(draft=q.to("meta")), ValueError), (dict(tokens=x.to("meta")), ValueError),
                       (dict(uniform=u.to("meta")), ValueError)):
        with pytest.raises(error):
            pk.DraftBuffers(**dict(dict(target=p, tokens=x, uniform=u, draft=q), **how))
    rows = torch.zeros(2, 8, 100)[:, ::2]
    assert list(pk.DraftBuffers(rows, x, u).shape.target_stride) == [800, 200]


def test_calls_for_another_device_than_the_current_one_are_refused(monkeypatch):
    monkeypatch.setattr(pk.binding, "_device", lambda: 0)
    pk.binding._here(None)
    pk.binding._here(0)
    with pytest.raises(ValueError):
        pk.binding._here(1)
    cache, other = _cache(), _cache()
    q = torch.zeros(2, 4, 3, 64, dtype=torch.bfloat16)
    seqs = pk.PagedSequences.allocate(50, 16, 3, 4, "cpu")
    kids, drafts = seqs.another(3), pk.DraftBuffers(torch.zeros(2, 4, 100), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 4))
    buf = pk.PagedBuffers(cache, [1, 2], 60, q=q)
    for x in (cache, other, seqs, kids, drafts):   # (as if their tensors were the second GPU's)
        assert x._index is None
        x._index = 1
    lens, lists = _ints(1, 2, 3), (torch.zeros(2, 2, 5, dtype=torch.int32), torch.zeros(2, 2, dtype=torch.int32))
    for call in (buf.cross_attn, lambda: other.compact(cache, *lists), lambda: other.copy(cache, lens=_ints(1, 2)), lambda: seqs.resize(lens),
                 lambda: kids.fork(seqs, lens, lens), drafts.verify):
        with pytest.raises(ValueError, match="current one"):
            call()


# ---- the plain forms, by hand -----------------------------------------------------------------------------------------

def test_the_plain_verification_draws_from_the_target():
    """Tokens drafted from q and verified are distributed as p: every cell of an exhaustive grid of random numbers counted."""
    p, q = np.array([0.5, 0.125, 0.25, 0.125]), np.array([0.125, 0.5, 0.25, 0.125])
    N = 16   # a grid that divides every probability
    counts = np.zeros(4)
    grid = (np.arange(N) + 0.5) / N
    for x in range(4):
        for u in grid:
            for r in grid:
                _, out = G.verify(np.stack([p, p]), [q], [x], [u, r], 1)
                counts[out[0]] += q[x] / N / N
    assert np.allclose(counts, p, atol=1e-12)


@pytest.mark.parametrize("value", [-np.inf, np.inf, np.nan])
@pytest.mark.parametrize("u", [0.5, 0.0, -0.5, np.inf, -np.inf, np.nan])
def test_the_plain_verification_refuses_tokens_whose_draft_probability_is_no_number(value, u):
    a, out = G.verify([[0.75, 0.25], [0.5, 0.5]], [[value, 0.0]], [0], [u, 0.5], 1)
    assert a == 0 and out.tolist() == [1, -1]


def test_the_plain_book_keeps_its_counts():
    ref = [0] * 10
    a = G.Book(ref, 4, 2, 5)
    assert a.resize([9, 4]) == 0 and a.rows == [[0, 1, 2], [3]] and ref[:4] == [1] * 4
    b = G.Book(ref, 4, 3, 5)
    assert b.fork(a, [0, 0, 7], [9, 4]) == ([8, 8, 0], [9, 9, 0], 0)
    assert b.rows == [[0, 1, 4], [0, 1, 5], []] and ref == [3, 3, 1, 1, 1, 1, 0, 0, 0, 0]
    assert a.resize([0, 20]) == 0 and a.rows == [[], [3, 2, 6, 7, 8]]   # the third page of the first came back in time
    assert a.resize([8, 20]) == 1 and a.rows[0] == [9] and a.table()[0].tolist() == [9, -1, -1, -1, -1]
