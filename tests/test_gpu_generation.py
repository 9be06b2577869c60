"""Generation over caches in pages on the GPU against plain float64 and whole numbers: cross attention, verification of drafted tokens, who
holds the pages, rows that move, and a run of them together."""
from fractions import Fraction

import numpy as np
import pytest
import torch

from tests import generation_plain as G
from tests import paged_plain as P

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _pk():
    import paper_2602_08722_amd as pk
    pk.load_library()
    return pk


def _ids(c):
    return "-".join(f"{k}{v}" for k, v in c.items()).replace(" ", "")


def _rows(rng, n, n_kv, d, dtype):
    return P.store(rng.standard_normal((n, n_kv, d)), dtype).astype(np.float64)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ---- cross attention ---------------------------------------------------------------------------------------------------

def _cross_problem(case, seed, layout="heads", scale=1.0, **how):
    rng = np.random.default_rng(seed)
    n_q, n_kv, d, C, lens, dtype = (case[k] for k in ("n_q", "n_kv", "d", "C", "lens", "dtype"))
    chunks = [C] * len(lens) if case.get("chunks") is None else [max(c, 0) for c in case["chunks"]]
    pool = P.Pool(rng, [_rows(rng, max(n, 0), n_kv, d, dtype) for n in lens], [_rows(rng, max(n, 0), n_kv, d, dtype) for n in lens], n_kv, d,
                  case["page_len"], dtype, case["fp8"], layout=layout, **how)
    q = P.store(rng.standard_normal((len(lens), n_q, C, d)) * scale, dtype)
    return pool, q, chunks


def _cross_buffers(case, pool, q, q_layout="heads", max_kv=None):
    tq = P.to_dev(q, case["dtype"], DEV)
    if q_layout == "tokens":
        tq = tq.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    buf = _pk().PagedBuffers(pool.cache(), case["lens"], max(max(case["lens"]), 0) if max_kv is None else max_kv, q=tq, chunk_lens=case.get("chunks"))
    buf.out.fill_(float("nan"))
    buf.lse.fill_(float("nan"))
    buf.workspace.fill_(0xFF)   # NaN, whatever it is read as
    return buf


def _check_cross(case, buf, pool, q, chunks):
    """bf16: every probability, and the output, is rounded once: |error| <= 2^-8 (P |V| + |O|), and a few units of float32 rounding on top
    (2^-8 * 1.05 holds them); over many values roundings are evenly spread, which takes their root mean square to at most 1 / sqrt(3) of
    that.  f32: a logit of d products is off by d * 2^-24 * sum |q k| / sqrt(d) at most, here below 5e-5, and a probability by as much relatively.  lse:
    of unrounded probabilities in float32 in either case."""
    got, got_lse = buf.out.float().cpu().numpy().astype(np.float64), buf.lse.cpu().numpy().astype(np.float64)
    for i, n in enumerate(chunks):
        want, lse, weight = G.cross(q[i, :, :n].astype(np.float64), pool.k[i], pool.v[i])
        bound = 1.05 * 2.0 ** -8 * (weight + np.abs(want)) + 1e-6 if case["dtype"] == "bf16" else 1e-4 * weight + 1e-7
        err = np.abs(got[i, :, :n] - want)
        assert np.all(err <= bound), f"sequence {i}: {np.nanmax(err)} (NaN: {np.isnan(err).sum()}), {np.argwhere(~(err <= bound))[:4].tolist()}"
        if case["dtype"] == "bf16" and n > 1 and len(pool.k[i]) > 0:
            assert np.linalg.norm(err) <= 1.05 * 2.0 ** -8 * np.sqrt((np.sum(weight ** 2) + np.sum(want ** 2)) / 3), f"sequence {i}"
        if len(pool.k[i]) == 0:
            assert np.all(got[i] == 0.0) and np.all(np.isneginf(got_lse[i])), f"sequence {i}: no states"
        else:
            assert np.all(np.abs(got_lse[i, :, :n] - lse) <= 1e-4), f"sequence {i}: lse"
        assert np.all(got[i, :, n:] == 0.0) and np.all(np.isneginf(got_lse[i, :, n:])), f"sequence {i}: rows past the chunk"


CROSS_CASES = [
    # single tokens and a few: states of every length around tiles and pages, none among them, more sequences than lanes
    dict(dtype="bf16", fp8=False, n_q=12, n_kv=12, d=64, page_len=64, C=1, lens=[300, 1]),
    dict(dtype="bf16", fp8=True, n_q=8, n_kv=2, d=128, page_len=16, C=1, lens=[0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 500]),
    dict(dtype="bf16", fp8=False, n_q=7, n_kv=1, d=64, page_len=8, C=4, lens=[777, 0]),
    dict(dtype="bf16", fp8=True, n_q=16, n_kv=1, d=128, page_len=128, C=2, lens=[5000, 40]),
    dict(dtype="bf16", fp8=True, n_q=8, n_kv=2, d=128, page_len=64, C=5, lens=[300, 20, 0, 9], chunks=[0, 5, 2, -1]),
    dict(dtype="bf16", fp8=False, n_q=8, n_kv=8, d=128, page_len=1, C=1, lens=[70]),
    dict(dtype="bf16", fp8=True, n_q=4, n_kv=2, d=64, page_len=16, C=2, lens=[(37 * i) % 211 for i in range(150)], chunks=[(5 * i) % 3 for i in range(150)]),
    dict(dtype="bf16", fp8=False, n_q=32, n_kv=8, d=128, page_len=16, C=1, lens=[(61 * i) % 517 for i in range(40)]),
    dict(dtype="bf16", fp8=False, n_q=16, n_kv=1, d=128, page_len=32, C=1, lens=[0] * 30 + [20000] + [0, 40] * 15),   # a long one among many
    dict(dtype="bf16", fp8=False, n_q=8, n_kv=2, d=128, page_len=16, C=1, lens=[0, 0]),
    dict(dtype="bf16", fp8=False, n_q=4, n_kv=1, d=64, page_len=64, C=1, lens=[30000]),
    # blocks for each sequence and KV head that fill half of the chip, all of it, and more than that
    dict(dtype="bf16", fp8=False, n_q=16, n_kv=4, d=64, page_len=64, C=1, lens=[2900 - 89 * i for i in range(32)]),
    dict(dtype="bf16", fp8=True, n_q=12, n_kv=4, d=128, page_len=32, C=2, lens=[65 * i for i in range(25)], chunks=[1 + i % 2 for i in range(25)]),
    dict(dtype="bf16", fp8=False, n_q=12, n_kv=12, d=128, page_len=16, C=1, lens=[2047 - 90 * i for i in range(20)]),
    dict(dtype="bf16", fp8=True, n_q=12, n_kv=12, d=64, page_len=64, C=1, lens=[(53 * i) % 997 for i in range(30)]),
    dict(dtype="bf16", fp8=False, n_q=12, n_kv=12, d=64, page_len=16, C=1, lens=[(17 * i) % 131 for i in range(70)]),
    dict(dtype="bf16", fp8=True, n_q=40, n_kv=40, d=128, page_len=16, C=1, lens=[33 * i for i in range(24)]),
    dict(dtype="bf16", fp8=False, n_q=520, n_kv=520, d=64, page_len=16, C=1, lens=[2000, 0, 31]),
    # one and two rows of a KV head over few states, and over more of many sequences
    dict(dtype="bf16", fp8=False, n_q=12, n_kv=12, d=64, page_len=64, C=1, lens=[600, 1, 0, 31, 32, 33, 256, 257]),
    dict(dtype="bf16", fp8=True, n_q=5, n_kv=5, d=128, page_len=16, C=2, lens=[50, 15, 16, 17], chunks=[2, 1, 0, 2]),
    dict(dtype="bf16", fp8=False, n_q=4, n_kv=2, d=64, page_len=8, C=1, lens=[150, 7]),
    dict(dtype="bf16", fp8=True, n_q=24, n_kv=24, d=64, page_len=32, C=1, lens=[33 * i for i in range(30)]),
    dict(dtype="bf16", fp8=False, n_q=20, n_kv=10, d=128, page_len=1, C=1, lens=[600 - 17 * i for i in range(28)], chunks=[i % 2 for i in range(28)]),
    # chunks: row blocks of four and eight, shared lists, whole ones
    dict(dtype="bf16", fp8=False, n_q=10, n_kv=10, d=64, page_len=64, C=270, lens=[300 - 23 * i for i in range(13)]),       # four (260 groups of eight)
    dict(dtype="bf16", fp8=True, n_q=10, n_kv=10, d=128, page_len=16, C=270, lens=[20 * i for i in range(13)], chunks=[270 - 20 * i for i in range(13)]),
    dict(dtype="bf16", fp8=True, n_q=9, n_kv=3, d=64, page_len=16, C=300, lens=[9 * i for i in range(20)]),                 # eight
    dict(dtype="bf16", fp8=True, n_q=8, n_kv=2, d=128, page_len=64, C=200, lens=[700]),
    dict(dtype="bf16", fp8=False, n_q=8, n_kv=2, d=64, page_len=16, C=77, lens=[0, 130]),
    dict(dtype="bf16", fp8=True, n_q=8, n_kv=2, d=128, page_len=32, C=129, lens=[1, 511, 64, 65, 128, 129]),
    dict(dtype="bf16", fp8=False, n_q=12, n_kv=4, d=64, page_len=16, C=100, lens=[1237, 0, 63], chunks=[100, 31, 65]),
    dict(dtype="bf16", fp8=True, n_q=6, n_kv=2, d=128, page_len=256, C=64, lens=[3000, 10, 0], chunks=[1, 64, 0]),
    dict(dtype="bf16", fp8=False, n_q=32, n_kv=2, d=128, page_len=64, C=300, lens=[260]),
    dict(dtype="bf16", fp8=True, n_q=16, n_kv=16, d=64, page_len=64, C=640, lens=[129]),
    dict(dtype="bf16", fp8=False, n_q=32, n_kv=8, d=64, page_len=16, C=1100, lens=[100]),       # more than 1024 row blocks
    dict(dtype="bf16", fp8=False, n_q=32, n_kv=8, d=128, page_len=16, C=1100, lens=[31]),
    dict(dtype="bf16", fp8=True, n_q=32, n_kv=8, d=128, page_len=16, C=1100, lens=[200]),
    dict(dtype="bf16", fp8=False, n_q=32, n_kv=8, d=64, page_len=16, C=1100, lens=[0]),
    dict(dtype="bf16", fp8=False, n_q=4, n_kv=1, d=64, page_len=32, C=20, lens=[3000 - 43 * i for i in range(70)]),
    dict(dtype="bf16", fp8=True, n_q=4, n_kv=1, d=128, page_len=32, C=20, lens=[40 * i for i in range(70)], chunks=[20 - i % 7 for i in range(70)]),
    dict(dtype="bf16", fp8=True, n_q=12, n_kv=4, d=128, page_len=64, C=333, lens=[6000, 0, 3100], chunks=[333, 101, 0]),
    dict(dtype="bf16", fp8=False, n_q=16, n_kv=8, d=64, page_len=64, C=1060, lens=[9000, 1500], chunks=[1060, 700]),
    dict(dtype="bf16", fp8=False, n_q=16, n_kv=16, d=128, page_len=64, C=33, lens=[0, 0, 0]),
    # float32: a wave a row, units of 32, shared lists
    dict(dtype="f32", fp8=False, n_q=4, n_kv=2, d=64, page_len=16, C=1, lens=[0, 20, 1]),
    dict(dtype="f32", fp8=True, n_q=4, n_kv=2, d=128, page_len=16, C=3, lens=[0, 30, 2], chunks=[3, 2, 0]),
    dict(dtype="f32", fp8=True, n_q=4, n_kv=2, d=128, page_len=32, C=1, lens=[2000, 0]),
    dict(dtype="f32", fp8=False, n_q=9, n_kv=3, d=64, page_len=32, C=133, lens=[1999, 700, 0], chunks=[133, 57, 90]),
    dict(dtype="f32", fp8=False, n_q=8, n_kv=2, d=128, page_len=64, C=100, lens=[333, 0], chunks=[100, 37]),
    dict(dtype="f32", fp8=True, n_q=6, n_kv=2, d=64, page_len=16, C=70, lens=[64, 900], chunks=[0, 70]),
    dict(dtype="f32", fp8=False, n_q=16, n_kv=1, d=64, page_len=8, C=33, lens=[31]),
    dict(dtype="f32", fp8=False, n_q=4, n_kv=2, d=128, page_len=16, C=1, lens=[0, 0]),
    dict(dtype="f32", fp8=True, n_q=4, n_kv=2, d=64, page_len=16, C=70, lens=[0]),
    dict(dtype="f32", fp8=False, n_q=4, n_kv=2, d=64, page_len=16, C=40, lens=[(97 * i) % 700 for i in range(140)], chunks=[(11 * i) % 41 for i in range(140)]),
    dict(dtype="f32", fp8=False, n_q=2, n_kv=1, d=128, page_len=16, C=3, lens=[9000 - 700 * i for i in range(13)]),
    dict(dtype="f32", fp8=True, n_q=32, n_kv=8, d=64, page_len=16, C=600, lens=[700, 300], chunks=[600, 100]),   # more row blocks than a round
    # one to four rows of a KV head over many states, of lengths around tiles and pages, more blocks than compute units
    dict(dtype="f32", fp8=False, n_q=12, n_kv=12, d=64, page_len=64, C=1, lens=[300, 1, 0, 31, 32, 33, 256, 257]),
    dict(dtype="f32", fp8=True, n_q=5, n_kv=5, d=64, page_len=16, C=3, lens=[1000, 15, 16, 17], chunks=[3, 1, 0, 2]),
    dict(dtype="f32", fp8=False, n_q=8, n_kv=2, d=128, page_len=8, C=1, lens=[(37 * i) % 300 for i in range(40)]),
    dict(dtype="f32", fp8=True, n_q=4, n_kv=2, d=128, page_len=128, C=2, lens=[700, 130], chunks=[1, 2]),
    dict(dtype="f32", fp8=False, n_q=2, n_kv=1, d=128, page_len=1, C=1, lens=[127, 128, 129]),
    dict(dtype="f32", fp8=False, n_q=24, n_kv=24, d=64, page_len=32, C=1, lens=[60 * i for i in range(30)]),
    dict(dtype="f32", fp8=True, n_q=10, n_kv=10, d=128, page_len=64, C=4, lens=[2500 - 90 * i for i in range(28)], chunks=[i % 5 for i in range(28)]),
    dict(dtype="f32", fp8=False, n_q=12, n_kv=12, d=128, page_len=16, C=40, lens=[16]),
    dict(dtype="f32", fp8=True, n_q=6, n_kv=2, d=64, page_len=8, C=90, lens=[12, 0, 1, 7], chunks=[90, 5, 0, 61]),
    dict(dtype="f32", fp8=False, n_q=8, n_kv=2, d=128, page_len=16, C=1000, lens=[2, 3], chunks=[1000, 999]),
]


@pytest.mark.parametrize("case", CROSS_CASES, ids=_ids)
def test_cross_attention(case):
    pool, q, chunks = _cross_problem(case, 41)
    buf = _cross_buffers(case, pool, q)
    buf.cross_attn()
    torch.cuda.synchronize()
    _check_cross(case, buf, pool, q, chunks)


@pytest.mark.parametrize("case", [
    dict(dtype="bf16", fp8=True, n_q=8, n_kv=2, d=128, page_len=16, C=1, lens=[300, 77]),
    dict(dtype="bf16", fp8=False, n_q=8, n_kv=2, d=64, page_len=16, C=90, lens=[300, 77]),
    dict(dtype="f32", fp8=True, n_q=8, n_kv=2, d=128, page_len=16, C=40, lens=[300, 77]),
    dict(dtype="f32", fp8=False, n_q=8, n_kv=4, d=64, page_len=16, C=2, lens=[300, 77]),
    dict(dtype="f32", fp8=True, n_q=8, n_kv=4, d=128, page_len=16, C=1, lens=[300, 77]),
], ids=_ids)
def test_cross_attention_over_other_strides_and_entries(case):
    """Heads inside tokens, gaps between rows, table entries past a sequence's length that name no page, and room for more states."""
    pool, q, chunks = _cross_problem(case, 42, layout="tokens", tail_entries=2 ** 31 - 1, table_cols=60)
    buf = _cross_buffers(case, pool, q, q_layout="tokens", max_kv=900)
    buf.cross_attn()
    torch.cuda.synchronize()
    _check_cross(case, buf, pool, q, chunks)


@pytest.mark.parametrize("case", [
    dict(dtype="bf16", fp8=False, n_q=8, n_kv=2, d=128, page_len=16, C=1, lens=[500, 77]),
    dict(dtype="bf16", fp8=True, n_q=8, n_kv=2, d=64, page_len=16, C=2, lens=[5000, 900]),
    dict(dtype="bf16", fp8=False, n_q=8, n_kv=2, d=64, page_len=16, C=150, lens=[700, 77]),
    dict(dtype="bf16", fp8=True, n_q=32, n_kv=8, d=128, page_len=64, C=280, lens=[600]),
], ids=_ids)
@pytest.mark.parametrize("rising", [False, True])
def test_cross_attention_of_wide_logits(case, rising):
    """Logits of a standard deviation of 8, and such that grow along the states, so that a row's maximum moves on in every tile."""
    pool, q, chunks = _cross_problem(case, 44, scale=8.0)
    if rising:   # (the rows as they are kept, in the other order: the ones that the first query likes least come first; no input of other cases)
        for i, n in enumerate(case["lens"]):
            k, v = pool.k[i], pool.v[i]
            order = np.argsort(k[:, 0] @ q[i, 0, 0].astype(np.float64))
            at = torch.tensor(np.arange(n), device=DEV)
            pages, slots = torch.tensor(pool.table[i], device=DEV)[at // case["page_len"]], at % case["page_len"]
            o = torch.tensor(order, device=DEV)
            for x in (pool.k_pages, pool.v_pages):
                bits = x.view(torch.uint8) if x.element_size() == 1 else x
                bits[pages, :, slots] = bits[pages[o], :, slots[o]]
            if case["fp8"]:
                for s in (pool.k_scale, pool.v_scale):
                    s[pages, :, slots] = s[pages[o], :, slots[o]]
            pool.k[i], pool.v[i] = k[order], v[order]
    buf = _cross_buffers(case, pool, q)
    buf.cross_attn()
    torch.cuda.synchronize()
    _check_cross(case, buf, pool, q, chunks)


def test_calls_on_two_streams_at_once():
    """Two buffers over one cache, and two pools of pages, each on a stream of its own."""
    pk = _pk()
    cases = [dict(dtype="bf16", fp8=True, n_q=8, n_kv=2, d=128, page_len=16, C=C, lens=[4000, 90]) for C in (1, 70)]
    pool, q, chunks = _cross_problem(cases[0], 45)
    many = P.store(np.random.default_rng(46).standard_normal((2, 8, 70, 128)), "bf16")
    bufs = [_cross_buffers(case, pool, x) for case, x in zip(cases, (q, many))]
    seqs = [pk.PagedSequences.allocate(4000, 16, 5, 400) for _ in range(2)]
    lens = [_ints([100, 0, 4000, 33, 17]), _ints([7, 6000, 1, 0, 800])]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        for s, buf, seq, n in zip(streams, bufs, seqs, lens):
            with torch.cuda.stream(s):
                seq.resize(n)
                buf.cross_attn()
                seq.resize(torch.zeros_like(n))
                seq.resize(n)
    torch.cuda.synchronize()
    for case, buf, x in zip(cases, bufs, (q, many)):
        _check_cross(case, buf, pool, x, [case["C"]] * 2)
    for seq, n in zip(seqs, lens):
        book = G.Book([0] * 4000, 16, 5, 400)
        book.resize(n.tolist())
        assert np.array_equal(seq.page_table.cpu().numpy(), book.table()) and seq.ref.tolist() == book.ref


@pytest.mark.parametrize("case", [
    dict(dtype=dtype, fp8=fp8, n_q=n_q, n_kv=8, d=128, page_len=64, C=C, lens=[T])
    for dtype, fp8, n_q, C, T in (("bf16", False, 8, 1, 300), ("bf16", True, 16, 1, 50), ("bf16", False, 32, 1, 400), ("bf16", True, 32, 1, 5000),
                                  ("bf16", False, 32, 70, 700), ("bf16", True, 32, 300, 300), ("f32", False, 8, 1, 700), ("f32", True, 32, 1, 300),
                                  ("f32", False, 32, 40, 300), ("f32", True, 8, 3, 5))
], ids=_ids)
def test_cross_attention_beyond_four_gib_of_a_pool(case):
    row = 1 if case["fp8"] else 2 if case["dtype"] == "bf16" else 4
    pool, q, chunks = _cross_problem(case, 47, n_pages=3 * (1 << 31) // (8 * 64 * 128 * row))   # (pages from all over it)
    buf = _cross_buffers(case, pool, q)
    buf.cross_attn()
    torch.cuda.synchronize()
    _check_cross(case, buf, pool, q, chunks)


@pytest.mark.parametrize("C,dtype", [(1, "bf16"), (70, "bf16"), (1, "f32"), (30, "f32")])
def test_cross_attention_from_a_graph_as_lengths_move(C, dtype):
    """Recorded once, replayed with other queries and lengths, a length of none among them."""
    case = dict(dtype=dtype, fp8=True, n_q=8, n_kv=2, d=128, page_len=16, C=C, lens=[400, 90])
    pool, q, chunks = _cross_problem(case, 43)
    buf = _cross_buffers(case, pool, q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        buf.cross_attn()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        buf.cross_attn()
    whole = [(k, v) for k, v in zip(pool.k, pool.v)]
    for lens in ([400, 90], [17, 0], [0, 33], [399, 90]):
        q = P.store(np.random.default_rng(sum(lens)).standard_normal(q.shape), dtype)
        buf.q.copy_(P.to_dev(q, dtype, DEV))
        buf.kv_lens.copy_(_ints(lens))
        buf.out.fill_(float("nan"))
        buf.lse.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        pool.k, pool.v = ([w[j][:n] for w, n in zip(whole, lens)] for j in range(2))
        _check_cross(case, buf, pool, q, chunks)
        float(torch.randn(1 << 16, device=DEV).sum())


@pytest.mark.parametrize("d,C,lens", [(64, 270, [5000, 4000]), (128, 270, [5000, 2500])])
def test_float32_attention_over_pages_in_its_own_workspace(d, C, lens):
    """Where cross attention wants more partials: the call that does not takes what it needs, and leaves what lies behind."""
    pk = _pk()
    case = dict(dtype="f32", fp8=False, n_q=8, n_kv=2, d=d, page_len=16, C=C, lens=[n + C for n in lens])
    pool, q, chunks = _cross_problem(case, 48)
    buf = _cross_buffers(dict(case, lens=lens), pool, q)
    want, lse = buf.attn().clone(), buf.lse.clone()
    need = 512 * 32 * (d + 2) * 4   # at most 512 partials of 32 rows
    assert buf.workspace.numel() > need
    whole, buf.workspace = buf.workspace, buf.workspace[:need]
    whole.fill_(0xFF)
    buf.out.fill_(float("nan"))
    buf.attn()
    torch.cuda.synchronize()
    assert torch.equal(buf.out, want) and torch.equal(buf.lse, lse) and bool((whole[need:] == 0xFF).all())
    for i, n in enumerate(lens):
        out, _, weight = P.attention(q[i].astype(np.float64), pool.k[i], pool.v[i], n)
        assert np.all(np.abs(buf.out[i].cpu().numpy() - out) <= 1e-4 * weight + 1e-7)
    with pytest.raises(pk.QuokaError):
        buf.cross_attn()
    wide = torch.full((whole.numel() + 65536,), 0xFF, dtype=torch.uint8, device=DEV)   # what cross attention asks for, and no more
    buf.workspace = wide[:whole.numel()]
    buf.out.fill_(float("nan"))
    buf.cross_attn()
    torch.cuda.synchronize()
    pool.k, pool.v = ([x[:n] for x, n in zip(y, lens)] for y in (pool.k, pool.v))
    _check_cross(case, buf, pool, q, chunks)
    assert bool((wide[whole.numel():] == 0xFF).all())


# ---- verification ------------------------------------------------------------------------------------------------------

def _softmax(z):
    e = np.exp(z - z.max(-1, keepdims=True))
    return e / e.sum(-1, keepdims=True)


def _verify_problem(rng, b, n, V, dtype, lookup):
    """Targets, and drafts from near them."""
    z = 2.5 * rng.standard_normal((b, n + 1, V))
    p = P.store(_softmax(z), dtype)
    zq = z[:, :n] + (0 if lookup else 0.4 * rng.standard_normal((b, n, V)))
    q = None if lookup else P.store(_softmax(zq), dtype)
    tokens = (zq + rng.gumbel(size=zq.shape)).argmax(-1)
    uniform = rng.random((b, n + 1), dtype=np.float32)
    return p, q, tokens, uniform


def _verified(p, q, tokens, uniform, dtype, lens=None, strided=False):
    def dev(x):
        if x is None:
            return None
        t = P.to_dev(x, dtype, DEV)
        if strided:   # rows further apart than they are long, at an odd element
            wide = torch.full((t.shape[0], t.shape[1], t.shape[2] + 5), float("nan"), dtype=t.dtype, device=DEV)
            wide[..., 3:-2] = t
            t = wide[..., 3:-2]
        return t

    buf = _pk().DraftBuffers(dev(p), _ints(tokens.tolist()), torch.from_numpy(np.asarray(uniform, np.float32)).to(DEV), draft=dev(q), draft_lens=lens)
    buf.workspace.fill_(0xFF)
    buf.n_accepted.fill_(77)
    buf.tokens_out.fill_(77)
    n_accepted, out = buf.verify()
    torch.cuda.synchronize()
    return n_accepted.cpu().numpy(), out.cpu().numpy()


def _check_verified(got, p, q, tokens, uniform, lens=None):
    for i in range(len(p)):
        n = tokens.shape[1] if lens is None else min(max(lens[i], 0), tokens.shape[1])
        a, out = G.verify(p[i], None if q is None else q[i], tokens[i], uniform[i], n)
        assert got[0][i] == a and got[1][i].tolist() == out.tolist(), (i, got[0][i], a, got[1][i], out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lookup", [False, True])
@pytest.mark.parametrize("b,n,V,lens", [
    (1, 1, 1, None), (3, 2, 7, None), (1, 4, 4095, None), (2, 3, 4096, [3, 0]), (2, 3, 4097, [-1, 9]), (5, 7, 32003, [7, 0, 3, 1, 6]), (1, 5, 70001, None),
    (40, 2, 513, None), (2, 70, 300, None), (2, 130, 64, [130, 65]), (1, 2, 300007, None),
])
def test_verification(b, n, V, lens, lookup, dtype):
    rng = np.random.default_rng(b * 1000 + n + V)
    for rep in range(3):
        p, q, tokens, uniform = _verify_problem(rng, b, n, V, dtype, lookup)
        if rep == 1:
            uniform[:, :n] = 0.0   # accepts whatever has any probability
        got = _verified(p, q, tokens, uniform, dtype, lens, strided=rep == 2)
        _check_verified(got, p, q, tokens, uniform, lens)


@pytest.mark.parametrize("dtype,V", [("f32", V + i) for V in (4096, 8192, 16384, 24576) for i in (0, 1)] +
                         [("bf16", V + i) for V in (8192, 16384) for i in (0, 1)] + [("f32", 63), ("f32", 257), ("bf16", 1), ("bf16", 4095)])
@pytest.mark.parametrize("lookup", [False, True])
def test_verification_of_vocabularies_around_a_blocks_pieces(dtype, V, lookup):
    rng = np.random.default_rng(V)
    for lens in (None, [0, 3, 1, 2, 3]):
        p, q, tokens, uniform = _verify_problem(rng, 5, 3, V, dtype, lookup)
        uniform[0, :3] = 0.0    # accepts what has any probability
        uniform[1, :3] = 1.0
        uniform[:, 3] = [0.0, 1.0, 0.5, 1.0 - 2.0 ** -24, 1e-30]
        _check_verified(_verified(p, q, tokens, uniform, dtype, lens), p, q, tokens, uniform, lens)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [32768, 32769, 25000])
def test_verification_of_many_sequences(dtype, V):
    rng = np.random.default_rng(V + 1)
    lens = [i % 3 for i in range(64)]
    p, q, tokens, uniform = _verify_problem(rng, 64, 2, V, dtype, False)
    q[5], uniform[5] = p[5, :2], 1.0   # nothing is left behind a refusal
    _check_verified(_verified(p, q, tokens, uniform, dtype, lens), p, q, tokens, uniform, lens)


@pytest.mark.parametrize("V", [1000, 40000])
def test_verification_of_rows_far_apart(V):
    """Strides past 32 bits: sequences more than 2^31 elements from each other, at an odd element."""
    rng = np.random.default_rng(9)
    p, q, tokens, uniform = _verify_problem(rng, 2, 2, V, "bf16", False)
    far = (1 << 31) + 12345
    base = torch.zeros(far + 6 * V + 7, dtype=torch.bfloat16, device=DEV)
    target, draft = (base.as_strided(x.shape, (far, V + 1, 1), at) for x, at in ((p, 1), (q, 3 * V + 5)))
    target.copy_(P.to_dev(p, "bf16", DEV))
    draft.copy_(P.to_dev(q, "bf16", DEV))
    buf = _pk().DraftBuffers(target, _ints(tokens.tolist()), torch.from_numpy(uniform).to(DEV), draft=draft)
    got = buf.verify()
    torch.cuda.synchronize()
    _check_verified([x.cpu().numpy() for x in got], p, q, tokens, uniform)


@pytest.mark.parametrize("V", [5, 33000])
def test_verification_of_what_distributions_should_not_hold(V):
    """NaN, infinities, negative entries, rows without any weight, tokens outside the vocabulary, random numbers outside [0, 1)."""
    rng = np.random.default_rng(3)
    for rep in range(40):
        b, n = 6, 3
        p, q, tokens, uniform = _verify_problem(rng, b, n, V, "f32", rep % 3 == 0)
        for x in (p,) if q is None else (p, q):
            for value in (np.nan, np.inf, -np.inf, -1.0, 0.0):
                at = rng.random(x.shape) < (0.2 if V < 10 else 0.01)
                x[at] = value
        tokens[rng.random(tokens.shape) < 0.1] = -1
        tokens[rng.random(tokens.shape) < 0.1] = V
        tokens[rng.random(tokens.shape) < 0.05] = 2 ** 31 - 1
        p[0] = 0.0
        p[1, :, 1:] = np.nan
        if q is not None:
            q[2] = p[2, :n]     # nothing is left behind a refusal: p itself
        uniform[3] = [1.0, 1.5, 0.0, rng.choice(np.array([1.0, 2.0, np.nan, -0.5, np.inf], np.float32))]
        uniform[2, :n] = 1.0    # refuses
        got = _verified(p, q, tokens, uniform, "f32")
        _check_verified(got, p, q, tokens, uniform)


@pytest.mark.parametrize("V", [4, 4096, 40960])
def test_borders_of_a_verification(V):
    """Equal parts, whose sums are exact: a random number at the very end of a part points into the next (where v / V is no float32 number, the
    one next to it points where it lies); u q == p refuses, one step below accepts."""
    p = np.full((1, 2, V), 1.0 / V, dtype=np.float32)
    one = np.zeros((1, 1), dtype=np.int64)
    for v in sorted({0, 1, 2, 3, V // 2, V - 1}):
        got = _verified(p, p[:, :1], one, np.array([[0.5, v / V]], np.float32), "f32")
        part = int(Fraction(float(np.float32(v / V))) * V)   # parts of equal width: the number of whole ones below the random number
        assert part == v or V & (V - 1) != 0
        assert got[0][0] == 1 and got[1][0].tolist() == [0, part]
    q = np.zeros((1, 1, V), dtype=np.float32)
    q[0, 0, 0] = 0.5
    p[0, 0, 0] = 0.25
    for u, a in ((0.5, 0), (np.nextafter(np.float32(0.5), np.float32(0)), 1)):
        got = _verified(p, q, one, np.array([[u, 0.0]], np.float32), "f32")
        assert got[0][0] == a and got[1][0, a] == (0 if a == 1 else 1)   # (refused: nothing is left at 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [8, 40000])
def test_tokens_drafted_with_a_probability_that_is_no_number_are_refused(V, dtype):
    """q is -inf, inf or NaN at the drafted token, whatever the random number: not accepted, and the token weighs nothing behind it.  (All of p
    lies on tokens 1, the drafted one, and 3: what is drawn is 3.)  A second token that could be accepted stays unread."""
    p, q = np.zeros((1, 3, V), np.float32), np.zeros((1, 2, V), np.float32)
    p[0, :, 1], p[0, :, 3] = 0.75, 0.25
    q[0, :, 1] = 0.5
    tokens = np.array([[1, 1]], dtype=np.int64)
    for value in (-np.inf, np.inf, np.nan):
        for u in (0.5, 1.0, 2.0 ** -40, 0.0, -0.5, np.inf, -np.inf, np.nan):
            q[0, 0, 1] = value
            n_accepted, out = _verified(p, q, tokens, np.array([[u, 0.25, 0.5]], np.float32), dtype)
            assert n_accepted.tolist() == [0] and out.tolist() == [[3, -1, -1]], (value, u)
    q[0, 0, 1] = 0.5   # (and with a number in its place: u q < p)
    n_accepted, out = _verified(p, q, tokens, np.array([[0.5, 0.25, 0.5]], np.float32), dtype)
    assert n_accepted.tolist() == [2] and out.tolist() == [[1, 1, 1]]


def test_verification_takes_distributions_that_sequences_share():
    """Strides of zero: one target for all sequences of the batch."""
    rng = np.random.default_rng(8)
    p, q, tokens, uniform = _verify_problem(rng, 1, 3, 1000, "f32", False)
    tokens, uniform = np.repeat(tokens, 9, 0), rng.random((9, 4), dtype=np.float32)
    dev = [P.to_dev(x, "f32", DEV).expand(9, -1, -1) for x in (p, q)]
    n_accepted, out = _pk().DraftBuffers(dev[0], _ints(tokens.tolist()), torch.from_numpy(uniform).to(DEV), draft=dev[1]).verify()
    _check_verified((n_accepted.cpu().numpy(), out.cpu().numpy()), np.repeat(p, 9, 0), np.repeat(q, 9, 0), tokens, uniform)


# ---- who holds the pages -----------------------------------------------------------------------------------------------

def _same(seqs, book, lacking, what):
    assert seqs.lacking.item() == lacking, what
    assert seqs.held.tolist() == [len(r) for r in book.rows], what
    assert np.array_equal(seqs.page_table.cpu().numpy(), book.table()), what
    assert seqs.ref.tolist() == book.ref, what


@pytest.mark.parametrize("n_pages,page_len,batch,max_pages", [(1, 1, 1, 1), (40, 16, 5, 9), (300, 64, 70, 6), (5000, 16, 33, 150), (9000, 1, 300, 60),
                                                              (70000, 32, 9, 9000), (4096, 256, 1, 4096), (20000, 16, 1500, 12),
                                                              (32769, 16, 40, 300), (131072, 8, 150, 200), (131073, 16, 3, 50)])
def test_pages_that_come_and_go(n_pages, page_len, batch, max_pages):
    """Calls of every kind in a row, more than there are pages for among them; the table's entries hold anything beforehand."""
    pk, rng = _pk(), np.random.default_rng(n_pages)
    ref = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    counts = [0] * n_pages
    for i in range(0, n_pages, 7):   # other holders', for good
        if n_pages > 1:
            counts[i] = 1
    ref.copy_(_ints(counts))
    a, b = (pk.PagedSequences(ref, torch.full((batch, max_pages), -1, dtype=torch.int32, device=DEV),
                              torch.zeros(batch, dtype=torch.int32, device=DEV), page_len) for _ in range(2))
    a.workspace.fill_(0xFF)
    books = [G.Book(counts, page_len, batch, max_pages) for _ in range(2)]
    each = max(int(0.4 * n_pages / batch), 1) * page_len   # tokens that half of the pool has room for
    lens = [0] * batch
    for step in range(8):
        kind = step % 4
        if kind == 3:   # the other batch goes on from this one, parents repeated, some missing, some unborn
            parents = [int(x) for x in rng.integers(-1, batch + 1, batch)]
            cached = [int(x) for x in rng.integers(-5, max(max(lens), 1) + page_len + 2, batch)]
            b.fork(a, _ints(parents), _ints(cached))
            first, kids, lacking = books[1].fork(books[0], parents, cached)
            torch.cuda.synchronize()
            assert b.first.tolist() == first and b.lens.tolist() == kids, step
            _same(b, books[1], lacking, step)
            a, b = b, a
            books.reverse()
            lens = kids
            continue
        if kind == 0:
            lens = [int(x) for x in rng.integers(-2, 2 * each + 2, batch)]
        elif kind == 1:
            lens = [max(t + int(x), 0) for t, x in zip(lens, rng.integers(-3 * page_len, 2 * page_len, batch))]
        else:
            lens = [(0, t, 2 ** 31 - 1)[int(x)] if rng.random() < 0.3 else t for t, x in zip(lens, rng.integers(0, 3, batch))]
        a.resize(_ints(lens))
        lacking = books[0].resize(lens)
        torch.cuda.synchronize()
        _same(a, books[0], lacking, step)
        lens = [min(max(t, 0), len(r) * page_len) for t, r in zip(lens, books[0].rows)]
    for seqs, book in ((a, books[0]), (b, books[1])):   # and all of it back
        seqs.resize(torch.zeros(batch, dtype=torch.int32, device=DEV))
        assert book.resize([0] * batch) == 0
    torch.cuda.synchronize()
    assert ref.tolist() == counts and set(counts) <= {0, 1}


@pytest.mark.parametrize("batch,kids,n_pages", [(3, 5, 100), (40, 90, 40000), (7, 300, 3000), (2, 1100, 2500)])
def test_children_with_less_room_than_their_parents(batch, kids, n_pages):
    """Tables of other widths, and fewer free pages than last pages that want one; the same fork again changes nothing."""
    pk, rng = _pk(), np.random.default_rng(70)
    seqs = pk.PagedSequences.allocate(n_pages, 16, batch, 20, DEV)
    lens = [int(x) for x in rng.integers(0, 320, batch)]
    counts = [0] * n_pages
    book, theirs = G.Book(counts, 16, batch, 20), G.Book(counts, 16, kids, 11)
    seqs.resize(_ints(lens))
    assert book.resize(lens) == 0
    child = seqs.another(kids, 11)
    parents = [int(x) for x in rng.integers(0, batch, kids)]
    for _ in range(3):
        child.fork(seqs, _ints(parents), _ints(lens))
        first, got, lacking = theirs.fork(book, parents, lens)
        torch.cuda.synchronize()
        assert child.first.tolist() == first and child.lens.tolist() == got
        _same(child, theirs, lacking, "")
    child.resize(torch.zeros(kids, dtype=torch.int32, device=DEV))
    theirs.resize([0] * kids)
    _same(seqs, book, 0, "")


@pytest.mark.parametrize("n_pages,batch,max_pages", [(20000, 30, 100), (32769, 30, 100), (65536, 300, 20), (131072, 100, 40), (140000, 30, 100)])
@pytest.mark.parametrize("busy", [0.5, 0.99])
def test_free_pages_among_others_pages(n_pages, batch, max_pages, busy):
    """Pages that other tables hold, here and there, at the pool's start and nearly everywhere; some calls want more than there are."""
    rng = np.random.default_rng(n_pages)
    seqs = _pk().PagedSequences.allocate(n_pages, 16, batch, max_pages)
    ref = (rng.random(n_pages) < busy).astype(np.int64) * rng.integers(1, 4, n_pages)
    ref[:n_pages // 3] = 1
    seqs.ref.copy_(_ints(ref.tolist()))
    book = G.Book(ref.tolist(), 16, batch, max_pages)
    for step in range(4):
        lens = rng.integers(0, 16 * max_pages + 40, batch)
        lacking = book.resize(lens.tolist())
        seqs.resize(_ints(lens.tolist()))
        _same(seqs, book, lacking, step)
    kids, kid_book = seqs.another(batch), G.Book(book.ref, 16, batch, max_pages)
    parents = rng.integers(-1, batch, batch)
    first, got, lacking = kid_book.fork(book, parents.tolist(), lens.tolist())
    kids.fork(seqs, _ints(parents.tolist()), _ints(lens.tolist()))
    _same(kids, kid_book, lacking, "fork")
    assert kids.first.tolist() == first and kids.lens.tolist() == got


def test_owners_that_hold_nonsense_stay_inside_the_arrays():
    """Counts of held pages and entries outside the pool: what is beside the arrays stays as it is."""
    pk = _pk()
    room = torch.full((4096,), 5, dtype=torch.int32, device=DEV)
    ref, table, held = room[1000:1050], room[2000:2024].view(3, 8), room[3000:3003]
    ref.zero_()
    seqs = pk.PagedSequences(ref, table, held, 16)
    for nonsense in ([-7, 2 ** 31 - 1, 100], [8, 9, -2 ** 31]):
        table.copy_(_ints([[-1, 50, 51, 2 ** 31 - 1, -2 ** 31, 3, 4, 10 ** 9]] * 3))
        held.copy_(_ints(nonsense))
        seqs.resize(_ints([17, 0, 1000]))
        other = seqs.another(4)
        other.fork(seqs, _ints([0, 1, 2, 2]), _ints([30, 1000, 2 ** 31 - 1]))
        torch.cuda.synchronize()
        assert all(0 <= n <= 8 for n in held.tolist() + other.held.tolist())
    keep = torch.ones(4096, dtype=torch.bool, device=DEV)
    for a, b in ((1000, 1050), (2000, 2024), (3000, 3003)):
        keep[a:b] = False
    assert bool((room[keep] == 5).all())


# ---- rows that move ----------------------------------------------------------------------------------------------------

def _pool_bits(pool):
    k, v = (x.view(torch.uint8) if pool.fp8 else x.view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32) for x in (pool.k_pages, pool.v_pages))
    return [x.clone() for x in (k, v, pool.k_scale, pool.v_scale) if x is not None]


def _moved(before, after, src, dst):
    """Every row (page, head, slot) of dst holds what the one of src held in `before`, and nothing else has changed."""
    for x, y in zip(before, after):
        want = x.clone()
        if len(src):
            s, d = (torch.tensor(np.array(i), device=DEV).unbind(1) for i in (src, dst))
            want[d] = x[s]
        assert torch.equal(want, y)


MOVE_CASES = [dict(dtype="bf16", fp8=True, n_kv=2, d=128, page_len=16), dict(dtype="bf16", fp8=True, n_kv=3, d=64, page_len=64),
              dict(dtype="bf16", fp8=False, n_kv=2, d=128, page_len=1), dict(dtype="bf16", fp8=False, n_kv=8, d=64, page_len=32),
              dict(dtype="f32", fp8=False, n_kv=2, d=128, page_len=16), dict(dtype="f32", fp8=False, n_kv=1, d=64, page_len=128),
              dict(dtype="f32", fp8=True, n_kv=2, d=128, page_len=16)]


def _two_tables(case, rng, lens, room, layout):
    """A pool with the sequences' rows, and a second table [.., room[b] positions] over pages that none of them holds."""
    n_kv, d, page_len = case["n_kv"], case["d"], case["page_len"]
    extra = sum(-(-r // page_len) for r in room)
    rows = [[_rows(rng, n, n_kv, d, case["dtype"]) for n in lens] for _ in range(2)]
    pool = P.Pool(rng, *rows, n_kv, d, page_len, case["dtype"], case["fp8"], layout=layout, spare=extra + 2)
    unused = rng.permutation(sorted(set(range(pool.k_pages.shape[0])) - set(pool.table[pool.table >= 0].tolist())))
    to = np.full((len(room), max(max(-(-r // page_len) for r in room), 1)), -1, dtype=np.int64)
    at = 0
    for i, r in enumerate(room):
        n = -(-r // page_len)
        to[i, :n] = unused[at:at + n]
        at += n
    return pool, to


@pytest.mark.parametrize("layout", ["heads", "tokens"])
@pytest.mark.parametrize("case", MOVE_CASES, ids=_ids)
def test_listed_rows_move_and_nothing_else(case, layout):
    """Lists of other lengths for each head (none, one, all), out of order and repeated; entries behind a list's length name nothing; one
    sequence has too few pages, and one none: their rows are dropped."""
    pk, rng = _pk(), np.random.default_rng(51)
    lens, P_len, n_kv = [300, 1, 77, 130, 0], case["page_len"], case["n_kv"]
    room = [300, 1, 40, 0, 5]
    pool, to = _two_tables(case, rng, lens, room, layout)
    B = 300
    idx, cnt = np.full((5, n_kv, B), -9, np.int64), np.zeros((5, n_kv), np.int64)
    src, dst = [], []
    for b, t in enumerate(lens):
        for kv in range(n_kv):
            n = (0, 1, t, t // 3)[int(rng.integers(0, 4))] if t else 0
            if b == 0:
                n = (t, t // 2, 1)[kv % 3]
            cnt[b, kv] = n
            picked = rng.permutation(t)[:n] if kv % 2 else np.sort(rng.choice(t, n, replace=True)) if t else []
            idx[b, kv, :n] = picked
            for j, pos in enumerate(picked):
                page = to[b, j // P_len] if j // P_len < to.shape[1] else -1
                if page >= 0:
                    src.append((pool.table[b, pos // P_len], kv, pos % P_len))
                    dst.append((page, kv, j % P_len))
    before = _pool_bits(pool)
    cache = pool.cache()
    target = pk.PagedCache(pool.k_pages, pool.v_pages, _ints(to.tolist()), pool.k_scale, pool.v_scale)
    # (as many pages a row as the longest list may take: entries past the others are -1)
    wide = torch.full((5, -(-B // P_len)), -1, dtype=torch.int32, device=DEV)
    wide[:, :to.shape[1]] = target.page_table[:, :wide.shape[1]]
    target.page_table = wide
    target.compact(cache, _ints(idx.tolist()), _ints(cnt.tolist()))
    torch.cuda.synchronize()
    src, dst = ([(int(p), k, int(s)) for p, k, s in x] for x in (src, dst))
    _moved([x for x in before], _pool_bits(pool), [list(x) for x in src], [list(x) for x in dst])


def test_listed_rows_move_between_pools_and_page_lengths():
    """Into a pool of its own, of longer pages and other strides; malformed entries are cut to the cache, and none leaves it."""
    pk, rng = _pk(), np.random.default_rng(52)
    case = dict(dtype="bf16", fp8=True, n_kv=2, d=128, page_len=16)
    k, v = ([_rows(rng, 200, 2, 128, "bf16")] for _ in range(2))
    pool = P.Pool(rng, k, v, 2, 128, 16, "bf16", True)
    there = P.Pool(rng, [np.zeros((0, 2, 128))], [np.zeros((0, 2, 128))], 2, 128, 64, "bf16", True, layout="tokens", n_pages=5, table_cols=4)
    there.dev_table.copy_(_ints([[4, 0, 2, 9]]))   # the last is no page
    idx = np.stack([np.sort(rng.choice(200, 150, replace=False)) for _ in range(2)])[None]
    target = there.cache()
    target.compact(pool.cache(), _ints(idx.tolist()), _ints([[150, 149]]))
    torch.cuda.synchronize()
    got, want = there.k_pages.view(torch.uint8), pool.k_pages.view(torch.uint8)
    for kv, n in ((0, 150), (1, 149)):
        for j in range(n):
            t = int(idx[0, kv, j])
            at, of = (int([4, 0, 2][j // 64]), kv, j % 64), (int(pool.table[0, t // 16]), kv, t % 16)
            assert torch.equal(got[at], want[of]) and there.k_scale[at] == pool.k_scale[of] and there.v_scale[at] == pool.v_scale[of]
    assert bool((got[2, 1, 21:] == 0x7F).all()) and bool((got[[1, 3]] == 0x7F).all())
    del case
    pool.dev_table[0, 3] = 10 ** 9
    pool.dev_table[0, 5] = -3
    target.compact(pool.cache(), torch.full((1, 2, 150), 2 ** 31 - 1, dtype=torch.int32, device=DEV), _ints([[150, 2 ** 31 - 1]]))
    target.compact(pool.cache(), torch.full((1, 2, 150), -5, dtype=torch.int32, device=DEV), _ints([[-3, 150]]))
    target.compact(pool.cache(), _ints((idx * 0 + 50).tolist()), _ints([[150, 150]]))
    torch.cuda.synchronize()
    assert bool((there.k_pages.view(torch.uint8)[[1, 3]] == 0x7F).all())


@pytest.mark.parametrize("dtype", [torch.float8_e4m3fn, torch.bfloat16])
def test_listed_rows_of_the_longest_caches_move(dtype):
    """Positions up to the last that a cache of 2^24 - 1 tokens has, through a table that repeats a few pages; rows of different bits."""
    pk, page_len, d = _pk(), 65536, 128
    table = torch.zeros(1, 256, dtype=torch.int32, device=DEV)
    table[0, 128], table[0, 255] = 1, 2
    cache = pk.PagedCache.allocate(3, page_len, 1, d, table, dtype=dtype)
    for i, x in enumerate((cache.k_pages, cache.v_pages)):
        bits = x.view(torch.uint8) if x.element_size() == 1 else x.view(torch.int16)
        bits.copy_(torch.randint(0, 100, bits.shape, device=DEV, generator=torch.Generator(DEV).manual_seed(i)).to(bits.dtype))
    for x in (cache.k_scale, cache.v_scale):
        if x is not None:
            x.copy_(torch.randint(100, 150, x.shape, device=DEV).to(torch.uint8))
    to = pk.PagedCache.allocate(1, 16, 1, d, torch.zeros(1, 1, dtype=torch.int32, device=DEV), dtype=dtype)
    at = [2 ** 23 - 3, 2 ** 23 - 2, 2 ** 23 - 1, 2 ** 23, 2 ** 23 + 77, 2 ** 24 - 65537, 2 ** 24 - 65536, 2 ** 24 - 2]
    to.compact(cache, _ints([[at]]), _ints([[len(at)]]))
    pages = table[0].tolist()
    for src, dst in ((cache.k_pages, to.k_pages), (cache.v_pages, to.v_pages), (cache.k_scale, to.k_scale), (cache.v_scale, to.v_scale)):
        if src is None:
            continue
        for j, t in enumerate(at):
            x, y = (z.reshape(-1).view(torch.uint8) for z in (dst[0, 0, j].clone(), src[pages[t // page_len], 0, t % page_len].clone()))
            assert torch.equal(x, y), (j, t)


@pytest.mark.parametrize("layout", ["heads", "tokens"])
@pytest.mark.parametrize("case", MOVE_CASES, ids=_ids)
def test_copied_rows_keep_their_positions(case, layout):
    """Rows first .. lens - 1 of the parents: a page's rest, none, whole sequences; parents repeated and missing, more rows than are asked for."""
    pk, rng = _pk(), np.random.default_rng(53)
    lens, P_len, n_kv = [290, 5, 64], case["page_len"], case["n_kv"]
    parents = [0, 0, 1, 2, 2, -1, 3, 0]
    until = [290, 290, 5, 64, 0, 9, 9, -4]
    for first, most in ((None, 1000), ([t // P_len * P_len for t in until], None), ([280, 285, 6, 1, 0, 0, 0, -2 ** 31], 3), ([-5, 290, 2 ** 31 - 1, 0, 0, 0, 0, 0], 290)):
        pool, to = _two_tables(case, rng, lens, [max(t, 1) for t in until], layout)
        src, dst = [], []
        for b, (p, t) in enumerate(zip(parents, until)):
            f = 0 if first is None else max(first[b], 0)
            for pos in range(f, min(max(t, 0), f + (P_len if most is None else most))):
                if 0 <= p < 3:
                    src += [[int(pool.table[p, pos // P_len]), kv, pos % P_len] for kv in range(n_kv)]
                    dst += [[int(to[b, pos // P_len]), kv, pos % P_len] for kv in range(n_kv)]
        before = _pool_bits(pool)
        target = pk.PagedCache(pool.k_pages, pool.v_pages, _ints(to.tolist()), pool.k_scale, pool.v_scale)
        target.copy(pool.cache(), _ints(parents), None if first is None else _ints(first), _ints(until), max_rows=most)
        torch.cuda.synchronize()
        _moved(before, _pool_bits(pool), src, dst)


def test_rows_that_the_source_has_no_page_for_are_dropped():
    """Entries that name no page of the pool, and positions past the source's table: what is in their place stays as it was."""
    pk, rng = _pk(), np.random.default_rng(56)
    pool = P.Pool(rng, [_rows(rng, 64, 2, 64, "bf16")], [_rows(rng, 64, 2, 64, "bf16")], 2, 64, 16, "bf16", False)
    source = pool.cache()
    pool.dev_table[0, 1] = -1
    pool.dev_table[0, 3] = pool.k_pages.shape[0]
    there = [torch.full((8, 2, 16, 64), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    target = pk.PagedCache(*there, _ints([list(range(8))]))
    one, shape = target._moves(source, 64, 3), bytes(target._moves(source, 64, 3))
    target.copy(source, lens=_ints([128]), max_rows=128)   # (the source's table has four pages)
    for page in range(8):
        for x, y in zip(there, (pool.k_pages, pool.v_pages)):
            assert torch.equal(x[page], y[int(pool.table[0, page])]) if page in (0, 2) else bool((x[page] == 7.0).all())
    for x in there:
        x.fill_(7.0)
    idx = torch.arange(60, 0, -1, dtype=torch.int32, device=DEV).expand(1, 2, 60).contiguous()
    target.compact(source, idx, _ints([[60, 60]]))
    for j in range(60):
        t = 60 - j
        for x, y in zip(there, (pool.k_pages, pool.v_pages)):
            got = x[j // 16, :, j % 16]
            assert torch.equal(got, y[int(pool.table[0, t // 16]), :, t % 16]) if t // 16 in (0, 2) else bool((got == 7.0).all())
    assert bytes(one) == shape   # (calls share nothing that they change)


def test_tensors_of_the_host_are_refused():
    pk = _pk()
    ints = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    cache, other = (pk.PagedCache(torch.zeros(4, 2, 16, 64), torch.zeros(4, 2, 16, 64), ints([0, 1])) for _ in range(2))
    seqs = pk.PagedSequences.allocate(4, 16, 1, 4, "cpu")
    drafts = pk.DraftBuffers(torch.zeros(1, 3, 9), ints([0, 1]), torch.zeros(1, 3))
    for call in (lambda: other.copy(cache, lens=ints(3)), lambda: other.compact(cache, torch.zeros(1, 2, 3, dtype=torch.int32), torch.ones(1, 2, dtype=torch.int32)),
                 lambda: seqs.resize(ints(3)), lambda: seqs.another(1).fork(seqs, ints(0), ints(3)), drafts.verify):
        with pytest.raises(ValueError, match="no GPU"):
            call()


def test_a_cache_is_copied_into_another_pool():
    """No parents and one page table for both: the same sequences in a pool of other strides."""
    pk, rng = _pk(), np.random.default_rng(54)
    pool = P.Pool(rng, [_rows(rng, n, 2, 64, "bf16") for n in (100, 33)], [_rows(rng, n, 2, 64, "bf16") for n in (100, 33)], 2, 64, 16, "bf16", False)
    other = torch.full_like(pool.k_pages, 7.0), torch.full_like(pool.v_pages, 7.0)
    to = pk.PagedCache(*other, pool.dev_table)
    to.copy(pool.cache(), lens=_ints([100, 33]), max_rows=100)
    back = [torch.empty(2, 2, 100, 64, dtype=torch.bfloat16, device=DEV) for _ in range(4)]
    for cache, out in ((to, back[:2]), (pool.cache(), back[2:])):
        pk.PagedBuffers(cache, [100, 33], 100).read(*out)
    torch.cuda.synchronize()
    for x, y in zip(back[:2], back[2:]):
        assert torch.equal(x[0], y[0]) and torch.equal(x[1, :, :33], y[1, :, :33])
    assert bool((other[0].float() == 7.0).any())


def test_rows_beyond_four_gib_of_a_pool_move():
    pk = _pk()
    n_kv, d, page_len = 8, 128, 64
    n_pages = (1 << 32) // (n_kv * page_len * d * 2) + 7
    pages = [torch.zeros(n_pages, n_kv, page_len, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    src, dst = [n_pages - 1, n_pages - 5], [n_pages - 2, n_pages - 4]
    for p in pages:
        p[src] = torch.randn(2, n_kv, page_len, d, device=DEV).bfloat16()
    cache, to = (pk.PagedCache(*pages, _ints([t])) for t in (src, dst))
    idx = torch.arange(5, 105, dtype=torch.int32, device=DEV).expand(1, n_kv, 100).contiguous()
    to.compact(cache, idx, torch.full((1, n_kv), 100, dtype=torch.int32, device=DEV))
    for p in pages:
        rows, got = (p[x].transpose(0, 1).reshape(n_kv, -1, d) for x in (src, dst))
        assert torch.equal(got[:, :100], rows[:, 5:105]) and not got[:, 100:].any()
    to.copy(cache, lens=_ints([127]), max_rows=128)
    for p in pages:
        rows, got = (p[x].transpose(0, 1).reshape(n_kv, -1, d) for x in (src, dst))
        assert torch.equal(got[:, :127], rows[:, :127]) and not got[:, 127:].any()


# ---- together ----------------------------------------------------------------------------------------------------------

def _pages_step(pk, fp8):
    """Beams over two prompts: state of a small generation loop, all of whose calls can be recorded."""
    n_kv, n_q, d, page_len, n = 2, 8, 128, 16, 3
    rng = np.random.default_rng(60)
    prompts, batch, V = [45, 32], 5, 700
    seqs = pk.PagedSequences.allocate(80, page_len, 2, 12, DEV)
    kids = seqs.another(batch)
    dtype = torch.float8_e4m3fn if fp8 else torch.bfloat16
    cache = pk.PagedCache.allocate(80, page_len, n_kv, d, seqs.page_table, dtype=dtype)
    kid_cache = pk.PagedCache(cache.k_pages, cache.v_pages, kids.page_table, cache.k_scale, cache.v_scale)
    k, v = ([_rows(rng, t, n_kv, d, "bf16") for t in prompts] for _ in range(2))
    new = [torch.zeros(2, n_kv, 45, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    for t, x in zip(new, (k, v)):
        for i in range(2):
            t[i, :, :prompts[i]] = P.to_dev(x[i].transpose(1, 0, 2), "bf16", DEV)
    seqs.resize(_ints(prompts))
    pk.PagedBuffers(cache, [0, 0], 0, k_chunk=new[0], v_chunk=new[1], chunk_lens=prompts).write()
    return dict(locals())


def _as_kept(x, fp8):
    if not fp8:
        return x
    y, e = P.quantise(x)
    return np.ldexp(y, (e - 127)[..., None])


@pytest.mark.parametrize("fp8", [False, True])
def test_drafts_of_beams_are_attended_verified_and_cut(fp8):
    """Two prompts go on in five beams; in each step every beam drafts three tokens, which are written, attended and verified, and the pages of
    refused ones are given back.  Outputs are those of attention over rows of each beam's own."""
    pk = _pk()
    s = _pages_step(pk, fp8)
    rng, n, batch, V = s["rng"], s["n"], s["batch"], s["V"]
    seqs, kids = s["seqs"], s["kids"]
    parents = [0, 1, 0, 0, 1]
    kids.fork(seqs, _ints(parents), _ints(s["prompts"]))
    s["kid_cache"].copy(s["cache"], _ints(parents), kids.first, kids.lens)
    seqs.resize(_ints([0, 0]))   # the prompts' own table is given up; what the beams share stays
    lens = kids.lens
    assert lens.tolist() == [s["prompts"][p] for p in parents] and (kids.ref > 0).sum().item() == 2 + 2 + 3
    kept_k, kept_v = ([list(_as_kept(x[p], fp8)) for p in parents] for x in (s["k"], s["v"]))
    for step in range(6):
        kids.resize(lens + (n + 1))
        q, k, v = (P.store(rng.standard_normal((batch, h, n + 1, s["d"])), "bf16") for h in (s["n_q"], s["n_kv"], s["n_kv"]))
        buf = pk.PagedBuffers(s["kid_cache"], lens, 100, q=P.to_dev(q, "bf16", DEV), k_chunk=P.to_dev(k, "bf16", DEV), v_chunk=P.to_dev(v, "bf16", DEV))
        buf.write()
        out = buf.attn().float().cpu().numpy()
        p, dq, tokens, uniform = _verify_problem(rng, batch, n, V, "f32", False)
        n_accepted, toks = pk.DraftBuffers(P.to_dev(p, "f32", DEV), _ints(tokens.tolist()), torch.from_numpy(uniform).to(DEV), draft=P.to_dev(dq, "f32", DEV)).verify()
        assert kids.lacking.item() == 0
        _check_verified((n_accepted.cpu().numpy(), toks.cpu().numpy()), p, dq, tokens, uniform)
        for i in range(batch):
            kk = np.stack(kept_k[i] + list(_as_kept(k[i].transpose(1, 0, 2).astype(np.float64), fp8)))
            vv = np.stack(kept_v[i] + list(_as_kept(v[i].transpose(1, 0, 2).astype(np.float64), fp8)))
            want, _, weight = P.attention(q[i].astype(np.float64), kk, vv, len(kept_k[i]))
            assert np.all(np.abs(out[i] - want) <= 1.05 * 2.0 ** -8 * (weight + np.abs(want)) + 1e-6), (step, i)
            m = len(kept_k[i]) + int(n_accepted[i]) + 1
            kept_k[i], kept_v[i] = list(kk[:m]), list(vv[:m])
        lens = lens + n_accepted + 1
        kids.resize(lens)
        assert lens.tolist() == [len(x) for x in kept_k] and kids.held.tolist() == [-(-len(x) // 16) for x in kept_k]
    kids.resize(torch.zeros_like(lens))
    assert not kids.ref.any()


def test_a_recorded_step_of_forks_drafts_and_cuts():
    """Fork, copy, room, write, attention, verification, cut: recorded once and replayed, each replay against the eager calls from the same
    state."""
    pk = _pk()
    s = _pages_step(pk, True)
    seqs, kids, n, batch, d = s["seqs"], s["kids"], s["n"], s["batch"], s["d"]
    parents, lens = _ints([0, 1, 0, 0, 1]), _ints(s["prompts"])
    shape = lambda h: torch.randn(batch, h, n + 1, d, device=DEV).bfloat16()  # noqa: E731
    q, k, v = shape(s["n_q"]), shape(s["n_kv"]), shape(s["n_kv"])
    probs = [torch.rand(batch, n + 1, s["V"], device=DEV), torch.rand(batch, n, s["V"], device=DEV)]
    tokens, uniform = torch.zeros(batch, n, dtype=torch.int32, device=DEV), torch.rand(batch, n + 1, device=DEV)
    room, stay = _ints([0] * batch), _ints([0] * batch)
    buf = pk.PagedBuffers(s["kid_cache"], kids.lens, 100, q=q, k_chunk=k, v_chunk=v)
    assert buf.kv_lens.data_ptr() == kids.lens.data_ptr()
    drafts = pk.DraftBuffers(probs[0], tokens, uniform, draft=probs[1])

    def step():
        kids.fork(seqs, parents, lens)
        s["kid_cache"].copy(s["cache"], parents, kids.first, kids.lens)
        torch.add(kids.lens, n + 1, out=room)
        kids.resize(room)
        buf.write()
        buf.attn()
        drafts.verify()
        torch.add(kids.lens, drafts.n_accepted, out=stay)
        stay.add_(1)
        kids.resize(stay)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    torch.cuda.synchronize()
    watched = (buf.out, buf.lse, drafts.n_accepted, drafts.tokens_out, kids.page_table, kids.held, kids.ref, kids.lens, kids.lacking)
    for rep in range(4):
        for t in (q, k, v):
            t.copy_(torch.randn_like(t))
        for t in (*probs, uniform):
            t.copy_(torch.rand_like(t))
        parents.copy_(_ints([[0, 1, 0, 0, 1], [1, 1, 1, 1, 1], [-1, 0, 9, 1, 0], [0, 0, 0, 0, 0]][rep]))
        lens.copy_(_ints([[45, 32], [45, 31], [40, 1], [0, 32]][rep]))
        buf.out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in watched]
        float(torch.randn(1 << 16, device=DEV).sum())
        buf.out.fill_(float("nan"))
        step()
        torch.cuda.synchronize()
        for i, (x, y) in enumerate(zip(got, watched)):
            assert torch.equal(x, y), (rep, i)


def test_a_cache_is_cut_down_to_selected_keys():
    """The keys that the method selects for a chunk move to pages of their own, the others are given back: cross attention over them, with the
    chunk's queries, is attention over the list."""
    pk, rng = _pk(), np.random.default_rng(61)
    n_kv, n_q, d, T, B, C = 2, 8, 128, 700, 150, 40
    seqs = pk.PagedSequences.allocate(200, 16, 1, 60, DEV)
    cache = pk.PagedCache.allocate(200, 16, n_kv, d, seqs.page_table)
    rows = [torch.randn(1, n_kv, T + C, d, device=DEV).bfloat16() for _ in range(2)]
    q = torch.randn(1, n_q, C, d, device=DEV).bfloat16()
    seqs.resize(_ints([T + C]))
    pk.PagedBuffers(cache, [0], 0, k_chunk=rows[0][:, :, :T], v_chunk=rows[1][:, :, :T]).write()
    buf = pk.PagedBuffers(cache, [T], T, q=q, k_chunk=rows[0][:, :, T:].contiguous(), v_chunk=rows[1][:, :, T:].contiguous(), budgets=[B], n_retain=16)
    buf.chunk_attn()
    fewer = seqs.another(1)
    fewer.resize(buf.k_cnt[:, 0].contiguous())
    kept = pk.PagedCache(cache.k_pages, cache.v_pages, fewer.page_table, cache.k_scale, cache.v_scale)
    kept.compact(cache, buf.k_idx, buf.k_cnt)
    whole = [torch.empty(1, n_kv, T, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    pk.PagedBuffers(cache, [T], T).read(*whole)
    seqs.resize(_ints([0]))
    got = [torch.empty(1, n_kv, B, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    pk.PagedBuffers(kept, buf.k_cnt[:, 0], B).read(*got)
    for x, y in zip(got, whole):
        assert torch.equal(x, torch.gather(y, 2, buf.k_idx.long().unsqueeze(-1).expand(-1, -1, -1, d)))
    assert (seqs.ref > 0).sum().item() == -(-B // 16)
    over = pk.PagedBuffers(kept, buf.k_cnt[:, 0], B, q=q)
    over.cross_attn()
    torch.cuda.synchronize()
    k, v = (x[0].float().cpu().numpy().transpose(1, 0, 2).astype(np.float64) for x in got)
    want, lse, weight = G.cross(q[0].float().cpu().numpy().astype(np.float64), k, v)
    assert np.all(np.abs(over.out[0].float().cpu().numpy() - want) <= 1.05 * 2.0 ** -8 * (weight + np.abs(want)) + 1e-6)
    assert np.all(np.abs(over.lse[0].cpu().numpy() - lse) <= 1e-4)
