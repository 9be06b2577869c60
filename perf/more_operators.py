"""Timed cases of generation over caches in pages: attention of tokens over an encoder's states, verification of drafted tokens,
and the upkeep of the pages themselves (sequences that grow, are cut and are given up; sequences that go on from others; caches
cut down to chosen rows).

A case is what a serving program calls once a step (or once a prompt) on the buffers that it keeps.  Sizes are those of this
repository's workloads, benchmark and tests, or generic ones of the same ranges.

Fields of a case
  op         "cross": attention of a chunk over the cached rows alone, none of which is the chunk's own
             "verify": how many drafted tokens the target's probabilities accept, and the token after them
             "resize": sequences cut to the tokens that stay, then given room for the next ones
             "fork": sequences that go on from others: whole pages are shared, the rows of the last one copied
             "compact": the listed rows of every KV head, one behind the other, in other pages
  batch      sequences; page_len: tokens per page
  cross, compact, fork
    dtype    "bf16" or "f32";  pages: "raw": rows as they are, "fp8": 8-bit elements and a scale for each row
    n_q, n_kv, d     query heads, KV heads, head size
    kv_max, kv_min   cached tokens per sequence: the first one kv_max, the last one kv_min, the others in between
  cross      chunk, chunk_min: queries per sequence, likewise
  compact    keep: rows of a list, of each KV head
  fork       parents: sequences that the batch goes on from
  verify     vocab, drafts: tokens drafted (drafts_min: for the last sequence), dtype of the probabilities,
             lookup: the drafts come without probabilities of their own
  resize     pool: pages there are; kv_max, kv_min; cut: most tokens that a sequence loses; grow: tokens of room it then gets;
             done: one sequence in so many is given up and another prompt of kv_max takes its place (0: none)
"""
import math

import torch

own = False   # False: the operators in plain torch; True: the framework's entry points

SPARE_PAGES = 5   # pages of a pool that no sequence holds


def _cross(name, dtype="bf16", pages="raw", batch=1, n_q=32, n_kv=8, d=128, chunk=1, chunk_min=None, page_len=64, kv_max=8192,
           kv_min=None):
    return _named(name, op="cross", dtype=dtype, pages=pages, batch=batch, n_q=n_q, n_kv=n_kv, d=d, chunk=chunk,
                  chunk_min=chunk if chunk_min is None else chunk_min, page_len=page_len, kv_max=kv_max,
                  kv_min=kv_max if kv_min is None else kv_min)


def _verify(name, batch, vocab, drafts, drafts_min=None, dtype="f32", lookup=False):
    return _named(name, op="verify", batch=batch, vocab=vocab, drafts=drafts, drafts_min=drafts if drafts_min is None else drafts_min,
                  dtype=dtype, lookup=lookup)


def _resize(name, batch, pool, page_len, kv_max, kv_min, cut, grow, done=0):
    return _named(name, op="resize", batch=batch, pool=pool, page_len=page_len, kv_max=kv_max, kv_min=kv_min, cut=cut, grow=grow, done=done)


def _fork(name, batch, parents, page_len, kv_max, kv_min, dtype="bf16", pages="raw", n_kv=8, d=128):
    return _named(name, op="fork", batch=batch, parents=parents, page_len=page_len, kv_max=kv_max, kv_min=kv_min, dtype=dtype,
                  pages=pages, n_q=n_kv, n_kv=n_kv, d=d)


def _compact(name, batch, keep, page_len, kv_max, kv_min, dtype="bf16", pages="raw", n_kv=8, d=128):
    return _named(name, op="compact", batch=batch, keep=keep, page_len=page_len, kv_max=kv_max, kv_min=kv_min, dtype=dtype, pages=pages,
                  n_q=n_kv, n_kv=n_kv, d=d)


def _named(name, **fields):
    return dict(fields, name=name) if name else fields


def listed():
    return [
        # one generated token of eight sequences over their encoder's states, heads of their own: latency
        _cross("cross_token", batch=8, n_q=12, n_kv=12, d=64, kv_max=1500, kv_min=200),
        # one token of a full serving batch over long states in 8 bits: a gigabyte of them
        _cross("cross_token_full", pages="fp8", batch=32, kv_max=32768, kv_min=1024),
        # a prompt's chunk over the states of a long document
        _cross("cross_prompt", chunk=2048, kv_max=16384),
        # nothing divides anything: three heads a group, ragged float32 chunks, states of one sequence missing
        _cross("cross_odd", dtype="f32", batch=3, n_q=9, n_kv=3, d=64, chunk=333, chunk_min=57, page_len=32, kv_max=1999, kv_min=0),
        # one sequence's tokens from a prompt lookup, an odd vocabulary: the smallest verification
        _verify("verify_lookup", batch=1, vocab=32003, drafts=4, lookup=True),
        # a full batch of drafts with their probabilities, some shorter than others
        _verify("verify_batch", batch=64, vocab=131072, drafts=7, drafts_min=2),
        # sixteen sequences after a verified step: rejected tokens go, the next step's come
        _resize("resize_step", batch=16, pool=8192, page_len=16, kv_max=4096, kv_min=100, cut=7, grow=8),
        # a large pool of long sequences, of which some have ended and give way to new prompts
        _resize("resize_prompts", batch=256, pool=262144, page_len=16, kv_max=16384, kv_min=300, cut=40, grow=48, done=8),
        # sixteen beams, four from each of four hypotheses of unequal length
        _fork("fork_beams", batch=16, parents=4, page_len=64, kv_max=4001, kv_min=900),
        # samples of long prompts, many of each
        _fork("fork_samples", batch=256, parents=32, page_len=64, kv_max=32700, kv_min=5000, n_kv=4, d=64),
        # ragged float32 heads of 64, small pages, a few rows each
        _compact("compact_odd", batch=3, keep=333, page_len=16, kv_max=1999, kv_min=237, dtype="f32", n_kv=3, d=64),
        # a quarter of a batch's long prompts stays cached
        _compact("compact_prompts", batch=4, keep=8192, page_len=64, kv_max=32768, kv_min=20001),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    largest = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("cross", "verify", "resize", "fork", "compact")}
    while True:
        kind = rng.choice(["cross", "cross", "token", "token", "verify", "verify", "resize", "resize", "fork", "fork", "compact", "compact"])
        d = rng.choice([64, 128, 128])
        n_kv, g = rng.choice([(8, 4), (8, 4), (4, 8), (4, 3), (2, 7), (1, 16), (8, 1), (12, 1)])
        page_len = rng.choice([16, 16, 32, 64, 64, 128, 256])
        spread = rng.choice([1, 2, 8])
        if kind in ("cross", "token"):
            kv = _log_int(rng, 1, 65536)
            dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
            chunk = rng.choice([1, 1, 1, 2, 5]) if kind == "token" else _log_int(rng, 6, 2048)
            c = _cross("", dtype=dtype, pages=rng.choice(["raw", "raw", "fp8"]), batch=rng.choice([1, 1, 2, 3, 8, 13]), n_q=n_kv * g,
                       n_kv=n_kv, d=d, chunk=chunk, chunk_min=-(-chunk // spread), page_len=page_len, kv_max=kv,
                       kv_min=rng.choice([kv, kv // spread, 0]))
            if c["batch"] * c["n_q"] * chunk * kv > 1 << 30:   # (the plain form keeps every score of a call at once)
                continue
        elif kind == "verify":
            drafts = rng.choice([1, 2, 3, 4, 5, 7, 8, 12])
            c = _verify("", batch=_log_int(rng, 1, 64), vocab=_log_int(rng, 1000, 262144), drafts=drafts, drafts_min=rng.choice([drafts, 0]),
                        dtype=rng.choice(["f32", "f32", "bf16"]), lookup=rng.random() < 0.4)
            if c["batch"] * (drafts + 1) * c["vocab"] > 1 << 27:
                continue
        elif kind == "resize":
            batch, kv = _log_int(rng, 1, 256), _log_int(rng, 50, 16384)
            pool = _log_int(rng, 256, 262144)
            c = _resize("", batch=batch, pool=pool, page_len=page_len, kv_max=kv, kv_min=kv // spread, cut=rng.choice([3, 9, 40, 300]),
                        grow=rng.choice([1, 5, 17, 64, 700]), done=rng.choice([0, 0, 4, 8]))
            if 1.2 * _pages_at_most(c) > pool:
                continue
        elif kind == "fork":
            kv = _log_int(rng, 20, 32768)
            batch = _log_int(rng, 1, 256)
            c = _fork("", batch=batch, parents=max(1, batch // rng.choice([1, 2, 4, 9])), page_len=page_len, kv_max=kv, kv_min=kv // spread,
                      dtype=rng.choice(["bf16", "bf16", "f32"]), n_kv=n_kv, d=d)
        else:
            kv = _log_int(rng, 30, 32768)
            c = _compact("", batch=rng.choice([1, 2, 3, 8]), keep=max(1, kv // rng.choice([2, 4, 8, 25])), page_len=page_len, kv_max=kv,
                         kv_min=kv // spread, dtype=rng.choice(["bf16", "bf16", "f32"]), n_kv=n_kv, d=d)
        if "kv_max" in c and c["op"] in ("cross", "fork", "compact"):
            rows = c["batch" if c["op"] != "fork" else "parents"] * (c["kv_max"] + page_len) + c["batch"] * page_len
            if 2 * rows * c["n_kv"] * d > 1 << 30:
                continue
        if _cost(c) <= largest[c["op"]]:
            return c


def _spread(hi, lo, n):
    """`hi` first, `lo` last, the others spread over [lo, hi] without order."""
    got = [hi - int((hi - lo) * ((i * 0.6180339887) % 1.0)) for i in range(n)]
    return got[:-1] + [lo] if n > 1 else got


def _pages_of(tokens, page_len):
    return -(-tokens // page_len)


# ---- inputs -------------------------------------------------------------------------------------------------------------

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _quantised(x):
    """float32 rows [..., d] -> (e4m3 [..., d], biased exponents uint8 [...]): elements times the smallest power of two that brings the
    row's largest magnitude to 448 or less."""
    bits = x.abs().amax(-1).view(torch.int32)
    e = (((bits + 0x1FFFFF) >> 23) - 8).clamp(1, 254)
    return (x * torch.exp2((127 - e).float()).unsqueeze(-1)).to(torch.float8_e4m3fn), e.to(torch.uint8)


def _table(lens, page_len, n_pages, gen, cols):
    """A page table [b, cols]: pages of every sequence in random order, -1 past them; and the pages that are left."""
    dev = torch.device("cuda")
    order = torch.randperm(n_pages, device=dev, generator=gen).to(torch.int32)
    table = torch.full((len(lens), cols), -1, dtype=torch.int32, device=dev)
    at = 0
    for i, t in enumerate(lens):
        n = _pages_of(t, page_len)
        table[i, :n] = order[at:at + n]
        at += n
    return table, order[at:]


def _pool(case, table, lens, n_pages, gen):
    """Keys and values of unit variance in the pages of the table; rows that no token owns are zero."""
    dev = torch.device("cuda")
    n_kv, d, P, dt, fp8 = case["n_kv"], case["d"], case["page_len"], TYPES[case["dtype"]], case["pages"] == "fp8"
    got = {}
    for which in ("k", "v"):
        pages = torch.zeros(n_pages, n_kv, P, d, dtype=torch.float8_e4m3fn if fp8 else dt, device=dev)
        scale = torch.zeros(n_pages, n_kv, P, dtype=torch.uint8, device=dev) if fp8 else None
        for i, n in enumerate(lens):
            used = _pages_of(n, P)
            if used == 0:
                continue
            x = torch.randn(used, n_kv, P, d, device=dev, generator=gen)
            x[-1:, :, n - (used - 1) * P:] = 0.0
            mine = table[i, :used].long()
            if fp8:
                q, e = _quantised(x.to(dt).float())
                pages.view(torch.uint8)[mine] = q.view(torch.uint8)
                scale[mine] = e
            else:
                pages[mine] = x.to(dt)
        got[which + "_pages"], got[which + "_scale"] = pages, scale
    return got


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    return {"cross": _prepare_cross, "verify": _prepare_verify, "resize": _prepare_resize, "fork": _prepare_fork,
            "compact": _prepare_compact}[case["op"]](case, gen)


def _lens(case):
    return _spread(case["kv_max"], case["kv_min"], case["batch"])


def _chunks(case):
    return _spread(case["chunk"], case["chunk_min"], case["batch"])


def _prepare_cross(case, gen):
    lens, chunks, P = _lens(case), _chunks(case), case["page_len"]
    n_pages = sum(_pages_of(t, P) for t in lens) + SPARE_PAGES
    table, _ = _table(lens, P, n_pages, gen, max(_pages_of(case["kv_max"], P), 1))
    s = {"op": "cross", "table": table, "kv_max": case["kv_max"], "lens": _ints(lens),
         "chunk_lens": None if min(chunks) == case["chunk"] else _ints(chunks), **_pool(case, table, lens, n_pages, gen)}
    s["q"] = torch.randn(case["batch"], case["n_q"], case["chunk"], case["d"], device="cuda", generator=gen).to(TYPES[case["dtype"]])
    return s


def _drafts(case):
    return _spread(case["drafts"], case["drafts_min"], case["batch"])


def _prepare_verify(case, gen):
    """Peaked target distributions, drafts from a model that mostly agrees (or, looked up, tokens that are mostly the likeliest)."""
    b, V, n = case["batch"], case["vocab"], case["drafts"]
    dt = TYPES[case["dtype"]]
    target = torch.empty(b, n + 1, V, dtype=dt, device="cuda")
    draft = None if case["lookup"] else torch.empty(b, n, V, dtype=dt, device="cuda")
    tokens = torch.empty(b, n, dtype=torch.int32, device="cuda")
    for i in range(b):
        logits = 2.5 * torch.randn(n + 1, V, device="cuda", generator=gen)
        target[i] = torch.softmax(logits, -1).to(dt)
        if case["lookup"]:
            sharp = logits[:n]
        else:
            sharp = logits[:n] + 0.4 * torch.randn(n, V, device="cuda", generator=gen)
            draft[i] = torch.softmax(sharp, -1).to(dt)
        u = torch.rand(n, V, device="cuda", generator=gen).clamp_(min=1e-9)
        tokens[i] = (sharp - torch.log(-torch.log(u))).argmax(-1).to(torch.int32)
    drafts = _drafts(case)
    return {"op": "verify", "target": target, "draft": draft, "tokens": tokens,
            "uniform": torch.rand(b, n + 1, device="cuda", generator=gen),
            "draft_lens": None if min(drafts) == n else _ints(drafts)}


def _resize_lens(case):
    """Tokens that the sequences have room for before a pass, that stay, and that they get room for."""
    room = _lens(case)
    stay = [max(t - (i * 7919) % (case["cut"] + 1), 0) for i, t in enumerate(room)]
    after = [t + case["grow"] for t in stay]
    if case["done"]:
        for i in range(0, case["batch"], case["done"]):
            stay[i], after[i] = 0, case["kv_max"]
    return room, stay, after


def _pages_at_most(case):
    """Of the table's rows together, at any time of a pass."""
    room, _, after = _resize_lens(case)
    return max(sum(_pages_of(t, case["page_len"]) for t in lens) for lens in (room, after))


def _prepare_resize(case, gen):
    """Every third page of what is left is another batch's, so that free pages lie scattered."""
    room, stay, after = _resize_lens(case)
    P = case["page_len"]
    cols = max(_pages_of(max(max(room), max(after)), P), 1)
    table, left = _table(room, P, case["pool"], gen, cols)
    ref = torch.zeros(case["pool"], dtype=torch.int32, device="cuda")
    ref[table[table >= 0].long()] = 1
    spare = case["pool"] - _pages_at_most(case)
    ref[left[:spare // 3].long()] = 1
    return {"op": "resize", "page_len": P, "ref": ref, "table": table, "held": _ints([_pages_of(t, P) for t in room]),
            "stay": _ints(stay), "after": _ints(after)}


def _fork_parents(case, gen):
    """Parents of the batch: each of them, in order, by turns, and the last quarter without order."""
    b, n = case["batch"], case["parents"]
    parents = torch.arange(b, device="cuda") * n // b
    some = b // 4
    if some:
        parents[b - some:] = torch.randint(0, n, (some,), device="cuda", generator=gen)
    return parents.to(torch.int32)


def _prepare_fork(case, gen):
    P, lens = case["page_len"], _spread(case["kv_max"], case["kv_min"], case["parents"])
    cols = max(_pages_of(case["kv_max"], P), 1)
    n_pages = sum(_pages_of(t, P) for t in lens) + case["batch"] + SPARE_PAGES
    table, _ = _table(lens, P, n_pages, gen, cols)
    ref = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    ref[table[table >= 0].long()] = 1
    b = case["batch"]
    return {"op": "fork", "page_len": P, "ref": ref, "table": table, "held": _ints([_pages_of(t, P) for t in lens]), "lens": _ints(lens),
            "parents": _fork_parents(case, gen), "child_table": torch.full((b, cols), -1, dtype=torch.int32, device="cuda"),
            "child_held": torch.zeros(b, dtype=torch.int32, device="cuda"), **_pool(case, table, lens, n_pages, gen)}


def _prepare_compact(case, gen):
    P, lens, n_kv = case["page_len"], _lens(case), case["n_kv"]
    kept = [min(case["keep"], t) for t in lens]
    n_pages = sum(_pages_of(t, P) + _pages_of(k, P) for t, k in zip(lens, kept)) + SPARE_PAGES
    table, left = _table(lens, P, n_pages, gen, max(_pages_of(case["kv_max"], P), 1))
    to = torch.full((case["batch"], max(_pages_of(max(kept), P), 1)), -1, dtype=torch.int32, device="cuda")
    at = 0
    k_idx = torch.zeros(case["batch"], n_kv, max(kept), dtype=torch.int32, device="cuda")
    for i, (t, k) in enumerate(zip(lens, kept)):
        to[i, :_pages_of(k, P)] = left[at:at + _pages_of(k, P)]
        at += _pages_of(k, P)
        if k:   # ascending positions without order in their gaps, as a selection leaves them
            k_idx[i, :, :k] = torch.rand(n_kv, t, device="cuda", generator=gen).topk(k, dim=-1).indices.sort(-1).values.to(torch.int32)
    return {"op": "compact", "table": table, "to": to, "k_idx": k_idx, "k_cnt": _ints([[k] * n_kv for k in kept]),
            **_pool(case, table, lens, n_pages, gen)}


# ---- the plain forms ----------------------------------------------------------------------------------------------------

def _values(s, which, positions):
    """Rows of the pool at `positions` [b, n_kv or 1, S] as float32 [b, n_kv, S, d]."""
    pages, scale = s[which + "_pages"], s[which + "_scale"]
    n_kv, P = pages.shape[1], pages.shape[2]
    page = torch.gather(s["table"].long().unsqueeze(1).expand(-1, positions.shape[1], -1), 2, positions // P).clamp(min=0)
    head = torch.arange(n_kv, device=pages.device).view(1, n_kv, 1)
    if scale is None:
        return pages[page, head, positions % P].float()
    rows = pages.view(torch.uint8)[page, head, positions % P].view(torch.float8_e4m3fn).float()
    return rows * torch.exp2(scale[page, head, positions % P].float() - 127.0).unsqueeze(-1)


def _plain_cross(s):
    q = s["q"]
    b, n_q, C, d = q.shape
    n_kv = s["k_pages"].shape[1]
    at = torch.arange(s["kv_max"], device=q.device).view(1, 1, -1).expand(b, 1, -1)
    k, v = _values(s, "k", at), _values(s, "v", at)
    seen = (at < s["lens"].view(b, 1, 1)).view(b, 1, 1, 1, -1)
    scores = torch.matmul(q.float().view(b, n_kv, -1, d), k.transpose(-1, -2).contiguous()).view(b, n_kv, n_q // n_kv, C, -1)
    scores = (scores / math.sqrt(d)).masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(top.clamp(min=-3e38)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(b, n_kv, -1, p.shape[-1]), v).view(b, n_kv, -1, C, d) / total.clamp(min=1e-30)
    lse = (top + total.log()).squeeze(-1)
    if s["chunk_lens"] is not None:
        live = torch.arange(C, device=q.device) < s["chunk_lens"].view(b, 1, 1, 1)
        out = out.masked_fill(~live.unsqueeze(-1), 0.0)
        lse = lse.masked_fill(~live, -math.inf)
    return {"out": out.view(b, n_q, C, d).to(q.dtype), "lse": lse.view(b, n_q, C)}


def _plain_verify(s):
    """In 64 bits: a token's part of the line that the random number points into is as narrow as its probability."""
    target, draft, tokens, uniform = s["target"], s["draft"], s["tokens"].long(), s["uniform"].double()
    b, n = tokens.shape
    dev = target.device
    lens = torch.full((b,), n, device=dev) if s["draft_lens"] is None else s["draft_lens"].long()
    p_x = torch.gather(target[:, :n], 2, tokens.unsqueeze(-1)).squeeze(-1).double()
    q_x = torch.ones_like(p_x) if draft is None else torch.gather(draft, 2, tokens.unsqueeze(-1)).squeeze(-1).double()
    good = (uniform[:, :n] * q_x < p_x) & (torch.arange(n, device=dev) < lens.unsqueeze(1))
    a = good.long().cumprod(1).sum(1)
    rows = torch.arange(b, device=dev)
    weight = target[rows, a].double()
    refused, at = a < lens, a.clamp(max=n - 1)
    if draft is None:
        q = torch.zeros_like(weight).scatter_(1, tokens[rows, at].unsqueeze(1), 1.0)
    else:
        q = draft[rows, at].double()
    left = (weight - q).clamp(min=0.0)
    weight = torch.where((refused & (left.sum(1) > 0)).unsqueeze(1), left, weight)
    line = weight.cumsum(1)
    point = uniform[:, n:] * line[:, -1:]
    y = torch.searchsorted(line, point, right=True).clamp(max=target.shape[2] - 1)
    out = torch.full((b, n + 1), -1, dtype=torch.int32, device=dev)
    place = torch.arange(n, device=dev)
    out[:, :n] = torch.where(place < a.unsqueeze(1), s["tokens"], out[:, :n])
    out.scatter_(1, a.unsqueeze(1), y.to(torch.int32))
    return {"n_accepted": a.to(torch.int32), "tokens": out}


def _take(ref, table, held, want):
    """Entries `want` [b, cols], the next ones of their rows, get the lowest free pages, sequence after sequence, as long as there are any.
    -> how many of each row, and how many entries got none."""
    free = (ref <= 0).nonzero().squeeze(1)
    at = want.nonzero()
    n = min(at.shape[0], free.shape[0])
    row, col = at[:n, 0], at[:n, 1]
    table[row, col] = free[:n].to(torch.int32)
    ref[free[:n]] = 1
    got = torch.zeros_like(held).index_add_(0, row, torch.ones_like(row, dtype=held.dtype))
    return got, torch.full((1,), at.shape[0] - n, dtype=torch.int32, device=table.device)


def _give(ref, table, drop):
    pages = table[drop].long()
    ref.index_add_(0, pages, torch.full_like(pages, -1, dtype=ref.dtype))
    table[drop] = -1


def _plain_resize(s, lens):
    ref, table, held, P = s["ref"], s["table"], s["held"], s["page_len"]
    n = ((lens + P - 1) // P).clamp(0, table.shape[1])
    e = torch.arange(table.shape[1], device=table.device)
    had, has = e < held.unsqueeze(1), e < n.unsqueeze(1)
    _give(ref, table, had & ~has)
    got, lacking = _take(ref, table, held, has & ~had)
    held.copy_(torch.minimum(held, n) + got)
    s["lacking"] = lacking


def _plain_fork(s):
    ref, table, held, P = s["ref"], s["child_table"], s["child_held"], s["page_len"]
    e = torch.arange(table.shape[1], device=table.device)
    _give(ref, table, e < held.unsqueeze(1))
    parents = s["parents"].long()
    lens = torch.minimum(s["lens"], s["held"] * P)[parents]
    whole = lens // P
    shared = e < whole.unsqueeze(1)
    table[shared] = s["table"][parents][shared]
    pages = table[shared].long()
    ref.index_add_(0, pages, torch.ones_like(pages, dtype=ref.dtype))
    got, lacking = _take(ref, table, held, (e == whole.unsqueeze(1)) & (lens % P > 0).unsqueeze(1))
    held.copy_(whole + got)
    first = whole * P
    lens = torch.where(got > 0, lens, first)
    # the rows of the last pages
    at = first.long().unsqueeze(1) + torch.arange(P, device=table.device)
    seq, row = (at < lens.unsqueeze(1)).nonzero().unbind(1)
    last = whole.long()[seq]
    src, dst = s["table"].long()[parents[seq], last], table.long()[seq, last]
    for name in ("k_pages", "v_pages", "k_scale", "v_scale"):
        if s[name] is not None:
            s[name][dst, :, row] = s[name][src, :, row]
    return first, lens, lacking


def _plain_compact(s):
    n_kv, P = s["k_pages"].shape[1], s["k_pages"].shape[2]
    seq, head, j = (torch.arange(s["k_idx"].shape[2], device="cuda") < s["k_cnt"].unsqueeze(-1)).nonzero().unbind(1)
    at = s["k_idx"].long()[seq, head, j]
    src, dst = s["table"].long()[seq, at // P], s["to"].long()[seq, j // P]
    for name in ("k_pages", "v_pages", "k_scale", "v_scale"):
        if s[name] is not None:
            s[name][dst, head, j % P] = s[name][src, head, at % P]


# ---- one pass -----------------------------------------------------------------------------------------------------------

def _handles(s):
    """What a program makes once from its tensors and keeps."""
    if "own" not in s:
        import paper_2602_08722_amd as quoka

        pool = (s["k_pages"], s["v_pages"]) if "k_pages" in s else None
        scales = (s["k_scale"], s["v_scale"]) if pool else None
        if s["op"] == "cross":
            cache = quoka.PagedCache(*pool, s["table"], *scales)
            s["own"] = quoka.PagedBuffers(cache, s["lens"], s["kv_max"], q=s["q"], chunk_lens=s["chunk_lens"])
        elif s["op"] == "verify":
            s["own"] = quoka.DraftBuffers(s["target"], s["tokens"], s["uniform"], draft=s["draft"], draft_lens=s["draft_lens"])
        elif s["op"] == "resize":
            s["own"] = quoka.PagedSequences(s["ref"], s["table"], s["held"], s["page_len"])
        elif s["op"] == "fork":
            s["own"] = (quoka.PagedSequences(s["ref"], s["table"], s["held"], s["page_len"]),
                        quoka.PagedSequences(s["ref"], s["child_table"], s["child_held"], s["page_len"]),
                        quoka.PagedCache(*pool, s["table"], *scales), quoka.PagedCache(*pool, s["child_table"], *scales))
        else:
            s["own"] = (quoka.PagedCache(*pool, s["table"], *scales), quoka.PagedCache(*pool, s["to"], *scales))
    return s["own"]


def _pool_of(s):
    return {k: s[k] for k in ("k_pages", "v_pages") if s[k] is not None}


def run(s):
    if s["op"] == "cross":
        if not own:
            return _plain_cross(s)
        buf = _handles(s)
        out = buf.cross_attn()
        return {"out": out, "lse": buf.lse}
    if s["op"] == "verify":
        if not own:
            return _plain_verify(s)
        n_accepted, tokens = _handles(s).verify()
        return {"n_accepted": n_accepted, "tokens": tokens}
    if s["op"] == "resize":
        if own:
            seqs = _handles(s)
            seqs.resize(s["stay"])
            seqs.resize(s["after"])
            lacking = seqs.lacking
        else:
            _plain_resize(s, s["stay"])
            _plain_resize(s, s["after"])
            lacking = s["lacking"]
        return {"table": s["table"], "held": s["held"], "ref": s["ref"], "lacking": lacking}
    if s["op"] == "fork":
        if own:
            parents, children, cache, child_cache = _handles(s)
            children.fork(parents, s["parents"], s["lens"])
            child_cache.copy(cache, s["parents"], children.first, children.lens)
            first, lens, lacking = children.first, children.lens, children.lacking
        else:
            first, lens, lacking = _plain_fork(s)
        return {"table": s["child_table"], "held": s["child_held"], "ref": s["ref"], "first": first, "lens": lens, "lacking": lacking,
                **_pool_of(s)}
    if own:
        cache, to = _handles(s)
        to.compact(cache, s["k_idx"], s["k_cnt"])
    else:
        _plain_compact(s)
    return _pool_of(s)


# ---- the definitions, one sequence at a time ----------------------------------------------------------------------------

def exact(case, seed):
    return {"cross": _exact_cross, "verify": _exact_verify, "resize": _exact_resize, "fork": _exact_fork,
            "compact": _exact_compact}[case["op"]](case, prepare(case, seed))


def _exact_cross(case, s):
    b, n_q, C, d = s["q"].shape
    P, g = case["page_len"], n_q // case["n_kv"]
    out = torch.zeros(b, n_q, C, d, dtype=torch.float64, device="cuda")
    lse = torch.full((b, n_q, C), -math.inf, dtype=torch.float64, device="cuda")
    for i, (T, n) in enumerate(zip(_lens(case), _chunks(case))):
        if T == 0:
            continue
        rows = s["table"].long()[i, :_pages_of(T, P)]
        for kv in range(case["n_kv"]):
            kk, vv = (s[w + "_pages"][rows, kv].to(torch.float64) for w in ("k", "v"))
            if s["k_scale"] is not None:
                kk, vv = (torch.ldexp(x, (s[w + "_scale"][rows, kv].to(torch.int64) - 127).unsqueeze(-1)) for x, w in ((kk, "k"), (vv, "v")))
            kk, vv = kk.reshape(-1, d)[:T], vv.reshape(-1, d)[:T]
            for h in range(kv * g, kv * g + g):
                z = s["q"][i, h, :n].to(torch.float64) @ kk.t() / math.sqrt(d)
                lse[i, h, :n] = torch.logsumexp(z, -1)
                out[i, h, :n] = torch.softmax(z, -1) @ vv
    return {"out": out, "lse": lse}


def _exact_verify(case, s):
    import numpy as np

    n = case["drafts"]
    tokens, uniform = s["tokens"].cpu().numpy(), s["uniform"].cpu().numpy().astype(np.float64)
    n_acc, out = np.zeros(case["batch"], np.int32), np.full((case["batch"], n + 1), -1, np.int32)
    for i, k in enumerate(_drafts(case)):
        p = s["target"][i].double().cpu().numpy()
        q = None if s["draft"] is None else s["draft"][i].double().cpu().numpy()
        a = 0
        while a < k and uniform[i, a] * (1.0 if q is None else q[a, tokens[i, a]]) < p[a, tokens[i, a]]:
            out[i, a] = tokens[i, a]
            a += 1
        w = p[a].copy()
        if a < k:
            if q is None:
                w[tokens[i, a]] = max(w[tokens[i, a]] - 1.0, 0.0)
            else:
                w = np.maximum(w - q[a], 0.0)
            if not w.sum() > 0:
                w = p[a]
        line = np.cumsum(w)
        n_acc[i], out[i, a] = a, np.argmax(line > uniform[i, n] * line[-1])
    return {"n_accepted": torch.from_numpy(n_acc), "tokens": torch.from_numpy(out)}


def _book(s, table, held):
    """Tables as lists of the pages that each sequence holds, and the pages' counts."""
    held = held.tolist()
    return [row[:n] for row, n in zip(table.tolist(), held)], s["ref"].tolist()


def _as_table(rows, cols):
    return torch.tensor([row + [-1] * (cols - len(row)) for row in rows], dtype=torch.int32)


def _exact_resize(case, s):
    rows, ref = _book(s, s["table"], s["held"])
    lacking = 0
    for lens in (s["stay"].tolist(), s["after"].tolist()):
        want = [_pages_of(t, case["page_len"]) for t in lens]
        for row, n in zip(rows, want):
            for page in row[n:]:
                ref[page] -= 1
            del row[n:]
        free, lacking = iter([i for i, r in enumerate(ref) if r <= 0]), 0
        for row, n in zip(rows, want):
            while len(row) < n:
                page = next(free, None)
                if page is None:
                    lacking += n - len(row)
                    break
                ref[page] = 1
                row.append(page)
    return {"table": _as_table(rows, s["table"].shape[1]), "held": torch.tensor([len(r) for r in rows], dtype=torch.int32),
            "ref": torch.tensor(ref, dtype=torch.int32), "lacking": torch.tensor([lacking], dtype=torch.int32)}


def _exact_fork(case, s):
    P = case["page_len"]
    rows, ref = _book(s, s["table"], s["held"])
    lens, children = s["lens"].tolist(), []
    pools = {k: v.double() for k, v in _pool_of(s).items()}
    free = iter([i for i, r in enumerate(ref) if r <= 0])
    for parent in s["parents"].tolist():
        n = lens[parent] // P
        row = rows[parent][:n]
        for page in row:
            ref[page] += 1
        if lens[parent] % P:
            page = next(free)
            ref[page] = 1
            row.append(page)
            for pool in pools.values():
                pool[page, :, :lens[parent] % P] = pool[rows[parent][n], :, :lens[parent] % P]
        children.append(row)
    kids = [lens[p] for p in s["parents"].tolist()]
    return {"table": _as_table(children, s["child_table"].shape[1]), "held": torch.tensor([len(r) for r in children], dtype=torch.int32),
            "ref": torch.tensor(ref, dtype=torch.int32), "first": torch.tensor([t // P * P for t in kids], dtype=torch.int32),
            "lens": torch.tensor(kids, dtype=torch.int32), "lacking": torch.zeros(1, dtype=torch.int32), **pools}


def _exact_compact(case, s):
    P = case["page_len"]
    pools = {k: v.double() for k, v in _pool_of(s).items()}
    for i, t in enumerate(_lens(case)):
        n = min(case["keep"], t)
        old, new = s["table"][i, :_pages_of(t, P)].long(), s["to"][i, :_pages_of(n, P)].long()
        for kv in range(case["n_kv"]):
            at = s["k_idx"][i, kv, :n].long()
            for name, pool in pools.items():
                rows = s[name][old, kv].reshape(-1, case["d"])[at].double()
                for e, page in enumerate(new.tolist()):
                    part = rows[e * P:(e + 1) * P]
                    pool[page, kv, :part.shape[0]] = part
    return pools


def work(case):
    """What one pass cannot do without.  cross: queries, and each state once; the output and the sums' logarithms; two products.  verify:
    the drafted tokens' probabilities, and the two rows (looked up: the one) that the last token comes from.  resize, fork: the entries that
    change, with their pages' counts, and the rows of the last pages, read and written; compact: the rows that stay, likewise."""
    op = case["op"]
    if op == "verify":
        es = 2 if case["dtype"] == "bf16" else 4
        dists = 1 if case["lookup"] else 2
        return {"bytes": float(case["batch"] * (dists * es * (case["vocab"] + case["drafts"]) + 12 * (case["drafts"] + 1))),
                "flops": float(2 * case["batch"] * case["vocab"])}
    P = case["page_len"]
    if op == "resize":
        room, stay, after = _resize_lens(case)
        moves = sum(abs(_pages_of(x, P) - _pages_of(y, P)) for a, b in ((room, stay), (stay, after)) for x, y in zip(a, b))
        return {"bytes": 24.0 * case["batch"] + 12.0 * moves, "flops": 0.0}
    row = case["d"] + 1 if case["pages"] == "fp8" else case["d"] * (2 if case["dtype"] == "bf16" else 4)
    if op == "fork":
        lens = _spread(case["kv_max"], case["kv_min"], case["parents"])
        total = 0.0
        for i in range(case["batch"]):
            t = lens[i * case["parents"] // case["batch"]]
            total += 32.0 + 16.0 * (t // P) + 4.0 * case["n_kv"] * (t % P) * row
        return {"bytes": total, "flops": 0.0}
    total = {"bytes": 0.0, "flops": 0.0}
    if op == "compact":
        for t in _lens(case):
            total["bytes"] += min(case["keep"], t) * case["n_kv"] * (4.0 + 4.0 * row)
        return total
    es = 2 if case["dtype"] == "bf16" else 4
    for T, C in zip(_lens(case), _chunks(case)):
        total["bytes"] += (2.0 * case["d"] * es + 4.0) * case["n_q"] * C + 2.0 * case["n_kv"] * T * row
        total["flops"] += 4.0 * case["n_q"] * case["d"] * C * T
    return total


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 8e12, w["flops"] / (1.5e14 if case.get("dtype") == "f32" and case["op"] == "cross" else 2.5e15))
