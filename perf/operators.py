"""Timed cases of the paged KV cache: writing a chunk's keys and values into pages (quantised or as they are), reading
pages back, and attention of a chunk over them.

A case is one call of a public entry point (`PagedBuffers.write`, `.read`, `.attn` or `.sparse_attn`) on the buffers that
a serving or prefill loop keeps.  Sizes are those of this repository's workloads, benchmark and tests, or generic ones of
the same ranges.

Fields of a case
  op         "write": the chunk's keys and values into the pages; "read": the pages as contiguous keys and values;
             "attn": attention over all cached tokens and the chunk; "sparse": over a list of them and the chunk
  dtype      "bf16" or "f32": of queries, new keys and values, and outputs
  pages      "fp8": 8-bit elements and a scale for each row; "raw": rows as they are
  batch, n_q, n_kv, d, chunk      sequences, query heads, KV heads, head size, tokens per chunk
  page_len   tokens per page
  kv_max, kv_min                  cached tokens per sequence: the first one kv_max, the others spread down to kv_min
  chunk_min  new tokens per sequence: the first one has `chunk`, the others spread down to chunk_min
  budget     entries of a key list ("sparse")
  values     "read": whether values are read back too, or keys alone (what a selection of keys needs)
"""
import math

import torch

own = False   # False: the operators in plain torch; True: the framework's entry points

SPARE_PAGES = 5   # pages of the pool that no sequence owns


def _case(name, op, dtype="bf16", pages="fp8", batch=1, n_q=32, n_kv=8, d=128, chunk=1, page_len=64, kv_max=8192,
          kv_min=None, chunk_min=None, budget=0, values=True):
    case = dict(op=op, dtype=dtype, pages=pages, batch=batch, n_q=n_q, n_kv=n_kv, d=d, chunk=chunk, page_len=page_len,
                kv_max=kv_max, kv_min=kv_max if kv_min is None else kv_min,
                chunk_min=chunk if chunk_min is None else chunk_min, budget=budget, values=values)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # the new token of each of sixteen sequences, once a step and layer of generation: a launch and little else
        _case("write_tokens", "write", batch=16, page_len=16, kv_max=4096, kv_min=100),
        # prefill chunks of eight sequences, quantised on their way into the cache
        _case("write_chunks", "write", batch=8, chunk=2048, kv_max=2048, kv_min=300),
        # ragged chunks of small float32 heads, kept as they are
        _case("write_odd", "write", dtype="f32", pages="raw", batch=3, n_q=9, n_kv=3, d=64, chunk=333, chunk_min=57,
              page_len=32, kv_max=1999, kv_min=237),
        # a long context's keys, read back for the selection of keys
        _case("read_keys_128k", "read", kv_max=131072, values=False),
        # keys and values of three ragged sequences, as they are kept: what leaves a pool of small pages
        _case("read_odd", "read", pages="raw", batch=3, n_q=12, n_kv=4, d=64, page_len=16, kv_max=19999, kv_min=1237),
        # one generated token after an 8K prompt: the smallest attention call, latency
        _case("token_8k", "attn", kv_max=8192),
        # one token for eight sequences of mixed length, 16-bit pages
        _case("tokens_batch", "attn", pages="raw", batch=8, page_len=16, kv_max=65536, kv_min=4096),
        # one token for a full serving batch, 8-bit pages: 1 GiB of cache
        _case("tokens_full", "attn", batch=32, kv_max=32768, kv_min=1024),
        # a chunk after a short context
        _case("chunk_8k", "attn", chunk=1024, kv_max=8192),
        # nothing divides anything: three heads a group, ragged chunks, small heads, 16-bit pages
        _case("chunk_odd", "attn", pages="raw", batch=3, n_q=12, n_kv=4, d=64, chunk=333, chunk_min=101, page_len=16,
              kv_max=9999, kv_min=1237),
        # a long-context chunk over the keys that a selection kept: the largest call
        _case("sparse_128k", "sparse", chunk=4096, kv_max=131072, budget=8192),
        # a float32 layer of ordinary size
        _case("f32_4k", "attn", dtype="f32", pages="raw", n_q=8, n_kv=2, chunk=512, kv_max=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    largest = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("write", "read", "attn", "sparse")}
    while True:
        kind = rng.choice(["write", "write", "read", "read", "token", "token", "token", "chunk", "chunk", "sparse", "f32"])
        d = rng.choice([64, 128, 128])
        n_kv, g = rng.choice([(8, 4), (8, 4), (4, 8), (4, 3), (2, 7), (1, 16), (8, 1)])
        batch = rng.choice([1, 1, 2, 3, 8, 13])
        how = dict(pages=rng.choice(["fp8", "fp8", "raw"]), batch=batch, n_q=n_kv * g, n_kv=n_kv, d=d,
                   page_len=rng.choice([16, 32, 64, 64, 128, 256]))
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        spread = rng.choice([1, 2, 8])
        if kind == "write":
            kv, chunk = rng.randint(0, 4096), _log_int(rng, 1, 4096)
            c = _case("", "write", dtype=dtype, chunk=chunk, chunk_min=-(-chunk // spread), kv_max=kv, kv_min=kv // spread, **how)
        elif kind == "read":
            kv = _log_int(rng, 300, 131072)
            c = _case("", "read", dtype=dtype, kv_max=kv, kv_min=kv // spread, values=rng.random() < 0.6, **how)
        elif kind == "token":
            kv = _log_int(rng, 512, 131072)
            c = _case("", rng.choice(["attn", "attn", "sparse"]), chunk=rng.choice([1, 1, 1, 2, 5, 8]), kv_max=kv,
                      kv_min=kv // spread, budget=max(1, kv // rng.choice([4, 8, 25])), **how)
        elif kind == "chunk":
            kv, chunk = _log_int(rng, 256, 16384), _log_int(rng, 33, 1500)
            c = _case("", "attn", chunk=chunk, chunk_min=-(-chunk // spread), kv_max=kv, kv_min=kv // spread, **how)
        elif kind == "sparse":
            kv, chunk = _log_int(rng, 1024, 131072), _log_int(rng, 64, 4096)
            c = _case("", "sparse", chunk=chunk, chunk_min=-(-chunk // spread), kv_max=kv, kv_min=kv // spread,
                      budget=max(1, kv // rng.choice([4, 8, 25])), **how)
        else:
            kv, chunk = _log_int(rng, 256, 8192), _log_int(rng, 1, 600)
            how.update(batch=rng.choice([1, 1, 2]), n_q=2 * g, n_kv=2)
            c = _case("", rng.choice(["attn", "sparse"]), dtype="f32", chunk=chunk, kv_max=kv, kv_min=kv // spread,
                      budget=max(1, kv // 8), **how)
        # (the plain form keeps every score of a call at once)
        scores = c["batch"] * c["n_q"] * c["chunk"] * (c["chunk"] + (c["budget"] if c["op"] == "sparse" else c["kv_max"]))
        if c["op"] in ("attn", "sparse") and scores > 1 << 31:
            continue
        if 2 * c["batch"] * c["n_kv"] * (c["kv_max"] + c["chunk"]) * d <= 1 << 29 and _cost(c) <= largest[c["op"]]:
            return c


def _spread(hi, lo, n):
    """`hi` first, the others spread over [lo, hi] without order."""
    return [hi - int((hi - lo) * ((i * 0.6180339887) % 1.0)) for i in range(n)]


def _lens(case):
    return _spread(case["kv_max"], case["kv_min"], case["batch"])


def _chunks(case):
    return _spread(case["chunk"], case["chunk_min"], case["batch"])


def _keys_per_list(case, kv_len):
    return min(case["budget"], kv_len)


# ---- the 8-bit format: a row is e4m3 elements times a power of two, the smallest one that brings the row's largest magnitude
# to 448 or less; the power is kept as its biased exponent, 1 .. 254

def _quantised(x):
    """float32 rows [..., d] -> (e4m3 [..., d], biased exponents uint8 [...])."""
    bits = x.abs().amax(-1).view(torch.int32)
    # the largest magnitude's exponent, one more where its significand exceeds that of 448 = 1.75 * 2^8
    e = (((bits + 0x1FFFFF) >> 23) - 8).clamp(1, 254)
    return (x * torch.exp2((127 - e).float()).unsqueeze(-1)).to(torch.float8_e4m3fn), e.to(torch.uint8)


def _values(pages, scale):
    """Rows of a pool as float32, or what they stand for."""
    if scale is None:
        return pages.float()
    return pages.float() * torch.exp2(scale.float() - 127.0).unsqueeze(-1)


def prepare(case, seed):
    """The pool and its page table, with every sequence's cached tokens in pages in random order, and a chunk's queries,
    keys and values of unit variance.  Rows of the pool that no token owns are zero."""
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    b, n_q, n_kv, d, C, P = (case[k] for k in ("batch", "n_q", "n_kv", "d", "chunk", "page_len"))
    lens, chunks = _lens(case), _chunks(case)
    fp8 = case["pages"] == "fp8"
    needs_new = case["op"] != "read"
    counts = [-(-(t + (c if needs_new else 0)) // P) for t, c in zip(lens, chunks)]
    n_pages = sum(counts) + SPARE_PAGES
    order = torch.randperm(n_pages, device=dev, generator=gen).to(torch.int32)
    max_pages = -(-(case["kv_max"] + (C if needs_new else 0)) // P)
    table = torch.full((b, max_pages), -1, dtype=torch.int32, device=dev)
    at = 0
    for i, n in enumerate(counts):
        table[i, :n] = order[at:at + n]
        at += n

    # a write starts from the tokens before the chunk; attention finds the chunk's own rows in the pages
    held = [t + (c if case["op"] in ("attn", "sparse") else 0) for t, c in zip(lens, chunks)]

    def pool():
        pages = torch.zeros(n_pages, n_kv, P, d, dtype=torch.float8_e4m3fn if fp8 else dt, device=dev)
        scale = torch.zeros(n_pages, n_kv, P, dtype=torch.uint8, device=dev) if fp8 else None
        for i, n in enumerate(held):
            used = -(-n // P)
            x = torch.randn(used, n_kv, P, d, device=dev, generator=gen)
            x[-1:, :, n - (used - 1) * P:] = 0.0
            own_pages = table[i, :used].long()
            if fp8:
                q, e = _quantised(x.to(dt).float())
                pages.view(torch.uint8)[own_pages] = q.view(torch.uint8)
                scale[own_pages] = e
            else:
                pages[own_pages] = x.to(dt)
        return pages, scale

    k_pages, k_scale = pool()
    v_pages, v_scale = pool()
    state = {"op": case["op"], "k_pages": k_pages, "v_pages": v_pages, "k_scale": k_scale, "v_scale": v_scale, "table": table,
             "kv_max": case["kv_max"], "lens": torch.tensor(lens, dtype=torch.int32, device=dev),
             "chunk_lens": None if min(chunks) == C else torch.tensor(chunks, dtype=torch.int32, device=dev)}
    if case["op"] == "write":
        state["k_new"] = torch.randn(b, n_kv, C, d, device=dev, generator=gen).to(dt)
        state["v_new"] = torch.randn(b, n_kv, C, d, device=dev, generator=gen).to(dt)
        # sequence and position in its chunk of every new token
        pairs = [(i, c) for i, n in enumerate(chunks) for c in range(n)]
        state["new"] = tuple(torch.tensor(x, device=dev) for x in zip(*pairs))
    elif case["op"] == "read":
        state["k_out"] = torch.zeros(b, n_kv, case["kv_max"], d, dtype=dt, device=dev)
        state["v_out"] = torch.zeros_like(state["k_out"]) if case["values"] else None
        state["live"] = (torch.arange(case["kv_max"], device=dev) < state["lens"][:, None])[:, None, :, None]
    else:
        state["q"] = torch.randn(b, n_q, C, d, device=dev, generator=gen).to(dt)
        state["k_idx"] = None
        if case["op"] == "sparse":   # ascending positions without order in their gaps, as a selection leaves them
            state["k_idx"] = torch.zeros(b, n_kv, case["budget"], dtype=torch.int32, device=dev)
            cnt = []
            for i, t in enumerate(lens):
                n = _keys_per_list(case, t)
                picked = torch.rand(n_kv, t, device=dev, generator=gen).topk(n, dim=-1).indices if n else None
                if n:
                    state["k_idx"][i, :, :n] = picked.sort(-1).values.to(torch.int32)
                cnt.append([n] * n_kv)
            state["k_cnt"] = torch.tensor(cnt, dtype=torch.int32, device=dev)
    return state


def _buffers(s):
    """The framework's handle on the state's tensors, made once per state as a program makes it."""
    if "buf" not in s:
        import paper_2602_08722_amd as quoka

        cache = quoka.PagedCache(s["k_pages"], s["v_pages"], s["table"], s["k_scale"], s["v_scale"])
        s["buf"] = quoka.PagedBuffers(cache, s["lens"], s["kv_max"], q=s.get("q"), k_chunk=s.get("k_new"),
                                      v_chunk=s.get("v_new"), chunk_lens=s["chunk_lens"], k_idx=s.get("k_idx"),
                                      k_cnt=s.get("k_cnt"))
    return s["buf"]


def _rows(s, which, positions):
    """Rows of the pool at `positions` [b, n_kv or 1, S] as float32 [b, n_kv, S, d]."""
    pages, scale = s[which + "_pages"], s[which + "_scale"]
    n_kv, P = pages.shape[1], pages.shape[2]
    page_of = torch.minimum(positions // P, torch.tensor(s["table"].shape[1] - 1, device=positions.device))
    page = torch.gather(s["table"].long().unsqueeze(1).expand(-1, positions.shape[1], -1), 2, page_of).clamp(min=0)
    head = torch.arange(n_kv, device=pages.device).view(1, n_kv, 1)
    raw = pages.view(torch.uint8) if scale is not None else pages
    rows = raw[page, head, positions % P]
    if scale is None:
        return rows.float()
    return _values(rows.view(torch.float8_e4m3fn), scale[page, head, positions % P])


def _plain_write(s):
    seq, tok = s["new"]
    P = s["k_pages"].shape[2]
    at = s["lens"].long()[seq] + tok
    page, slot = s["table"].long()[seq, at // P], at % P

    def put(pages, scale, new):
        rows = new[seq, :, tok]
        if scale is None:
            pages[page, :, slot] = rows
            return
        q, e = _quantised(rows.float())
        pages.view(torch.uint8)[page, :, slot] = q.view(torch.uint8)
        scale[page, :, slot] = e

    put(s["k_pages"], s["k_scale"], s["k_new"])
    put(s["v_pages"], s["v_scale"], s["v_new"])


def _plain_read(s):
    at = torch.arange(s["kv_max"], device=s["lens"].device).view(1, 1, -1).expand(s["lens"].shape[0], -1, -1)

    def get(which, out):
        out.copy_(torch.where(s["live"], _rows(s, which, at).to(out.dtype), out))

    get("k", s["k_out"])
    if s["v_out"] is not None:
        get("v", s["v_out"])


def _plain_attn(s):
    q = s["q"]
    b, n_q, C, d = q.shape
    n_kv = s["k_pages"].shape[1]
    dev = q.device
    lens = s["lens"].long().view(b, 1, 1)
    mine = torch.arange(C, device=dev).view(1, 1, C)
    if s["k_idx"] is None:
        before = torch.arange(s["kv_max"], device=dev).view(1, 1, -1).expand(b, 1, -1)
        seen = before < lens
    else:
        before = s["k_idx"].long()
        seen = torch.arange(before.shape[2], device=dev) < s["k_cnt"].long().unsqueeze(-1)
    heads = before.shape[1]
    at = torch.cat([before, (lens + mine).expand(b, heads, C)], -1)
    k, v = _rows(s, "k", at), _rows(s, "v", at)
    # [b, heads, C, S]: every row sees the cached keys, and the chunk's up to itself
    causal = (mine <= mine.view(1, C, 1)).expand(b, heads, C, C)
    seen = torch.cat([seen.unsqueeze(2).expand(-1, -1, C, -1), causal], -1)
    scores = torch.matmul(q.float().view(b, n_kv, -1, d), k.transpose(-1, -2)).view(b, n_kv, n_q // n_kv, C, -1) / math.sqrt(d)
    scores = scores.masked_fill_(~seen.unsqueeze(2), -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(b, n_kv, -1, p.shape[-1]), v).view(b, n_kv, -1, C, d) / total
    lse = (top + total.log()).squeeze(-1)
    if s["chunk_lens"] is not None:   # rows past a sequence's chunk have no key
        live = torch.arange(C, device=dev) < s["chunk_lens"].view(b, 1, 1, 1)
        out = out.masked_fill(~live.unsqueeze(-1), 0.0)
        lse = lse.masked_fill(~live, -math.inf)
    return out.view(b, n_q, C, d).to(q.dtype), lse.view(b, n_q, C)


def _pool_of(s):
    return {k: s[k] for k in ("k_pages", "v_pages", "k_scale", "v_scale") if s[k] is not None}


def run(s):
    if s["op"] == "write":
        if own:
            _buffers(s).write()
        else:
            _plain_write(s)
        return _pool_of(s)
    if s["op"] == "read":
        if own:
            _buffers(s).read(s["k_out"], s["v_out"])
        else:
            _plain_read(s)
        return {"k": s["k_out"]} if s["v_out"] is None else {"k": s["k_out"], "v": s["v_out"]}
    if own:
        buf = _buffers(s)
        out = buf.attn() if s["op"] == "attn" else buf.sparse_attn()
        return {"out": out, "lse": buf.lse}
    out, lse = _plain_attn(s)
    return {"out": out, "lse": lse}


def exact(case, seed):
    """From the definitions, in float64: row by row of the pool for what is written and read, sequence by sequence and head
    by head for attention."""
    s = prepare(case, seed)
    lens, chunks, P = _lens(case), _chunks(case), case["page_len"]
    table = s["table"].long()

    def held(which):
        """What a pool's rows stand for."""
        x = s[which + "_pages"].to(torch.float64)
        e = s[which + "_scale"]
        return x if e is None else torch.ldexp(x, (e.to(torch.int64) - 127).unsqueeze(-1))

    if case["op"] == "write":
        got = {}
        for which in ("k", "v"):
            pages, scale = s[which + "_pages"].to(torch.float64), s[which + "_scale"]
            new = s[which + "_new"].to(torch.float64)
            for i, n in enumerate(chunks):
                at = torch.arange(lens[i], lens[i] + n, device=table.device)
                rows = new[i, :, :n].transpose(0, 1)
                if scale is not None:
                    top = rows.abs().amax(-1, keepdim=True)
                    e = torch.ceil(torch.log2(torch.clamp(top, min=1e-300) / 448.0))
                    e = torch.where(torch.ldexp(torch.full_like(e, 448.0), e) < top, e + 1, e)
                    e = torch.where(torch.ldexp(torch.full_like(e, 448.0), e - 1) >= top, e - 1, e).clamp(-126, 127)
                    y = torch.ldexp(rows, -e)
                    # steps of 2^-3 of the element's own power of two, and of 2^-9 below 2^-6
                    step = torch.exp2((torch.floor(torch.log2(torch.clamp(y.abs(), min=2.0 ** -6))) - 3.0))
                    rows = torch.round(y / step) * step
                pages[table[i, at // P], :, at % P] = rows
            got[which + "_pages"] = pages
        return {k: got.get(k) for k in ("k_pages", "v_pages", "k_scale", "v_scale") if s[k] is not None}
    if case["op"] == "read":
        got = {}
        for which in ("k", "v") if case["values"] else ("k",):
            pool, out = held(which), s[which + "_out"].to(torch.float64)
            for i, n in enumerate(lens):
                rows = pool[table[i, :-(-n // P)]].transpose(0, 1).reshape(case["n_kv"], -1, case["d"])
                out[i, :, :n] = rows[:, :n]
            got[which] = out
        return got
    b, n_q, C, d = s["q"].shape
    g = n_q // case["n_kv"]
    out = torch.zeros(b, n_q, C, d, dtype=torch.float64, device="cuda")
    lse = torch.full((b, n_q, C), -math.inf, dtype=torch.float64, device="cuda")
    for i in range(b):
        T, n = lens[i], chunks[i]
        rows = table[i, :-(-(T + n) // P)]
        hidden = torch.ones(n, n, device="cuda", dtype=torch.bool).triu(1)
        for kv in range(case["n_kv"]):
            def of(which):
                x = s[which + "_pages"][rows, kv].to(torch.float64)
                e = s[which + "_scale"]
                x = x if e is None else torch.ldexp(x, (e[rows, kv].to(torch.int64) - 127).unsqueeze(-1))
                x = x.reshape(-1, d)
                cached = x[:T] if s["k_idx"] is None else x[s["k_idx"][i, kv, :_keys_per_list(case, T)].long()]
                return torch.cat([cached, x[T:T + n]])

            k, v = of("k"), of("v")
            for h in range(kv * g, kv * g + g):
                z = s["q"][i, h, :n].to(torch.float64) @ k.t() / math.sqrt(d)
                z[:, -n:].masked_fill_(hidden, -math.inf)
                lse[i, h, :n] = torch.logsumexp(z, -1)
                out[i, h, :n] = torch.softmax(z, -1) @ v
    return {"out": out, "lse": lse}


def work(case):
    """What one pass cannot do without.  write: the new rows read, and written as they are kept.  read: the other way.
    Attention: queries, and each attended row of the pool once; the output and the row sums' logarithms; two products."""
    es = 2 if case["dtype"] == "bf16" else 4
    n_q, n_kv, d = case["n_q"], case["n_kv"], case["d"]
    row = d + 1 if case["pages"] == "fp8" else d * es
    total = {"bytes": 0.0, "flops": 0.0}
    for T, C in zip(_lens(case), _chunks(case)):
        if case["op"] == "write":
            total["bytes"] += 2.0 * n_kv * C * (d * es + row)
        elif case["op"] == "read":
            total["bytes"] += (2.0 if case["values"] else 1.0) * n_kv * T * (d * es + row)
        else:
            keys = T if case["op"] == "attn" else _keys_per_list(case, T)
            total["bytes"] += 2.0 * n_q * C * d * es + 4.0 * n_q * C + 2.0 * n_kv * (keys + C) * row
            total["flops"] += 4.0 * n_q * d * (C * keys + C * (C + 1) / 2.0)
            if case["op"] == "sparse":
                total["bytes"] += 4.0 * n_kv * keys
    return total


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 8e12, w["flops"] / (2.5e15 if case["dtype"] == "bf16" else 1.5e14))
