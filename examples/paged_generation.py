"""One layer of a serving loop over a cache in pages: two prompts are prefilled chunk by chunk with selected keys, then tokens are
generated with attention over everything that is cached, all from 8-bit pages.

    python examples/paged_generation.py [--prompt 4000] [--tokens 16]

Queries, keys and values are random (there is no model here); the program prints how far the outputs are from attention over the
unquantised rows, and how many bytes the cache takes in either form.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2602_08722_amd as quoka  # noqa: E402


def main(prompt=4000, tokens=16, chunk=512, batch=2, n_q=32, n_kv=8, d=128, page_len=64, budget=0.25):
    quoka.load_library()
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(0)
    total = prompt + tokens

    def rows(heads):
        return torch.randn(batch, heads, total, d, device=dev, generator=gen).bfloat16()

    q, k, v = rows(n_q), rows(n_kv), rows(n_kv)

    # a pool with room for both sequences; a real program hands pages out as sequences grow
    per_sequence = -(-total // page_len)
    table = torch.randperm(batch * per_sequence, device=dev, generator=gen).to(torch.int32).view(batch, per_sequence)
    cache = quoka.PagedCache.allocate(batch * per_sequence, page_len, n_kv, d, table)

    # prefill: write the chunk, select keys among the cached ones, attend over them and the chunk
    for at in range(0, prompt, chunk):
        end = min(at + chunk, prompt)
        buf = quoka.PagedBuffers(cache, [at] * batch, at, q=q[:, :, at:end], k_chunk=k[:, :, at:end], v_chunk=v[:, :, at:end],
                                 budgets=[int(budget * at)] * batch, n_retain=64)
        out = buf.chunk_attn()

    # generation: one token a step; the buffers stay, the lengths move on
    step = quoka.PagedBuffers(cache, [prompt] * batch, total, q=torch.empty_like(q[:, :, :1]).contiguous(),
                              k_chunk=torch.empty_like(k[:, :, :1]).contiguous(), v_chunk=torch.empty_like(v[:, :, :1]).contiguous())
    outs = []
    for t in range(prompt, total):
        step.q.copy_(q[:, :, t:t + 1])
        step.k_chunk.copy_(k[:, :, t:t + 1])
        step.v_chunk.copy_(v[:, :, t:t + 1])
        step.write()
        outs.append(step.attn().clone())
        step.kv_lens += 1
    out = torch.cat(outs, 2)

    # the same tokens over the rows themselves
    n = total - prompt
    scores = q[:, :, prompt:].float().view(batch, n_kv, -1, n, d) @ k.float().transpose(-1, -2).unsqueeze(2) / d ** 0.5
    hidden = torch.arange(total, device=dev) > torch.arange(prompt, total, device=dev)[:, None]
    want = scores.masked_fill(hidden, -torch.inf).softmax(-1) @ v.float().unsqueeze(2)
    want = want.view(batch, n_q, n, d)
    off = ((out.float() - want).norm() / want.norm()).item()
    held = 2 * cache.k_pages.numel() + 2 * cache.k_scale.numel()
    print(f"{batch} x ({prompt} + {tokens}) tokens: relative difference from unquantised attention {off:.3f}; "
          f"cache {held / 2**20:.1f} MiB, in bfloat16 {4 * cache.k_pages.numel() / 2**20:.1f}")
    return off


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--prompt", type=int, default=4000)
    p.add_argument("--tokens", type=int, default=16)
    a = p.parse_args()
    main(a.prompt, a.tokens)
