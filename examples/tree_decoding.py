"""Speculative decoding with drafted trees over the quantized cache, several samples of one prompt: how the entry points for prompts,
forks, trees and cuts are used together.

One attention block with random projections stands for the model, and a random tree for the drafting model; which branch is accepted is drawn.
The program checks what speculative decoding promises: the output of an accepted node is that of the decode step that would
have come to the same token.

    python examples/tree_decoding.py [--prompt 1000] [--samples 4] [--nodes 24] [--rounds 8]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2505_18610_amd as kq  # noqa: E402

D, Q_HEADS, KV_HEADS, HIDDEN = 128, 16, 4, 512


def rotated(x, positions):
    """Rotary embedding, pairs (i, i + 64), of fp32 [..., n, 128] at positions [n]."""
    i = torch.arange(D // 2, device=x.device, dtype=torch.float64)
    angle = positions.double()[:, None] * (1.0e6 ** (-2.0 * i / D))
    c, s = angle.cos().float(), angle.sin().float()
    a, b = x[..., :D // 2], x[..., D // 2:]
    return torch.cat([a * c - b * s, a * s + b * c], -1)


class Block:
    """The projections of one attention block."""

    def __init__(self, seed):
        g = torch.Generator("cuda").manual_seed(seed)
        self.w = torch.randn((Q_HEADS + 2 * KV_HEADS) * D, HIDDEN, generator=g, device="cuda") / HIDDEN ** 0.5

    def qkv(self, x, positions):
        """x [n, hidden] -> fp16 queries, keys, values [heads, n, 128], rotated."""
        y = (x @ self.w.t()).view(x.shape[0], -1, D).transpose(0, 1)
        q, k, v = y.split([Q_HEADS, KV_HEADS, KV_HEADS])
        return rotated(q, positions).half(), rotated(k, positions).half(), v.half().contiguous()


def new_cache(batch, tokens, budget):
    cfg = kq.KvqConfig(1, batch, Q_HEADS, KV_HEADS, tokens, page_tokens=64, policy=kq.KVQ_POLICY_PAPER, window=128)
    arena = torch.empty(kq.kvq_arena_bytes(cfg, 2 * budget + (16 << 20)), dtype=torch.uint8, device="cuda")
    return kq.KvqCache(cfg, [budget], [4], arena=arena)


def append(cache, k, v):
    """Appends [batch, heads, n, 128]; a full budget is met by lowering the block's width, as the method asks."""
    while True:
        try:
            return cache.kvq_quantize_append(0, k.contiguous(), v.contiguous())
        except kq.KvqError as e:
            if e.status != kq.KVQ_E_BUDGET:
                raise
            cache.kvq_progressive_requant(0)


def drafted_tree(n, g):
    """Parents of n nodes (-1: the last accepted token), their depths, and the words of who sees whom."""
    draws = torch.rand(n, generator=g).tolist()
    parents = [int(d * (i + 1)) - 1 for i, d in enumerate(draws)]
    depth, sees = [], [0] * n
    for i, p in enumerate(parents):
        depth.append(depth[p] + 1 if p >= 0 else 0)
        sees[i] = (sees[p] if p >= 0 else 0) | 1 << i
    words = [[(s >> 32 * w & 0xffffffff) for w in range((n + 31) // 32)] for s in sees]
    mask = torch.tensor(words, dtype=torch.int64)
    return parents, depth, torch.where(mask >= 1 << 31, mask - (1 << 32), mask).to(torch.int32).cuda()


def main(argv=None):
    p = argparse.ArgumentParser()
    for name, value in (("prompt", 1000), ("samples", 4), ("nodes", 24), ("rounds", 8)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args(argv)
    g, host = torch.Generator("cuda").manual_seed(1), torch.Generator().manual_seed(1)
    block, B, n = Block(0), a.samples, a.nodes
    most = a.prompt + a.rounds * n
    # half of what the longest state would take at 16 bits: the block is lowered on the way
    budget = KV_HEADS * (a.prompt // 2 + 512) * kq.kvq_bytes_per_token_head(16)

    # the prompt: its attention, and its keys and values into a cache of one sequence
    prompt = torch.randn(a.prompt, HIDDEN, generator=g, device="cuda")
    q, k, v = block.qkv(prompt, torch.arange(a.prompt, device="cuda"))
    out = torch.empty_like(q)
    kq.kvq_prompt_attention(q.transpose(0, 1), k.transpose(0, 1), v.transpose(0, 1), out.transpose(0, 1), [0, a.prompt])
    one = new_cache(1, most, budget)
    for t in range(0, a.prompt, 256):
        append(one, k[None, :, t:t + 256], v[None, :, t:t + 256])

    # every sample goes on from it
    cache = new_cache(B, most, B * budget)
    kq.kvq_cache_fork(cache, one, 0)
    workspace = torch.empty(cache.kvq_tree_workspace_bytes(n), dtype=torch.uint8, device="cuda")
    copy = new_cache(B, most, B * budget)

    worst, accepted = 0.0, 0
    for step in range(a.rounds):
        length = cache.kvq_cache_describe(0)[2]
        parents, depth, mask = drafted_tree(n, host)
        positions = length + torch.tensor(depth, device="cuda")
        q, k, v = (torch.stack(x) for x in zip(*(block.qkv(torch.randn(n, HIDDEN, generator=g, device="cuda"), positions) for _ in range(B))))
        out = torch.empty_like(q)
        cache.kvq_tree_attention(0, q, k, v, mask, out, workspace=workspace)

        # the accepted branch: a drawn node and its ancestors, in the order of the sequence
        node, path = int(torch.randint(0, n, (1,), generator=host)), []
        while node >= 0:
            path.insert(0, node)
            node = parents[node]
        # the same by decode steps on a copy of the state, to compare
        kq.kvq_cache_fork(copy, cache, 0)
        for i in path:
            append(copy, k[:, :, i:i + 1], v[:, :, i:i + 1])
            want = torch.empty(B, Q_HEADS, D, dtype=torch.float16, device="cuda")
            copy.kvq_decode_attention(0, q[:, :, i].contiguous(), want)
            if copy.kvq_cache_describe(0)[0][:-1] == cache.kvq_cache_describe(0)[0][:-1]:  # (nothing was lowered meanwhile)
                worst = max(worst, float((out[:, :, i].float() - want.float()).abs().max()))
        # a state that keeps too much is cut back: here the copy, to where it was
        widths = copy.kvq_cache_describe(0)[0]
        copy.kvq_cache_truncate(0, length if widths[-1][2] == 16 and widths[-1][0] <= length else length // 64 * 64)

        append(cache, k[:, :, path], v[:, :, path])
        accepted += len(path)

    length = cache.kvq_cache_describe(0)[2]
    K, V = (torch.empty(B, KV_HEADS, length, D, dtype=torch.float16, device="cuda") for _ in range(2))
    cache.kvq_cache_read(0, 0, K, V)
    torch.cuda.synchronize()
    print("%d samples, %d tokens accepted in %d rounds, widths %s, largest difference to decode steps %.1e"
          % (B, accepted, a.rounds, [s[2] for s in cache.kvq_cache_describe(0)[0]], worst))
    assert length == a.prompt + accepted and torch.isfinite(K).all() and torch.isfinite(V).all()
    assert worst < 4e-3, worst
    return worst


if __name__ == "__main__":
    main()
