"""A decoder member's attention layer from the library's operators: prompts, then drafted trees verified over the paged cache.

    python examples/decoder_step.py [--hidden 1024] [--heads 16] [--kv-heads 4] [--head-dim 64]

One layer with random 4-bit weights: the projection to queries, keys and values (q4_matmul), norms, rotation and cache write (qk_norm_rope),
attention over the packed prompts (prompt_attention) or of the nodes over the cache (tree_attention), and the projection back (q4_matmul).
The program runs ragged prompts, drafts a tree behind each of them, and checks that every branch of the trees comes out as if its tokens had
been part of the prompt, then prints how long the two kinds of pass take.
"""
import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2410_21120_amd as fi  # noqa: E402


class PagedCache:
    """Pages of one layer's keys and values, handed out as sequences grow."""

    def __init__(self, pages, page_size, kv_heads, head_dim, dtype, device):
        self.page_size = page_size
        self.k, self.v = (torch.zeros((pages, page_size, kv_heads, head_dim), dtype=dtype, device=device) for _ in range(2))
        self.free, self.owned, self.length = list(range(pages - 1, -1, -1)), [], []

    def add_sequence(self):
        self.owned.append([])
        self.length.append(0)
        return len(self.owned) - 1

    def slots(self, seq, count):
        """Slots of the next `count` places behind the committed tokens (a draft's places are not committed)."""
        last = self.length[seq] + count
        while len(self.owned[seq]) * self.page_size < last:
            self.owned[seq].append(self.free.pop())
        return [self.owned[seq][p // self.page_size] * self.page_size + p % self.page_size for p in range(self.length[seq], last)]

    def table(self, seqs):
        columns = max(1, max(len(self.owned[s]) for s in seqs))
        return torch.tensor([self.owned[s] + [0] * (columns - len(self.owned[s])) for s in seqs], dtype=torch.int32, device=self.k.device)


class DecoderAttention:
    """One layer.  Weights are drawn from the seed; rows are [tokens, hidden] in the layer's type."""

    def __init__(self, hidden, q_heads, kv_heads, head_dim, dtype=torch.bfloat16, group=64, seed=0, device="cuda:0"):
        self.hidden, self.q_heads, self.kv_heads, self.head_dim, self.group = hidden, q_heads, kv_heads, head_dim, group
        g = torch.Generator().manual_seed(seed)

        def weights(outputs, inputs):
            w = torch.randint(0, 256, (outputs, inputs // 2), generator=g, dtype=torch.uint8)
            scales = (0.5 + torch.rand((outputs, inputs // group), generator=g)) / (4.6 * math.sqrt(inputs))
            return w.to(device), scales.to(device), torch.randint(6, 11, scales.shape, generator=g, dtype=torch.uint8).to(device)

        self.qkv, self.out = weights((q_heads + 2 * kv_heads) * head_dim, hidden), weights(hidden, q_heads * head_dim)
        self.q_norm, self.k_norm = ((1 + 0.1 * torch.randn(head_dim, generator=g)).to(device) for _ in range(2))
        self.inv_freq = (10000.0 ** -(torch.arange(head_dim // 2) / (head_dim // 2))).float().to(device)
        self.dtype, self.device = dtype, device

    def project(self, x, positions, slots, cache):
        """Normed and rotated queries, keys and values of the rows; keys and values are in the cache, too, where slots are given."""
        hq, hk = self.q_heads, self.kv_heads
        rows = fi.q4_matmul(x, *self.qkv, group=self.group).view(x.shape[0], hq + 2 * hk, self.head_dim)
        q, k, v = rows[:, :hq], rows[:, hq:hq + hk], rows[:, hq + hk:]
        norms = dict(q_weight=self.q_norm, k_weight=self.k_norm)
        # the prompt's attention reads the rows' own keys and values, in place of the projection's; the cache gets a copy
        fi.qk_norm_rope(q, k, None, positions, self.inv_freq, q_out=q, k_out=k, **norms)
        cache.k.view(-1, hk, self.head_dim)[slots], cache.v.view(-1, hk, self.head_dim)[slots] = k, v
        return q, k, v

    def prompt(self, x, cu, positions, slots, cache):
        """Whole prompts, packed by the offsets cu."""
        q, k, v = self.project(x, positions, slots, cache)
        attended = fi.prompt_attention(q, k, v, cu)
        return fi.q4_matmul(attended.view(x.shape[0], -1), *self.out, group=self.group)

    def step(self, x, cu_nodes, positions, slots, cache, table, cached, mask, max_nodes, max_length):
        """Nodes of drafted trees (or single tokens) behind what the cache holds: four launches and what shares their work out."""
        hq, hk = self.q_heads, self.kv_heads
        rows = fi.q4_matmul(x, *self.qkv, group=self.group).view(x.shape[0], hq + 2 * hk, self.head_dim)
        q, _, _ = fi.qk_norm_rope(rows[:, :hq], rows[:, hq:hq + hk], rows[:, hq + hk:], positions, self.inv_freq, q_weight=self.q_norm, k_weight=self.k_norm, slots=slots,
                                  q_out=rows[:, :hq], k_out=cache.k, v_out=cache.v)
        attended = fi.tree_attention(q, cache.k, cache.v, table, cached, cu_nodes, mask, max_nodes=max_nodes, max_length=max_length)
        return fi.q4_matmul(attended.view(x.shape[0], -1), *self.out, group=self.group)


def offsets(counts, device):
    return torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32, device=device)


def ancestors(parents):
    """Mask words of a tree of at most 64 nodes: a node sees itself and the nodes above it."""
    seen = []
    for i, p in enumerate(parents):
        seen.append((seen[p] if p >= 0 else 0) | 1 << i)
    return [m - (1 << 64) if m >> 63 else m for m in seen]


def run_prompts(layer, cache, xs):
    """Packs the prompts xs (one [tokens, hidden] each), runs them and commits them; returns the rows' results per sequence."""
    device, lengths, seqs = layer.device, [x.shape[0] for x in xs], [cache.add_sequence() for _ in xs]
    slots = torch.tensor([s for seq, n in zip(seqs, lengths) for s in cache.slots(seq, n)], device=device)
    positions = torch.cat([torch.arange(n) for n in lengths]).to(torch.int32).to(device)
    y = layer.prompt(torch.cat(xs), offsets(lengths, device), positions, slots, cache)
    for seq, n in zip(seqs, lengths):
        cache.length[seq] = n
    return seqs, list(y.split(lengths))


def tree_arguments(layer, cache, seqs, trees):
    """What a step over the trees (a list of parents per sequence) needs beside its rows."""
    device, counts = layer.device, [len(t) for t in trees]
    depth = [[0] * len(t) for t in trees]
    for d, t in zip(depth, trees):
        for i, p in enumerate(t):
            d[i] = d[p] + 1 if p >= 0 else 0
    cached = [cache.length[s] for s in seqs]
    slots = torch.tensor([s for seq, n in zip(seqs, counts) for s in cache.slots(seq, n)], device=device)
    positions = torch.tensor([c + i for c, d in zip(cached, depth) for i in d], dtype=torch.int32, device=device)
    mask = torch.tensor([[m] for t in trees for m in ancestors(t)], dtype=torch.int64, device=device)
    return (offsets(counts, device), positions, slots, cache, cache.table(seqs), torch.tensor(cached, dtype=torch.int32, device=device), mask, max(counts),
            max(c + n for c, n in zip(cached, counts)))


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--heads", type=int, default=16)
    ap.add_argument("--kv-heads", type=int, default=4)
    ap.add_argument("--head-dim", type=int, default=64)
    a = ap.parse_args(argv)
    layer = DecoderAttention(a.hidden, a.heads, a.kv_heads, a.head_dim)
    cache = PagedCache(400, 16, a.kv_heads, a.head_dim, layer.dtype, layer.device)
    g = torch.Generator().manual_seed(1)

    def rows(n):
        return torch.randn((n, a.hidden), generator=g).to(layer.dtype).to(layer.device)

    prompts = [rows(n) for n in (300, 17, 1, 150)]
    trees = [[-1, 0, 0, 1, 2, -1, 5], [-1], [-1, 0, 1, 1, 3], [-1, 0, 1]]   # parents; two branches behind the first prompt's last token
    seqs, _ = run_prompts(layer, cache, prompts)
    drafts = [rows(len(t)) for t in trees]
    step = tree_arguments(layer, cache, seqs, trees)
    got = list(layer.step(torch.cat(drafts), *step).split([len(t) for t in trees]))

    worst = 0.0
    for x, t, d, y in zip(prompts, trees, drafts, got):   # every node, as the last token of a prompt of its own
        for node in range(len(t)):
            path, at = [], node
            while at >= 0:
                path.append(at)
                at = t[at]
            alone = PagedCache(40, 16, a.kv_heads, a.head_dim, layer.dtype, layer.device)
            _, whole = run_prompts(layer, alone, [torch.cat([x, d[path[::-1]]])])
            off = float((whole[0][-1].float() - y[node].float()).norm() / whole[0][-1].float().norm())
            worst = max(worst, off) if math.isfinite(off) else math.inf   # (max() drops a NaN)
    print(f"{sum(len(t) for t in trees)} nodes of {len(trees)} trees against prompts that end in them: relative difference {worst:.1e} at most")

    def timed(call, n=50):
        call()
        torch.cuda.synchronize()
        began = time.perf_counter()
        for _ in range(n):
            call()
        torch.cuda.synchronize()
        return (time.perf_counter() - began) / n * 1e6

    x, nodes = torch.cat(prompts), torch.cat(drafts)
    lengths = [p.shape[0] for p in prompts]
    cu, positions = offsets(lengths, layer.device), torch.cat([torch.arange(n) for n in lengths]).to(torch.int32).to(layer.device)
    slots = torch.arange(len(x), device=layer.device)
    scratch = PagedCache(400, 16, a.kv_heads, a.head_dim, layer.dtype, layer.device)
    print(f"prompts of {lengths} tokens: {timed(lambda: layer.prompt(x, cu, positions, slots, scratch)):.0f} us; "
          f"trees of {[len(t) for t in trees]} nodes: {timed(lambda: layer.step(nodes, *step)):.0f} us")
    return worst


if __name__ == "__main__":
    sys.exit(0 if main() <= 0.02 else 1)
