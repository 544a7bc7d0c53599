"""The decoder operators together, as examples/decoder_step.py runs them: prompts, then trees over the cache that the prompts left."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("decoder_step", os.path.join(ROOT, "examples", "decoder_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("hidden,heads,kv_heads,head_dim", [(1024, 16, 4, 64), (512, 4, 1, 128), (640, 8, 8, 80)])
def test_trees_continue_the_prompts(hidden, heads, kv_heads, head_dim):
    """A node's result is that of a prompt which ends in it.  Both round the projections, the attention and its weights to bf16 (2^-8 each) over sums in another order:
    four such roundings, as they add up in the 2-norm, stay below 2 %."""
    argv = ["--hidden", str(hidden), "--heads", str(heads), "--kv-heads", str(kv_heads), "--head-dim", str(head_dim)]
    assert _example().main(argv) <= 0.02


def test_layer_against_64_bits():
    """Prompt and tree pass of a small layer in fp32 against the formulas in 64 bits on the CPU."""
    import torch
    ex = _example()
    layer = ex.DecoderAttention(256, 4, 2, 32, dtype=torch.float32, group=32, seed=3)
    cache = ex.PagedCache(30, 4, 2, 32, torch.float32, layer.device)
    g = torch.Generator().manual_seed(2)
    prompts = [torch.randn((n, 256), generator=g) for n in (11, 1, 30)]
    trees = [[-1, 0, 0], [-1, -1], [-1, 0, 1, 0]]
    drafts = [torch.randn((len(t), 256), generator=g) for t in trees]
    seqs, got_prompts = ex.run_prompts(layer, cache, [p.cuda() for p in prompts])
    got_nodes = layer.step(torch.cat(drafts).cuda(), *ex.tree_arguments(layer, cache, seqs, trees)).cpu().split([len(t) for t in trees])

    def dense(weights):
        w, s, z = (t.cpu() for t in weights)
        q = torch.stack([w & 15, w >> 4], -1).flatten(1).double().view(w.shape[0], -1, 32)
        return ((q - z.double()[..., None]) * s.double()[..., None]).flatten(1)

    w_qkv, w_out = dense(layer.qkv), dense(layer.out)

    def rotated(x, weight, positions):
        x = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * weight.cpu().double()
        angle = (positions[:, None].float() * layer.inv_freq.cpu()).double()[:, None]
        a, b = x[..., :16], x[..., 16:]
        return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)

    for p, t, d, yp, yt in zip(prompts, trees, drafts, got_prompts, got_nodes):
        n, m = len(p), len(t)
        depth = []
        for parent in t:
            depth.append(depth[parent] + 1 if parent >= 0 else 0)
        positions = torch.tensor(list(range(n)) + [n + i for i in depth])
        rows = (torch.cat([p, d]).double() @ w_qkv.t()).view(n + m, 8, 32)
        q, k, v = rotated(rows[:, :4], layer.q_norm, positions), rotated(rows[:, 4:6], layer.k_norm, positions), rows[:, 6:]
        seen = torch.ones((n + m, n + m), dtype=torch.bool).tril()
        for i in range(m):
            seen[n + i, n:] = False
            at = i
            while at >= 0:
                seen[n + i, n + at] = True
                at = t[at]
        out = torch.stack([torch.softmax((q[:, h] @ k[:, h // 2].t() * 32 ** -0.5).masked_fill(~seen, float("-inf")), 1) @ v[:, h // 2] for h in range(4)], 1)
        want = out.flatten(1) @ w_out.t()
        for got, ref in ((yp.cpu(), want[:n]), (yt, want[n:])):
            # fp32 throughout: products of 256 and 128 terms, scores of 32; some hundred units of 2^-24 of the norm at most
            assert float((got.double() - ref).norm() / ref.norm()) <= 256 * 2.0 ** -24
