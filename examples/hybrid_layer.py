"""A decoder layer around a Test-Time Control block, as it is served: attention over a paged cache in 4 bits, then the block.

    x += W_o attention(positions(W_q LN x), cache(positions(W_k LN x), W_v LN x));   x = ttc_block(x)

With --memory N there is a layer of linear attention between the two, N heads whose states fade by a decay that each token sets:

    h = LN x;   x += W_r (silu(W_g h) * RMS_by_heads(linear_attention(W_q h, W_k h, W_v h, -softplus(W_d h))))

Prompts of several sequences go through the layer at once, then each sequence grows by one token a step; the step's launches are captured
into a HIP graph once and replayed.  Run from the repository root:

    python examples/hybrid_layer.py [--sequences 4] [--prompt 300] [--steps 32] [--memory 4]

It prints what the prompt and a step take, and how far the last step's features are from those of the same tokens given as one prompt (both
read keys and values from a 4-bit cache, so the difference is rounding in bfloat16).
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2603_09221_amd import binding, synth  # noqa: E402


class HybridLayer:
    """Seeded random weights: `features` wide, `heads_q` query heads of `d` over `heads` cache heads, a block of `block_heads` heads of 16;
    between them `memory_heads` heads of linear attention, keys of `d` / 2 and values of `d`, if there are any."""

    def __init__(self, features=1024, heads_q=8, heads=2, d=128, block_heads=4, horizon=8, longest=8192, device="cuda:0", seed=0, memory_heads=0):
        gen = torch.Generator(device=device).manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn((cols, rows), generator=gen, device=device) / cols ** 0.5).bfloat16()

        self.heads_q, self.heads, self.d, self.horizon = heads_q, heads, d, horizon
        self.W_qkv, self.W_o = weight((heads_q + 2 * heads) * d, features), weight(features, heads_q * d)
        self.block = synth.make_block_weights(features, block_heads, 16, 16, seed=seed, device=device)
        self.block["W_in"], self.block["W_out"] = self.block["W_in"].bfloat16(), self.block["W_out"].bfloat16()
        freqs, scale = binding.rope_frequencies(d)
        self.table = binding.ttc_rope_table(longest, freqs, scale=scale, device=device)
        self.memory_heads = memory_heads
        if memory_heads:
            self.W_memory, self.W_r = weight(memory_heads * (3 * d + 1), features), weight(features, memory_heads * d)

    def states(self, count, device="cuda:0"):
        return torch.zeros((count, self.memory_heads, self.d // 2, self.d), device=device)

    def memory(self, y, x, states, kv_len, cu_q, max_q):
        """x + y and what the memory layer adds to it; the sequences' states go on in place."""
        heads, d, tokens = self.memory_heads, self.d, x.shape[0]
        around = binding.ttc_residual_norm(y, residual=x, pre="layer")
        q, k, v, gate, decay = (around["h"] @ self.W_memory).split([heads * d // 2, heads * d // 2, heads * d, heads * d, heads], dim=1)
        k = k.view(tokens, heads, -1) / d ** 0.5
        o = binding.ttc_linear_attention(q.view(tokens, heads, -1), k, v.view(tokens, heads, -1), -torch.nn.functional.softplus(decay.float()),
                                         cu_q=cu_q, max_q=max_q, state=states, kv_len=kv_len, out={"state": states})["out"]
        gated = binding.ttc_residual_norm(o.view(tokens, -1), gate=gate, activation="silu", post="rms", groups=heads)["r"]
        return binding.ttc_residual_norm(gated @ self.W_r, residual=around["r"], out={"r": around["r"]})["r"]

    def forward(self, x, cache, slots, positions, pages, kv_len, cu_q=None, max_q=None, max_kv=None, states=None):
        """x (tokens, features) bfloat16 of new tokens: into the cache at slots, through attention, the memory layer if there is one, and the block."""
        tokens = x.shape[0]
        h = torch.nn.functional.layer_norm(x, x.shape[1:]) @ self.W_qkv
        q, k, v = h.view(tokens, -1, self.d).split([self.heads_q, self.heads, self.heads], dim=1)
        q = binding.ttc_kv_append(cache, k, v, slots, positions, self.table, q=q)
        a = binding.ttc_attention(q, cache, pages, kv_len, cu_q=cu_q, max_q=max_q, max_kv=max_kv, want_lse=False)["out"]
        y = a.reshape(tokens, -1) @ self.W_o
        x = self.memory(y, x, states, kv_len, cu_q, max_q) if self.memory_heads else x + y
        return binding.ttc_block_forward(x, self.block, self.horizon)["x_out"]


class Sequences:
    """Pages of one layer's cache dealt out to sequences in turn, and the device-side numbers of a step."""

    def __init__(self, layer, count, longest, page=64, device="cuda:0"):
        self.page, width = page, -(-longest // page)
        self.cache = binding.make_kv_cache(count * width, layer.heads, layer.d, page, device)
        self.pages = torch.arange(count * width, dtype=torch.int32, device=device).view(width, count).T.contiguous()
        self.length = torch.zeros(count, dtype=torch.int32, device=device)
        self.states = layer.states(count, device) if layer.memory_heads else None

    def grow(self, new, tokens):
        """new[s] tokens more for every sequence, `tokens` of all: what ttc_kv_place says of them; the lengths go on in place."""
        pages = self.cache.shape[0]
        return binding.ttc_kv_place(self.length, new, self.pages, self.page, tokens, pages=pages, out={"kv_len": self.length})

    def place(self, sequence, position):
        """Slots of tokens from their sequences and positions (int64 tensors)."""
        return self.pages[sequence, position // self.page].long() * self.page + position % self.page


def prompt(layer, seqs, x, lengths):
    """The tokens x of all sequences, one behind the other, onto what their caches hold."""
    at = seqs.grow(torch.tensor(lengths, dtype=torch.int32, device=x.device), x.shape[0])
    return layer.forward(x, seqs.cache, at["slots"], at["positions"], seqs.pages, seqs.length, at["cu_q"], max(lengths), states=seqs.states)


class Step:
    """One token a sequence, captured once; replay(x) takes the tokens' features and returns the layer's."""

    def __init__(self, layer, seqs, features, device="cuda:0"):
        count = seqs.length.shape[0]
        # what the captured launches read outside the graph's own memory lives as long as the graph does
        self.layer, self.seqs, self.one = layer, seqs, torch.ones(count, dtype=torch.int32, device=device)
        self.x = torch.zeros((count, features), dtype=torch.bfloat16, device=device)
        kept = [(t, t.clone()) for t in (seqs.length, seqs.cache, seqs.states) if t is not None]

        def run():
            at = seqs.grow(self.one, count)
            return layer.forward(self.x, seqs.cache, at["slots"], at["positions"], seqs.pages, seqs.length, states=seqs.states)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run()
        torch.cuda.current_stream().wait_stream(side)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.y = run()
        for t, before in kept:      # as before the run that went ahead of the capture
            t.copy_(before)

    def replay(self, x):
        self.x.copy_(x)
        self.graph.replay()
        return self.y


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--sequences", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=300, help="tokens of the longest prompt; the others are shorter")
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--features", type=int, default=1024)
    ap.add_argument("--memory", type=int, default=0, help="heads of a memory layer between attention and block")
    a = ap.parse_args(argv)
    lengths = [max(1, a.prompt - 37 * i) for i in range(a.sequences)]
    longest = a.prompt + a.steps
    layer = HybridLayer(a.features, longest=longest, memory_heads=a.memory)
    gen = torch.Generator(device="cuda:0").manual_seed(1)
    tokens = [torch.randn((n + a.steps, a.features), generator=gen, device="cuda:0").bfloat16() for n in lengths]

    seqs = Sequences(layer, a.sequences, longest)
    torch.cuda.synchronize()
    t = time.perf_counter()
    prompt(layer, seqs, torch.cat([x[:n] for x, n in zip(tokens, lengths)]), lengths)
    torch.cuda.synchronize()
    print("prompt of %d tokens: %.3f ms" % (sum(lengths), 1e3 * (time.perf_counter() - t)))
    step = Step(layer, seqs, a.features)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for i in range(a.steps):
        y = step.replay(torch.stack([x[n + i] for x, n in zip(tokens, lengths)]))
    torch.cuda.synchronize()
    print("a step of %d sequences: %.1f us" % (a.sequences, 1e6 * (time.perf_counter() - t) / a.steps))

    again = Sequences(layer, a.sequences, longest)
    whole = prompt(layer, again, torch.cat(tokens), [n + a.steps for n in lengths])
    ends = torch.tensor([n + a.steps for n in lengths], device="cuda:0").cumsum(0) - 1
    off = float((whole[ends].float() - y.float()).norm() / whole[ends].float().norm())
    print("last step against the same tokens as one prompt: relative difference %.2g" % off)
    return off


if __name__ == "__main__":
    sys.exit(0 if main() < 0.02 else 1)
