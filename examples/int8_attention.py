"""The attention half of a decoder block on int8 codes: a prompt, single tokens as a graph, and trees of drafted tokens, over one paged cache.

    python examples/int8_attention.py
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1609_07061_amd as q  # noqa: E402
from examples.int8_feed_forward import EPS, codes_of_rows  # noqa: E402


class Attention:
    """h = x + residual; h + output(attention(norm(h))).  Weights and cache int8, activations bf16.  Sequences own their pages; every buffer is allocated once."""

    def __init__(self, width, heads, kv, size, pages, page, sequences, most_tokens, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        init = lambda n, k: codes_of_rows(torch.randn(n, k, device="cuda", generator=g) / math.sqrt(k))
        self.heads, self.kv, self.size, self.page = heads, kv, size, page
        self.gamma = torch.ones(width, device="cuda").bfloat16()
        self.gamma_q, self.gamma_k = torch.ones(size, device="cuda").bfloat16(), torch.ones(size, device="cuda").bfloat16()
        self.qkv, self.output = init((heads + 2 * kv) * size, width), init(width, heads * size)
        self.freq = 10000.0 ** (-torch.arange(size // 2, device="cuda", dtype=torch.float64) / (size // 2))
        self.cache = q.qnn_new_cache(pages, kv, page, size)
        self.table = torch.arange(pages, device="cuda", dtype=torch.int32).view(sequences, pages // sequences)
        self.lengths = torch.zeros(sequences, device="cuda", dtype=torch.int32)
        new = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device="cuda")
        T, longest = most_tokens, pages // sequences * page
        self.codes, self.scale, self.h = new(T, width, dtype=torch.int8), new(T, dtype=torch.float32), new(T, width)
        self.rows, self.mixed, self.y = new(T, (heads + 2 * kv) * size), new(T, heads, size), new(T, width)
        self.mixed_codes, self.mixed_scale = new(T, heads * size, dtype=torch.int8), new(T, dtype=torch.float32)
        need = q.qnn_cache_attention_workspace_bytes(T, sequences, heads, kv, size, T, longest)  # (enough for fewer tokens, shared among the sequences in any way)
        self.workspace = new(max(need, 1), dtype=torch.uint8)
        self.longest = longest

    def forward(self, x, residual, starts, positions, most_new, tree=None):
        """x, residual: [tokens][width]; starts: where each sequence's tokens begin; positions of the tokens; tree: masks of drafted tokens.  The sequences' lengths have
        the new tokens in already."""
        T, heads, kv, size = x.shape[0], self.heads, self.kv, self.size
        codes, scale, h, rows = self.codes[:T], self.scale[:T], self.h[:T], self.rows[:T]
        q.qnn_rms_norm_quant(x, self.gamma, EPS, residual, codes, scale, h)
        q.qnn_int8_gemm(codes, scale, *self.qkv, out=rows)
        parts = rows.view(T, heads + 2 * kv, size)
        queries, keys, values = parts[:, :heads], parts[:, heads:heads + kv], parts[:, heads + kv:]
        q.qnn_cache_append(self.cache, self.table, starts, self.lengths, keys, values, self.gamma_k, EPS, positions, self.freq, q=queries, gamma_q=self.gamma_q, q_out=queries)
        mixed = q.qnn_cache_attention(queries, self.cache, self.table, starts, self.lengths, 1 / math.sqrt(size), tree=tree, most_new=most_new, longest=self.longest,
                                      out=self.mixed[:T], workspace=self.workspace)
        codes, scale = q.qnn_rows_quant(mixed.view(T, heads * size), self.mixed_codes[:T], self.mixed_scale[:T])
        return q.qnn_int8_gemm(codes, scale, *self.output, out=self.y[:T]), h


def build(sequences=4, most_tokens=96, width=256, heads=8, kv=2, size=64, page=16, pages=64, seed=0):
    return Attention(width, heads, kv, size, pages, page, sequences, most_tokens, seed)


def tokens_of(layer, count, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return tuple(torch.randn(count, layer.h.shape[1], device="cuda", generator=g).bfloat16() for _ in range(2))


def ints(values):
    return torch.tensor(values, device="cuda", dtype=torch.int32)


def serve(steps=5):
    """A prompt for every sequence, then `steps` tokens each as replays of one graph -> (outputs of the steps, what the same calls gave outside the graph)."""
    layer = build()
    prompts = [20, 7, 33, 1]
    starts = [0]
    for n in prompts:
        starts.append(starts[-1] + n)
    x, r = tokens_of(layer, starts[-1], 1)
    layer.lengths.copy_(ints(prompts))
    layer.forward(x, r, ints(starts), torch.cat([torch.arange(n, device="cuda", dtype=torch.int32) for n in prompts])[None], max(prompts))
    one, positions = ints([0, 1, 2, 3, 4]), layer.lengths.clone()[None]
    x, r = (t.clone() for t in tokens_of(layer, 4, 2))

    def step():
        layer.lengths.add_(1)
        torch.sub(layer.lengths, 1, out=positions[0])
        return layer.forward(x, r, one, positions, 1)[0]

    kept = [t.clone() for t in (*layer.cache, layer.lengths)]
    want = []
    for i in range(steps):
        new = tokens_of(layer, 4, 10 + i)
        x.copy_(new[0]), r.copy_(new[1])
        want.append(step().clone())
    for t, k in zip((*layer.cache, layer.lengths), kept):
        t.copy_(k)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    got = []
    for i in range(steps):
        new = tokens_of(layer, 4, 10 + i)
        x.copy_(new[0]), r.copy_(new[1])
        graph.replay()
        got.append(out.clone())
    return torch.stack(got), torch.stack(want)


def check_drafts():
    """A tree of drafted tokens for one sequence -> (outputs along one of its branches, what the branch's tokens gave one after the other)."""
    layer = build(sequences=1, pages=16)
    x, r = tokens_of(layer, 30, 3)
    layer.lengths.fill_(30)
    layer.forward(x, r, ints([0, 30]), torch.arange(30, device="cuda", dtype=torch.int32)[None], 30)
    parents = [-1, 0, 0, 1, 2, 4]  # two branches: 0 1 3 and 0 2 4 5
    masks, depth = [], []
    for i, p in enumerate(parents):
        masks.append((masks[p] if p >= 0 else 0) | 1 << i)
        depth.append(depth[p] + 1 if p >= 0 else 0)
    drafted = tokens_of(layer, len(parents), 4)
    layer.lengths.fill_(30 + len(parents))
    y = layer.forward(*drafted, ints([0, len(parents)]), ints([30 + d for d in depth])[None], len(parents), torch.tensor(masks, device="cuda"))[0].clone()
    branch = [0, 2, 4, 5]
    alone = []
    for i, t in enumerate(branch):
        layer.lengths.fill_(31 + i)
        alone.append(layer.forward(drafted[0][t:t + 1], drafted[1][t:t + 1], ints([0, 1]), ints([[30 + i]]), 1)[0].clone())
    return y[branch], torch.cat(alone)


def main():
    got, want = serve()
    print(f"{len(got)} tokens of 4 sequences as a graph: {'same' if torch.equal(got, want) else 'DIFFERENT'} as outside of it")
    tree, alone = check_drafts()
    print(f"a branch of drafted tokens against its tokens one by one: largest difference {(tree.float() - alone.float()).abs().max():.2e} of {alone.float().abs().max():.2f}")


if __name__ == "__main__":
    main()
