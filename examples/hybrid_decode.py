"""Speculative decoding of a small gated-delta hybrid, every step of a round on the library's calls.

A random-weight model alternates gated-delta layers (state per head) and softmax layers (paged cache).  A round drafts a tree
for every sequence, runs the model over all nodes at once, draws the target's token at every node, keeps the longest matching
path and commits it: the states by treewy_commit, the caches by treewy_cache_append.  Drawing the target's own token at each
node and keeping the child that equals it leaves the target's distribution as it is; with one random number for each position the
tokens are those of plain decoding, which is the same loop with a tree of one node:

    python examples/hybrid_decode.py [--sequences 4] [--tokens 48] [--dtype f32|bf16]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_20961_amd import hybrid, treewy  # noqa: E402


class Model:
    """`blocks` pairs of a gated-delta layer (heads of 128) and a softmax layer (grouped heads, half of each rotating)."""

    def __init__(self, blocks=2, width=128, vocab=512, gdn_heads=2, q_heads=4, kv_heads=2, d=64, positions=4096,
                 dtype=torch.float32, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda *s: torch.randn(*s, generator=g, device="cuda") / math.sqrt(s[0])
        self.width, self.vocab, self.d, self.dtype = width, vocab, d, dtype
        self.gdn_heads, self.q_heads, self.kv_heads = gdn_heads, q_heads, kv_heads
        self.embed = torch.randn(vocab, width, generator=g, device="cuda")
        self.gdn = [dict(qkv=w(width, 3 * gdn_heads * 128), gates=w(width, 2 * gdn_heads), out=0.4 * w(gdn_heads * 128, width))
                    for _ in range(blocks)]
        self.att = [dict(qkv=w(width, (q_heads + 2 * kv_heads) * d), out=0.4 * w(q_heads * d, width)) for _ in range(blocks)]
        a = torch.arange(positions, device="cuda")[:, None] * 1e4 ** (-torch.arange(0, d // 2, 2, device="cuda") / (d // 2))
        self.cos, self.sin = a.cos().contiguous(), a.sin().contiguous()


class Sequences:
    """What a batch keeps between rounds: states, caches, lengths, and each sequence's next token, drawn but not run yet."""

    def __init__(self, m, first, most, page=16):
        B = len(first)
        pages = -(-most // page)
        dev = dict(device="cuda")
        self.S = [torch.zeros(B, m.gdn_heads, 128, 128, **dev) for _ in m.gdn]
        self.pages = [[torch.zeros(B * pages, m.kv_heads, page, m.d, dtype=m.dtype, **dev) for _ in "kv"] for _ in m.att]
        self.table = torch.randperm(B * pages, **dev).reshape(B, pages).int()
        self.len = torch.zeros(B, dtype=torch.int32, **dev)
        self.next = first.int().cuda()


def norm(x):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)


def forward(m, s, tokens, parent):
    """Logits [B, N, vocab] of every node, and what a commit needs of each layer."""
    B, N = tokens.shape
    heads = lambda x, n, d: x.to(m.dtype).reshape(B, N, n, d).transpose(1, 2)
    x, kept = m.embed[tokens.long()], []
    for i, (g, a) in enumerate(zip(m.gdn, m.att)):
        h = norm(x)
        q, k, v = (heads(t, m.gdn_heads, 128).float() for t in (h @ g["qkv"]).split(m.gdn_heads * 128, -1))
        q, k = (t / (t.norm(dim=-1, keepdim=True) + 1e-6) for t in (q, k))
        q, k, v = (t.to(m.dtype).contiguous() for t in (q, k, v))
        gates = torch.sigmoid(h @ g["gates"] + 2.0).transpose(1, 2).contiguous()
        alpha, beta = (0.9 + 0.0999 * gates[:, :m.gdn_heads]).contiguous(), gates[:, m.gdn_heads:].contiguous()
        o, U = treewy.treewy_verify(s.S[i], q, k, v, alpha, beta, parent)
        x = x + o.transpose(1, 2).reshape(B, N, -1).float() @ g["out"]
        kept.append((U, k, alpha))
        qkv = (norm(x) @ a["qkv"]).to(m.dtype).reshape(B, N, -1, m.d)
        q, k, v = (t.transpose(1, 2) for t in qkv.split((m.q_heads, m.kv_heads, m.kv_heads), 2))
        o = torch.empty(B, N, m.q_heads, m.d, dtype=m.dtype, device="cuda").transpose(1, 2)
        hybrid.treewy_tree_attention(q, k, v, parent, *s.pages[i], s.table, s.len, cos=m.cos, sin=m.sin, o=o)
        x = x + o.transpose(1, 2).reshape(B, N, -1).float() @ a["out"]
        kept.append((k, v))
    return norm(x) @ m.embed.T / math.sqrt(m.width), kept


def draft(m, s, widths):
    """A tree of each sequence's next token and, level by level, the embedding's likeliest followers (no layer is run)."""
    tokens, parent, level = [s.next], [-1], [0]
    for w in widths:
        new = []
        for n in level:
            best = (norm(m.embed[tokens[n].long()]) @ m.embed.T).topk(w, -1).indices.int()
            for j in range(w):
                new.append(len(tokens))
                tokens.append(best[:, j])
                parent.append(n)
        level = new
    B = len(s.next)
    return torch.stack(tokens, 1).contiguous(), torch.tensor(parent, dtype=torch.int32, device="cuda").expand(B, -1).contiguous()


def round_(m, s, widths, numbers, sampling):
    """One round: the accepted tokens [B, L] (-1 past a path) and how many, with the state, caches and next tokens moved on."""
    tokens, parent = draft(m, s, widths)
    B, N = tokens.shape
    depth = [0] * N
    for t, p in enumerate(parent[0].tolist()):
        depth[t] = depth[p] + 1 if p >= 0 else 0
    logits, kept = forward(m, s, tokens, parent)
    at = s.len.long()[:, None] + torch.tensor(depth, device="cuda")
    u = numbers.gather(1, at)                            # one number per position, whichever node stands there
    rows = {n: v.repeat_interleave(N) for n, v in sampling.items()}
    drawn, _ = hybrid.treewy_sample(logits.reshape(B * N, -1), u.reshape(-1), **rows)
    L = len(widths) + 1
    path, plen, bonus = treewy.treewy_accept_greedy(parent, tokens, drawn.reshape(B, N), s.next, L)
    new_len = torch.empty_like(s.len)
    for i in range(len(m.gdn)):
        U, k, alpha = kept[2 * i]
        s.S[i] = treewy.treewy_commit(s.S[i], U, k, alpha, path, plen, parent=parent)
        hybrid.treewy_cache_append(*kept[2 * i + 1], *s.pages[i], s.table, s.len, cos=m.cos, sin=m.sin, path=path, count=plen,
                                   new_len=new_len)
    s.len, s.next = new_len, bonus
    return torch.where(path >= 0, tokens.gather(1, path.long().clamp(min=0)), -1), plen


def decode(m, first, numbers, sampling, count, widths=()):
    """At least `count` tokens of every sequence, and the number of rounds (widths (): plain decoding)."""
    s = Sequences(m, first, numbers.shape[1] + 8)
    out, rounds = [[] for _ in first], 0
    while min(map(len, out)) < count:
        got, n = round_(m, s, widths, numbers, sampling)
        for o, row, k in zip(out, got.tolist(), n.tolist()):
            o.extend(row[:k])
        rounds += 1
    return [o[:count] for o in out], rounds


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--sequences", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=48)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    a = ap.parse_args(argv)
    m = Model(dtype=torch.float32 if a.dtype == "f32" else torch.bfloat16)
    g = torch.Generator(device="cuda").manual_seed(1)
    B = a.sequences
    first = torch.randint(0, m.vocab, (B,), generator=g, device="cuda")
    numbers = torch.rand(B, 8 * a.tokens + 64, generator=g, device="cuda")
    full = lambda x, t=torch.float32: torch.full((B,), x, dtype=t, device="cuda")
    sampling = dict(temperature=full(0.7), top_k=full(40, torch.int32), top_p=full(0.95), min_p=full(0.01))
    plain, steps = decode(m, first, numbers, sampling, a.tokens)
    tree, rounds = decode(m, first, numbers, sampling, a.tokens, widths=(3, 2, 2))
    same = sum(x == y for p, t in zip(plain, tree) for x, y in zip(p, t))
    print("%d tokens of %d sequences: %d steps one by one, %d rounds of 22-node trees; %d of %d tokens agree"
          % (a.tokens, B, steps, rounds, same, a.tokens * B))
    return plain, tree, steps, rounds


if __name__ == "__main__":
    main()
