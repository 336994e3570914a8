"""Speculative decoding with a drafted tree: the draft's layer, the choice of candidates and their verification through the library.

    python examples/decode_step.py [--rounds 4]

A draft layer (queries, keys and values from the features, rotary positions, attention over a paged cache, the gated block, the
trimmed head) grows a tree of candidates for each request (vt_rope_append, vt_tree_attention, vt_draft_head, vt_tree_select), the target
scores it, and what stays is decided by vt_verify_tokens.  The target is a stand-in: the logits of a full head on the draft's own hidden states
(vt_debug_logits) with noise, and torch.softmax.  Candidates are the best ones, so the form of the verification for drawn ones is not shown.  Weights
are random.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2603_05210_b200 as vt  # noqa: E402


class DraftLayer:
    """One layer with its cache: token embeddings in, hidden states out."""

    def __init__(self, B: int, d: int = 512, f: int = 1024, Hq: int = 8, heads: int = 2, D: int = 64, V: int = 4000, Vd: int = 3200, page: int = 16,
                 max_len: int = 256, max_tokens: int = 16):
        gen = torch.Generator(device="cuda").manual_seed(11)

        def normal(*shape, std):
            return (torch.randn(*shape, device="cuda", generator=gen) * std).bfloat16()

        self.embed, self.head = normal(V, d, std=1.0), normal(V, d, std=4 * d ** -0.5)
        self.W_qkv, self.W_o = normal((Hq + 2 * heads) * D, d, std=d ** -0.5), normal(d, Hq * D, std=(Hq * D) ** -0.5)
        self.gate, self.up, self.down = normal(f, d, std=d ** -0.5), normal(f, d, std=d ** -0.5), normal(d, f, std=f ** -0.5)
        self.keep = torch.randperm(V, device="cuda", generator=gen)[:Vd].int()
        self.head_kept = vt.vt_compact_head(self.head, self.keep)
        self.Hq, self.heads, self.D, self.max_tokens = Hq, heads, D, max_tokens
        per = max_len // page
        shape = (B * per, page, heads, D)
        self.cache = vt.VtCache(torch.zeros(shape, dtype=torch.bfloat16, device="cuda"), torch.zeros(shape, dtype=torch.bfloat16, device="cuda"),
                                torch.randperm(B * per, device="cuda", generator=gen).int().view(B, per), torch.zeros(B, dtype=torch.int32, device="cuda"))
        self.rope = vt.vt_rope_table(D)
        self.workspace = vt.new_workspace(vt.vt_tree_attention_workspace_bytes(Hq, heads, D, max_tokens))

    def __call__(self, tokens: torch.Tensor, positions: torch.Tensor, cu: torch.Tensor, mask: torch.Tensor | None) -> torch.Tensor:
        """Hidden states [N, d] of tokens that follow the cache's; their keys and values are stored behind it (lens stays)."""
        x = self.embed[tokens.long()]
        qkv = vt.vt_fuse_features(x, self.W_qkv).view(len(tokens), self.Hq + 2 * self.heads, self.D)
        q, k, v = qkv.split((self.Hq, self.heads, self.heads), dim=1)
        q = vt.vt_rope_append(q, k, v, positions, cu, self.cache, self.rope)
        a, _ = vt.vt_tree_attention(q, cu, self.cache, max_tokens=self.max_tokens, mask=mask, workspace=self.workspace)
        x = x + vt.vt_fuse_features(a.view(len(tokens), -1), self.W_o)
        return x + vt.vt_gated_ffn(x, self.gate, self.up, self.down)


def grow(layer: DraftLayer, root: torch.Tensor, lens: torch.Tensor, depth: int = 3, k: int = 4, width: int = 4):
    """Trees of 1 + depth * width tokens behind each request's root: (tokens, parents) [B, n].  Deeper tokens see their own way up alone."""
    B = len(root)
    tokens, parents = root[:, None], torch.full((B, 1), -1, dtype=torch.int32, device="cuda")
    scores = torch.zeros(B, 1, device="cuda")
    for level in range(depth):
        n = tokens.shape[1]
        cu = torch.arange(B + 1, dtype=torch.int32, device="cuda") * n
        mask, positions = vt.vt_tree_mask(parents.flatten().contiguous(), cu, layer.max_tokens, lens=lens)
        h = layer(tokens.flatten(), positions, cu, mask).view(B, n, -1)
        first = 0 if level == 0 else n - width
        for b in range(B):
            ids, lp = vt.vt_draft_head(h[b, first:].contiguous(), layer.head_kept, layer.keep, k)
            rows, _, chosen, best = vt.vt_tree_select(lp, ids, scores[b, first:].contiguous(), width)
            if b == 0:
                new = [torch.empty(B, width, dtype=torch.int32, device="cuda") for _ in range(2)] + [torch.empty(B, width, device="cuda")]
            new[0][b], new[1][b], new[2][b] = chosen, rows + first, best
        tokens, parents, scores = (torch.cat([a, c], 1) for a, c in zip((tokens, parents, scores), new))
    return tokens.contiguous(), parents.contiguous()


def main(rounds: int = 4, B: int = 3, prompt: int = 20, verbose: bool = True) -> list[list[int]]:
    layer = DraftLayer(B)
    gen = torch.Generator(device="cuda").manual_seed(5)
    V = layer.embed.shape[0]
    text = [torch.randint(V, (prompt + 3 * b,), device="cuda", generator=gen).tolist() for b in range(B)]

    def append(new: list[list[int]]) -> None:
        """Certain tokens go into the cache for good; the last one of a request is the next tree's root."""
        counts = [len(t) for t in new]
        cu = torch.tensor([0] + counts).cumsum(0).int().cuda()
        at = torch.cat([torch.arange(c) + int(n) for c, n in zip(counts, layer.cache.lens.tolist())]).int().cuda()
        layer.max_tokens, most = max(counts), layer.max_tokens
        layer.workspace = vt.new_workspace(vt.vt_tree_attention_workspace_bytes(layer.Hq, layer.heads, layer.D, max(most, layer.max_tokens)))
        layer(torch.tensor(sum(new, []), dtype=torch.int32, device="cuda"), at, cu, None)
        layer.cache.lens.add_(torch.tensor(counts, dtype=torch.int32, device="cuda"))
        layer.max_tokens = most

    append([t[:-1] for t in text])
    for _ in range(rounds):
        lens = layer.cache.lens
        tokens, parents = grow(layer, torch.tensor([t[-1] for t in text], dtype=torch.int32, device="cuda"), lens)
        n = tokens.shape[1]
        cu = torch.arange(B + 1, dtype=torch.int32, device="cuda") * n
        flat = parents.flatten().contiguous()
        mask, positions = vt.vt_tree_mask(flat, cu, layer.max_tokens, lens=lens)
        h = layer(tokens.flatten(), positions, cu, mask)                       # the target's pass over the whole tree
        logits = vt.vt_debug_logits(h, layer.head)
        logits += 0.5 * torch.randn(logits.shape, device="cuda", generator=gen)
        r = vt.vt_verify_tokens(torch.softmax(logits, 1), tokens.flatten(), flat, cu, torch.rand(B * n, device="cuda", generator=gen),
                                torch.rand(B, device="cuda", generator=gen), max_tokens=n)
        kept = [row[:c + 1] for row, c in zip(r.tokens.tolist(), r.n_accepted.tolist())]
        append([[t[-1]] + new[:-1] for t, new in zip(text, kept)])             # the root and what was accepted
        for t, new in zip(text, kept):
            t += new
        if verbose:
            print("accepted", r.n_accepted.tolist(), "lengths", [len(t) for t in text])
    assert vt.vt_last_status(layer.workspace) == vt.VT_OK
    assert layer.cache.lens.tolist() == [len(t) - 1 for t in text]
    return text


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--rounds", type=int, default=4)
    main(ap.parse_args().rounds)
