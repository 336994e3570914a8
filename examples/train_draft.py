"""A draft layer trained on a trimmed vocabulary and then used to check drafted tokens: every step through the library.

    python examples/train_draft.py [--steps 30]

The draft vocabulary is chosen from a token stream (vt_select_vocab) and the head cut down to it (vt_compact_head).  A training
step fuses three layers' features (vt_fuse_features), runs the gated feed-forward block around a residual (vt_gated_ffn), scores
the next tokens under the trimmed head (vt_score_tokens; a token outside the kept set is not scored), and takes both gradients
back (vt_score_tokens_backward, vt_gated_ffn_backward).  At the end the draft head proposes tokens (vt_draft_head) and the full
head scores them (vt_score_tokens), which is what accepting them is decided by.  Data and weights are synthetic.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2603_05210_b200 as vt  # noqa: E402
from paper_2603_05210_b200 import inputs  # noqa: E402


class Draft:
    """Fusion, one gated block, trimmed head; plain stochastic gradient descent on fp32 copies of the weights."""

    def __init__(self, W_head: torch.Tensor, d: int, f: int, rows: int, entropy_bonus: float = 0.0, lr: float = 1.0):
        gen = torch.Generator(device="cuda").manual_seed(7)

        def normal(r, c, std):
            return torch.randn(r, c, device="cuda", generator=gen) * std

        self.master = {"gate": normal(f, d, d ** -0.5), "up": normal(f, d, d ** -0.5), "down": normal(d, f, 0.1 * f ** -0.5),
                       "head": W_head.float()}
        self.W = {n: w.bfloat16() for n, w in self.master.items()}
        self.W_fuse = normal(d, 3 * d, (3 * d) ** -0.5).bfloat16()
        self.lr, self.entropy_bonus = lr, entropy_bonus
        V = W_head.shape[0]
        self.saved = torch.empty((rows, 2 * f), device="cuda")
        self.workspace = vt.new_workspace(max(
            vt.vt_workspace_bytes(rows, 1), vt.vt_gated_ffn_workspace_bytes(rows, d, f), vt.vt_gated_ffn_backward_workspace_bytes(rows, d, f),
            vt.vt_score_workspace_bytes(rows, d, V, 0), vt.vt_score_backward_workspace_bytes(rows, d, V)))

    def hidden(self, features: torch.Tensor, saved: torch.Tensor | None = None):
        x = vt.vt_fuse_features(features, self.W_fuse, workspace=self.workspace)
        y = vt.vt_gated_ffn(x, self.W["gate"], self.W["up"], self.W["down"], saved=saved, workspace=self.workspace)
        return x, x + y

    def step(self, features: torch.Tensor, tokens: torch.Tensor) -> torch.Tensor:
        """One update on `features` [rows, 3d] and draft indices `tokens` [rows] (-1: not in the draft vocabulary); the loss."""
        x, h = self.hidden(features, self.saved)
        r = vt.vt_score_tokens(h, self.W["head"], tokens, workspace=self.workspace)
        n = (tokens >= 0).sum().clamp(min=1)
        loss = -(r.logprobs.sum() + self.entropy_bonus * r.entropy.sum()) / n
        grad_logprobs = (-1.0 / n).expand_as(r.logprobs).contiguous()
        grad_h, grad_head = vt.vt_score_tokens_backward(h, self.W["head"], tokens, r.lse, r.entropy, grad_logprobs,
                                                        self.entropy_bonus * grad_logprobs, workspace=self.workspace)
        _, grad_gate, grad_up, grad_down = vt.vt_gated_ffn_backward(x, self.W["gate"], self.W["up"], self.W["down"], self.saved, grad_h,
                                                                    workspace=self.workspace)
        for name, grad in (("gate", grad_gate), ("up", grad_up), ("down", grad_down), ("head", grad_head)):
            self.master[name] -= self.lr * grad.float()
            self.W[name].copy_(self.master[name])
        return loss


def main(steps: int = 30, rows: int = 512, d: int = 512, f: int = 1024, V_full: int = 20000, verbose: bool = True) -> list[float]:
    stream = torch.from_numpy(inputs.zipf_token_stream(V_full, 1.1, 200_000, seed=1)).cuda()
    chosen = vt.vt_select_vocab(stream, V_full, d, 2.0 * (3 * d * d + 3 * d * f), 0.5, 0.9, 64, V_full)
    keep = chosen["ranked_ids"][:chosen["k_star"]].contiguous()
    W_full = torch.from_numpy(inputs.normal_bf16((V_full, d), 0.02, 2).view("int16")).cuda().view(torch.bfloat16)
    index_of = torch.full((V_full,), -1, dtype=torch.int32, device="cuda")
    index_of[keep.long()] = torch.arange(len(keep), dtype=torch.int32, device="cuda")
    draft = Draft(vt.vt_compact_head(W_full, keep), d, f, rows)

    gen = torch.Generator(device="cuda").manual_seed(3)
    features = torch.randn(rows, 3 * d, device="cuda", generator=gen).bfloat16()
    targets = stream[:rows].contiguous()
    losses = []
    for i in range(steps):
        losses.append(float(draft.step(features, index_of[targets.long()])))
        if verbose and i % 10 == 0:
            print(f"step {i:3d}  loss {losses[-1]:.4f}")

    # serving: eight rows propose one token each, the full head says how likely each is and what it would have preferred
    _, h = draft.hidden(features[:8].contiguous())
    proposed, draft_logprobs = vt.vt_draft_head(h, draft.W["head"], keep, 1)
    full = vt.vt_score_tokens(h, W_full, proposed[:, 0].contiguous(), k=4)
    accept = (full.logprobs - draft_logprobs[:, 0]).exp().clamp(max=1.0)
    if verbose:
        print(f"{len(keep)} of {V_full} tokens kept (coverage {chosen['C']:.3f}); loss {losses[0]:.4f} -> {losses[-1]:.4f}")
        print("acceptance probabilities of the proposed tokens:", [round(float(a), 4) for a in accept])
    assert vt.vt_last_status(draft.workspace) == vt.VT_OK
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=30)
    main(ap.parse_args().steps)
