"""Rotary positions, cache, attention and verification together, as a decode step uses them."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import vt_step_oracle as so

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def vt():
    import paper_2603_05210_b200 as vt
    vt.lib()
    return vt


def f64(t):
    return t.detach().double().cpu().numpy()


def test_positions_cache_and_attention(vt):
    """A prompt in chunks, then a tree, through vt_rope_append and vt_tree_attention; the oracle goes from the unturned projections.
    Keys and queries are rounded to bf16 once after the turn, 2^-8 each: scores move by at most 2 * 2^-8 X, X = scale sum |q||k|, weights by twice that;
    with the bounds of the attention alone (2^-8 |out| + A 2^-8 and less) an element is within 2^-8 |out| + A (4 * 2^-8 Xmax + 2^-7)."""
    torch.manual_seed(1)
    B, Hq, heads, D, page = 2, 6, 3, 64, 16
    rope, w = vt.vt_rope_table(D, scaling="linear", factor=2.0), so.rope_frequencies(D, scaling="linear", factor=2.0)
    shape = (40, page, heads, D)
    cache = vt.VtCache(*(torch.full(shape, float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)),
                       torch.randperm(40, device="cuda").int().view(B, 20), torch.zeros(B, dtype=torch.int32, device="cuda"))
    history = [[] for _ in range(B)]
    for counts, tree in (([70, 33], False), ([1, 90], False), ([9, 5], True)):
        N = sum(counts)
        cu = torch.tensor([0] + counts).cumsum(0).int().cuda()
        qkv = (torch.randn(N, Hq + 2 * heads, D, device="cuda") * 0.7).bfloat16()
        q, k, v = qkv.split((Hq, heads, heads), dim=1)
        parents = torch.cat([torch.tensor([max(i - 1 - (i % 3), 0) if i else -1 for i in range(c)]) for c in counts]).int().cuda()
        mask, positions = vt.vt_tree_mask(parents, cu, max(counts), lens=cache.lens)
        if not tree:
            mask = None
            positions = torch.cat([torch.arange(c, device="cuda") + n for c, n in zip(counts, cache.lens)]).int()
        turned = vt.vt_rope_append(q, k, v, positions, cu, cache, rope)
        out, _ = vt.vt_tree_attention(turned, cu, cache, max_tokens=max(counts), mask=mask)
        tq, tk = so.rope(f64(q), positions.tolist(), w), so.rope(f64(k), positions.tolist(), w)
        for b in range(B):
            lo, hi = int(cu[b]), int(cu[b + 1])
            keys = np.concatenate([*(h[0] for h in history[b]), tk[lo:hi]])
            values = np.concatenate([*(h[1] for h in history[b]), f64(v)[lo:hi]])
            L = len(keys) - (hi - lo)
            bits = None if mask is None else mask[lo:hi].cpu().numpy().astype(np.int64) & 0xFFFFFFFF
            want, _, size = so.attention(tq[lo:hi], keys[None], values[None], np.zeros((1, 1), int), [L], [0, hi - lo], bits, D ** -0.5, hi - lo)
            X = D ** -0.5 * np.abs(tq[lo:hi]).sum(-1) * np.abs(keys).max()
            err = np.abs(f64(out)[lo:hi] - want) - 2.0 ** -8 * np.abs(want) - size * (4 * 2.0 ** -8 * X + 2.0 ** -7)[..., None]
            assert np.all(err <= 0), err.max()
            history[b].append((tk[lo:hi], f64(v)[lo:hi]))
        cache.lens.add_(torch.tensor(counts, dtype=torch.int32, device="cuda"))


def test_a_step_captured_whole(vt):
    """Append, attention and verification in one graph, replayed with other inputs, equal the calls one by one."""
    torch.manual_seed(2)
    B, T, Hq, heads, D, V = 3, 8, 4, 2, 64, 700
    N = B * T
    cache = vt.VtCache(*(torch.randn(30, 16, heads, D, device="cuda").bfloat16() for _ in range(2)), torch.randperm(30, device="cuda").int().view(B, 10),
                       torch.tensor([5, 0, 100], dtype=torch.int32, device="cuda"))
    cu = torch.arange(0, N + 1, T, dtype=torch.int32, device="cuda")
    parents = torch.tensor([-1, 0, 0, 1, 1, 2, 3, 5] * B, dtype=torch.int32, device="cuda")
    x = {"qkv": torch.randn(N, Hq + 2 * heads, D, device="cuda").bfloat16(), "P": torch.softmax(3 * torch.randn(N, V, device="cuda"), 1),
         "tokens": torch.randint(V, (N,), device="cuda").int(), "ua": torch.rand(N, device="cuda"), "us": torch.rand(B, device="cuda")}
    rope, ws = vt.vt_rope_table(D, interleaved=True), vt.new_workspace(vt.vt_tree_attention_workspace_bytes(Hq, heads, D, T))

    def step():
        q, k, v = x["qkv"].split((Hq, heads, heads), dim=1)
        mask, positions = vt.vt_tree_mask(parents, cu, T, lens=cache.lens)
        q = vt.vt_rope_append(q, k, v, positions, cu, cache, rope)
        a, lse = vt.vt_tree_attention(q, cu, cache, max_tokens=T, mask=mask, workspace=ws)
        return a, lse, *vt.vt_verify_tokens(x["P"], x["tokens"], parents, cu, x["ua"], x["us"], max_tokens=T)

    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        with torch.cuda.graph(g, stream=side):
            got = step()
    torch.cuda.synchronize()
    for i in range(3):
        x["qkv"].normal_()
        x["P"].copy_(torch.softmax(3 * torch.randn(N, V, device="cuda"), 1))
        x["tokens"].copy_(x["P"].argmax(1).int()[parents.clamp(min=0).long() + cu[:-1].repeat_interleave(T).long()])
        x["ua"].uniform_(), x["us"].uniform_()
        cache.lens.copy_(torch.tensor([5 + i, 31 * i, 100], dtype=torch.int32))
        want = step()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert vt.vt_last_status(ws) == vt.VT_OK


def test_example():
    spec = importlib.util.spec_from_file_location("decode_step", os.path.join(ROOT, "examples", "decode_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    text = m.main(rounds=3, verbose=False)
    assert text == m.main(rounds=3, verbose=False)               # the same run twice
    assert all(len(t) > 20 + 3 * b for b, t in enumerate(text)) and all(0 <= i < 4000 for t in text for i in t)
