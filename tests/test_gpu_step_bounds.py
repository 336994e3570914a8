"""Offsets below 0 count as 0, in every call of a decode step alike."""
import pytest
import torch

from .test_gpu_rope import paged, vt  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("first", [-1, -3, -1000, -2 ** 31])
def test_offsets_below_zero(vt, first):  # noqa: F811
    def dev(a):
        return torch.tensor(a, dtype=torch.int32, device="cuda")

    parents, lens = dev([2, 0, 1, 0, 2, -1, 0, 0]), dev([4, 9, 3])
    for counts, below in (([6, 0, 2], [first, 6, 6, 8]), ([0, 6, 2], [first, first // 2, 6, 8])):
        cu = dev([0] + [sum(counts[:i + 1]) for i in range(3)])
        want = vt.vt_tree_mask(parents, cu, 8, lens=lens)
        got = vt.vt_tree_mask(parents, dev(below), 8, lens=lens)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        torch.manual_seed(1)
        cache, _ = paged(vt, [4, 9, 3], counts, 2, 64, 16)
        q, k, v = (torch.randn(8, h, 64, device="cuda").bfloat16() for h in (4, 2, 2))
        rope, kc, vc = vt.vt_rope_table(64), cache.k.clone(), cache.v.clone()
        out = vt.vt_rope_append(q, k, v, want[1], cu, cache, rope)
        want_k, want_v, want_a = cache.k.clone(), cache.v.clone(), vt.vt_tree_attention(out, cu, cache, max_tokens=8, mask=want[0])
        cache.k.copy_(kc), cache.v.copy_(vc)
        again = vt.vt_rope_append(q, k, v, want[1], dev(below), cache, rope)
        got_a = vt.vt_tree_attention(again, dev(below), cache, max_tokens=8, mask=want[0])
        assert torch.equal(again, out) and torch.equal(cache.k, want_k) and torch.equal(cache.v, want_v)
        assert torch.equal(got_a[0], want_a[0]) and torch.equal(got_a[1], want_a[1])
