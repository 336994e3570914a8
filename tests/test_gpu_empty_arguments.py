"""An empty tensor has no address. It must not pass for an argument that was not given."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def dev(a, dtype=torch.int32):
    return torch.tensor(a, dtype=dtype, device="cuda")


def test_a_mask_without_words():
    import paper_2603_05210_b200 as vt
    q, kv = torch.randn(3, 2, 64, device="cuda").bfloat16(), torch.randn(2, 16, 1, 64, device="cuda").bfloat16()
    cache, cu = vt.VtCache(kv, kv, dev([[0, 1]]), dev([9])), dev([0, 3])
    with pytest.raises(ValueError):
        vt.vt_tree_attention(q, cu, cache, max_tokens=3, mask=torch.empty(3, 0, dtype=torch.int32, device="cuda"))
    empty = vt.vt_tree_attention(q[:0], dev([0, 0]), cache, max_tokens=3, mask=torch.empty(0, 1, dtype=torch.int32, device="cuda"))
    assert empty[0].shape == (0, 2, 64)


def test_a_draft_without_a_vocabulary():
    import paper_2603_05210_b200 as vt
    probs = torch.full((2, 8), 0.125, device="cuda")
    args = (probs, dev([0, 1]), dev([-1, 0]), dev([0, 2]), torch.zeros(2, device="cuda"), torch.zeros(1, device="cuda"))
    for d2t in (None, dev([])):
        with pytest.raises(ValueError):
            vt.vt_verify_tokens(*args, max_tokens=2, draft_probs=torch.empty(2, 0, device="cuda"), draft_ids=dev([0, 0]), d2t=d2t)
    none = vt.vt_verify_tokens(probs[:0], dev([]), dev([]), dev([0, 0]), torch.zeros(0, device="cuda"), torch.zeros(1, device="cuda"), max_tokens=2,
                               draft_probs=torch.empty(0, 4, device="cuda"), draft_ids=dev([]))
    assert none.n_accepted.tolist() == [0] and none.tokens.tolist() == [[-1, -1]]
