"""The unwinding of the products behind scoring and the feed-forward block, without any fault: each ring stage is made to count on 16
bytes more than its copies bring (host side), so its wait runs out after two milliseconds.  Every CTA must then let what is in flight
end, give its memory back and return; the status word reports it, and the next calls, on the same workspace, are right."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vt():
    import paper_2603_05210_b200 as vt
    vt.lib()
    assert torch.cuda.is_available()
    return vt


@pytest.fixture
def withheld(vt):
    yield vt.vt_test_withhold_copies
    vt.vt_test_withhold_copies(0)


def rand(*shape, std=1.0):
    return (torch.randn(*shape, device="cuda") * std).bfloat16()


# few rows: single CTAs, sums divided in clusters; 60: several; 300: pairs; 1100: pairs with several tiles each
@pytest.mark.parametrize("M", [2, 60, 300, 1100])
def test_block(vt, withheld, M):
    d, f = 512, 1096
    x, g, u, dn, dy = rand(M, d), rand(f, d, std=d ** -0.5), rand(f, d, std=d ** -0.5), rand(d, f, std=f ** -0.5), rand(M, d)
    ws = vt.new_workspace(max(vt.vt_gated_ffn_workspace_bytes(M, d, f), vt.vt_gated_ffn_backward_workspace_bytes(M, d, f)))
    saved = torch.empty(M, 2 * f, device="cuda")
    want = vt.vt_gated_ffn(x, g, u, dn, saved=saved), *vt.vt_gated_ffn_backward(x, g, u, dn, saved, dy)
    for _ in range(2):
        withheld(2000)
        vt.vt_gated_ffn(x, g, u, dn, workspace=ws)
        assert vt.vt_last_status(ws) == vt.VT_ERR_TIMEOUT
        vt.vt_gated_ffn_backward(x, g, u, dn, saved, dy, workspace=ws)
        assert vt.vt_last_status(ws) == vt.VT_ERR_TIMEOUT
        withheld(0)
        got = vt.vt_gated_ffn(x, g, u, dn, workspace=ws), *vt.vt_gated_ffn_backward(x, g, u, dn, saved, dy, workspace=ws)
        assert vt.vt_last_status(ws) == vt.VT_OK
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("M,V,k", [(3, 3000, 0), (3, 3000, 8), (40, 30000, 8), (300, 9000, 20), (1100, 5000, 4)])
def test_scoring(vt, withheld, M, V, k):
    d = 512
    h, W, t, g = rand(M, d), rand(V, d, std=0.03), torch.randint(V, (M,), device="cuda").int(), torch.randn(M, device="cuda")
    ws = vt.new_workspace(max(vt.vt_score_workspace_bytes(M, d, V, k), vt.vt_score_backward_workspace_bytes(M, d, V)))
    want = vt.vt_score_tokens(h, W, t, k=k)
    want_grads = vt.vt_score_tokens_backward(h, W, t, want.lse, want.entropy, g, g)
    for _ in range(2):
        withheld(2000)
        vt.vt_score_tokens(h, W, t, k=k, workspace=ws)
        assert vt.vt_last_status(ws) == vt.VT_ERR_TIMEOUT
        vt.vt_score_tokens_backward(h, W, t, want.lse, want.entropy, g, g, workspace=ws)
        assert vt.vt_last_status(ws) == vt.VT_ERR_TIMEOUT
        withheld(0)
        got = vt.vt_score_tokens(h, W, t, k=k, workspace=ws)
        grads = vt.vt_score_tokens_backward(h, W, t, want.lse, want.entropy, g, g, workspace=ws)
        assert vt.vt_last_status(ws) == vt.VT_OK
        assert all(a is b or torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(a, b) for a, b in zip(grads, want_grads))
    for bad in (-1, 100_001):
        with pytest.raises(vt.VtError):
            withheld(bad)
