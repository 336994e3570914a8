"""What the binding of the scoring and feed-forward operators refuses although its tensors are on the device."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vt():
    import paper_2603_05210_b200 as vt
    vt.lib()
    assert torch.cuda.is_available()
    return vt


def calls(vt):
    """The four operators on small inputs, each as a function of its workspace, with the bytes it needs."""
    M, d, V, f = 3, 64, 100, 72
    h, W, t = torch.randn(M, d, device="cuda").bfloat16(), torch.randn(V, d, device="cuda").bfloat16(), torch.arange(M, device="cuda", dtype=torch.int32)
    r = vt.vt_score_tokens(h, W, t)
    g, u, dn = torch.randn(f, d, device="cuda").bfloat16(), torch.randn(f, d, device="cuda").bfloat16(), torch.randn(d, f, device="cuda").bfloat16()
    saved = torch.empty(M, 2 * f, device="cuda")
    vt.vt_gated_ffn(h, g, u, dn, saved=saved)
    return [(lambda ws: vt.vt_score_tokens(h, W, t, workspace=ws), vt.vt_score_workspace_bytes(M, d, V, 0)),
            (lambda ws: vt.vt_score_tokens_backward(h, W, t, r.lse, None, r.lse, workspace=ws), vt.vt_score_backward_workspace_bytes(M, d, V)),
            (lambda ws: vt.vt_gated_ffn(h, g, u, dn, workspace=ws), vt.vt_gated_ffn_workspace_bytes(M, d, f)),
            (lambda ws: vt.vt_gated_ffn_backward(h, g, u, dn, saved, h, workspace=ws), vt.vt_gated_ffn_backward_workspace_bytes(M, d, f))]


def test_workspaces(vt):
    for call, need in calls(vt):
        with pytest.raises(ValueError):
            call(torch.empty(need, dtype=torch.uint8))                                     # host memory
        with pytest.raises(ValueError):
            call(torch.empty(2 * need, dtype=torch.uint8, device="cuda")[::2])             # every other byte
        with pytest.raises(vt.VtError) as e:
            call(torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
        assert e.value.status == vt.VT_ERR_WORKSPACE
        call(torch.empty((need + 3) // 4, dtype=torch.float32, device="cuda"))             # its bytes count, whatever its type


def test_activations(vt):
    M, d, f = 3, 64, 72
    x, g, u, dn = (torch.randn(r, c, device="cuda").bfloat16() for r, c in ((M, d), (f, d), (f, d), (d, f)))
    saved = torch.empty(M, 2 * f, device="cuda")
    for name, number in (("silu", vt.VT_ACT_SILU), ("gelu", vt.VT_ACT_GELU)):
        assert torch.equal(vt.vt_gated_ffn(x, g, u, dn, act=name, saved=saved), vt.vt_gated_ffn(x, g, u, dn, act=number))
    for bad in ("relu", "SiLU", 2, -1, None):
        with pytest.raises(ValueError):
            vt.vt_gated_ffn(x, g, u, dn, act=bad)
        with pytest.raises(ValueError):
            vt.vt_gated_ffn_backward(x, g, u, dn, saved, x, act=bad)
