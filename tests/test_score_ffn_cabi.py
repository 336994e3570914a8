"""Refusals of the scoring and feed-forward entry points, and the checks of their binding, without a GPU."""
import math

import pytest
import torch


@pytest.fixture(scope="module")
def vt():
    from paper_2603_05210_b200.build import build
    build()
    import paper_2603_05210_b200 as vt
    vt.lib()
    return vt


FAKE = 0x10000        # a non-NULL, 256-byte aligned address that is never dereferenced on the host
BIG = 1 << 40


def score(vt, **kw):
    a = dict(h=FAKE, ldh=4096, W=FAKE, tokens=FAKE, M=8, d=4096, V=32000, scale=1.0, k=8, lp=FAKE, H=FAKE, lse=FAKE, ti=FAKE, tl=FAKE,
             ws=FAKE, n=BIG)
    a.update(kw)
    return vt.lib().vt_score_tokens(a["h"], a["ldh"], a["W"], a["tokens"], a["M"], a["d"], a["V"], a["scale"], a["k"], a["lp"], a["H"],
                                    a["lse"], a["ti"], a["tl"], a["ws"], a["n"], None)


def test_score_refuses(vt):
    for bad in (dict(h=None), dict(W=None), dict(ti=None), dict(tl=None), dict(tokens=None)):
        assert score(vt, **bad) == vt.VT_ERR_NULL, bad
    for bad in (dict(d=0), dict(d=4100), dict(M=0), dict(V=0), dict(k=-1), dict(k=9, V=8), dict(k=vt.VT_MAX_K + 1), dict(ldh=4088), dict(ldh=4100),
                dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf)):
        assert score(vt, **bad) == vt.VT_ERR_SHAPE, bad
    for bad in (dict(h=FAKE + 8), dict(W=FAKE + 2), dict(tokens=FAKE + 1), dict(lp=FAKE + 2), dict(ti=FAKE + 2)):
        assert score(vt, **bad) == vt.VT_ERR_ALIGN, bad
    need = vt.vt_score_workspace_bytes(8, 4096, 32000, 8)
    for bad in (dict(ws=None), dict(ws=FAKE + 16), dict(n=need - 1)):
        assert score(vt, **bad) == vt.VT_ERR_WORKSPACE, bad


def score_back(vt, **kw):
    a = dict(h=FAKE, ldh=4096, W=FAKE, tokens=FAKE, lse=FAKE, H=FAKE, gl=FAKE, ge=FAKE, M=8, d=4096, V=32000, scale=1.0, dh=FAKE, dW=FAKE,
             ws=FAKE, n=BIG)
    a.update(kw)
    return vt.lib().vt_score_tokens_backward(a["h"], a["ldh"], a["W"], a["tokens"], a["lse"], a["H"], a["gl"], a["ge"], a["M"], a["d"], a["V"],
                                             a["scale"], a["dh"], a["dW"], a["ws"], a["n"], None)


def test_score_backward_refuses(vt):
    for bad in (dict(h=None), dict(W=None), dict(tokens=None), dict(lse=None), dict(gl=None), dict(H=None), dict(dh=None, dW=None)):
        assert score_back(vt, **bad) == vt.VT_ERR_NULL, bad
    for bad in (dict(d=12), dict(M=0), dict(V=0), dict(ldh=8), dict(scale=0.0)):
        assert score_back(vt, **bad) == vt.VT_ERR_SHAPE, bad
    for bad in (dict(h=FAKE + 8), dict(dh=FAKE + 8), dict(dW=FAKE + 2), dict(lse=FAKE + 2), dict(ge=FAKE + 1)):
        assert score_back(vt, **bad) == vt.VT_ERR_ALIGN, bad
    need = vt.vt_score_backward_workspace_bytes(8, 4096, 32000)
    assert need >= 8 * 32000 * 2
    for bad in (dict(ws=None), dict(ws=FAKE + 8), dict(n=need - 1)):
        assert score_back(vt, **bad) == vt.VT_ERR_WORKSPACE, bad


def ffn(vt, **kw):
    a = dict(x=FAKE, ldx=4096, g=FAKE, u=FAKE, dn=FAKE, M=8, d=4096, f=2048, act=0, y=FAKE, saved=FAKE, ws=FAKE, n=BIG)
    a.update(kw)
    return vt.lib().vt_gated_ffn(a["x"], a["ldx"], a["g"], a["u"], a["dn"], a["M"], a["d"], a["f"], a["act"], a["y"], a["saved"], a["ws"],
                                 a["n"], None)


def test_ffn_refuses(vt):
    for bad in (dict(x=None), dict(g=None), dict(u=None), dict(dn=None), dict(y=None)):
        assert ffn(vt, **bad) == vt.VT_ERR_NULL, bad
    for bad in (dict(d=0), dict(d=20), dict(f=0), dict(f=2044), dict(M=0), dict(ldx=2048), dict(ldx=4100), dict(act=2), dict(act=-1)):
        assert ffn(vt, **bad) == vt.VT_ERR_SHAPE, bad
    for bad in (dict(x=FAKE + 8), dict(g=FAKE + 2), dict(u=FAKE + 2), dict(dn=FAKE + 2), dict(y=FAKE + 8), dict(saved=FAKE + 8)):
        assert ffn(vt, **bad) == vt.VT_ERR_ALIGN, bad
    need = vt.vt_gated_ffn_workspace_bytes(8, 4096, 2048)
    for bad in (dict(ws=None), dict(ws=FAKE + 8), dict(n=need - 1)):
        assert ffn(vt, **bad) == vt.VT_ERR_WORKSPACE, bad


def ffn_back(vt, **kw):
    a = dict(x=FAKE, ldx=4096, g=FAKE, u=FAKE, dn=FAKE, saved=FAKE, dy=FAKE, ldy=4096, M=8, d=4096, f=2048, act=1, gx=FAKE, gg=FAKE, gu=FAKE,
             gd=FAKE, ws=FAKE, n=BIG)
    a.update(kw)
    return vt.lib().vt_gated_ffn_backward(a["x"], a["ldx"], a["g"], a["u"], a["dn"], a["saved"], a["dy"], a["ldy"], a["M"], a["d"], a["f"],
                                          a["act"], a["gx"], a["gg"], a["gu"], a["gd"], a["ws"], a["n"], None)


def test_ffn_backward_refuses(vt):
    for bad in (dict(x=None), dict(g=None), dict(saved=None), dict(dy=None), dict(gx=None, gg=None, gu=None, gd=None)):
        assert ffn_back(vt, **bad) == vt.VT_ERR_NULL, bad
    for bad in (dict(d=20), dict(f=12), dict(M=0), dict(ldy=8), dict(ldy=4100), dict(act=7)):
        assert ffn_back(vt, **bad) == vt.VT_ERR_SHAPE, bad
    for bad in (dict(dy=FAKE + 8), dict(gx=FAKE + 2), dict(gg=FAKE + 8), dict(saved=FAKE + 4)):
        assert ffn_back(vt, **bad) == vt.VT_ERR_ALIGN, bad
    need = vt.vt_gated_ffn_backward_workspace_bytes(8, 4096, 2048)
    for bad in (dict(ws=None), dict(ws=FAKE + 8), dict(n=need - 1)):
        assert ffn_back(vt, **bad) == vt.VT_ERR_WORKSPACE, bad


def test_sizes(vt):
    assert vt.vt_score_workspace_bytes(0, 64, 10, 0) == 0 and vt.vt_score_workspace_bytes(1, 64, 10, 11) == 0
    assert vt.vt_score_workspace_bytes(1, 60, 10, 1) == 0 and vt.vt_score_backward_workspace_bytes(1, 64, 0) == 0
    assert vt.vt_gated_ffn_workspace_bytes(4, 64, 12) == 0 and vt.vt_gated_ffn_backward_workspace_bytes(0, 64, 64) == 0
    assert vt.vt_gated_ffn_workspace_bytes(100, 64, 128) >= 100 * 128 * 2
    assert vt.vt_gated_ffn_backward_workspace_bytes(100, 64, 128) >= 3 * 100 * 128 * 2
    # few logits are kept, many are not: the workspace stays far below M * V * 4 there
    assert vt.vt_score_workspace_bytes(4, 64, 32000, 4) >= 4 * 32000 * 4
    assert vt.vt_score_workspace_bytes(4096, 4096, 32000, 4) < 4096 * 32000 * 4 // 4


def test_binding_refuses_what_is_not_on_the_device_or_does_not_fit(vt):
    h, W, t = torch.zeros(2, 8, dtype=torch.bfloat16), torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        vt.vt_score_tokens(h, W, t)
    with pytest.raises(TypeError):
        vt.vt_score_tokens(h.float(), W, t)
    with pytest.raises(ValueError):
        vt.vt_score_tokens_backward(h, W, t, torch.zeros(2), torch.zeros(2), torch.zeros(2))
    with pytest.raises(ValueError):
        vt.vt_gated_ffn(h, W, W, W.T.contiguous())
    with pytest.raises(ValueError):
        vt.vt_gated_ffn_backward(h, W, W, W.T.contiguous(), torch.zeros(2, 8), h)


def test_docstrings_say_where_a_time_out_is_seen(vt):
    for name in ("vt_score_tokens", "vt_score_tokens_backward", "vt_gated_ffn", "vt_gated_ffn_backward"):
        assert "vt_last_status" in getattr(vt, name).__doc__, name
