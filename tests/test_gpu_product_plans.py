"""Scoring and the feed-forward block at sizes whose products run as CTA pairs, over several rounds of tiles, with more row tiles
than share their columns (8), and with divided sums: the forms that calls of thousands of rows take.  Each test first asserts that
its products do take them, so that a change of the plans cannot quietly leave one untested.  Data, bounds and their derivation are
those of test_gpu_ffn.py and test_gpu_score.py."""
import numpy as np
import pytest
import torch

from oracle import vt_score_oracle as so
from tests import test_gpu_ffn as tf
from tests import test_gpu_score as ts

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vt():
    import paper_2603_05210_b200 as vt
    vt.lib()
    assert torch.cuda.is_available()
    return vt


def forms(rows):
    """Per product: P a CTA pair, S a divided sum, C one CTA to a tile; + where a CTA or pair takes several tiles in turn."""
    return [("P" if pair else "S" if splits > 1 else "C") + ("+" if items > at_once else "") for pair, _, splits, items, at_once in rows]


# gate and up, y, da, dx, the weight gradients
BLOCKS = [((20000, 128, 264), ["P+", "P+", "P+", "P+", "S"]), ((2500, 520, 1352), ["P+", "P", "P", "P", "P"]),
          ((1500, 1024, 2000), ["P+", "P", "P", "P", "P+"]), ((600, 264, 8192), ["P+", "S", "P+", "S", "P+"])]


@pytest.mark.parametrize("size,expected", BLOCKS)
@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_block(vt, size, expected, kind):
    M, d, f = size
    args = tf.case(M, d, f, M + d)
    x, Wg, Wu, Wd, dy = (t.cuda() for t in args)
    y, saved = tf.Guarded((M, d), torch.bfloat16), tf.Guarded((M, 2 * f), torch.float32)
    ws = vt.new_workspace(max(vt.vt_gated_ffn_workspace_bytes(M, d, f), vt.vt_gated_ffn_backward_workspace_bytes(M, d, f)))
    vt.vt_test_products()
    vt.vt_gated_ffn(x, Wg, Wu, Wd, act=kind, out=y.t, saved=saved.t, workspace=ws)
    outs = {"grad_x": tf.Guarded((M, d), torch.bfloat16), "grad_W_gate": tf.Guarded((f, d), torch.bfloat16),
            "grad_W_up": tf.Guarded((f, d), torch.bfloat16), "grad_W_down": tf.Guarded((d, f), torch.bfloat16)}
    vt.vt_gated_ffn_backward(x, Wg, Wu, Wd, saved.t, dy, act=kind, workspace=ws, **{n: g.t for n, g in outs.items()})
    assert forms(vt.vt_test_products()) == expected
    assert vt.vt_last_status(ws) == vt.VT_OK and y.intact() and saved.intact() and all(g.intact() for g in outs.values())
    tf.compare({"y": y.t} | {n: g.t for n, g in outs.items()}, tf.bounds(*args, kind))
    again = vt.vt_gated_ffn_backward(x, Wg, Wu, Wd, saved.t, dy, act=kind)
    assert all(torch.equal(a, g.t) for a, g in zip(again, outs.values())), "not the same bits twice"


# scores, G, dh, dW
SCORES = [((20000, 136, 300), ["P+", "P+", "P+", "S"]), ((4608, 512, 4100), ["P", "P+", "P", "P"]), ((2500, 1032, 1500), ["P", "P", "P", "P"]),
          ((700, 512, 20000), ["P", "P+", "S", "P+"])]


@pytest.mark.parametrize("size,expected", SCORES)
def test_scores_and_gradients(vt, size, expected):
    M, d, V = size
    rng = np.random.default_rng(30)
    h, W, tokens = ts.case(M, d, V, M + V)
    tokens[::7] = -1
    scale = 0.8
    gl, ge = rng.normal(size=M).astype(np.float32), rng.normal(size=M).astype(np.float32)
    hd, Wd, t = ts.dev(h), ts.dev(W), ts.dev(tokens, torch.int32)
    ws = vt.new_workspace(max(vt.vt_score_workspace_bytes(M, d, V, 0), vt.vt_score_backward_workspace_bytes(M, d, V)))
    vt.vt_test_products()
    r = vt.vt_score_tokens(hd, Wd, t, scale=scale, workspace=ws)
    gh, gW = ts.Guarded((M, d), torch.bfloat16), ts.Guarded((V, d), torch.bfloat16)
    ups = torch.from_numpy(gl).cuda(), torch.from_numpy(ge).cuda()
    vt.vt_score_tokens_backward(hd, Wd, t, r.lse, r.entropy, *ups, scale=scale, workspace=ws, grad_h=gh.t, grad_W=gW.t)
    assert forms(vt.vt_test_products()) == expected
    assert vt.vt_last_status(ws) == vt.VT_OK and gh.intact() and gW.intact()
    ts.check({n: getattr(r, n).cpu().numpy() for n in ("logprobs", "entropy", "lse")}, so.score(h, W, tokens, 0, scale), V)
    want_h, want_W = so.score_backward(h, W, tokens, gl, ge, scale)
    _, A = so.grad_logits(h, W, tokens, gl, ge, scale)
    keep = so.scored_rows(tokens, M, V)
    slack = 2.0 ** -8 + 2.0 ** -14
    for got, want, terms in ((gh.t, want_h, A @ np.abs(W)), (gW.t, want_W, A[keep].T @ np.abs(h[keep]))):
        err = np.abs(got.double().cpu().numpy() - want)
        assert (err <= 2.0 ** -8 * np.abs(want) + slack * terms + 1e-30).all()
        assert np.linalg.norm(err) <= 2.0 ** -8 * np.linalg.norm(want)
    again = vt.vt_score_tokens_backward(hd, Wd, t, r.lse, r.entropy, *ups, scale=scale)
    assert torch.equal(again[0], gh.t) and torch.equal(again[1], gW.t), "not the same bits twice"


@pytest.mark.parametrize("M,V,k", [(20000, 300, 8), (4608, 4100, 20), (3000, 9000, 4), (3000, 9000, 30)])
def test_alternatives_of_many_rows(vt, M, V, k):
    h, W, tokens = ts.case(M, 136, V, M + k)
    vt.vt_test_products()
    got = ts.run(vt, ts.dev(h), ts.dev(W), ts.dev(tokens, torch.int32), k)
    assert forms(vt.vt_test_products())[0][0] == "P"
    ts.check(got, so.score(h, W, tokens, k), V)
