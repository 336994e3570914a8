"""The fp64 oracles of token scoring and of the gated feed-forward block against closed forms, loops and differences."""
import math

import numpy as np
import pytest

from oracle import vt_ffn_oracle as fo
from oracle import vt_score_oracle as so


def test_uniform_logits_have_closed_forms():
    M, d, V = 3, 5, 7
    r = so.score(np.zeros((M, d)), np.random.default_rng(0).normal(size=(V, d)), [0, 3, 6], k=4)
    assert np.allclose(r["lse"], math.log(V)) and np.allclose(r["logprobs"], -math.log(V)) and np.allclose(r["entropy"], math.log(V))
    assert (r["top_ids"] == np.arange(4)).all() and np.allclose(r["top_logprobs"], -math.log(V))


def test_two_tokens_by_hand():
    # logits 0 and s: p = 1 / (1 + e^s), e^s / (1 + e^s)
    for s in (-3.0, 0.5, 20.0):
        r = so.score(np.array([[1.0]]), np.array([[0.0], [s]]), [1], k=2)
        q = 1.0 / (1.0 + math.exp(-s))
        assert math.isclose(r["logprobs"][0], -math.log1p(math.exp(-s)), rel_tol=1e-12)
        H = -(q * math.log(q) + (1 - q) * math.log1p(-q)) if q < 1 else 0.0
        assert math.isclose(r["entropy"][0], H, rel_tol=1e-6, abs_tol=1e-12)
        assert list(r["top_ids"][0]) == ([1, 0] if s > 0 else [0, 1])


def test_a_common_shift_of_the_logits_moves_only_the_log_sum_exp():
    rng = np.random.default_rng(9)
    h, W, t = rng.normal(size=(4, 6)), rng.normal(size=(9, 6)), [0, 3, 5, 8]
    plain = so.score(h, W, t, k=3)
    assert np.allclose(plain["lse"], [math.log(sum(math.exp(sum(a * b for a, b in zip(x, w))) for w in W)) for x in h])
    for c in (-1000.0, 7.0, 1000.0):
        r = so.score(np.hstack([h, np.full((4, 1), c)]), np.hstack([W, np.ones((9, 1))]), t, k=3)
        assert np.allclose(r["lse"], plain["lse"] + c) and (r["top_ids"] == plain["top_ids"]).all()
        assert all(np.allclose(r[n], plain[n], atol=1e-11) for n in ("logprobs", "entropy", "top_logprobs"))


def test_scale_is_a_temperature():
    rng = np.random.default_rng(1)
    h, W, t = rng.normal(size=(4, 6)), rng.normal(size=(9, 6)), [0, 1, 2, 3]
    a, b = so.score(h, W, t, k=3, scale=0.5), so.score(0.5 * h, W, t, k=3)
    assert all(np.allclose(a[n], b[n]) for n in a)


def test_rows_without_a_token_inside_are_neutral():
    rng = np.random.default_rng(2)
    h, W = rng.normal(size=(4, 6)), rng.normal(size=(9, 6))
    h[[0, 2]] = np.nan
    t = [-1, 4, 9, 0]
    r = so.score(h, W, t, k=2)
    for n in ("logprobs", "entropy", "lse"):
        assert (r[n][[0, 2]] == 0).all() and (r[n][[1, 3]] != 0).all()
    assert (r["top_ids"][[0, 2]] == -1).all()
    dh, dW = so.score_backward(h, W, t, np.ones(4), np.ones(4))
    assert (dh[[0, 2]] == 0).all() and np.isfinite(dW).all()
    only, dW_only = so.score_backward(h[[1, 3]], W, [4, 0], np.ones(2), np.ones(2))
    assert np.allclose(dW, dW_only) and np.allclose(dh[[1, 3]], only)


def test_the_gradient_of_a_row_of_logits_sums_to_nothing():
    rng = np.random.default_rng(3)
    G, A = so.grad_logits(rng.normal(size=(5, 4)), rng.normal(size=(11, 4)), rng.integers(0, 11, 5), rng.normal(size=5), rng.normal(size=5), 1.3)
    assert np.abs(G.sum(1)).max() < 1e-12 and (np.abs(G) <= A + 1e-15).all()


@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_score_gradients_against_differences(scale):
    rng = np.random.default_rng(4)
    h, W, t = rng.normal(size=(3, 5)), rng.normal(size=(8, 5)), [2, -1, 7]
    gl, ge = rng.normal(size=3), rng.normal(size=3)

    def loss(h, W):
        r = so.score(h, W, t, scale=scale)
        return float(gl @ r["logprobs"] + ge @ r["entropy"])

    dh, dW = so.score_backward(h, W, t, gl, ge, scale)
    eps = 1e-5
    for a, g in ((h, dh), (W, dW)):
        for i in np.ndindex(a.shape):
            keep = a[i]
            a[i] = keep + eps
            up = loss(h, W)
            a[i] = keep - eps
            down = loss(h, W)
            a[i] = keep
            assert abs((up - down) / (2 * eps) - g[i]) < 1e-8


def test_activations_by_hand():
    assert fo.act(np.array([0.0]), "silu")[0] == 0.0 and fo.act(np.array([0.0]), "gelu")[0] == 0.0
    assert math.isclose(fo.act(np.array([1.0]), "silu")[0], 1 / (1 + math.exp(-1)), rel_tol=1e-12)
    assert math.isclose(fo.act(np.array([1.0]), "gelu")[0], 0.8411919906082768, rel_tol=1e-9)
    for kind in ("silu", "gelu"):
        assert math.isclose(fo.act(np.array([30.0]), kind)[0], 30.0, rel_tol=1e-9) and abs(fo.act(np.array([-30.0]), kind)[0]) < 1e-10
        assert math.isclose(fo.act_slope(np.array([0.0]), kind)[0], 0.5)


def test_block_by_loops():
    rng = np.random.default_rng(5)
    M, d, f = 2, 3, 4
    x, Wg, Wu, Wd = rng.normal(size=(M, d)), rng.normal(size=(f, d)), rng.normal(size=(f, d)), rng.normal(size=(d, f))
    y = np.zeros((M, d))
    for m in range(M):
        for j in range(f):
            g = sum(x[m, c] * Wg[j, c] for c in range(d))
            u = sum(x[m, c] * Wu[j, c] for c in range(d))
            for i in range(d):
                y[m, i] += Wd[i, j] * u * g / (1 + math.exp(-g))
    assert np.allclose(y, fo.forward(x, Wg, Wu, Wd, "silu")["y"])


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_block_gradients_against_differences(kind):
    rng = np.random.default_rng(6)
    M, d, f = 2, 3, 4
    args = [rng.normal(size=s) for s in ((M, d), (f, d), (f, d), (d, f))]
    dy = rng.normal(size=(M, d))
    r = fo.backward(*args, dy, kind)
    eps = 1e-6
    for a, name in zip(args, ("grad_x", "grad_W_gate", "grad_W_up", "grad_W_down")):
        for i in np.ndindex(a.shape):
            keep = a[i]
            a[i] = keep + eps
            up = (dy * fo.forward(*args, kind)["y"]).sum()
            a[i] = keep - eps
            down = (dy * fo.forward(*args, kind)["y"]).sum()
            a[i] = keep
            assert abs((up - down) / (2 * eps) - r[name][i]) < 1e-7
