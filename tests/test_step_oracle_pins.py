"""Pins of the decode-step oracle: closed forms, invariances, brute force, and the law that verification has to obey."""
import itertools
import math

import numpy as np
import pytest

from oracle import vt_step_oracle as so


# ------------------------------------------------------------------------------------------ rotary positions
@pytest.mark.parametrize("scaling", ["none", "linear", "base", "wavelength", "ramp"])
def test_frequencies_lie_between_the_stretched_and_the_plain_ones(scaling):
    f = so.rope_frequencies(64)
    assert f[0] == 1.0 and math.isclose(f[16], 10000.0 ** -0.5)
    w = so.rope_frequencies(64, scaling=scaling, factor=8.0)
    assert np.all(w <= f * (1 + 1e-15)) and np.all(w >= f / 8 * (1 - 1e-12)) and np.all(np.diff(w) < 0)
    assert np.allclose(so.rope_frequencies(64, scaling=scaling, factor=1.0), f, rtol=1e-14)
    if scaling in ("wavelength", "ramp"):        # fast pairs keep their speed, slow ones are stretched in full
        assert w[0] == f[0] and math.isclose(w[-1], f[-1] / 8)
    if scaling == "base":                        # the slowest pair is stretched in full
        assert math.isclose(w[-1], f[-1] / 8, rel_tol=1e-12)


@pytest.mark.parametrize("interleaved", [False, True])
def test_turns_depend_on_the_difference_of_positions_alone(interleaved):
    rng = np.random.default_rng(1)
    w = so.rope_frequencies(32)
    q, k = rng.standard_normal((1, 1, 48)), rng.standard_normal((1, 1, 48))
    dots = [float((so.rope(q, [a], w, interleaved) * so.rope(k, [b], w, interleaved)).sum()) for a, b in ((5, 2), (105, 102), (3, 0))]
    assert np.allclose(dots, dots[0])
    y = so.rope(q, [77], w, interleaved, amplitude=1.5)
    assert np.array_equal(y[..., 32:], q[..., 32:])
    assert np.allclose(so.rope(y, [77], w, interleaved, amplitude=1 / 1.5, inverse=True), q)
    assert math.isclose(np.linalg.norm(y[..., :32]), 1.5 * np.linalg.norm(q[..., :32]))


def test_pairs_by_hand():
    x = np.arange(1.0, 5.0).reshape(1, 1, 4)
    w = np.array([math.pi / 2, 0.0])
    assert np.allclose(so.rope(x, [1], w)[0, 0], [-3, 2, 1, 4])
    assert np.allclose(so.rope(x, [1], w, interleaved=True)[0, 0], [-2, 1, 3, 4])


def test_the_gradient_is_the_inverse_turn():
    rng = np.random.default_rng(2)
    w = so.rope_frequencies(16, scaling="linear", factor=3.0)
    x, g = rng.standard_normal((2, 3, 16)), rng.standard_normal((2, 3, 16))
    back = so.rope(g, [9, 4], w, amplitude=1.2, inverse=True)
    for n, h, j in itertools.product(range(2), range(3), range(16)):
        d = np.zeros_like(x)
        d[n, h, j] = 1e-6
        diff = ((so.rope(x + d, [9, 4], w, amplitude=1.2) - so.rope(x - d, [9, 4], w, amplitude=1.2)) * g).sum() / 2e-6
        assert abs(diff - back[n, h, j]) < 1e-7


# ------------------------------------------------------------------------------------------ trees, attention
def test_masks_are_the_ways_to_the_root():
    mask, depth = so.tree_mask([-1, 0, 0, 1, 3, 9, -1, 0], [0, 6, 8], 1)
    assert [bin(int(m))[2:] for m in mask[:, 0]] == ["1", "11", "101", "1011", "11011", "100000", "1", "11"]
    assert depth.tolist() == [0, 1, 1, 2, 3, 0, 0, 1]            # a parent that does not come earlier is none
    chain, _ = so.tree_mask(list(range(-1, 69)), [0, 70], 3)
    assert [int(m).bit_count() for m in chain[69]] == [32, 32, 6]


def attend(L, T, Hq=2, heads=1, D=4, page=3, mask=None, seed=0, pages=9):
    rng = np.random.default_rng(seed)
    table = rng.permutation(pages)[None].astype(np.int32)
    k, v, q = rng.standard_normal((pages, page, heads, D)), rng.standard_normal((pages, page, heads, D)), rng.standard_normal((T, Hq, D))
    return q, k, v, table, so.attention(q, k, v, table, [L], [0, T], mask, 0.5, T)


def test_attention_against_loops():
    L, T = 7, 4
    m = np.array([[0b1], [0b10], [0b0101], [0]])
    q, k, v, table, (out, lse, _) = attend(L, T, mask=m)
    for t, h in itertools.product(range(T), range(2)):
        seen = [i for i in range(L + T) if i < L or m[t, 0] >> (i - L) & 1]
        x = [0.5 * sum(q[t, h, d] * k[table[0, i // 3], i % 3, 0, d] for d in range(4)) for i in seen]
        total = sum(math.exp(e) for e in x)
        assert math.isclose(lse[t, h], math.log(total), rel_tol=1e-12)
        for d in range(4):
            assert math.isclose(out[t, h, d], sum(math.exp(e) * v[table[0, i // 3], i % 3, 0, d] for e, i in zip(x, seen)) / total, rel_tol=1e-10)


def test_attention_limits():
    *_, (out, lse, _) = attend(0, 2, mask=np.array([[0], [0b10]]))
    assert np.all(out[0] == 0) and np.all(lse[0] == -np.inf)     # nothing attended
    q, k, v, table, (out, lse, _) = attend(0, 1)
    assert np.allclose(out[0], v[table[0, 0], 0, 0])             # one position: its value
    chain = np.array([[0b1], [0b11], [0b111]])
    a, b = attend(5, 3, mask=chain)[-1], attend(5, 3)[-1]
    assert np.allclose(a[0], b[0]) and np.allclose(a[1], b[1])   # no mask: the chain
    q, k, v, table, (out, lse, _) = attend(6, 1)
    again = so.attention(q, k, v + 3.0, table, [6], [0, 1], None, 0.5, 1)
    assert np.allclose(again[0], out + 3.0)                      # weights add up to 1


# ------------------------------------------------------------------------------------------ verification
def chain_case(p, q, token):
    """One drafted token behind the root; d2t is the identity."""
    return dict(probs=np.array([p, p], dtype=np.float64), tokens=[0, token], parents=[-1, 0], cu=[0, 2], max_tokens=2)


def test_accepting_by_hand():
    p, q = [0.5, 0.3, 0.2], [0.1, 0.6, 0.3]
    case = chain_case(p, q, 1)
    draft = dict(draft_probs=np.array([q, q]), draft_ids=[0, 1])
    for u, n in ((0.49, 1), (0.51, 0)):                          # p / q = 0.5
        got = so.verify(**case, u_accept=[0, u], u_sample=[0.0], **draft)
        assert got[0][0] == n
    n, path, out = so.verify(**case, u_accept=[0, 0.9], u_sample=[0.99], **draft)
    assert n[0] == 0 and out[0].tolist() == [0, -1]              # max(p - q, 0) holds id 0 alone
    n, path, out = so.verify(**case, u_accept=[0, 0.1], u_sample=[0.6], **draft)
    assert path[0].tolist() == [1, -1] and out[0].tolist() == [1, 1]
    # picked without chance: accepted with probability p, and left out afterwards
    assert so.verify(**case, u_accept=[0, 0.29], u_sample=[0.0])[0][0] == 1
    n, _, out = so.verify(**case, u_accept=[0, 0.31], u_sample=[0.72])
    assert n[0] == 0 and out[0].tolist() == [2, -1]              # 0.5 and 0.2 remain: 0.72 * 0.7 > 0.5


def first_token_law(p, q, children, drawn):
    """The exact distribution of the token that follows the root, over all draws of children and all random numbers."""
    V = len(p)
    law = np.zeros(V)
    draws = itertools.product(range(V), repeat=children) if drawn else [tuple(np.argsort(-np.array(q))[:children])]
    for draw in draws:
        weight = math.prod(q[c] for c in draw) if drawn else 1.0
        # acceptance probabilities in turn, found by bisection on u; the token that follows from its distribution by bisection, too
        alive = 1.0
        base = dict(probs=np.array([p] * (children + 1)), tokens=[0, *draw], parents=[-1] + [0] * children, cu=[0, children + 1],
                    max_tokens=children + 1)
        if drawn:
            base |= dict(draft_probs=np.array([q] * (children + 1)), draft_ids=[0, *draw])
        for c in range(children):
            lo, hi = 0.0, 1.0
            for _ in range(45):
                u = (lo + hi) / 2
                ok = so.verify(u_accept=[0] + [2.0] * c + [u] + [2.0] * (children - c - 1), u_sample=[0.0], **base)[1][0, 0] == c + 1
                lo, hi = (u, hi) if ok else (lo, u)
            law[draw[c]] += weight * alive * lo
            alive *= 1 - lo
        edges = [0.0]
        for y in range(V):
            lo, hi = 0.0, 1.0
            for _ in range(45):
                u = (lo + hi) / 2
                got = so.verify(u_accept=[2.0] * (children + 1), u_sample=[u], **base)[2][0, 0]
                lo, hi = (u, hi) if got <= y else (lo, u)
            law[y] += weight * alive * (lo - edges[-1])
            edges.append(lo)
    return law


@pytest.mark.parametrize("drawn,children", [(True, 1), (True, 2), (False, 1), (False, 3)])
def test_the_outcome_is_distributed_as_the_target(drawn, children):
    p, q = [0.45, 0.3, 0.15, 0.1], [0.1, 0.2, 0.5, 0.2]
    assert np.allclose(first_token_law(p, q, children, drawn), p, atol=1e-9)


def test_trees_and_what_does_not_fit():
    rng = np.random.default_rng(5)
    P = rng.dirichlet(np.ones(6), size=8)
    tokens, parents = [0, 3, 4, 5, 1, 2, 9, 0], [-1, 0, 0, 1, 2, 7, 0, 1]
    n, path, out = so.verify(P, tokens, parents, [0, 8], [0.0] * 8, [0.0], 8)
    assert path[0, :2].tolist() == [1, 3] and n[0] == 2          # the first child each time
    u = [0.0, 1.0, 0, 0, 0, 0, 0, 0]
    assert so.verify(P, tokens, parents, [0, 8], u, [0.0], 8)[1][0, :2].tolist() == [2, 4]
    u = [0.0, 1.0, 1.0, 0, 0, 0, 0, 0]
    assert so.verify(P, tokens, parents, [0, 8], u, [0.0], 8)[0][0] == 0      # token 9 lies outside, 5's parent comes later
    n, path, out = so.verify(P, tokens, parents, [0, 0, 8], [0.0] * 8, [0.0, 0.0], 8)
    assert n.tolist() == [0, 2] and out[0].tolist() == [-1] * 8
