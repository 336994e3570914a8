"""More pins of the decode-step oracle: what planted mistakes showed the others not to notice."""
import math

import numpy as np

from oracle import vt_step_oracle as so


def test_ramp_by_hand():
    # 8192 / (2 pi 32) = 40.74 and 8192 / (2 pi) = 1303.8: pairs 12.88 and 24.92 of 64 / 2 make 32 turns and one
    f, w = so.rope_frequencies(64), so.rope_frequencies(64, scaling="ramp", factor=8.0)
    assert np.allclose(w[:13], f[:13], rtol=1e-14) and np.allclose(w[25:], f[25:] / 8, rtol=1e-14)
    for i in range(13, 25):
        assert math.isclose(w[i] / f[i], 1 - (i - 12) / 13 * 7 / 8, rel_tol=1e-12)
    # other ends: 4 turns (pair 20.1) to 8 (pair 17.7)
    w = so.rope_frequencies(64, scaling="ramp", factor=2.0, low=4.0, high=8.0)
    assert np.allclose(w[18:21] / f[18:21], [1 - 1 / 8, 1 - 2 / 8, 1 - 3 / 8], rtol=1e-12) and w[17] == f[17] and math.isclose(w[21], f[21] / 2)


def test_wavelength_by_hand():
    f, w = so.rope_frequencies(64), so.rope_frequencies(64, scaling="wavelength", factor=8.0)
    turns = 8192 * 10.0 ** (-4 * 21 / 32) / (2 * math.pi)        # 3.09: between one and four
    assert math.isclose(turns, 3.0918, rel_tol=1e-3) and w[20] == f[20]
    assert math.isclose(w[21] / f[21], (turns - 1) / 3 + (4 - turns) / 3 / 8, rel_tol=1e-12)


def test_groups_of_query_heads_lie_together():
    rng = np.random.default_rng(3)
    k, v, q = rng.standard_normal((2, 4, 2, 4)), rng.standard_normal((2, 4, 2, 4)), rng.standard_normal((1, 6, 4))
    out, lse, _ = so.attention(q, k, v, np.array([[1, 0]]), [5], [0, 1], None, 0.5, 1)
    for h in range(6):                                           # 0, 1, 2 on key head 0; 3, 4, 5 on 1
        one = so.attention(q[:, h:h + 1], k[:, :, h // 3:h // 3 + 1], v[:, :, h // 3:h // 3 + 1], np.array([[1, 0]]), [5], [0, 1], None, 0.5, 1)
        assert np.allclose(out[:, h], one[0][:, 0]) and np.allclose(lse[:, h], one[1][:, 0])


def test_the_draft_map():
    # the draft's ids 0, 1, 2 are the target's 3, 0, 2; draft 1 (target 0) is turned down
    p, q, d2t = [0.1, 0.4, 0.2, 0.3], [0.5, 0.3, 0.2], [3, 0, 2]
    case = dict(probs=np.array([p, p]), tokens=[0, 0], parents=[-1, 0], cu=[0, 2], max_tokens=2, draft_probs=np.array([q, q]), draft_ids=[0, 1], d2t=d2t)
    assert so.verify(u_accept=[0, 0.33], u_sample=[0.0], **case)[0][0] == 1              # 0.1 / 0.3
    for u, y in ((0.0, 1), (0.99, 1)):                           # max(p - q, 0) = 0, 0.4, 0, 0
        assert so.verify(u_accept=[0, 0.34], u_sample=[u], **case)[2][0].tolist() == [y, -1]


def test_children_come_after_their_parents():
    P = np.full((4, 3), 1 / 3)
    # token 1 names the later token 3, token 2 names itself: neither is anybody's child
    n, path, _ = so.verify(P, [0, 1, 1, 2], [-1, 3, 2, 0], [0, 4], [0.0] * 4, [0.0], 4)
    assert n[0] == 1 and path[0].tolist() == [3, -1, -1, -1]


def test_draft_indices_outside_the_draft():
    P, q = np.full((3, 2), 0.5), np.full((3, 2), 0.5)
    for bad in (-1, 2):
        got = so.verify(P, [0, 1, 1], [-1, 0, 0], [0, 3], [0.0] * 3, [0.0], 3, draft_probs=q, draft_ids=[0, bad, 1])
        assert got[1][0].tolist() == [2, -1, -1]
