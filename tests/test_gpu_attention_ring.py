"""Attention where every CTA goes through several items, with few rows and heads of 128: five ring stages, two issuers (see test_attention_ring.py)."""
import numpy as np
import pytest
import torch

from .test_gpu_tree_attention import Case, vt  # noqa: F401

pytestmark = pytest.mark.gpu


def lengths(rng, B, most):
    """Ragged, odd and even numbers of tiles, some of a tile or two."""
    tiles = rng.integers(1, most // 128 + 1, B)
    tiles[::5] = rng.integers(1, 3, len(tiles[::5]))
    return np.maximum(tiles * 128 - rng.integers(0, 128, B), 0).tolist()


# one token a request, and chains and trees of up to eight; four query heads to a key head
@pytest.mark.parametrize("B,T,tree,page", [(64, 1, False, 64), (90, 1, False, 16), (40, 8, False, 32), (36, 8, True, 128)])
def test_many_items_a_cta(vt, B, T, tree, page):  # noqa: F811
    rng = np.random.default_rng(B)
    counts = [T] + rng.integers(1, T + 1, B - 1).tolist()
    c = Case(vt, lengths(rng, B, 1700 if T == 1 else 1000), counts, 32, 8, 128, page, tree=tree)
    ws = vt.new_workspace(vt.vt_tree_attention_workspace_bytes(32, 8, 128, T))
    out, lse = c.run(workspace=ws)
    c.check(out, lse)
    # the same bits, whatever else the memory is busy with
    busy, side = torch.empty(2, 1 << 26, device="cuda"), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    same = []
    for i in range(100):
        if i % 2:
            with torch.cuda.stream(side):
                busy[1].copy_(busy[0])
        again = c.run(workspace=ws)
        same += [(again[0] == out).all(), (again[1] == lse).all()]
    assert bool(torch.stack(same).all())
    assert vt.vt_last_status(ws) == vt.VT_OK


def test_long_items_behind_one_another(vt):  # noqa: F811
    # more tiles than the ring has places in most items: a stream can fall behind by a whole turn
    rng = np.random.default_rng(5)
    c = Case(vt, (128 * rng.integers(9, 24, 24) + rng.integers(1, 128, 24)).tolist(), [1] * 24, 16, 16, 128, 64)
    out, lse = c.run()
    c.check(out, lse)
    again = [c.run() for _ in range(50)]
    assert all(torch.equal(a, out) and torch.equal(b, lse) for a, b in again)


def test_a_wait_that_runs_out_with_two_issuers_and_a_short_ring(vt):  # noqa: F811
    # each copy is made to fall 16 bytes short of what is waited for (host side): every role leaves, and the next call is right
    c = Case(vt, [3000, 700] * 12, [1, 3] * 12, 16, 4, 128, 32)
    ws = vt.new_workspace(vt.vt_tree_attention_workspace_bytes(16, 4, 128, 3))
    want = c.run()
    try:
        vt.vt_test_withhold_copies(2000)
        c.run(workspace=ws)
        assert vt.vt_last_status(ws) == vt.VT_ERR_TIMEOUT
    finally:
        vt.vt_test_withhold_copies(0)
    got = c.run(workspace=ws)
    assert vt.vt_last_status(ws) == vt.VT_OK
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
