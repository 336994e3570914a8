"""vt_score_tokens and vt_score_tokens_backward against the fp64 oracle.

Inputs.  Hidden states and weights lie on binary grids (h on 1/16, W on 1/1024, 8 significant bits at most), on which every
fp32 sum of products is exact in any order: ids, and ties among equal logits, must then be the oracle's exactly.

Tolerances, derived.  The logits are exact, so what is left is the softmax in fp32.
  B_z   the exponents' arguments: (x - max) * scale * log2(e) is rounded twice, relative 2^-23 of a magnitude that matters up
        to ~25 (beyond it p < 2^-36): 25 * 2^-23 * ln 2 ~ 2e-6; ex2.approx adds 2^-22.  As every p has its own error of either
        sign, 2e-6 bounds log s with room; the sums add a few 2^-24.
  lse, logprob, top logprob   |error| <= 4e-6 + 2^-22 |value|        (one more rounding of scale * max, one of the difference)
  entropy                     log s - E[z - max] / s: |error| <= 4e-6 + 2^-21 (1 + ln V), the same relative errors on E
  G     p = exp(scale x - lse): |scale x - lse| <= ~30 rounded at 2^-24 * 64, plus lse's error: relative 1e-5 < 2^-16; rounded
        once to bf16 (2^-8 at most); so  |dh - exact| <= 2^-8 |dh| + (2^-8 + 2^-14) sum_v A |W|, A the magnitudes of G's terms,
        and the same for dW with |h|; the fp32 sums' own errors are far below the slack of 2^-14."""
import numpy as np
import pytest
import torch

from oracle import vt_score_oracle as so
from tests.gpu_util import Guarded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vt():
    import paper_2603_05210_b200 as vt
    vt.lib()
    assert torch.cuda.is_available()
    return vt


def grid(rng, shape, rms, step):
    return np.clip(np.round(rng.normal(size=shape) * rms / step), -255, 255) * step


def case(M, d, V, seed, lean=8.0):
    rng = np.random.default_rng(seed)
    W = grid(rng, (V, d), 0.02 if d >= 256 else 0.1, 1 / 1024)
    tokens = rng.integers(0, V, M)
    norm = np.maximum(np.linalg.norm(W[tokens], axis=1, keepdims=True), 1e-6)
    h = np.clip(np.round((rng.normal(size=(M, d)) + rng.uniform(0, lean, (M, 1)) * W[tokens] / norm) * 16), -255, 255) / 16
    tokens = np.where(rng.random(M) < 0.6, tokens, rng.integers(0, V, M)).astype(np.int32)
    return h, W, tokens


def dev(a, dtype=torch.bfloat16):
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch.float64).to(dtype).cuda() if dtype.is_floating_point \
        else torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def run(vt, h, W, tokens, k, scale=1.0, ws=None):
    M, V = h.shape[0], W.shape[0]
    outs = {"entropy": Guarded((M,), torch.float32), "lse": Guarded((M,), torch.float32)}
    if tokens is not None:
        outs["logprobs"] = Guarded((M,), torch.float32)
    if k:
        outs |= {"top_ids": Guarded((M, k), torch.int32), "top_logprobs": Guarded((M, k), torch.float32)}
    if ws is None:      # whatever an allocator hands out must do
        ws = torch.full((vt.vt_score_workspace_bytes(M, h.shape[1], V, k),), 0xFF, dtype=torch.uint8, device="cuda")
        ws[:512] = 0
    vt.vt_score_tokens(h, W, tokens, k=k, scale=scale, workspace=ws, **{n: g.t for n, g in outs.items()})
    assert vt.vt_last_status(ws) == vt.VT_OK
    assert all(g.intact() for g in outs.values()), "write outside an output"
    return {n: g.t.cpu().numpy() for n, g in outs.items()}


def check(got, want, V):
    for n in ("lse", "logprobs", "top_logprobs"):
        if n in got:
            err = np.abs(got[n] - want[n])
            assert (err <= 4e-6 + 2.0 ** -22 * np.abs(want[n])).all(), (n, err.max())
    assert (np.abs(got["entropy"] - want["entropy"]) <= 4e-6 + 2.0 ** -21 * (1 + np.log(V))).all()
    if "top_ids" in got:
        assert np.array_equal(got["top_ids"], want["top_ids"])


SHAPES = [(1, 8, 1, 1), (1, 8, 2, 2), (2, 24, 7, 7), (1, 64, 100, 64), (8, 136, 255, 20), (31, 64, 256, 8), (32, 512, 257, 1), (33, 200, 1000, 3),
          (64, 256, 2001, 20), (65, 64, 4099, 8), (127, 1024, 999, 4), (128, 72, 5000, 0), (129, 512, 777, 64), (255, 264, 3001, 8),
          (256, 64, 1500, 20), (257, 520, 513, 5), (600, 128, 2048, 0), (3, 5120, 1111, 8)]


@pytest.mark.parametrize("M,d,V,k", SHAPES)
def test_scores(vt, M, d, V, k):
    h, W, tokens = case(M, d, V, M + d + V)
    scale = [1.0, 0.6, 1.7][(M + V) % 3]
    if M > 2:
        tokens[::3] = np.resize([-1, V, 2 ** 31 - 1, -2 ** 31], len(tokens[::3]))
    want = so.score(h, W, tokens, k, scale)
    got = run(vt, dev(h), dev(W), dev(tokens, torch.int32), k, scale)
    check(got, want, V)
    again = run(vt, dev(h), dev(W), dev(tokens, torch.int32), k, scale)
    assert all(np.array_equal(got[n], again[n]) for n in got), "not the same bits twice"


@pytest.mark.parametrize("M,d,V,k", [(1, 64, 500, 3), (40, 64, 900, 8), (200, 128, 1000, 8)])
def test_without_given_tokens_every_row_is_scored(vt, M, d, V, k):
    h, W, _ = case(M, d, V, 5)
    check(run(vt, dev(h), dev(W), None, k), so.score(h, W, None, k), V)
    r = vt.vt_score_tokens(dev(h), dev(W), None, k=k)
    assert r.logprobs is None and r.top_ids.shape == (M, k)


# lists (72 MB of logits would be more than are kept) and kept logits, both with more ties than a join's buffer holds
@pytest.mark.parametrize("M,V,k", [(2, 5000, 20), (40, 30000, 8), (600, 30011, 20), (600, 30011, 64)])
def test_rows_of_equal_logits(vt, M, V, k):
    d = 64
    h, W, tokens = case(M, d, V, 6)
    h[::2] = 0.0                                # every token the same: ids 0 .. k-1, entropy ln V
    W[1::2] = W[: len(W[1::2])]                 # and pairs of equal rows elsewhere
    want = so.score(h, W, tokens, k)
    assert (want["top_ids"][0] == np.arange(k)).all()
    check(run(vt, dev(h), dev(W), dev(tokens, torch.int32), k), want, V)


def test_winners_in_one_place(vt):
    """All of a row's best tokens in one tile's range, in ascending and descending order, kept and listed."""
    for M, V, k in ((3, 6000, 64), (600, 30011, 20)):
        d = 64
        W = np.zeros((V, d))
        W[:, 0] = -0.25
        W[1000:1200, 0] = np.arange(200) / 1024
        W[2000:2200, 1] = np.arange(200)[::-1] / 1024
        h = np.zeros((M, d))
        h[::2, 0] = 1.0
        h[1::2, 1] = 1.0
        tokens = np.full(M, 1001, np.int32)
        check(run(vt, dev(h), dev(W), dev(tokens, torch.int32), k), so.score(h, W, tokens, k), V)


def test_near_certain_rows_keep_a_small_entropy(vt):
    """One token far ahead: H ~ 1e-4, where lse and E[z] are both ~50."""
    d, V = 64, 3000
    rng = np.random.default_rng(8)
    W = grid(rng, (V, d), 0.01, 1 / 1024)
    W[77] = 0.1875
    h = np.full((4, d), 1.0) * np.array([[4.0], [1.25], [1.0], [2.0]])
    tokens = np.array([77, 77, 5, 77], np.int32)
    want = so.score(h, W, tokens, 4)
    got = run(vt, dev(h), dev(W), dev(tokens, torch.int32), 4)
    check(got, want, V)
    small = want["entropy"] < 0.1
    assert small.any() and (np.abs(got["entropy"] - want["entropy"])[small] <= 1e-6 + 1e-4 * want["entropy"][small]).all()


def test_what_unscored_rows_hold_reaches_nothing(vt):
    M, d, V, k = 70, 64, 800, 4
    h, W, tokens = case(M, d, V, 9)
    tokens[10:20] = -1
    clean = run(vt, dev(h), dev(W), dev(tokens, torch.int32), k)
    bad = dev(h)
    bad[10] = float("nan")
    bad[11] = float("inf")
    bad[12] = -float("inf")
    bad[13] = torch.finfo(torch.bfloat16).min
    got = run(vt, bad, dev(W), dev(tokens, torch.int32), k)
    assert all(np.array_equal(clean[n], got[n]) for n in clean)
    assert (got["top_ids"][10:20] == -1).all() and (got["entropy"][10:20] == 0).all()
    gl, ge = torch.randn(M, device="cuda"), torch.randn(M, device="cuda")
    t = dev(tokens, torch.int32)
    lse, H = (torch.from_numpy(clean[n]).cuda() for n in ("lse", "entropy"))
    lse[10:20] = float("nan")                   # nor do their statistics and gradients
    gl[10:20] = float("inf")
    one = vt.vt_score_tokens_backward(dev(h), dev(W), t, lse, H, gl, ge)
    two = vt.vt_score_tokens_backward(bad, dev(W), t, lse, H, gl, ge)
    assert torch.isfinite(two[1].float()).all() and torch.equal(one[1], two[1]) and torch.equal(one[0], two[0])
    assert (two[0][10:20] == 0).all()


def test_a_nan_stays_in_its_row(vt):
    M, d, V, k = 300, 64, 800, 4
    h, W, tokens = case(M, d, V, 10)
    clean = run(vt, dev(h), dev(W), dev(tokens, torch.int32), k)
    bad = dev(h)
    bad[7, 3] = float("nan")
    got = run(vt, bad, dev(W), dev(tokens, torch.int32), k)
    assert np.isnan(got["lse"][7]) and np.isnan(got["logprobs"][7])
    rest = np.arange(M) != 7
    assert all(np.array_equal(clean[n][rest], got[n][rest]) for n in clean)


def test_all_rows_unscored(vt):
    M, d, V = 5, 64, 100
    h, W, _ = case(M, d, V, 11)
    t = torch.full((M,), -1, dtype=torch.int32, device="cuda")
    r = vt.vt_score_tokens(dev(h), dev(W), t, k=3)
    assert (r.logprobs == 0).all() and (r.top_ids == -1).all()
    dh, dW = vt.vt_score_tokens_backward(dev(h), dev(W), t, r.lse, r.entropy, torch.ones(M, device="cuda"))
    assert (dh == 0).all() and (dW == 0).all()


def wide(t, extra=24, fill=float("nan")):
    """The same rows inside a wider buffer."""
    b = torch.full((t.shape[0], t.shape[1] + extra), fill, dtype=t.dtype, device=t.device)
    b[:, 8:8 + t.shape[1]] = t
    return b[:, 8:8 + t.shape[1]]


@pytest.mark.parametrize("M", [1, 50, 300])
def test_rows_apart(vt, M):
    d, V, k = 136, 700, 5
    h, W, tokens = case(M, d, V, 12)
    hd, Wd, t = dev(h), dev(W), dev(tokens, torch.int32)
    a, b = vt.vt_score_tokens(hd, Wd, t, k=k), vt.vt_score_tokens(wide(hd), Wd, t, k=k)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    g = torch.randn(M, device="cuda")
    one, two = (vt.vt_score_tokens_backward(x, Wd, t, a.lse, a.entropy, g, g) for x in (hd, wide(hd)))
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])


GRADS = [(1, 8, 1), (1, 64, 100), (2, 24, 7), (16, 520, 999), (63, 64, 257), (100, 256, 3001), (128, 136, 1000), (129, 72, 513), (300, 264, 2050),
         (513, 64, 300)]


@pytest.mark.parametrize("M,d,V", GRADS)
@pytest.mark.parametrize("with_entropy", [False, True])
def test_gradients(vt, M, d, V, with_entropy):
    rng = np.random.default_rng(13)
    h, W, tokens = case(M, d, V, M * d)
    if M > 2:
        tokens[::4] = -1
    scale = 0.8
    gl = rng.normal(size=M).astype(np.float32)
    ge = rng.normal(size=M).astype(np.float32) if with_entropy else None
    hd, Wd, t = dev(h), dev(W), dev(tokens, torch.int32)
    r = vt.vt_score_tokens(hd, Wd, t, scale=scale)
    gh, gW = Guarded((M, d), torch.bfloat16), Guarded((V, d), torch.bfloat16)
    ws = torch.full((vt.vt_score_backward_workspace_bytes(M, d, V),), 0xFF, dtype=torch.uint8, device="cuda")
    ws[:512] = 0
    vt.vt_score_tokens_backward(hd, Wd, t, r.lse, r.entropy if with_entropy else None, torch.from_numpy(gl).cuda(),
                                None if ge is None else torch.from_numpy(ge).cuda(), scale=scale, workspace=ws, grad_h=gh.t, grad_W=gW.t)
    assert vt.vt_last_status(ws) == vt.VT_OK and gh.intact() and gW.intact()
    want_h, want_W = so.score_backward(h, W, tokens, gl, ge, scale)
    _, A = so.grad_logits(h, W, tokens, gl, ge, scale)
    keep = so.scored_rows(tokens, M, V)
    slack = 2.0 ** -8 + 2.0 ** -14
    for got, want, terms in ((gh.t, want_h, A @ np.abs(W)), (gW.t, want_W, A[keep].T @ np.abs(h[keep]))):
        err = np.abs(got.double().cpu().numpy() - want)
        assert (err <= 2.0 ** -8 * np.abs(want) + slack * terms + 1e-30).all()
        if want.size > 2000:                    # and on the whole far nearer than the bound: two roundings of bf16
            assert np.linalg.norm(err) <= 2.0 ** -8 * np.linalg.norm(want)
    for want_h_too, want_W_too in ((True, False), (False, True)):
        one = vt.vt_score_tokens_backward(hd, Wd, t, r.lse, r.entropy, torch.from_numpy(gl).cuda(), None if ge is None else torch.from_numpy(ge).cuda(),
                                          scale=scale, want_h=want_h_too, want_W=want_W_too)
        assert (one[0] is None) != want_h_too and (one[1] is None) != want_W_too
        assert torch.equal(one[0], gh.t) if want_h_too else torch.equal(one[1], gW.t)


@pytest.mark.parametrize("M,d,V", [(1, 8, 5), (2, 2056, 300), (40, 4104, 100), (300, 264, 5000), (700, 72, 259)])
@pytest.mark.parametrize("shared", [1, 3, 1000])
def test_given_entries_are_rounded_once(vt, M, d, V, shared):
    """Up to `shared` rows have the same token.  A given token's entry of G enters dh and dW unrounded: of it only the 2^-14 that stand for
    its own fp32 errors (2^-16) and the sums' are left, beside the other entries' rounding and the result's."""
    h, W, _ = case(M, d, V, 5 * M + d)
    rng = np.random.default_rng(M + shared)
    tokens = np.resize(np.repeat(rng.permutation(V)[:max(1, M // shared)], min(shared, M)), M).astype(np.int32)
    tokens[0] = V - 1
    if M > 2:
        tokens[rng.permutation(M)[: M // 5]] = -1
    gl = rng.normal(size=M).astype(np.float32)
    hd, Wd, t = dev(h), dev(W), dev(tokens, torch.int32)
    r = vt.vt_score_tokens(hd, Wd, t)
    gh, gW = Guarded((M, d), torch.bfloat16), Guarded((V, d), torch.bfloat16)
    ws = torch.full((vt.vt_score_backward_workspace_bytes(M, d, V),), 0xFF, dtype=torch.uint8, device="cuda")
    ws[:512] = 0
    vt.vt_score_tokens_backward(hd, Wd, t, r.lse, None, torch.from_numpy(gl).cuda(), None, workspace=ws, grad_h=gh.t, grad_W=gW.t)
    assert vt.vt_last_status(ws) == vt.VT_OK and gh.intact() and gW.intact()
    want_h, want_W = so.score_backward(h, W, tokens, gl)
    _, A = so.grad_logits(h, W, tokens, gl)
    keep = so.scored_rows(tokens, M, V)
    others, given = A.copy(), np.zeros_like(A)
    m = np.flatnonzero(keep)
    given[m, tokens[m]], others[m, tokens[m]] = A[m, tokens[m]], 0.0
    E = (2.0 ** -8 + 2.0 ** -14) * others + 2.0 ** -14 * given
    for got, want, terms in ((gh.t, want_h, E @ np.abs(W)), (gW.t, want_W, E[keep].T @ np.abs(h[keep]))):
        err = np.abs(got.double().cpu().numpy() - want)
        assert (err <= 2.0 ** -8 * np.abs(want) + terms + 1e-30).all()


def test_gradients_against_differences(vt):
    """The GPU's gradients along random directions against central differences of the oracle's loss.  The gradients' relative
    error is 2^-8 per element at most and averages out along a direction; the differences' is eps^2: 1 % of the norms' product
    over sqrt(size) bounds both."""
    M, d, V, scale = 20, 64, 150, 1.1
    rng = np.random.default_rng(14)
    h, W, tokens = case(M, d, V, 15)
    tokens[3] = -1
    gl, ge = rng.normal(size=M).astype(np.float32), rng.normal(size=M).astype(np.float32)

    def loss(h, W):
        r = so.score(h, W, tokens, scale=scale)
        return float(gl.astype(np.float64) @ r["logprobs"] + ge.astype(np.float64) @ r["entropy"])

    t = dev(tokens, torch.int32)
    r = vt.vt_score_tokens(dev(h), dev(W), t, scale=scale)
    gh, gW = (x.double().cpu().numpy() for x in vt.vt_score_tokens_backward(dev(h), dev(W), t, r.lse, r.entropy, torch.from_numpy(gl).cuda(),
                                                                            torch.from_numpy(ge).cuda(), scale=scale))
    eps = 1e-4
    for _ in range(5):
        v, w = rng.normal(size=h.shape), rng.normal(size=W.shape)
        for got, dh, dW, g in ((gh, v, 0 * w, gh), (gW, 0 * v, w, gW)):
            step = v if dh.any() else w
            diff = (loss(h + eps * dh, W + eps * dW) - loss(h - eps * dh, W - eps * dW)) / (2 * eps)
            assert abs(diff - (got * step).sum()) <= 0.01 * np.linalg.norm(g) * np.linalg.norm(step) / np.sqrt(g.size) + 1e-6


def test_on_another_stream_and_behind_a_late_producer(vt):
    M, d, V, k = 40, 256, 3000, 4
    h, W, tokens = case(M, d, V, 16)
    h2, W2, _ = case(M, d, V, 17)
    hd, Wd, t = dev(h), dev(W), dev(tokens, torch.int32)
    want = vt.vt_score_tokens(dev(h2), dev(W2), t, k=k)
    g = torch.randn(M, device="cuda")
    want_grads = vt.vt_score_tokens_backward(dev(h2), dev(W2), t, want.lse, want.entropy, g, g)
    src_h, src_W = dev(h2), dev(W2)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        vt.vt_test_late_copy(Wd, src_W, 300)
        vt.vt_test_late_copy(hd, src_h, 300)
        got = vt.vt_score_tokens(hd, Wd, t, k=k)
        grads = vt.vt_score_tokens_backward(hd, Wd, t, got.lse, got.entropy, g, g)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert all(torch.equal(a, b) for a, b in zip(want_grads, grads))


def test_back_to_back_calls_share_a_workspace_and_a_graph(vt):
    M, d, V, k = 12, 512, 2500, 6
    a, b = case(M, d, V, 18), case(M, d, V, 19)
    ins = [(dev(h), dev(W), dev(t, torch.int32)) for h, W, t in (a, b)]
    ws = vt.new_workspace(vt.vt_score_workspace_bytes(M, d, V, k))
    want = [vt.vt_score_tokens(*i, k=k) for i in ins]
    outs = [vt.vt_score_tokens(*ins[i % 2], k=k, workspace=ws) for i in range(6)]
    assert all(torch.equal(x, y) for i, o in enumerate(outs) for x, y in zip(o, want[i % 2]))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [vt.vt_score_tokens(*i, k=k, workspace=ws) for i in ins]
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for o, w in zip(got, want) for x, y in zip(o, w))


def test_offsets_past_32_bits(vt):
    """A head of 2.2e9 elements: ids, log probabilities and gradients at its far end."""
    M, d, V, k = 3, 8192, 270000, 3
    W = torch.zeros((V, d), dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, 131071, 262143, 262144, V - 1], device="cuda")
    W[rows, 0] = torch.tensor([1.0, 2.0, 3.0, 5.0, 4.0], device="cuda").bfloat16()
    h = torch.zeros((M, d), dtype=torch.bfloat16, device="cuda")
    h[:, 0] = torch.tensor([1.0, 2.0, -1.0], device="cuda").bfloat16()
    tokens = torch.tensor([V - 1, 262144, 5], dtype=torch.int32, device="cuda")
    r = vt.vt_score_tokens(h, W, tokens, k=k)
    x = (W[:, 0].double()[None] * h[:, 0].double()[:, None])
    logp = torch.log_softmax(x, 1)
    assert r.top_ids[:2].tolist() == [[262144, V - 1, 262143]] * 2 and r.top_ids[2].tolist() == [1, 2, 3]
    assert (r.logprobs.double() - logp.gather(1, tokens.long()[:, None])[:, 0]).abs().max() < 2e-5
    g = torch.ones(M, device="cuda")
    gh, gW = vt.vt_score_tokens_backward(h, W, tokens, r.lse, r.entropy, g)
    G = -logp.exp()
    G[torch.arange(M), tokens.long()] += 1
    want = (G.T @ h[:, 0].double())
    err = (gW[:, 0].double() - want).abs()
    assert (err <= 2.0 ** -7 * (G.abs().T @ h[:, 0].double().abs()) + 1e-12).all()
    assert (gW[:, 1:] == 0).all()
    assert (gh[:, 0].double() - G @ W[:, 0].double()).abs().max() < 2.0 ** -7 * float((G.abs() @ W[:, 0].double().abs()).max())


def test_more_rows_than_32_bit_thread_indices(vt):
    """2^24 + 5 rows: one thread per row and 256 per block pass 2^31 and 2^32.  A handful of rows are scored, the first, the last and
    those around 2^23 and 2^24; nothing of the others may appear anywhere.  Tolerances as above: h and W lie on binary grids, G
    is one rounding (the given entries none) from its value, the result one more."""
    M, d, V = 2 ** 24 + 5, 8, 9
    at = torch.tensor([0, 1, 2 ** 23 - 1, 2 ** 23, 2 ** 23 + 1, 2 ** 24 - 1, 2 ** 24, M - 1], device="cuda")
    given = torch.tensor([3, 8, 3, 0, 5, 3, 8, 7], dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(20)
    h = torch.full((M, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    h[at] = (torch.randint(-32, 33, (len(at), d), device="cuda", generator=gen) / 16).bfloat16()
    W = (torch.randint(-255, 256, (V, d), device="cuda", generator=gen) / 256).bfloat16()
    tokens = torch.full((M,), -1, dtype=torch.int32, device="cuda")
    tokens[at] = given
    r = vt.vt_score_tokens(h, W, tokens)
    rows, w = h[at].double(), W.double()
    logp = torch.log_softmax(rows @ w.T, 1)
    want = logp.gather(1, given.long()[:, None])[:, 0]
    assert ((r.logprobs[at].double() - want).abs() <= 4e-6 + 2.0 ** -22 * want.abs()).all()
    assert int((r.lse != 0).sum()) == len(at) and int((r.logprobs != 0).sum()) == len(at)
    gl = torch.ones(M, device="cuda")
    ws = vt.new_workspace(vt.vt_score_backward_workspace_bytes(M, d, V))
    dh, dW = vt.vt_score_tokens_backward(h, W, tokens, r.lse, None, gl, workspace=ws)
    assert vt.vt_last_status(ws) == vt.VT_OK
    p = logp.exp()
    G = -p
    G[torch.arange(len(at)), given.long()] += 1
    A = p.clone()
    A[torch.arange(len(at)), given.long()] += 1
    slack = 2.0 ** -8 + 2.0 ** -14
    for got, exact, terms in ((dh[at], G @ w, A @ w.abs()), (dW, G.T @ rows, A.T @ rows.abs())):
        assert ((got.double() - exact).abs() <= 2.0 ** -8 * exact.abs() + slack * terms).all()
    dh[at] = 0
    assert not dh.any()


@pytest.mark.parametrize("M,d,V", [(4096, 512, 300), (1000, 64, 45), (600, 1024, 130)])
def test_weight_gradients_from_divided_sums(vt, M, d, V):
    """Many rows and a small vocabulary: the sums of dW (and their fp32 copies for given tokens) are divided among a cluster's CTAs, whose
    tiles end inside a warp's rows.  Tolerances as in test_gradients."""
    rng = np.random.default_rng(21)
    h, W, tokens = case(M, d, V, M + V)
    tokens[::5] = -1
    gl, ge = rng.normal(size=M).astype(np.float32), rng.normal(size=M).astype(np.float32)
    hd, Wd, t = dev(h), dev(W), dev(tokens, torch.int32)
    r = vt.vt_score_tokens(hd, Wd, t)
    grads = [vt.vt_score_tokens_backward(hd, Wd, t, r.lse, r.entropy, torch.from_numpy(gl).cuda(), torch.from_numpy(ge).cuda()) for _ in range(2)]
    assert torch.equal(grads[0][0], grads[1][0]) and torch.equal(grads[0][1], grads[1][1])
    want_h, want_W = so.score_backward(h, W, tokens, gl, ge)
    _, A = so.grad_logits(h, W, tokens, gl, ge)
    keep = so.scored_rows(tokens, M, V)
    slack = 2.0 ** -8 + 2.0 ** -14
    for got, want, terms in zip(grads[0], (want_h, want_W), (A @ np.abs(W), A[keep].T @ np.abs(h[keep]))):
        err = np.abs(got.double().cpu().numpy() - want)
        assert (err <= 2.0 ** -8 * np.abs(want) + slack * terms + 1e-30).all()


@pytest.mark.parametrize("M", [3, 200])
@pytest.mark.parametrize("k", [0, 4, 20, 30])
@pytest.mark.parametrize("scale", [1e-44, 1e-38, 1e-37, 1e-30, 1e30, 2.5e38])
def test_any_finite_scale(vt, M, k, scale):
    """Scales that flatten every difference (columns past the vocabulary must still weigh nothing) and ones that leave one token alone."""
    V, d = 1003, 64
    h, W, tokens = case(M, d, V, 22)
    h, W = h / 16, W / 16                        # exact in bf16: |scale x| stays below the largest float
    scale = float(np.float32(scale))
    want = so.score(h, W, tokens, k, scale)
    assert np.abs(want["lse"]).max() < 3e38
    check(run(vt, dev(h), dev(W), dev(tokens, torch.int32), k, scale), want, V)


@pytest.mark.parametrize("M", [3, 200])
@pytest.mark.parametrize("k", [0, 4, 20, 30])
def test_logits_near_the_lowest_float(vt, M, k):
    """Every logit between -1.1e38 and -2.6e38, scaled to differences of a few units."""
    V, d = 90, 8
    h, W = np.zeros((M, d)), np.zeros((V, d))
    h[:, 0] = 1.0
    W[:, 0] = -(1.28125 + np.random.default_rng(23).permutation(V) / 64.0) * 2.0 ** 126
    tokens = (np.arange(M) % V).astype(np.int32)
    scale = 2.0 ** -126
    check(run(vt, dev(h), dev(W), dev(tokens, torch.int32), k, scale), so.score(h, W, tokens, k, scale), V)


@pytest.mark.parametrize("M,d,V", [(2500, 520, 300), (5000, 64, 40), (40, 72, 9)])
def test_tokens_given_to_many_rows(vt, M, d, V):
    """A quarter of the rows have one token, two others 33 and 32 (around where a token's rows begin to share it), the rest any; rows that
    are not scored between them.  Bounds as in test_given_entries_are_rounded_once, and the same bits twice."""
    h, W, _ = case(M, d, V, 24)
    rng = np.random.default_rng(25)
    tokens = rng.integers(3, V, M)
    places = rng.permutation(M)
    tokens[places[: M // 4]] = 0
    tokens[places[M // 4: M // 4 + min(33, M // 4)]] = 1
    tokens[places[M // 2: M // 2 + min(32, M // 4)]] = 2
    tokens[places[M - M // 10:]] = -1
    tokens = tokens.astype(np.int32)
    gl = rng.normal(size=M).astype(np.float32)
    hd, Wd, t = dev(h), dev(W), dev(tokens, torch.int32)
    r = vt.vt_score_tokens(hd, Wd, t)
    (dh, dW), again = (vt.vt_score_tokens_backward(hd, Wd, t, r.lse, None, torch.from_numpy(gl).cuda()) for _ in range(2))
    assert torch.equal(dh, again[0]) and torch.equal(dW, again[1])
    want_h, want_W = so.score_backward(h, W, tokens, gl)
    _, A = so.grad_logits(h, W, tokens, gl)
    keep = so.scored_rows(tokens, M, V)
    others, given = A.copy(), np.zeros_like(A)
    m = np.flatnonzero(keep)
    given[m, tokens[m]], others[m, tokens[m]] = A[m, tokens[m]], 0.0
    E = (2.0 ** -8 + 2.0 ** -14) * others + 2.0 ** -14 * given
    for got, want, terms in ((dh, want_h, E @ np.abs(W)), (dW, want_W, E[keep].T @ np.abs(h[keep]))):
        err = np.abs(got.double().cpu().numpy() - want)
        assert (err <= 2.0 ** -8 * np.abs(want) + terms + 1e-30).all()


def test_repeated_tokens_do_not_hold_a_gradient_up(vt):
    """All rows on one token against tokens all over the vocabulary: the same products, so at most half as much again, where a token's
    rows added one after the other took three times as long."""
    M, d, V = 8192, 512, 8000
    gen = torch.Generator(device="cuda").manual_seed(26)
    h = torch.randn(M, d, device="cuda", generator=gen).bfloat16()
    W = (torch.randn(V, d, device="cuda", generator=gen) * 0.02).bfloat16()
    ws = vt.new_workspace(max(vt.vt_score_workspace_bytes(M, d, V, 0), vt.vt_score_backward_workspace_bytes(M, d, V)))
    times = {}
    for name, t in (("any", torch.randint(V, (M,), device="cuda", generator=gen).int()), ("one", torch.full((M,), 77, dtype=torch.int32, device="cuda"))):
        r = vt.vt_score_tokens(h, W, t, workspace=ws)
        runs = []
        for _ in range(7):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(5):
                vt.vt_score_tokens_backward(h, W, t, r.lse, None, r.lse, workspace=ws)
            b.record()
            torch.cuda.synchronize()
            runs.append(a.elapsed_time(b))
        times[name] = min(runs)
    assert times["one"] <= 1.5 * times["any"], times
