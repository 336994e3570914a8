"""Verification of drafted tokens against the fp64 oracle: whole numbers, equal or not."""
import numpy as np
import pytest
import torch

from oracle import vt_step_oracle as so

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vt():
    import paper_2603_05210_b200 as vt
    vt.lib()
    assert torch.cuda.is_available()
    return vt


def make(counts, V, Vd, tree, seed, ld=None, ldq=None, like=0.5, identity=False):
    """probs, tokens, ... on the host; the draft's distribution resembles the target's more or less."""
    rng = np.random.default_rng(seed)
    N = int(sum(counts))
    cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)
    z = rng.normal(size=(N, V)) * 2
    peaks = rng.integers(0, V, (N, 3))
    z[np.arange(N)[:, None], peaks] += rng.uniform(4, 9, (N, 3))
    P = np.exp(z - z.max(1, keepdims=True))
    P = (P / P.sum(1, keepdims=True)).astype(np.float32)
    within = np.concatenate([np.arange(c) for c in counts]) if N else np.zeros(0, int)
    parents = np.maximum(within - (rng.integers(1, 5, N) if tree else 1), 0)
    parents[within == 0] = -1
    up = np.repeat(cu[:-1], counts) + np.maximum(parents, 0)
    a = dict(P=P, parents=parents, cu=cu, u_accept=rng.random(N).astype(np.float32), u_sample=rng.random(len(counts)).astype(np.float32))
    if Vd:
        d2t = np.arange(Vd) if identity else rng.permutation(V)[:Vd]
        zq = z[:, d2t] + like * rng.normal(size=(N, Vd))
        Q = np.exp(zq - zq.max(1, keepdims=True))
        Q = (Q / Q.sum(1, keepdims=True)).astype(np.float32)
        ids = np.array([rng.choice(Vd, p=Q[u].astype(np.float64) / Q[u].astype(np.float64).sum()) for u in up], dtype=np.int64)
        a |= dict(Q=Q, draft_ids=ids, d2t=None if identity else d2t, tokens=d2t[ids])
    else:
        best = np.argsort(-(z + like * rng.normal(size=z.shape)), axis=1)
        rank = np.array([np.sum(up[:n] == up[n]) - (1 if parents[n] >= 0 and (up[:n] == up[n]).any() and parents[n] == 0 else 0) for n in range(N)]) if N else np.zeros(0, int)
        a |= dict(tokens=best[up, np.clip(rank, 0, V - 1)] if N else np.zeros(0, int))
    return a


def dev(x, dtype=torch.int32):
    return None if x is None else torch.tensor(np.asarray(x), dtype=dtype, device="cuda")


def run(vt, a, max_tokens, pad=0):
    P = dev(a["P"], torch.float32)
    if pad:
        P = torch.cat([P, torch.full((P.shape[0], pad), 9.0, device="cuda")], 1)[:, :P.shape[1]]
    kw = {}
    if "Q" in a:
        Q = dev(a["Q"], torch.float32)
        if pad:
            Q = torch.cat([Q, torch.full((Q.shape[0], pad), 9.0, device="cuda")], 1)[:, :Q.shape[1]]
        kw = dict(draft_probs=Q, draft_ids=dev(a["draft_ids"]), d2t=dev(a["d2t"]))
    r = vt.vt_verify_tokens(P, dev(a["tokens"]), dev(a["parents"]), dev(a["cu"]), dev(a["u_accept"], torch.float32), dev(a["u_sample"], torch.float32),
                            max_tokens=max_tokens, **kw)
    return [t.cpu().numpy() for t in r]


def check(vt, a, max_tokens, pad=0):
    want = so.verify(a["P"], a["tokens"], a["parents"], a["cu"], a["u_accept"], a["u_sample"], max_tokens, a.get("Q"), a.get("draft_ids"), a.get("d2t"))
    got = run(vt, a, max_tokens, pad)
    for name, g, w in zip(("n_accepted", "path", "tokens"), got, want):
        assert np.array_equal(g, w), (name, np.argwhere(g != w)[:4], g[:2], w[:2])
    return want


# vocabularies around the shares of warps and CTAs, rows that are and are not 16 bytes apart
@pytest.mark.parametrize("V,Vd", [(1, 0), (1, 1), (2, 2), (5, 3), (127, 40), (128, 0), (1000, 300), (2047, 0), (2048, 2048), (2049, 700), (16385, 5000), (33000, 0)])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("pad", [0, 3])
def test_vocabularies(vt, V, Vd, tree, pad):
    counts = [1, 6, 0, 9, 2, 33]
    a = make(counts, V, Vd, tree, seed=V + Vd + tree)
    check(vt, a, 33, pad)


# rows that begin at each place between two 16-byte boundaries, their neighbours NaN; the last ids chosen, at the end of a CTA's or a warp's part
@pytest.mark.parametrize("V,Vd", [(16384, 0), (16383, 0), (2046, 0), (2045, 77), (16384, 900), (16381, 16381)])
@pytest.mark.parametrize("shift", [0, 1, 2, 3])
@pytest.mark.parametrize("odd", [0, 1])
def test_rows_anywhere(vt, V, Vd, shift, odd):
    a = make([3, 1, 12], V, Vd, True, seed=V + shift, identity=Vd == V)
    a["u_sample"] = np.float32([0.0, 1.0, 0.9999])
    want = so.verify(a["P"], a["tokens"], a["parents"], a["cu"], a["u_accept"], a["u_sample"], 12, a.get("Q"), a.get("draft_ids"), a.get("d2t"))
    ld = V + 5 if odd else -(-(V + 3) // 4) * 4
    flat = torch.full((16 * ld + 8,), float("nan"), device="cuda")
    P = flat[shift:shift + 16 * ld].view(16, ld)[:, :V]
    P.copy_(dev(a["P"], torch.float32))
    kw = dict(draft_probs=dev(a["Q"], torch.float32), draft_ids=dev(a["draft_ids"]), d2t=dev(a["d2t"])) if Vd else {}
    got = vt.vt_verify_tokens(P, dev(a["tokens"]), dev(a["parents"]), dev(a["cu"]), dev(a["u_accept"], torch.float32), dev(a["u_sample"], torch.float32),
                              max_tokens=12, **kw)
    for g, w in zip(got, want):
        assert np.array_equal(g.cpu().numpy(), w)


@pytest.mark.parametrize("drawn", [False, True])
def test_the_largest_vocabularies(vt, drawn):
    rng = np.random.default_rng(1)
    V, Vd = (393216, 50000) if drawn else (4194304, 0)
    P = rng.random((4, V), dtype=np.float32) ** 8
    P /= P.sum(1, keepdims=True, dtype=np.float64).astype(np.float32)
    a = dict(P=P, parents=[-1, 0, 0, 1], cu=[0, 4], u_accept=np.float32([0, .9, .9, .9]), u_sample=np.float32([0.77]), tokens=[0, 5, V - 1, 7])
    if drawn:
        d2t = rng.permutation(V)[:Vd]
        Q = rng.random((4, Vd), dtype=np.float32)
        Q /= Q.sum(1, keepdims=True)
        a |= dict(Q=Q, draft_ids=np.array([0, 5, 70, 7]), d2t=d2t, tokens=d2t[[0, 5, 70, 7]])
    check(vt, a, 4)


def test_the_largest_drawn_vocabulary_with_rows_anywhere_and_the_most_tokens(vt):
    rng = np.random.default_rng(4)
    V, Vd, N = 393216, 1000, 5
    P = rng.random((N, V), dtype=np.float32) ** 8
    P /= P.sum(1, keepdims=True, dtype=np.float64).astype(np.float32)
    Q = rng.random((N, Vd), dtype=np.float32)
    Q /= Q.sum(1, keepdims=True)
    d2t, ids = rng.permutation(V)[:Vd], np.array([0, 5, 70, 7, 999])
    a = dict(P=P, parents=[-1, 0, 0, 1, 0], cu=[0, 5], u_accept=np.float32([0, .99, .99, .99, .99]), u_sample=np.float32([0.999999]), tokens=d2t[ids])
    want = so.verify(P, a["tokens"], a["parents"], a["cu"], a["u_accept"], a["u_sample"], 1024, Q, ids, d2t)
    flat = torch.full((N * (V + 1) + 1,), float("nan"), device="cuda")
    rows = flat[1:].view(N, V + 1)[:, :V]
    rows.copy_(dev(P, torch.float32))
    got = vt.vt_verify_tokens(rows, dev(a["tokens"]), dev(a["parents"]), dev(a["cu"]), dev(a["u_accept"], torch.float32), dev(a["u_sample"], torch.float32),
                              max_tokens=1024, draft_probs=dev(Q, torch.float32), draft_ids=dev(ids), d2t=dev(d2t))
    for g, w in zip(got, want):
        assert np.array_equal(g.cpu().numpy(), w)


@pytest.mark.parametrize("drawn", [False, True])
def test_many_random_trees(vt, drawn):
    for seed in range(12):
        rng = np.random.default_rng(seed)
        counts = rng.integers(0, 40, 40).tolist()
        a = make(counts, 200 + 13 * seed, 90 if drawn else 0, True, seed, like=[0.0, 0.3, 2.0][seed % 3])
        check(vt, a, 40)


def test_long_chains_are_accepted_and_cut(vt):
    a = make([400, 1024, 7], 64, 0, False, 3)
    a["tokens"][1:] = a["P"].argmax(1)[:-1]
    a["tokens"][0] = 0
    a["u_accept"][:] = 0.0
    want = check(vt, a, 1024)
    assert want[0].tolist() == [399, 1023, 6]
    want = check(vt, a, 100)                     # what a request has beyond max_tokens is left out
    assert want[0].tolist() == [99, 99, 6]


def test_the_identity_map(vt):
    check(vt, make([5, 9], 77, 77, True, 4, identity=True), 9)
    check(vt, make([5, 9], 77, 30, True, 4, identity=True), 9)
    check(vt, make([5, 9], 9000, 8999, False, 4, identity=True), 9)


def test_edges_of_the_random_numbers(vt):
    last = np.float32(1) - np.float32(2.0 ** -24)
    for drawn in (0, 120):
        for ua in (0.0, last, 1.0):
            for us in (0.0, last, 1.0, -0.5, 2.0):
                a = make([7, 3], 300, drawn, True, 11)
                a["u_accept"][:] = ua
                a["u_sample"][:] = us
                a["P"][:, [0, 1, 299]] = 0                           # nothing at either end
                check(vt, a, 7)


def test_same_distribution_accepts_and_leaves_nothing(vt):
    # q = p: every draw is accepted; where a child is turned down all the same (u past 1), p itself is drawn from
    rng = np.random.default_rng(0)
    P = rng.dirichlet(np.ones(64), size=6).astype(np.float32)
    ids = np.array([0, 9, 11, 30, 2, 5])
    a = dict(P=P, Q=P.copy(), parents=[-1, 0, 1, 2, 3, 4], cu=[0, 6], u_accept=np.full(6, 0.999, np.float32), u_sample=np.float32([0.4]), tokens=ids,
             draft_ids=ids, d2t=None)
    assert check(vt, a, 6)[0][0] == 5
    a["u_accept"][2] = 1.5
    want = check(vt, a, 6)
    assert want[0][0] == 1 and want[2][0, 1] >= 0


def test_what_does_not_fit_is_left_out(vt):
    for drawn in (0, 60):
        a = make([12, 12], 90, drawn, True, 21)
        a["parents"][3], a["parents"][15], a["parents"][7] = 3, 99, -7
        a["tokens"][5], a["tokens"][17] = 90, -1
        if drawn:
            a["draft_ids"][2], a["draft_ids"][14] = 60, -4
        a["u_accept"][:] *= 0.3
        check(vt, a, 12)
    a = make([4], 40, 0, False, 1)
    a["P"][:] = 0
    want = check(vt, a, 4)                       # nothing to draw from
    assert want[2][0].tolist() == [-1] * 4
    a = make([4], 40, 0, False, 1)
    a["P"][0, :7], a["P"][0, 9] = np.nan, -3.0
    check(vt, a, 4)


def test_the_same_token_twice(vt):
    for drawn in (0, 10):
        a = make([6], 12, drawn, True, 2)
        a["parents"] = np.array([-1, 0, 0, 0, 0, 0])
        a["tokens"][1:] = a["tokens"][1]
        if drawn:
            a["draft_ids"][1:] = a["draft_ids"][1]
        a["u_accept"][1], a["u_accept"][2:] = 1.0, 0.0
        check(vt, a, 6)


def test_no_tokens_at_all(vt):
    a = make([0, 0, 0], 10, 0, False, 0)
    n, path, out = run(vt, a, 3)
    assert n.tolist() == [0, 0, 0] and (path == -1).all() and (out == -1).all()


def test_captured_on_another_stream_into_given_outputs(vt):
    a, b = make([9, 4], 500, 100, True, 1), make([9, 4], 500, 100, True, 2)
    t = {k: dev(v, torch.float32 if k in ("P", "Q", "u_accept", "u_sample") else torch.int32) for k, v in a.items()}
    out = vt.VtVerified(*(torch.empty(s, dtype=torch.int32, device="cuda") for s in ((2,), (2, 9), (2, 9))))

    def call():
        return vt.vt_verify_tokens(t["P"], t["tokens"], t["parents"], t["cu"], t["u_accept"], t["u_sample"], max_tokens=9, draft_probs=t["Q"],
                                   draft_ids=t["draft_ids"], d2t=t["d2t"], out=out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            call()
    torch.cuda.synchronize()
    for c in (a, b, a):
        for k, v in c.items():
            t[k].copy_(torch.tensor(np.asarray(v)))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay()
        torch.cuda.synchronize()
        want = so.verify(c["P"], c["tokens"], c["parents"], c["cu"], c["u_accept"], c["u_sample"], 9, c["Q"], c["draft_ids"], c["d2t"])
        assert all(np.array_equal(x.cpu().numpy(), w) for x, w in zip(out, want))
