"""Attention of drafted tokens over a paged cache against the fp64 oracle.

What may be off, for a row with scores x_i = scale q.k_i, weights w_i and A = sum_i w_i |v_i|:
  scores    fp32 sums of D exact products: E(D) = 2^-23 (D / 16 + 8) of scale sum |q_j k_j|, twice (its own and the largest's)
  exponents the argument x log2 e - m log2 e is off by 2^-23 of its parts' size, ex2 by 2^-22: relative error of a weight
            d = 2 E(D) X + 2^-23 |x|max + 2^-22,   X = scale max_i sum_j |q_j k_ij|
  lse       d, the sum's own 2^-24 (60 + tiles), 2^-22 |lse|
  out       each weight is rounded to bf16, 2^-8; the products' sums E(n); the result is rounded once, 2^-8:
            2^-8 |out| + A (2^-8 + 2 d + E(n) + 2^-20)"""
import itertools

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


def f64(t):
    return t.detach().double().cpu().numpy()


class Case:
    def __init__(self, vt, lens, counts, Hq, heads, D, page, tree=False, by_head=False, pad=0, words=None, max_pages=None, fused=True, seed=0):
        torch.manual_seed(seed + sum(lens) + 7 * sum(counts))
        used = [max(1, -(-(a + b) // page)) for a, b in zip(lens, counts)]
        n = sum(used) + 2
        shape = (n, heads, page, D) if by_head else (n, page, heads, D)
        self.k, self.v = (torch.randn(shape, device="cuda").bfloat16() for _ in range(2))
        if by_head:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        order, at = torch.randperm(n).tolist(), 0
        table = torch.full((len(lens), max_pages or max(used)), -1, dtype=torch.int32)
        for b, u in enumerate(used):
            u = min(u, table.shape[1])
            table[b, :u] = torch.tensor(order[at:at + u], dtype=torch.int32)
            at += u
        self.cache = vt.VtCache(self.k, self.v, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
        self.cu = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
        self.N, self.max_tokens = sum(counts), max(1, max(counts))
        wide = torch.randn(self.N + pad, Hq + (2 * heads if fused else 0), D, device="cuda") * torch.rand(self.N + pad, 1, 1, device="cuda").mul(2.5).add(0.2)
        self.q = wide.bfloat16()[:, :Hq]
        self.mask = None
        if tree:
            within = torch.arange(self.N) - torch.repeat_interleave(self.cu.cpu()[:-1], torch.tensor(counts)).long()
            parents = (within - 1 - torch.randint(0, 6, (self.N,))).clamp(min=0).masked_fill(within == 0, -1).int().cuda()
            self.mask, _ = vt.vt_tree_mask(parents, self.cu, 32 * (words or -(-self.max_tokens // 32)))
            if pad:
                self.mask = torch.cat([self.mask, torch.full((pad, self.mask.shape[1]), -1, dtype=torch.int32, device="cuda")])
        self.scale = D ** -0.5
        self.vt = vt

    def run(self, **kw):
        return self.vt.vt_tree_attention(self.q, self.cu, self.cache, max_tokens=self.max_tokens, mask=self.mask, scale=self.scale, **kw)

    def check(self, out, lse, rows=None):
        lens, cu = self.cache.lens.cpu().numpy(), self.cu.cpu().numpy()
        k, v = f64(self.cache.k), f64(self.cache.v)
        mask = None if self.mask is None else self.mask.cpu().numpy().astype(np.int64) & 0xFFFFFFFF
        want, want_lse, size = so.attention(f64(self.q)[:self.N], k, v, self.cache.page_table.cpu().numpy(), lens, cu, mask, self.scale, self.max_tokens)
        rows = np.arange(self.N) if rows is None else np.asarray(rows)
        D, n = self.q.shape[2], int(lens.max()) + self.max_tokens
        big = lambda D: 2.0 ** -23 * (D / 16 + 8)  # noqa: E731
        kmax = np.nan_to_num(np.abs(k), nan=0.0, posinf=0.0).max()
        X = self.scale * np.abs(f64(self.q)[rows]).sum(-1) * kmax                 # [rows, Hq], an upper bound
        d = 2 * big(D) * X + 2.0 ** -23 * X * 1.45 + 2.0 ** -22
        got, got_lse = f64(out)[rows], f64(lse)[rows]
        want, want_lse, size = want[rows], want_lse[rows], size[rows]
        empty = np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(got_lse), empty) and np.all(got[empty] == 0)
        tol = d + 2.0 ** -24 * (60 + n / 128) + 2.0 ** -22 * np.abs(np.where(empty, 0, want_lse))
        assert np.all(np.abs(got_lse - want_lse)[~empty] <= tol[~empty]), np.abs(got_lse - want_lse)[~empty].max()
        err = np.abs(got - want) - 2.0 ** -8 * np.abs(want) - size * (2.0 ** -8 + 2 * d + big(n) + 2.0 ** -20)[..., None]
        assert np.all(err <= 0), err.max()


# tokens a request, heads and groups (one row tile, two, several blocks; groups that do not divide 128), both widths
@pytest.mark.parametrize("T,Hq,heads", [(1, 1, 1), (1, 32, 8), (2, 3, 1), (8, 8, 8), (31, 5, 1), (33, 4, 1), (64, 8, 2), (65, 8, 2), (3, 128, 1), (2, 100, 1),
                                        (200, 6, 2), (130, 1, 1), (300, 2, 1)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tree", [False, True])
def test_layouts(vt, T, Hq, heads, D, tree):
    c = Case(vt, [150, 0, 400], [T, max(1, T // 3), T], Hq, heads, D, 16, tree=tree)
    c.check(*c.run())


# lengths at and around tiles and pages; pages smaller and larger than a tile
@pytest.mark.parametrize("page,by_head", [(8, False), (16, True), (32, False), (64, False), (128, True), (256, False), (384, False)])
@pytest.mark.parametrize("tree", [False, True])
def test_lengths(vt, page, by_head, tree):
    lens = [0, 1, 7, 8, 126, 127, 128, 129, 255, 256, 383, 384, 385, 640]
    c = Case(vt, lens, [1 + i % 5 for i in range(len(lens))], 4, 2, 64, page, tree=tree, by_head=by_head)
    c.check(*c.run())


def test_items_that_are_not_cut_and_items_in_many_pieces(vt):
    for lens, counts, kw in (([100, 300, 0, 500], [4, 3, 2, 1], {}), ([20000], [1], {}), ([9000, 130], [60, 60], {"tree": True}), ([15000, 3], [9, 70], {})):
        c = Case(vt, lens, counts, 8, 2, 128, 16, **kw)
        out, lse = c.run()
        c.check(out, lse)
        again = c.run()
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])         # the same bits


# ragged trees whose items weigh differently (one row tile and two, side by side in a run), runs that end between the places of a heavy tile
@pytest.mark.parametrize("seed", range(4))
def test_light_and_heavy_items_in_one_call(vt, seed):
    rng = np.random.default_rng(seed)
    B = int(rng.integers(2, 12))
    lens, counts = rng.integers(0, 2500, B).tolist(), rng.integers(0, 75, B).tolist()
    c = Case(vt, lens, counts, 8, 2, 128 if seed & 1 else 64, 32, tree=seed < 2)
    c.check(*c.run())


# more items than CTAs, as many, one less; some requests without tokens
@pytest.mark.parametrize("B", [36, 37, 38, 60])
def test_as_many_items_as_there_are_ctas(vt, B):
    rng = np.random.default_rng(B)
    lens, counts = rng.integers(0, 1500, B).tolist(), rng.integers(0, 12, B).tolist()
    lens[0], counts[0] = 9000, 12
    c = Case(vt, lens, counts, 16, 4, 64, 32, tree=True)
    c.check(*c.run())


def test_a_bound_far_above_the_tokens(vt):
    c = Case(vt, [700, 90], [1, 2], 8, 2, 128, 16, tree=True)
    c.max_tokens = 5000
    c.check(*c.run())


# one long item in up to as many pieces as there are CTAs, and in one more or fewer than are fetched at a time
@pytest.mark.parametrize("T,Hq,D,L", [(1, 8, 128, 40000), (1, 1, 64, 1100), (9, 4, 128, 2304), (33, 4, 64, 9000), (60, 4, 128, 2500)])
def test_one_item_in_many_pieces(vt, T, Hq, D, L):
    c = Case(vt, [L], [T], Hq, 1, D, 128, tree=T > 1)
    c.check(*c.run())


def test_many_requests(vt):
    rng = np.random.default_rng(3)
    lens, counts = rng.integers(0, 300, 700).tolist(), rng.integers(0, 4, 700).tolist()
    c = Case(vt, lens, counts, 2, 1, 64, 16, max_pages=80)
    c.check(*c.run())
    c = Case(vt, lens[:40], counts[:40], 2, 1, 64, 16)
    c.check(*c.run())


def test_rows_outside_the_requests_and_past_max_tokens_stay(vt):
    c = Case(vt, [40, 200, 5], [6, 0, 9], 4, 2, 64, 16, tree=True, pad=5)
    out, lse = torch.full((20, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda"), torch.full((20, 4), 3.0, device="cuda")
    c.run(out=out, lse=lse)
    c.check(out, lse)
    assert bool((out[15:] == 3).all()) and bool((lse[15:] == 3).all())
    out.fill_(3.0), lse.fill_(3.0)
    c.max_tokens = 4
    c.run(out=out, lse=lse)
    done = [0, 1, 2, 3, 6, 7, 8, 9]
    c.check(out, lse, rows=done)
    left = [i for i in range(20) if i not in done]
    assert bool((out[left] == 3).all()) and bool((lse[left] == 3).all())
    # requests need not begin at row 0
    c = Case(vt, [40, 20], [6, 9], 4, 2, 64, 16)
    ref = c.run()
    c.cu[0] = 2
    out.fill_(3.0)
    c.run(out=out[:15], lse=lse[:15])
    assert bool((out[:2] == 3).all()) and torch.equal(out[6:15], ref[0][6:])


def test_empty_rows_and_stray_mask_bits(vt):
    c = Case(vt, [0, 0, 130], [5, 40, 3], 2, 1, 64, 16, tree=True)
    c.mask[1] = 0
    c.mask[7] = 0
    c.mask[20] = -1                    # bits of tokens that the request does not have, too
    c.mask[46] = 0                     # attends what came earlier
    out, lse = c.run()
    c.check(out, lse)
    assert bool((lse[1] == -float("inf")).all()) and bool((out[7] == 0).all())
    c.mask = c.mask[:, :1].contiguous()           # tokens from 32 on: nobody's
    c.check(*c.run())


def test_the_end_of_the_table(vt):
    # positions past the table are not attended, wherever in a tile that is
    for tree, lens in itertools.product((False, True), ([500, 520, 700], [30, 516, 2 ** 31 - 1])):
        c = Case(vt, [300, 300, 300], [40, 10, 6], 4, 2, 64, 8, tree=tree, max_pages=65)
        c.cache.page_table.copy_(torch.randint(0, c.k.shape[0], c.cache.page_table.shape).int())
        c.cache.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        out, lse = c.run()
        c.cache.lens.clamp_(max=520)
        c.check(out, lse)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_nobody_attends_may_hold_anything(vt, bad):
    c = Case(vt, [70, 140, 3], [20, 9, 40], 4, 2, 64, 16, tree=True)
    want = c.run()
    for b, (L, T) in enumerate(zip([70, 140, 3], [20, 9, 40])):                  # behind the end, on pages in use
        at = L + T
        pg = int(c.cache.page_table[b, at // 16]) if at // 16 < c.cache.page_table.shape[1] else -1
        if pg >= 0 and at % 16:
            c.k[pg, at % 16:], c.v[pg, at % 16:] = bad, bad
    unused = [i for i in range(c.k.shape[0]) if i not in set(c.cache.page_table.flatten().tolist())]
    c.k[unused], c.v[unused] = bad, bad
    got = c.run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # a drafted token that one row alone attends: the others are not touched
    only = 4
    c.mask[:20] &= ~(1 << only)
    want = c.run()
    at = 70 + only
    pg = int(c.cache.page_table[0, at // 16])
    c.k[pg, at % 16], c.v[pg, at % 16] = bad, bad
    got = c.run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    c.mask[only] |= 1 << only
    got = c.run()
    keep = [i for i in range(69) if i != only]
    assert torch.equal(got[0][keep], want[0][keep]) and torch.equal(got[1][keep], want[1][keep])


def test_large_and_small_scores(vt):
    # one score far above all others, late or early, and scores far below zero: the maximum moves, weights vanish
    c = Case(vt, [1000, 129], [3, 2], 4, 1, 128, 16)
    for place, boost in ((0, 60.0), (999, 60.0), (500, 30.0)):
        k = c.k.clone()
        pg = int(c.cache.page_table[0, place // 16])
        c.k[pg, place % 16, 0] = (c.q[0, 0] * boost / c.q[0, 0].float().norm()).bfloat16()
        c.check(*c.run())
        c.k.copy_(k)
    c.k.mul_(-1.0).sub_(3.0)
    c.check(*c.run())
    c.scale = 1e-4
    c.check(*c.run())


def test_a_cache_past_32_bits(vt):
    heads, D, page = 8, 128, 128
    n = 2 ** 31 // (heads * D * page) + 40
    big = torch.zeros(n, page, heads, D, dtype=torch.bfloat16, device="cuda")
    small = Case(vt, [700], [6], 16, heads, D, page, tree=True)
    ids = torch.arange(n - 1, n - 1 - small.cache.page_table.shape[1], -1, dtype=torch.int32, device="cuda")
    for src in (small.k, small.v):
        big[ids.long()] = src[small.cache.page_table[0].long()]
        if src is small.k:
            keys = big[ids.long()].clone()
    cache = vt.VtCache(big, big, ids[None].contiguous(), small.cache.lens)
    out, lse = vt.vt_tree_attention(small.q, small.cu, cache, max_tokens=6, mask=small.mask)
    ref = vt.VtCache(big[ids.long()].contiguous(), big[ids.long()].contiguous(), torch.arange(len(ids), dtype=torch.int32, device="cuda")[None], small.cache.lens)
    want = vt.vt_tree_attention(small.q, small.cu, ref, max_tokens=6, mask=small.mask)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and not torch.equal(keys, big[ids.long()])
    rope = vt.vt_rope_table(D)
    k = torch.randn(6, heads, D, device="cuda").bfloat16()
    vt.vt_rope_append(small.q, k, k, torch.zeros(6, dtype=torch.int32, device="cuda"), small.cu, cache, rope)
    assert torch.equal(big[int(ids[5]), 60:66], k)


def test_pages_outside_the_cache_are_reported_and_read_as_zeros(vt):
    c = Case(vt, [100, 50], [3, 2], 2, 1, 64, 16)
    ws = vt.new_workspace(vt.vt_tree_attention_workspace_bytes(2, 1, 64, 3))
    c.run(workspace=ws)
    assert vt.vt_last_status(ws) == vt.VT_OK
    for bad in (-1, c.k.shape[0], 2 ** 31 - 1, -2 ** 31):
        c.cache.page_table[0, 2] = bad
        out, lse = c.run(workspace=ws)
        assert vt.vt_last_status(ws) == vt.VT_ERR_RANGE
        c.check(out, lse)
    c.cache.page_table[0, 2] = 0
    c.run(workspace=ws)
    assert vt.vt_last_status(ws) == vt.VT_OK


def test_captured_and_replayed_with_other_lengths(vt):
    a, b = Case(vt, [300, 20], [5, 7], 4, 2, 64, 16, tree=True, max_pages=64), Case(vt, [2000], [3], 8, 1, 128, 32)
    ws = vt.new_workspace(max(vt.vt_tree_attention_workspace_bytes(4, 2, 64, 7), vt.vt_tree_attention_workspace_bytes(8, 1, 128, 3)))
    side = torch.cuda.Stream()
    graphs, outs = [], []
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for c in (a, b):                          # both graphs use one workspace
            outs.append(c.run(workspace=ws))
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                c.run(workspace=ws, out=outs[-1][0], lse=outs[-1][1])
            graphs.append(g)
    torch.cuda.synchronize()
    for lens in ([300, 20], [0, 900], [64, 127]):
        a.cache.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        a.cache.page_table.copy_(torch.randint(0, a.k.shape[0], a.cache.page_table.shape).int())
        for o in outs:
            o[0].zero_(), o[1].zero_()
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.current_stream())
            for g in graphs + graphs[:1]:
                g.replay()
        torch.cuda.synchronize()
        a.check(*outs[0])
        b.check(*outs[1])
    assert vt.vt_last_status(ws) == vt.VT_OK


def test_two_streams_at_once(vt):
    cases = [Case(vt, [4000, 200], [5, 7], 8, 2, 128, 16, tree=True, seed=i) for i in range(2)]
    want = [c.run() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                got.append((c, c.run()))
    torch.cuda.synchronize()
    for c, g in got:
        ref = want[cases.index(c)]
        assert torch.equal(g[0], ref[0]) and torch.equal(g[1], ref[1])


def test_a_wait_that_runs_out_is_reported(vt):
    # each copy is made to fall 16 bytes short of what is waited for (host side): every role leaves, and the next call is right
    for lens, counts, D in (([300, 20], [5, 7], 64), ([5000], [60], 128)):
        c = Case(vt, lens, counts, 4, 1, D, 16, tree=True)
        ws = vt.new_workspace(vt.vt_tree_attention_workspace_bytes(4, 1, D, c.max_tokens))
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


def test_strided_outputs_and_workspaces(vt):
    c = Case(vt, [300, 20], [5, 7], 4, 2, 64, 16, tree=True)
    want = c.run()
    wide = torch.zeros(12, 4, 3, 64, dtype=torch.bfloat16, device="cuda")
    got, lse = c.run(out=wide[:, :, 1])
    assert torch.equal(got, want[0]) and torch.equal(lse, want[1]) and not wide[:, :, 0].any() and not wide[:, :, 2].any()
    need = vt.vt_tree_attention_workspace_bytes(4, 2, 64, 7)
    with pytest.raises(vt.VtError) as e:
        c.run(workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    assert e.value.status == vt.VT_ERR_WORKSPACE
    for bad in (torch.empty(need, dtype=torch.uint8), torch.empty(2 * need, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            c.run(workspace=bad)
    assert c.run()[0].shape == (12, 4, 64)
    none = c.vt.vt_tree_attention(c.q[:0], torch.zeros_like(c.cu), c.cache, max_tokens=4)
    assert none[0].shape == (0, 4, 64) and none[1].shape == (0, 4)
