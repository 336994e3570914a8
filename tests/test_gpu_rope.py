"""Rotary positions and the write into the cache against the fp64 oracle.

What an element may be off: half a step of bf16, 2^-8 |y|, and what the turn loses, (|x1| + |x2|) a times
  2^-24 pi + 2^-23  (the angle as a float in half turns, sincospif to 2 units)  + 3 * 2^-24 (two products, one sum)  < 6e-7."""
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


def check(got, x, positions, w, interleaved, amplitude, inverse=False):
    want, x = so.rope(f64(x), positions, w, interleaved, amplitude, inverse), f64(x)
    size, half = np.zeros_like(x), len(w)
    if interleaved:
        size[..., :2 * half] = np.repeat(np.abs(x[..., 0:2 * half:2]) + np.abs(x[..., 1:2 * half:2]), 2, axis=-1)
    else:
        size[..., :half] = size[..., half:2 * half] = np.abs(x[..., :half]) + np.abs(x[..., half:2 * half])
    err = np.abs(f64(got) - want)
    assert np.all(err <= 2.0 ** -8 * np.abs(want) + 6e-7 * abs(amplitude) * size), err.max()
    assert np.array_equal(f64(got)[..., 2 * half:], x[..., 2 * half:])


@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("linear", 4.0), ("base", 8.0), ("wavelength", 8.0), ("ramp", 32.0)])
@pytest.mark.parametrize("rot", [16, 64, 128, 1024])
def test_table(vt, scaling, factor, rot):
    r = vt.vt_rope_table(rot, scaling=scaling, factor=factor, base=500000.0 if rot == 64 else 10000.0, original_len=4096.0)
    w = so.rope_frequencies(rot, 500000.0 if rot == 64 else 10000.0, scaling, factor, original_len=4096.0)
    turns = r.table.cpu().numpy().astype(np.uint64).astype(np.float64) / 2.0 ** 64
    # an entry is a multiple of 2^-63 turns: off by half of that, 2 pi 2^-64 radians (and by what pow and the way back to floats lose)
    assert np.allclose(turns * 2 * np.pi, w, rtol=1e-14, atol=2 * np.pi * 2.0 ** -64)
    assert r.amplitude == (pytest.approx(0.1 * np.log(factor) + 1) if scaling == "ramp" else 1.0)


# few and many tokens (whole tokens on a block, or several blocks on a token), odd head counts, the whole head and parts of it
@pytest.mark.parametrize("N,Hq,Hkv,D,rot", [(1, 32, 8, 128, 128), (3, 1, 1, 16, 16), (5, 7, 3, 64, 32), (149, 5, 0, 96, 96), (1200, 3, 1, 128, 48),
                                            (2400, 2, 2, 256, 16), (4, 2, 1, 1024, 1024)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_turn_and_back(vt, N, Hq, Hkv, D, rot, interleaved):
    torch.manual_seed(N)
    rope = vt.vt_rope_table(rot, interleaved=interleaved, scaling="wavelength", factor=4.0, amplitude=1.25)
    w = so.rope_frequencies(rot, scaling="wavelength", factor=4.0)
    q = torch.randn(N, Hq, D, device="cuda").bfloat16()
    k = torch.randn(N, Hkv, D, device="cuda").bfloat16() if Hkv else None
    positions = torch.randint(0, 1_000_000, (N,), device="cuda").int()
    positions[0] = 2 ** 31 - 1
    positions[-1] = -5
    at = positions.tolist()
    for inverse in (False, True):
        yq, yk = vt.vt_rope(q, k, positions, rope, inverse=inverse)
        check(yq, q, at, w, interleaved, 1.25, inverse)
        if Hkv:
            check(yk, k, at, w, interleaved, 1.25, inverse)
    # in place, and on parts of a fused projection's output
    fused = torch.randn(N, Hq + 2 * Hkv + 1, D, device="cuda").bfloat16()
    before = fused.clone()
    fq, fk = fused[:, :Hq], fused[:, Hq:Hq + Hkv] if Hkv else None
    vt.vt_rope(fq, fk, positions, rope, out_q=fq, out_k=fk)
    check(fq, before[:, :Hq], at, w, interleaved, 1.25)
    if Hkv:
        check(fk, before[:, Hq:Hq + Hkv], at, w, interleaved, 1.25)
    assert torch.equal(fused[:, Hq + Hkv:], before[:, Hq + Hkv:])


def test_gradient_by_differences(vt):
    # y is linear in x: the gradient of sum(g y) is the inverse turn of g; both sides carry one rounding per element
    torch.manual_seed(4)
    N, H, D = 6, 2, 64
    rope = vt.vt_rope_table(D)
    positions = torch.randint(0, 5000, (N,), device="cuda").int()
    x, g = torch.randn(N, H, D, device="cuda").bfloat16(), torch.randn(N, H, D, device="cuda").bfloat16()
    back, _ = vt.vt_rope(g, None, positions, rope, inverse=True)
    for n, h, j in ((0, 0, 0), (3, 1, 40), (5, 0, 63)):
        d = torch.zeros_like(x)
        d[n, h, j] = 4.0
        hi, lo = (vt.vt_rope(x * 0 + s * d, None, positions, rope)[0] for s in (1, -1))
        diff = ((hi.double() - lo.double()) * g.double()).sum() / 8
        size = g[n, h].double().abs().sum()
        assert abs(diff - back[n, h, j].double()) <= 2.0 ** -7 * size


def paged(vt, lens, counts, heads, D, page, spare=2, by_head=False, max_pages=None):
    used = [max(1, -(-(a + b) // page)) for a, b in zip(lens, counts)]
    n = sum(used) + spare
    shape = (n, heads, page, D) if by_head else (n, page, heads, D)
    k, v = (torch.randn(shape, device="cuda").bfloat16() for _ in range(2))
    if by_head:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    order, table, at = torch.randperm(n).tolist(), torch.full((len(lens), max_pages or max(used)), -1, dtype=torch.int32), 0
    for b, u in enumerate(used):
        table[b, :u] = torch.tensor(order[at:at + u], dtype=torch.int32)
        at += u
    cache = vt.VtCache(k, v, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    cu = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
    return cache, cu


@pytest.mark.parametrize("page,by_head", [(8, False), (16, True), (64, False), (128, True), (384, False)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append(vt, page, by_head, interleaved):
    torch.manual_seed(page)
    lens, counts, heads, Hq, D, rot = [0, 5, 127, 300, 0], [3, 1, 40, 0, 200], 3, 6, 64, 32
    cache, cu = paged(vt, lens, counts, heads, D, page, by_head=by_head)
    N, pad = sum(counts), 4                       # padding rows behind the last request
    q, k, v = (torch.randn(N + pad, h, D, device="cuda").bfloat16() for h in (Hq, heads, heads))
    positions = torch.randint(0, 100_000, (N + pad,), device="cuda").int()
    rope, w = vt.vt_rope_table(rot, interleaved=interleaved), so.rope_frequencies(rot)
    kc, vc, out = cache.k.clone(), cache.v.clone(), torch.full_like(q, 7.0)
    assert vt.vt_rope_append(q, k, v, positions, cu, cache, rope, out_q=out) is out
    check(out[:N], q[:N], positions[:N].tolist(), w, interleaved, 1.0)
    assert bool((out[N:] == 7.0).all())
    turned = vt.vt_rope(k, None, positions, rope)[0]
    for b, (L, T) in enumerate(zip(lens, counts)):
        for t in range(T):
            at = L + t
            pg = int(cache.page_table[b, at // page])
            kc[pg, at % page], vc[pg, at % page] = turned[int(cu[b]) + t], v[int(cu[b]) + t]
    assert torch.equal(cache.k, kc) and torch.equal(cache.v, vc)      # the tokens' places and nothing else


def test_append_leaves_out_what_has_no_place(vt):
    torch.manual_seed(0)
    cache, cu = paged(vt, [14, 0, 2], [4, 2, 2], 1, 16, 16, max_pages=2)
    cache.lens[2] = 2 ** 31 - 3
    q, k, v = (torch.randn(8, 1, 16, device="cuda").bfloat16() for _ in range(3))
    cache.page_table[0, 1] = 10 ** 6              # token 2 and 3 of request 0
    cache.page_table[1, 0] = -1
    kc, vc = cache.k.clone(), cache.v.clone()
    rope = vt.vt_rope_table(16)
    positions = torch.zeros(8, dtype=torch.int32, device="cuda")
    out = vt.vt_rope_append(q, k, v, positions, cu, cache, rope)
    pg = int(cache.page_table[0, 0])
    kc[pg, 14:16], vc[pg, 14:16] = k[:2], v[:2]
    assert torch.equal(cache.k, kc) and torch.equal(cache.v, vc) and torch.equal(out, q)


def test_nothing_to_do(vt):
    cache, cu = paged(vt, [3], [0], 1, 16, 16)
    rope, empty = vt.vt_rope_table(16), torch.empty(0, 1, 16, dtype=torch.bfloat16, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert vt.vt_rope_append(empty, empty, empty, none, cu, cache, rope).shape == (0, 1, 16)
    assert vt.vt_rope(empty, None, none, rope)[0].shape == (0, 1, 16)


@pytest.mark.parametrize("N,words", [(1, 1), (70, 3), (300, 2)])
def test_tree_mask(vt, N, words):
    rng = np.random.default_rng(N)
    cuts = np.sort(rng.integers(0, N + 1, 4))
    cu = np.concatenate([[0], cuts, [N]])
    parents = np.array([rng.integers(-1, max(1, n - cu[np.searchsorted(cu, n, side="right") - 1])) for n in range(N)])
    parents[rng.integers(0, N)] = 10 ** 6
    lens = rng.integers(0, 50, len(cu) - 1)
    want, depth = so.tree_mask(parents, cu, words)

    def dev(a):
        return torch.tensor(a, dtype=torch.int32, device="cuda")

    mask, positions = vt.vt_tree_mask(dev(parents), dev(cu), 32 * words, lens=dev(lens))
    assert np.array_equal(mask.cpu().numpy().astype(np.int64) & 0xFFFFFFFF, want)
    owner = np.searchsorted(cu, np.arange(N), side="right") - 1
    assert np.array_equal(positions.cpu().numpy(), depth + lens[owner])
    assert np.array_equal(vt.vt_tree_mask(dev(parents), dev(cu), 32 * words)[1].cpu().numpy(), depth)


def test_a_table_of_another_size_is_refused(vt):
    rope = vt.vt_rope_table(64)
    q = torch.zeros(3, 2, 128, dtype=torch.bfloat16, device="cuda")
    positions = torch.arange(3, dtype=torch.int32, device="cuda")
    for wrong in (rope._replace(rot_dim=128), rope._replace(table=rope.table[:-1]), rope._replace(table=rope.table[::2], rot_dim=32),
                  rope._replace(table=rope.table.int()), rope._replace(table=rope.table.cpu())):
        with pytest.raises(ValueError):
            vt.vt_rope(q, None, positions, wrong)
