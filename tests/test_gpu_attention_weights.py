"""Few rows: the weights that multiply the values add up to what out is divided by.

A weight w_i (they add up to 1) is rounded to bf16, by 2^-8 at most; out = sum r_i v_i / sum r_i moves by 2^-8 sum w_i |v_i - out| at most, which for
a weight far above the others is next to nothing, and is rounded once, 2^-8 |out|.  Products and sums in fp32: sum w_i |v_i| (2 d + 2^-16), d as in
test_gpu_tree_attention.py; second-order terms are within the 2^-16."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vt():
    import paper_2603_05210_b200 as vt
    vt.lib()
    return vt


def attend(vt, q, k, v, scale, page=32):
    """q [T, Hq, D] on a chain behind k, v [n - T, heads, D], whose last T positions are theirs; the pages lie in reverse."""
    n, heads, D = k.shape
    T, pages = q.shape[0], -(-n // page)
    kc, vc = (torch.zeros(pages, page, heads, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kc.view(-1, heads, D)[:n], vc.view(-1, heads, D)[:n] = k, v
    table = torch.arange(pages - 1, -1, -1, dtype=torch.int32, device="cuda")[None].contiguous()
    cache = vt.VtCache(kc.flip(0).contiguous(), vc.flip(0).contiguous(), table, torch.tensor([n - T], dtype=torch.int32, device="cuda"))
    return vt.vt_tree_attention(q, torch.tensor([0, T], dtype=torch.int32, device="cuda"), cache, max_tokens=T, scale=scale)


def check(vt, q, k, v, scale):
    out, lse = attend(vt, q, k, v, scale)
    (T, Hq, D), (n, heads, _) = q.shape, k.shape
    G = Hq // heads
    qd, kd, vd = q.double(), k.double().repeat_interleave(G, 1), v.double().repeat_interleave(G, 1)
    x = torch.einsum("thd,ihd->thi", qd, kd) * scale
    sees = torch.arange(n, device="cuda")[None] <= torch.arange(n - T, n, device="cuda")[:, None]
    x = x.masked_fill(~sees[:, None], -float("inf"))
    want_lse = torch.logsumexp(x, -1)
    w = (x - want_lse[..., None]).exp()
    want = torch.einsum("thi,ihd->thd", w, vd)
    X = scale * torch.einsum("thd,ihd->thi", qd.abs(), kd.abs()).amax(-1)
    d = 2 * 2.0 ** -23 * (D / 16 + 8) * X + 2.0 ** -23 * X * 1.45 + 2.0 ** -22
    size = torch.einsum("thi,ihd->thd", w, vd.abs())
    moved = torch.stack([(w[:, h, :, None] * (vd[None, :, h] - want[:, h, None]).abs()).sum(1) for h in range(Hq)], 1)
    over = (out.double() - want).abs() - 2.0 ** -8 * (moved + want.abs()) - size * (2 * d[..., None] + 2.0 ** -16)
    assert bool((over <= 0).all()), float(over.max())
    off = (lse.double() - want_lse).abs() - d - 2.0 ** -24 * (60 + n / 128) - 2.0 ** -22 * want_lse.abs()
    assert bool((off <= 0).all()), float(off.max())


# one score above all others by less than what moves the maximum in use: its weight is no power of two.  In one piece and in many
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,first,late", [(300, 5, 261), (505, 40, 300), (5000, 5, 2309), (5000, 1, 4990)])
def test_one_weight_far_above_the_others(vt, D, n, first, late):
    torch.manual_seed(n)
    k, q = torch.zeros(n, 1, D), torch.zeros(1, 16, D)
    k[:, 0, 0] = -40.0
    k[first, 0, 0], k[late, 0, 0] = 0.0, 5.0                       # a weight of 2^7 or so
    q[0, :, 0] = 8.0 + 0.0625 * torch.arange(-12, 4)               # scale 1 / 8: scores from 4.06 to 5.09 on
    v = torch.rand(n, 1, D) + 1.0
    check(vt, *(a.cuda().bfloat16() for a in (q, k, v)), 0.125)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,Hq,heads,n", [(1, 8, 2, 700), (4, 4, 1, 3000), (8, 8, 2, 130), (1, 32, 1, 20000), (2, 2, 2, 2)])
@pytest.mark.parametrize("peak", [0.5, 3.0, 12.0])
def test_flat_and_peaked_rows(vt, D, T, Hq, heads, n, peak):
    torch.manual_seed(T + n)
    q, k, v = torch.randn(T, Hq, D) * peak, torch.randn(n, heads, D), torch.randn(n, heads, D)
    check(vt, *(a.cuda().bfloat16() for a in (q, k, v)), D ** -0.5)


@pytest.mark.parametrize("scale", [1e-38, 2.0 ** -126, 1e-30, 1e-4, 1.0])
def test_small_scales(vt, scale):
    torch.manual_seed(3)
    q, k, v = torch.randn(2, 4, 64), torch.randn(900, 2, 64), torch.randn(900, 2, 64)
    check(vt, *(a.cuda().bfloat16() for a in (q, k, v)), float(np.float32(scale)))
