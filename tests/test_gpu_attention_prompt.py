"""A prompt's chunk through the attention: many blocks of rows, each with keys of its own number.  Tolerances as in test_gpu_tree_attention.py."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,counts,Hq,heads", [([0], [2100], 8, 2), ([3000, 5], [1025, 640], 4, 1), ([129, 0, 4000], [1, 1500, 77], 6, 2)])
def test_chunks(D, lens, counts, Hq, heads):
    import paper_2603_05210_b200 as vt
    torch.manual_seed(sum(counts) + D)
    page, N = 64, sum(counts)
    used = [-(-(a + b) // page) for a, b in zip(lens, counts)]
    k, v = (torch.randn(sum(used), page, heads, D, device="cuda").bfloat16() for _ in range(2))
    order, at = torch.randperm(sum(used)).int().cuda(), 0
    table = torch.full((len(lens), max(used)), -1, dtype=torch.int32, device="cuda")
    for b, u in enumerate(used):
        table[b, :u] = order[at:at + u]
        at += u
    cu = torch.tensor([0] + counts).cumsum(0).int().cuda()
    q = (torch.randn(N, Hq, D, device="cuda") * 1.5).bfloat16()
    out, lse = vt.vt_tree_attention(q, cu, vt.VtCache(k, v, table, torch.tensor(lens, dtype=torch.int32, device="cuda")), max_tokens=max(counts))
    big = lambda n: 2.0 ** -23 * (n / 16 + 8)  # noqa: E731
    scale, G = D ** -0.5, Hq // heads
    for b, (L, T) in enumerate(zip(lens, counts)):
        n, rows = L + T, slice(int(cu[b]), int(cu[b + 1]))
        kb, vb = (t[table[b, :used[b]].long()].flatten(0, 1)[:n].double() for t in (k, v))
        sees = torch.arange(n, device="cuda")[None] <= L + torch.arange(T, device="cuda")[:, None]
        for h in range(Hq):
            x = (q[rows, h].double() @ kb[:, h // G].T * scale).masked_fill(~sees, -float("inf"))
            want_lse = torch.logsumexp(x, 1)
            w = (x - want_lse[:, None]).exp()
            want, size = w @ vb[:, h // G], w @ vb[:, h // G].abs()
            X = scale * (q[rows, h].double().abs() @ kb[:, h // G].abs().T).amax(1)
            d = 2 * big(D) * X + 2.0 ** -23 * X * 1.45 + 2.0 ** -22
            off = (lse[rows, h].double() - want_lse).abs() - d - 2.0 ** -24 * (60 + n / 128) - 2.0 ** -22 * want_lse.abs()
            assert bool((off <= 0).all()), float(off.max())
            err = (out[rows, h].double() - want).abs() - 2.0 ** -8 * want.abs() - size * (2.0 ** -8 + 2 * d + big(n) + 2.0 ** -20)[:, None]
            assert bool((err <= 0).all()), float(err.max())
