"""vt_gated_ffn and vt_gated_ffn_backward against the fp64 oracle.

Tolerances, derived.  u = 2^-8 is the most one rounding to bf16 moves a value, relatively.
  sums      fp32 sums of n exact products on the tensor cores: each addition moves by at most 2^-23 of the running sum, and at most
            n / 16 + 8 of them follow one another: |error| <= E(n) sum |products|, E(n) = 2^-23 (n / 16 + 8)
  g, u      by E(d); act and its slope are Lipschitz (act' <= 1.13, |act''| <= 1.2), the exponential and the quotient add a relative
            2^-18 at most
  a         |error| <= (u + 2^-18) |a| + 1.13 E(d) Sg |u| + E(d) Su |act(g)|,  Sg = |x| |Wg|^T, Su = |x| |Wu|^T; the same way dg, du
  y and the gradients   the error of their operands through absolute products, E(n) of the sum, and u of the result"""
import numpy as np
import pytest
import torch

from oracle import vt_ffn_oracle as fo
from tests.gpu_util import Guarded

pytestmark = pytest.mark.gpu
U = 2.0 ** -8


def E(n):
    return 2.0 ** -23 * (n / 16 + 8)


@pytest.fixture(scope="module")
def vt():
    import paper_2603_05210_b200 as vt
    vt.lib()
    assert torch.cuda.is_available()
    return vt


def case(M, d, f, seed, gain=1.0):
    g = torch.Generator().manual_seed(seed)

    def t(r, c, std):
        return (torch.randn(r, c, generator=g) * std).bfloat16()

    return t(M, d, gain), t(f, d, d ** -0.5), t(f, d, d ** -0.5), t(d, f, f ** -0.5), t(M, d, 1.0)


def f64(t):
    return t.double().cpu().numpy()


def bounds(x, Wg, Wu, Wd, dy, kind):
    """The oracle's results and how far the kernels' may be, element by element."""
    x, Wg, Wu, Wd, dy = (f64(t) for t in (x, Wg, Wu, Wd, dy))
    (M, d), f = x.shape, Wg.shape[0]
    r = fo.forward(x, Wg, Wu, Wd, kind) | fo.backward(x, Wg, Wu, Wd, dy, kind)
    eg, eu = E(d) * (abs(x) @ abs(Wg).T), E(d) * (abs(x) @ abs(Wu).T)
    act, slope = fo.act(r["g"], kind), fo.act_slope(r["g"], kind)
    e_act, e_slope = 1.13 * eg + 2.0 ** -18 * (abs(act) + 2.0 ** -10), 1.2 * eg + 2.0 ** -18
    e_da = E(d) * (abs(dy) @ abs(Wd))
    ea = U * abs(r["a"]) + abs(r["u"]) * e_act + eu * abs(act)
    edu = U * abs(r["du"]) + e_da * abs(act) + abs(r["da"]) * e_act
    edg = U * abs(r["dg"]) + e_da * abs(r["u"] * slope) + abs(r["da"]) * (eu * abs(slope) + abs(r["u"]) * e_slope)

    def out(name, ops):      # ops: (operand, its error, the exact other operand)
        err = sum((e + E(n) * abs(a)) @ abs(b) for a, e, b, n in ops)
        return r[name], U * abs(r[name]) + (1 + U) * err + 1e-30

    return {"y": out("y", [(r["a"], ea, Wd.T, f)]), "grad_x": out("grad_x", [(r["dg"], edg, Wg, 2 * f), (r["du"], edu, Wu, 2 * f)]),
            "grad_W_gate": out("grad_W_gate", [(r["dg"].T, edg.T, x, M)]), "grad_W_up": out("grad_W_up", [(r["du"].T, edu.T, x, M)]),
            "grad_W_down": (r["grad_W_down"], U * abs(r["grad_W_down"]) + (1 + U) * (abs(dy).T @ (ea + E(M) * abs(r["a"]))) + 1e-30)}


def compare(got, want):
    for n, t in got.items():
        value, most = want[n]
        err = np.abs(f64(t) - value)
        assert (err <= most).all(), (n, (err / most).max())
        if value.size > 2000:                    # on the whole, two roundings of bf16
            assert np.linalg.norm(err) <= U * np.linalg.norm(value), n


SHAPES = [(1, 8, 8), (1, 64, 64), (1, 4096, 1024), (2, 24, 136), (7, 200, 1000), (8, 512, 264), (31, 64, 520), (32, 72, 72), (33, 256, 1504),
          (63, 128, 2048), (64, 1000, 104), (65, 64, 776), (100, 264, 512), (127, 520, 328), (128, 64, 3000), (129, 512, 1000), (255, 136, 264),
          (256, 256, 256), (257, 64, 520), (300, 1000, 680), (700, 128, 264)]


@pytest.mark.parametrize("M,d,f", SHAPES)
@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_block_and_its_gradients(vt, M, d, f, kind):
    args = case(M, d, f, M + d + f, gain=2.0 if M % 2 else 1.0)
    x, Wg, Wu, Wd, dy = (t.cuda() for t in args)
    want = bounds(*args, kind)
    y, saved = Guarded((M, d), torch.bfloat16), Guarded((M, 2 * f), torch.float32)
    ws = torch.full((vt.vt_gated_ffn_workspace_bytes(M, d, f),), 0xFF, dtype=torch.uint8, device="cuda")
    ws[:512] = 0
    vt.vt_gated_ffn(x, Wg, Wu, Wd, act=kind, out=y.t, workspace=ws)
    plain = y.t.clone()
    vt.vt_gated_ffn(x, Wg, Wu, Wd, act=kind, out=y.t, saved=saved.t, workspace=ws)
    assert vt.vt_last_status(ws) == vt.VT_OK and y.intact() and saved.intact() and torch.equal(plain, y.t)
    outs = {"grad_x": Guarded((M, d), torch.bfloat16), "grad_W_gate": Guarded((f, d), torch.bfloat16),
            "grad_W_up": Guarded((f, d), torch.bfloat16), "grad_W_down": Guarded((d, f), torch.bfloat16)}
    ws = torch.full((vt.vt_gated_ffn_backward_workspace_bytes(M, d, f),), 0xFF, dtype=torch.uint8, device="cuda")
    ws[:512] = 0
    vt.vt_gated_ffn_backward(x, Wg, Wu, Wd, saved.t, dy, act=kind, workspace=ws, **{n: g.t for n, g in outs.items()})
    assert vt.vt_last_status(ws) == vt.VT_OK and saved.intact() and all(g.intact() for g in outs.values())
    compare({"y": y.t} | {n: g.t for n, g in outs.items()}, want)
    again = vt.vt_gated_ffn_backward(x, Wg, Wu, Wd, saved.t, dy, act=kind)
    assert all(torch.equal(a, g.t) for a, g in zip(again, outs.values())), "not the same bits twice"


def test_some_gradients_alone(vt):
    M, d, f = 50, 64, 136
    x, Wg, Wu, Wd, dy = (t.cuda() for t in case(M, d, f, 3))
    saved = torch.empty((M, 2 * f), device="cuda")
    vt.vt_gated_ffn(x, Wg, Wu, Wd, saved=saved)
    full = vt.vt_gated_ffn_backward(x, Wg, Wu, Wd, saved, dy)
    ws = vt.new_workspace(vt.vt_gated_ffn_backward_workspace_bytes(M, d, f))
    for some in ([0], [1], [2], [3], [1, 3], [0, 2, 3]):
        outs = [torch.empty_like(full[i]) if i in some else None for i in range(4)]
        st = vt.lib().vt_gated_ffn_backward(x.data_ptr(), d, Wg.data_ptr(), Wu.data_ptr(), Wd.data_ptr(), saved.data_ptr(), dy.data_ptr(), d, M, d, f,
                                            vt.VT_ACT_SILU, *[None if o is None else o.data_ptr() for o in outs], ws.data_ptr(), ws.numel(),
                                            torch.cuda.current_stream().cuda_stream)
        assert st == vt.VT_OK
        torch.cuda.synchronize()
        assert all(torch.equal(outs[i], full[i]) for i in some)


def test_extreme_projections(vt):
    """Projections far out on both sides: act(g) must go to g or to nothing, its slope to one or to nothing, with no NaN between."""
    d, f, M = 8, 64, 9
    x = torch.zeros((M, d))
    x[:, 0] = torch.tensor([0.0, 1.0, -1.0, 30.0, -30.0, 100.0, -100.0, 3e4, -3e4])
    Wg, Wu = torch.zeros((f, d)), torch.zeros((f, d))
    Wg[:, 0] = torch.linspace(-3, 3, f)
    Wu[:, 0] = 1.0 / 128
    Wd = torch.ones((d, f)) / 64
    dy = torch.ones((M, d))
    args = [t.bfloat16() for t in (x, Wg, Wu, Wd, dy)]
    for kind in ("silu", "gelu"):
        xd, g, u, dn, dyd = (t.cuda() for t in args)
        saved = torch.empty((M, 2 * f), device="cuda")
        y = vt.vt_gated_ffn(xd, g, u, dn, act=kind, saved=saved)
        grads = vt.vt_gated_ffn_backward(xd, g, u, dn, saved, dyd, act=kind)
        with np.errstate(over="ignore"):
            want = bounds(*args, kind)
        got = dict(zip(("y", "grad_x", "grad_W_gate", "grad_W_up", "grad_W_down"), (y, *grads)))
        for n, t in got.items():
            assert torch.isfinite(t.float()).all(), n
            assert (np.abs(f64(t) - want[n][0]) <= want[n][1]).all(), (kind, n)


def test_a_nan_stays_in_its_row(vt):
    for M in (3, 60, 300):
        x, Wg, Wu, Wd, _ = (t.cuda() for t in case(M, 64, 264, 4))
        clean = vt.vt_gated_ffn(x, Wg, Wu, Wd)
        x[1, 5] = float("nan")
        got = vt.vt_gated_ffn(x, Wg, Wu, Wd)
        rest = torch.arange(M, device="cuda") != 1
        assert torch.isnan(got[1].float()).all() and torch.equal(got[rest], clean[rest])


def wide(t, extra=24):
    b = torch.full((t.shape[0], t.shape[1] + extra), float("nan"), dtype=t.dtype, device=t.device)
    b[:, 8:8 + t.shape[1]] = t
    return b[:, 8:8 + t.shape[1]]


@pytest.mark.parametrize("M", [1, 40, 300])
def test_rows_apart(vt, M):
    d, f = 136, 520
    x, Wg, Wu, Wd, dy = (t.cuda() for t in case(M, d, f, 5))
    saved = [torch.empty((M, 2 * f), device="cuda") for _ in range(2)]
    a, b = (vt.vt_gated_ffn(v, Wg, Wu, Wd, saved=s) for v, s in zip((x, wide(x)), saved))
    assert torch.equal(a, b) and torch.equal(*saved)
    one, two = vt.vt_gated_ffn_backward(x, Wg, Wu, Wd, saved[0], dy), vt.vt_gated_ffn_backward(wide(x), Wg, Wu, Wd, saved[1], wide(dy))
    assert all(torch.equal(p, q) for p, q in zip(one, two))
    if M > 1:                                       # from the second row on, 8 bytes off a 16-byte boundary
        with pytest.raises(vt.VtError) as e:
            vt.vt_gated_ffn(wide(x, 20), Wg, Wu, Wd)
        assert e.value.status == vt.VT_ERR_SHAPE


def test_gradients_against_differences(vt):
    """Along random directions, against central differences of the oracle's loss: see the scoring test for the tolerance."""
    M, d, f = 20, 64, 136
    rng = np.random.default_rng(6)
    for kind in ("silu", "gelu"):
        args = case(M, d, f, 7)
        x, Wg, Wu, Wd, dy = (t.cuda() for t in args)
        saved = torch.empty((M, 2 * f), device="cuda")
        vt.vt_gated_ffn(x, Wg, Wu, Wd, act=kind, saved=saved)
        grads = [f64(g) for g in vt.vt_gated_ffn_backward(x, Wg, Wu, Wd, saved, dy, act=kind)]
        base, up = [f64(t) for t in args[:4]], f64(args[4])
        for i, g in enumerate(grads):
            for _ in range(3):
                v = rng.normal(size=g.shape)
                ends = [(up * fo.forward(*[b + s * 1e-4 * v if j == i else b for j, b in enumerate(base)], kind)["y"]).sum() for s in (1, -1)]
                assert abs((ends[0] - ends[1]) / 2e-4 - (g * v).sum()) <= 0.01 * np.linalg.norm(g) * np.linalg.norm(v) / np.sqrt(g.size) + 1e-5


@pytest.mark.parametrize("M", [4, 60, 260])
def test_behind_late_producers_on_another_stream(vt, M):
    """Every operand written by the kernels just ahead, W_down (which the second product fetches early) last of all."""
    d, f = 256, 1024
    old, new = case(M, d, f, 8), case(M, d, f, 9)
    src = [t.cuda() for t in new]
    want = vt.vt_gated_ffn(*src[:4])
    saved = torch.empty((M, 2 * f), device="cuda")
    vt.vt_gated_ffn(*src[:4], saved=saved)
    want_grads = vt.vt_gated_ffn_backward(*src[:4], saved, src[4])
    for last in range(4):
        dst = [t.cuda() for t in old]
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            for i in [j for j in range(5) if j != last] + [last]:
                vt.vt_test_late_copy(dst[i], src[i], 200)
            got = vt.vt_gated_ffn(*dst[:4])
        side.synchronize()
        assert torch.equal(got, want), last
        dst = [t.cuda() for t in old]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for i in [j for j in range(5) if j != last] + [last]:
                vt.vt_test_late_copy(dst[i], src[i], 200)
            grads = vt.vt_gated_ffn_backward(*dst[:4], saved, dst[4])
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(grads, want_grads)), last


def test_in_a_graph_with_one_workspace(vt):
    M, d, f = 33, 256, 512
    ins = [[t.cuda() for t in case(M, d, f, s)[:4]] for s in (10, 11)]
    want = [vt.vt_gated_ffn(*i) for i in ins]
    ws = vt.new_workspace(vt.vt_gated_ffn_workspace_bytes(M, d, f))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [vt.vt_gated_ffn(*i, workspace=ws) for i in ins * 2]
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[i % 2]) for i, g in enumerate(got))


def test_offsets_past_32_bits(vt):
    """Weights of 2.2e9 elements each (d = 33000, f = 66000): features at their far end."""
    M, d, f = 2, 33000, 66000
    Wg = torch.zeros((f, d), dtype=torch.bfloat16, device="cuda")
    Wu, Wd = torch.zeros_like(Wg), torch.zeros((d, f), dtype=torch.bfloat16, device="cuda")
    x = torch.zeros((M, d), dtype=torch.bfloat16, device="cuda")
    x[:, 0], x[:, d - 1] = 1.0, torch.tensor([2.0, -1.0], device="cuda").bfloat16()
    for j in (0, 65071, 65072, f - 1):
        Wg[j, d - 1], Wu[j, 0], Wd[d - 1, j], Wd[3, j] = 1.5, 0.5 + (j % 7), 1.0, 0.25
    y = vt.vt_gated_ffn(x, Wg, Wu, Wd)
    g = 1.5 * x[:, d - 1].double()
    a = (g / (1 + torch.exp(-g)))[:, None] * torch.tensor([0.5 + (j % 7) for j in (0, 65071, 65072, f - 1)], device="cuda").double()[None]
    assert torch.allclose(y[:, d - 1].double(), a.sum(1), rtol=2.0 ** -6) and torch.allclose(y[:, 3].double(), 0.25 * a.sum(1), rtol=2.0 ** -6)
    assert (y[:, 4:d - 1] == 0).all() and (y[:, :3] == 0).all()
