"""The workloads the scoring and feed-forward operators are measured on, each with its plain form.

Two operators, each forward alone (serving) and forward with its gradient (training):

  score        log probabilities of given tokens under a head, with entropy, log-sum-exp and the k best alternatives
  score_train  the same without alternatives, then the gradients of hidden states and head weights
  ffn          the gated feed-forward block, y = (act(x Wg^T) * (x Wu^T)) Wd^T
  ffn_train    the same, then the gradients of its input and its three weights
"""
import math

import torch

own = False

_SILU, _GELU = "silu", "gelu"


def listed():
    return [
        # one draft token against the smallest trimmed head: nothing but latency
        {"name": "score 1 row, 4096 ids", "op": "score", "M": 1, "d": 2048, "V": 4096, "k": 8, "scale": 1.0, "ignored": 0.0},
        # a drafted tree checked against the trimmed head of the benchmark
        {"name": "score 33 rows, 32000 ids", "op": "score", "M": 33, "d": 4096, "V": 32000, "k": 8, "scale": 1.0, "ignored": 0.0},
        # several requests' drafted tokens verified by the full head, with the twenty alternatives a server reports
        {"name": "score 61 rows, 128256 ids", "op": "score", "M": 61, "d": 4096, "V": 128256, "k": 20, "scale": 0.8, "ignored": 0.0},
        # scoring a batch of prompts, padding among it
        {"name": "score 4096 rows, 32000 ids", "op": "score", "M": 4096, "d": 4096, "V": 32000, "k": 4, "scale": 1.0, "ignored": 0.1},
        # a ragged fine-tuning batch on the paper's trimmed vocabulary
        {"name": "score_train 255 rows, 13264", "op": "score_train", "M": 255, "d": 2048, "V": 13264, "k": 0, "scale": 1.0, "ignored": 0.2},
        # a full training batch of the benchmark's head
        {"name": "score_train 4096 rows, 32000", "op": "score_train", "M": 4096, "d": 4096, "V": 32000, "k": 0, "scale": 1.0, "ignored": 0.1},
        # one token through the block: the weights' bytes
        {"name": "ffn 1 row, 14336", "op": "ffn", "M": 1, "d": 4096, "f": 14336, "act": _SILU},
        # a drafted tree through the narrow block that the paper's FLOP table implies
        {"name": "ffn 60 rows, 2048", "op": "ffn", "M": 60, "d": 4096, "f": 2048, "act": _SILU},
        # a ragged prompt through a small block of odd sizes
        {"name": "ffn 777 rows, 2728", "op": "ffn", "M": 777, "d": 1000, "f": 2728, "act": _GELU},
        # a long prompt
        {"name": "ffn 4096 rows, 14336", "op": "ffn", "M": 4096, "d": 4096, "f": 14336, "act": _SILU},
        # a ragged fine-tuning batch
        {"name": "ffn_train 300 rows, 5504", "op": "ffn_train", "M": 300, "d": 2048, "f": 5504, "act": _GELU},
        # a full training batch
        {"name": "ffn_train 4096 rows, 14336", "op": "ffn_train", "M": 4096, "d": 4096, "f": 14336, "act": _SILU},
    ]


def _products(case):
    """Multiply-adds of the operator's matrix products, forward and backward."""
    if case["op"].startswith("score"):
        return case["M"] * case["d"] * case["V"] * (3 if case["op"] == "score_train" else 1)
    return case["M"] * case["d"] * case["f"] * (9 if case["op"] == "ffn_train" else 3)


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = max(_products(c) for c in listed())
    while True:
        op = rng.choice(["score", "score_train", "ffn", "ffn_train"])
        case = {"op": op, "M": spread(16 if op.endswith("train") else 1, 4096), "d": 8 * spread(64, 640)}
        if op.startswith("score"):
            case["V"] = spread(2000, 32768 if op == "score_train" else 131072)
            case["k"] = rng.randint(0, 20) if op == "score" else 0
            case["scale"] = rng.choice([1.0, rng.uniform(0.5, 1.5)])
            case["ignored"] = rng.choice([0.0, rng.uniform(0.0, 0.5)])
        else:
            case["f"] = 8 * spread(128, 1792)
            case["act"] = rng.choice([_SILU, _GELU])
        if _products(case) <= most:
            return case


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 2 + 1)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    M, d = case["M"], case["d"]
    if case["op"].startswith("score"):
        V = case["V"]
        # Head weights of deviation 0.02, hidden states of unit deviation that lean towards the row of the token that
        # comes next, by a different amount for each row: distributions from nearly flat to nearly certain.  Both lie on
        # a binary grid (8 significant bits at most, as bf16 has), on which fp32 sums are exact in every order: the
        # best ids and the ties among them are then the same for everybody.
        W = (normal(V, d) * (0.02 * 1024)).round().clamp(-255, 255) / 1024
        leading = torch.randint(V, (M,), device="cuda", generator=gen)
        lean = torch.rand(M, 1, device="cuda", generator=gen) * 12.0
        h = normal(M, d) + lean * W[leading] / (0.02 * math.sqrt(d))
        h = (h * 16).round().clamp(-255, 255) / 16
        other = torch.randint(V, (M,), device="cuda", generator=gen)
        tokens = torch.where(torch.rand(M, device="cuda", generator=gen) < 0.7, leading, other)
        tokens = torch.where(torch.rand(M, device="cuda", generator=gen) < case["ignored"], -1, tokens)
        state = {"case": case, "h": h.bfloat16(), "W": W.bfloat16(), "tokens": tokens.int()}
        if case["op"] == "score_train":
            # gradients of a mean over the rows, weighted as an advantage would, and of a small entropy bonus
            state["grad_logprobs"] = -normal(M).abs() / M
            state["grad_entropy"] = -0.01 * (1 + normal(M).abs()) / M
        return state
    f = case["f"]
    state = {"case": case, "x": normal(M, d).bfloat16()}
    state["W_gate"] = (normal(f, d) / math.sqrt(d)).bfloat16()
    state["W_up"] = (normal(f, d) / math.sqrt(d)).bfloat16()
    state["W_down"] = (normal(d, f) / math.sqrt(f)).bfloat16()
    if case["op"] == "ffn_train":
        state["grad_y"] = (normal(M, d) / M).bfloat16()
    return state


def run(state):
    op = state["case"]["op"]
    if own:
        return {"score": _score_own, "score_train": _score_train_own, "ffn": _ffn_own, "ffn_train": _ffn_train_own}[op](state)
    return {"score": _score, "score_train": _score_train, "ffn": _ffn, "ffn_train": _ffn_train}[op](state)


# ---------------------------------------------------------------------------------------------- the framework's calls
def _score_own(state):
    import paper_2603_05210_b200 as vt
    case = state["case"]
    h, W, k = state["h"], state["W"], case["k"]
    if "workspace" not in state:
        state["workspace"] = vt.new_workspace(vt.vt_score_workspace_bytes(h.shape[0], h.shape[1], W.shape[0], k))
    r = vt.vt_score_tokens(h, W, state["tokens"], k=k, scale=case["scale"], workspace=state["workspace"])
    out = {"logprobs": r.logprobs, "entropy": r.entropy, "lse": r.lse}
    if k:
        out |= {"top_ids": r.top_ids, "top_logprobs": r.top_logprobs}
    return out


def _score_train_own(state):
    import paper_2603_05210_b200 as vt
    h, W, tokens, scale = state["h"], state["W"], state["tokens"], state["case"]["scale"]
    if "workspace" not in state:
        M, d, V = *h.shape, W.shape[0]
        state["workspace"] = vt.new_workspace(max(vt.vt_score_workspace_bytes(M, d, V, 0),
                                                  vt.vt_score_backward_workspace_bytes(M, d, V)))
    r = vt.vt_score_tokens(h, W, tokens, scale=scale, workspace=state["workspace"])
    grad_h, grad_W = vt.vt_score_tokens_backward(h, W, tokens, r.lse, r.entropy, state["grad_logprobs"], state["grad_entropy"],
                                                 scale=scale, workspace=state["workspace"])
    return {"logprobs": r.logprobs, "entropy": r.entropy, "lse": r.lse, "grad_h": grad_h, "grad_W": grad_W}


def _weights(state):
    return state["W_gate"], state["W_up"], state["W_down"]


def _ffn_own(state):
    import paper_2603_05210_b200 as vt
    x, act = state["x"], state["case"]["act"]
    if "workspace" not in state:
        state["workspace"] = vt.new_workspace(vt.vt_gated_ffn_workspace_bytes(*x.shape, state["case"]["f"]))
    return {"y": vt.vt_gated_ffn(x, *_weights(state), act=act, workspace=state["workspace"])}


def _ffn_train_own(state):
    import paper_2603_05210_b200 as vt
    x, act, f = state["x"], state["case"]["act"], state["case"]["f"]
    if "workspace" not in state:
        state["workspace"] = vt.new_workspace(max(vt.vt_gated_ffn_workspace_bytes(*x.shape, f),
                                                  vt.vt_gated_ffn_backward_workspace_bytes(*x.shape, f)))
    saved = torch.empty((x.shape[0], 2 * f), dtype=torch.float32, device=x.device)
    y = vt.vt_gated_ffn(x, *_weights(state), act=act, saved=saved, workspace=state["workspace"])
    gx, gg, gu, gd = vt.vt_gated_ffn_backward(x, *_weights(state), saved, state["grad_y"], act=act, workspace=state["workspace"])
    return {"y": y, "grad_x": gx, "grad_W_gate": gg, "grad_W_up": gu, "grad_W_down": gd}


# ---------------------------------------------------------------------------------------------- the plain forms, in 32 bits
def _score_parts(state):
    x = state["h"].float() @ state["W"].float().T
    z = x * state["case"]["scale"]
    shifted = z - z.amax(1, keepdim=True)
    log_p = shifted - shifted.exp().sum(1, keepdim=True).log()
    p = log_p.exp()
    entropy = -(p * log_p).sum(1)
    lse = z.amax(1) + (shifted.exp().sum(1)).log()
    scored = state["tokens"] >= 0
    at = state["tokens"].long().clamp(min=0)[:, None]
    zero = torch.zeros_like(lse)
    out = {"logprobs": torch.where(scored, log_p.gather(1, at)[:, 0], zero), "entropy": torch.where(scored, entropy, zero),
           "lse": torch.where(scored, lse, zero)}
    return x, log_p, p, entropy, scored, at, out


def _score(state):
    x, log_p, _, _, scored, _, out = _score_parts(state)
    k = state["case"]["k"]
    if k:
        # the largest logits, the lower id first among equals: one whole number that orders both
        V = x.shape[1]
        bits = (x + 0.0).view(torch.int32).long()
        order = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF)) * V + torch.arange(V - 1, -1, -1, device=x.device)
        ids = V - 1 - order.topk(k, dim=1).values % V
        out["top_ids"] = torch.where(scored[:, None], ids, -1).int()
        out["top_logprobs"] = torch.where(scored[:, None], log_p.gather(1, ids), torch.zeros_like(log_p[:, :1]))
    return out


def _score_train(state):
    _, log_p, p, entropy, scored, at, out = _score_parts(state)
    gl = (state["grad_logprobs"] * scored)[:, None]
    ge = (state["grad_entropy"] * scored)[:, None]
    G = -gl * p - ge * p * (log_p + entropy[:, None])
    G.scatter_add_(1, at, gl)
    G *= state["case"]["scale"]
    out["grad_h"] = (G @ state["W"].float()).bfloat16()
    out["grad_W"] = (G.T @ state["h"].float()).bfloat16()
    return out


_C, _A = math.sqrt(2.0 / math.pi), 0.044715


def _act(g, act):
    if act == _SILU:
        return g / (1 + torch.exp(-g))
    return 0.5 * g * (1 + torch.tanh(_C * (g + _A * g * g * g)))


def _act_grad(g, act):
    if act == _SILU:
        s = 1 / (1 + torch.exp(-g))
        return s * (1 + g * (1 - s))
    t = torch.tanh(_C * (g + _A * g * g * g))
    return 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * _C * (1 + 3 * _A * g * g)


def _ffn_parts(state):
    x = state["x"].float()
    g, u = x @ state["W_gate"].float().T, x @ state["W_up"].float().T
    a = _act(g, state["case"]["act"]) * u
    return x, g, u, a, (a @ state["W_down"].float().T).bfloat16()


def _ffn(state):
    return {"y": _ffn_parts(state)[-1]}


def _ffn_train(state):
    act = state["case"]["act"]
    x, g, u, a, y = _ffn_parts(state)
    gy = state["grad_y"].float()
    ga = gy @ state["W_down"].float()
    gg, gu = ga * u * _act_grad(g, act), ga * _act(g, act)
    return {"y": y, "grad_x": (gg @ state["W_gate"].float() + gu @ state["W_up"].float()).bfloat16(),
            "grad_W_gate": (gg.T @ x).bfloat16(), "grad_W_up": (gu.T @ x).bfloat16(), "grad_W_down": (gy.T @ a).bfloat16()}


# ---------------------------------------------------------------------------------------------- work and exact values
def work(case):
    M, d = case["M"], case["d"]
    train = case["op"].endswith("train")
    if case["op"].startswith("score"):
        bytes_ = 2 * d * (M + case["V"]) * (2 if train else 1) + M * (16 + 8 * case["k"] + (8 if train else 0))
    else:
        bytes_ = 2 * d * (2 * M + 3 * case["f"]) * (2 if train else 1)
    return {"bytes": bytes_, "flops": 2 * _products(case)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("score"):
        return _score_exact(case, s)
    x, Wg, Wu, Wd = (s[n].double() for n in ("x", "W_gate", "W_up", "W_down"))
    g = torch.einsum("md,fd->mf", x, Wg)
    u = torch.einsum("md,fd->mf", x, Wu)
    if case["act"] == _SILU:
        sig = torch.sigmoid(g)
        value, slope = g * sig, sig + g * sig * torch.sigmoid(-g)
    else:
        inner = math.sqrt(2 / math.pi) * (g + 0.044715 * g.pow(3))
        value = g * torch.sigmoid(2 * inner)                       # (1 + tanh b) / 2 = sigmoid(2 b)
        slope = torch.sigmoid(2 * inner) + 2 * g * torch.sigmoid(2 * inner) * torch.sigmoid(-2 * inner) * \
            math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g.pow(2))
    out = {"y": torch.einsum("mf,df->md", value * u, Wd)}
    if case["op"] == "ffn_train":
        gy = s["grad_y"].double()
        ga = torch.einsum("md,df->mf", gy, Wd)
        dg, du = ga * u * slope, ga * value
        out |= {"grad_x": torch.einsum("mf,fd->md", dg, Wg) + torch.einsum("mf,fd->md", du, Wu),
                "grad_W_gate": torch.einsum("mf,md->fd", dg, x), "grad_W_up": torch.einsum("mf,md->fd", du, x),
                "grad_W_down": torch.einsum("md,mf->df", gy, value * u)}
    return out


def _score_exact(case, s):
    h, W, tokens, M = s["h"].double(), s["W"].double(), s["tokens"].long(), case["M"]
    keep = torch.nonzero(tokens >= 0)[:, 0]                        # the scored rows alone; the others stay neutral
    x = torch.einsum("md,vd->mv", h[keep], W)
    z = case["scale"] * x
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    H = lse - (p * z).sum(1)
    rows = torch.arange(len(keep), device=h.device)

    def whole(v, fill=0.0):
        r = torch.full((M, *v.shape[1:]), fill, dtype=v.dtype, device=v.device)
        r[keep] = v
        return r

    out = {"logprobs": whole(z[rows, tokens[keep]] - lse), "entropy": whole(H), "lse": whole(lse)}
    if case["op"] == "score_train":
        gl, ge = s["grad_logprobs"].double()[keep, None], s["grad_entropy"].double()[keep, None]
        hot = torch.zeros_like(p)
        hot[rows, tokens[keep]] = 1.0
        G = case["scale"] * (gl * (hot - p) - ge * p * (z - lse[:, None] + H[:, None]))
        out |= {"grad_h": whole(torch.einsum("mv,vd->md", G, W)), "grad_W": torch.einsum("mv,md->vd", G, h[keep])}
    elif case["k"]:
        best, ids = torch.sort(x, dim=1, descending=True, stable=True)
        out["top_ids"] = whole(ids[:, :case["k"]].int(), -1)
        out["top_logprobs"] = whole(case["scale"] * best[:, :case["k"]] - lse[:, None])
    return out
