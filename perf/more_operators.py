"""The workloads the operators of a draft layer's decode step are measured on, each with its plain form.

  rope     rotary positions of queries and keys in training: the forward pass, then the gradients' way back
  append   the same in serving: queries rotated, keys rotated into a paged cache, values copied beside them
  attend   attention of drafted tokens (a tree of them, a chain, or one alone) over a paged cache that holds them at its end
  verify   which drafted tokens stay, given the target's probabilities and random numbers, and the token that follows them
"""
import math
import random

import torch

own = False


def listed():
    return [
        # a ragged fine-tuning batch of a small draft, half of each head rotated, pairs side by side
        {"name": "rope 300 tokens", "op": "rope", "B": 3, "T": 130, "ragged": True, "L": 900, "Hq": 32, "Hkv": 32, "D": 64, "rot": 32,
         "interleaved": True, "scaling": "none", "factor": 1.0},
        # a full training batch at the target's head layout and its long-context frequencies
        {"name": "rope 8192 tokens", "op": "rope", "B": 2, "T": 4096, "ragged": False, "L": 0, "Hq": 32, "Hkv": 8, "D": 128, "rot": 128,
         "interleaved": False, "scaling": "wavelength", "factor": 8.0},
        # one token of one request: nothing but latency
        {"name": "append 1 token", "op": "append", "B": 1, "T": 1, "ragged": False, "L": 700, "Hq": 32, "Hkv": 8, "D": 128, "rot": 128,
         "interleaved": False, "scaling": "none", "factor": 1.0, "page": 16},
        # a prompt's chunk behind a long context
        {"name": "append 4099 tokens", "op": "append", "B": 1, "T": 4099, "ragged": False, "L": 120000, "Hq": 32, "Hkv": 8, "D": 128, "rot": 128,
         "interleaved": False, "scaling": "ramp", "factor": 16.0, "page": 64},
        # the draft's own step: one token after a short prompt
        {"name": "attend 1 x 1 over 700", "op": "attend", "B": 1, "T": 1, "ragged": False, "L": 700, "Hq": 32, "Hkv": 8, "D": 128, "page": 16, "tree": False},
        # one request's drafted tree under the target
        {"name": "attend 1 x 60 over 4000", "op": "attend", "B": 1, "T": 60, "ragged": False, "L": 4000, "Hq": 32, "Hkv": 8, "D": 128, "page": 16, "tree": True},
        # many requests, a token each, none as long as another
        {"name": "attend 64 x 1 over 4096", "op": "attend", "B": 64, "T": 1, "ragged": True, "L": 4096, "Hq": 32, "Hkv": 8, "D": 128, "page": 64, "tree": False},
        # a small draft with a key head for every query head, chains of up to eight tokens
        {"name": "attend 24 x 8 over 2500", "op": "attend", "B": 24, "T": 8, "ragged": True, "L": 2500, "Hq": 32, "Hkv": 32, "D": 64, "page": 32, "tree": False},
        # a server's batch of drafted trees
        {"name": "attend 16 x 60 over 8000", "op": "attend", "B": 16, "T": 60, "ragged": True, "L": 8000, "Hq": 32, "Hkv": 8, "D": 128, "page": 64, "tree": True},
        # two long documents
        {"name": "attend 2 x 8 over 100000", "op": "attend", "B": 2, "T": 8, "ragged": False, "L": 100000, "Hq": 32, "Hkv": 8, "D": 128, "page": 128, "tree": True},
        # one request's chain, drawn from the draft's distribution over the trimmed vocabulary of the benchmark
        {"name": "verify 1 x 5, drawn", "op": "verify", "B": 1, "T": 6, "ragged": False, "V": 128256, "Vd": 32000, "tree": False},
        # a server's batch of trees of best candidates
        {"name": "verify 16 x 60, best", "op": "verify", "B": 16, "T": 60, "ragged": True, "V": 128256, "Vd": 0, "tree": True},
    ]


def _sizes(case):
    """Tokens and cached tokens of each request. They belong to the case: another seed has the same."""
    r = random.Random(str(sorted((k, v) for k, v in case.items() if k != "name")))
    B, T, L = case["B"], case["T"], case.get("L", 0)
    if not case["ragged"]:
        return [T] * B, [L] * B
    return [T] + [r.randint(1, T) for _ in range(B - 1)], [L] + [r.randint(0, L) for _ in range(B - 1)]


def _cost(case):
    """Bytes and multiply-adds of one pass."""
    lens, cached = _sizes(case)
    N = sum(lens)
    if case["op"] == "verify":
        return case["B"] * (4 * case["V"] + 8 * case["Vd"]) + 12 * N, case["B"] * (case["V"] + case["Vd"])
    D, Hq, Hkv = case["D"], case["Hq"], case["Hkv"]
    if case["op"] == "rope":
        return 2 * 4 * N * (Hq + Hkv) * D, 2 * 2 * N * (Hq + Hkv) * case["rot"]
    if case["op"] == "append":
        return 4 * N * (Hq + 2 * Hkv) * D, 2 * N * (Hq + Hkv) * case["rot"]
    keys = sum(c + t for c, t in zip(cached, lens))
    return 4 * keys * Hkv * D + 4 * N * Hq * D + 4 * N * Hq, sum(2 * (c + t) * t for c, t in zip(cached, lens)) * Hq * D


def work(case):
    bytes_, products = _cost(case)
    return {"bytes": bytes_, "flops": 2 * products}


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["rope", "append", "attend", "attend", "verify"])
        case = {"op": op, "B": spread(1, 64), "ragged": rng.random() < 0.7}
        if op == "verify":
            case |= {"T": rng.randint(1, 64), "V": spread(4000, 131072), "tree": rng.random() < 0.5}
            case["Vd"] = 0 if rng.random() < 0.5 else spread(1000, min(case["V"], 32768))
            if case["B"] * case["T"] * (case["V"] + case["Vd"]) > 16 * 60 * 128256:
                continue
            return case
        Hkv = rng.choice([1, 2, 4, 8, 16, 32])
        case |= {"Hkv": Hkv, "Hq": Hkv * rng.choice([1, 2, 3, 4, 5, 8]), "D": rng.choice([64, 128])}
        if op == "attend":
            case |= {"T": rng.choice([1, spread(1, 64)]), "L": spread(16, 100000), "page": rng.choice([16, 32, 64, 128]), "tree": rng.random() < 0.5}
        else:
            case |= {"T": spread(1, 4096), "L": spread(16, 120000), "rot": 16 * rng.randint(1, case["D"] // 16), "interleaved": rng.random() < 0.5,
                     "scaling": rng.choice(["none", "linear", "base", "wavelength", "ramp"]), "factor": rng.choice([2.0, 4.0, 8.0, 32.0])}
            if case["scaling"] == "none":
                case["factor"] = 1.0
            if op == "append":
                case["page"] = rng.choice([16, 32, 64, 128])
        if case["Hq"] > 64 or (op != "attend" and case["B"] * case["T"] * (case["Hq"] + 2 * Hkv) * case["D"] > 8192 * 48 * 128):
            continue
        largest = [c for c in listed() if c["op"] == op]
        if all(a <= max(b) for a, b in zip(_cost(case), zip(*(_cost(c) for c in largest)))):
            if op == "attend" and case["B"] * case["L"] * max(case["Hkv"] * case["D"], case["Hq"] * case["T"]) > 16 * 8000 * 32 * 64:
                continue                                           # the plain form lays every request out at the longest one's length
            return case


# ---------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 2 + 1)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    lens, cached = _sizes(case)
    B, T, N = case["B"], case["T"], sum(lens)
    cu = torch.tensor([0] + lens, dtype=torch.int32).cumsum(0).int().cuda()
    state = {"case": case, "cu": cu, "N": N}
    if case["op"] == "verify":
        return _prepare_verify(case, state, lens, gen)
    cached = torch.tensor(cached, dtype=torch.int32, device="cuda")
    request = torch.repeat_interleave(torch.arange(B, device="cuda"), torch.tensor(lens, device="cuda"))
    within = torch.arange(N, device="cuda") - cu[request]
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    if case["op"] in ("rope", "append"):
        state["positions"] = (cached[request] + within).int()
        # what a fused projection leaves: queries, keys and values of a token side by side
        heads = normal(N, Hq + 2 * Hkv, D).bfloat16()
        state["q"], state["k"], state["v"] = heads[:, :Hq], heads[:, Hq:Hq + Hkv], heads[:, Hq + Hkv:]
        if case["op"] == "rope":
            state["grad_q"], state["grad_k"] = (normal(N, Hq, D) / N).bfloat16(), (normal(N, Hkv, D) / N).bfloat16()
            return state
        cached %= 4 * case["page"]                                 # the cache holds the end of each context: its pages are what matters
    state["lens"], state["request"], state["within"] = cached, request, within
    page = case["page"]
    used = ((cached.cpu() + torch.tensor(lens) + page - 1) // page).tolist()
    order = torch.randperm(sum(used) + 3, device="cuda", generator=gen).int()
    table = torch.full((B, max(used)), -1, dtype=torch.int32, device="cuda")
    owner = torch.repeat_interleave(torch.arange(B), torch.tensor(used)).cuda()
    first = torch.tensor([0] + used).cumsum(0)[:-1].cuda()
    at = torch.arange(sum(used), device="cuda")
    table[owner, at - first[owner]] = order[:sum(used)]
    state["table"] = table
    shape = (sum(used) + 3, page, Hkv, D)
    if case["op"] == "append":
        state["k_cache"], state["v_cache"] = (torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        return state
    state["k_cache"] = torch.randn(shape, device="cuda", generator=gen, dtype=torch.bfloat16)
    state["v_cache"] = torch.randn(shape, device="cuda", generator=gen, dtype=torch.bfloat16)
    # some heads look at few positions, some at nearly all
    state["q"] = (normal(N, Hq, D) * (0.3 + 2.2 * torch.rand(N, Hq, 1, device="cuda", generator=gen))).bfloat16()
    state["max_tokens"], state["scale"] = T, D ** -0.5
    if case["tree"]:
        # token t's parent is one of the eight before it (token 0 stands for the last token that is certain)
        back = (torch.rand(N, device="cuda", generator=gen) * 8).long() + 1
        state["parents"] = (within - back).clamp(min=0).masked_fill(within == 0, -1).int()
        state["mask"] = _tree_mask(state["parents"], request, within, cu, T)
    return state


def _ancestors(parents, request, cu):
    """[N, N] truth values: whether the second token is the first or lies on its way to the root; doubling steps along the way."""
    N = len(parents)
    eye = torch.eye(N, dtype=torch.bool, device=parents.device)
    step = eye.float()
    up = (cu[request] + parents).long()
    has = parents >= 0
    step[has, up[has]] = 1.0                                       # itself and its parent
    for _ in range(max(1, (N - 1).bit_length())):
        step = ((step @ step) > 0).float()
    return step > 0


def _tree_mask(parents, request, within, cu, T):
    """Bit u % 32 of word u / 32 of a token's row: the token attends token u of its request."""
    N, words = len(parents), (T + 31) // 32
    anc = _ancestors(parents, request, cu)
    first = cu[request].long()[:, None]
    u = torch.arange(words * 32, device=parents.device)
    inside = first + u < N
    same = inside & (request[(first + u).clamp(max=N - 1)] == request[:, None])
    bits = (anc.gather(1, (first + u).clamp(max=N - 1)) & same).view(N, words, 32).long()
    value = (bits << torch.arange(32, device=parents.device)).sum(2)
    return torch.where(value >= 2 ** 31, value - 2 ** 32, value).int()


def _prepare_verify(case, state, lens, gen):
    B, T, V, Vd, N = case["B"], case["T"], case["V"], case["Vd"], state["N"]
    cu = state["cu"]

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=gen)

    request = torch.repeat_interleave(torch.arange(B, device="cuda"), torch.tensor(lens, device="cuda"))
    within = torch.arange(N, device="cuda") - cu[request]
    back = (uniform(N) * 8).long() + 1 if case["tree"] else torch.ones(N, dtype=torch.long, device="cuda")
    parents = (within - back).clamp(min=0).masked_fill(within == 0, -1).int()
    # the target's logits: a broad floor and a few tokens that stand out, more or less
    z = torch.randn(N, V, device="cuda", generator=gen) * 2.0
    peaks = torch.randint(Vd or V, (N, 6), device="cuda", generator=gen)
    d2t = torch.randperm(V, device="cuda", generator=gen)[:Vd].int() if Vd else None
    z.scatter_(1, d2t[peaks].long() if Vd else peaks, 8.0 + 8.0 * uniform(N, 6))
    up = (cu[request] + parents.clamp(min=0)).long()
    state |= {"request": request, "within": within, "parents": parents, "u_accept": uniform(N), "u_sample": uniform(B), "max_tokens": T}
    if Vd:
        q = torch.softmax(z[:, d2t.long()] + 0.7 * torch.randn(N, Vd, device="cuda", generator=gen), 1)
        drafted = torch.multinomial(q[up], 1, generator=gen)[:, 0].int()
        state |= {"draft_probs": q, "draft_ids": drafted, "d2t": d2t, "tokens": d2t[drafted.long()]}
    else:
        # the r-th child of a node holds the r-th best candidate after it, as the draft saw it
        siblings = (up[:, None] == up[None, :]) & (parents >= 0)[None, :] & (parents >= 0)[:, None]
        rank = torch.tril(siblings, -1).sum(1)
        best = (z + torch.randn(N, V, device="cuda", generator=gen)).topk(min(V, 64), dim=1).indices
        state["tokens"] = best[up, rank.clamp(max=best.shape[1] - 1)].int()
    state["probs"] = torch.softmax(z, 1)
    return state


# ---------------------------------------------------------------------------------------------- one pass
def run(state):
    op = state["case"]["op"]
    if own:
        return {"rope": _rope_own, "append": _append_own, "attend": _attend_own, "verify": _verify_own}[op](state)
    return {"rope": _rope, "append": _append, "attend": _attend, "verify": _verify}[op](state)


def _rope_plan(state):
    import paper_2603_05210_b200 as vt
    if "rope" not in state:
        c = state["case"]
        state["rope"] = vt.vt_rope_table(c["rot"], interleaved=c["interleaved"], scaling=c["scaling"], factor=c["factor"])
    return vt, state["rope"]


def _rope_own(state):
    vt, rope = _rope_plan(state)
    q, k = vt.vt_rope(state["q"], state["k"], state["positions"], rope)
    grad_q, grad_k = vt.vt_rope(state["grad_q"], state["grad_k"], state["positions"], rope, inverse=True)
    return {"q": q, "k": k, "grad_q": grad_q, "grad_k": grad_k}


def _cache_own(state):
    import paper_2603_05210_b200 as vt
    if "cache" not in state:
        state["cache"] = vt.VtCache(state["k_cache"], state["v_cache"], state["table"], state["lens"])
    return state["cache"]


def _append_own(state):
    vt, rope = _rope_plan(state)
    cache = _cache_own(state)
    q = vt.vt_rope_append(state["q"], state["k"], state["v"], state["positions"], state["cu"], cache, rope)
    return {"q": q, "k_cache": cache.k, "v_cache": cache.v}


def _attend_own(state):
    import paper_2603_05210_b200 as vt
    cache = _cache_own(state)
    if "workspace" not in state:
        c = state["case"]
        state["workspace"] = vt.new_workspace(vt.vt_tree_attention_workspace_bytes(c["Hq"], c["Hkv"], c["D"], state["max_tokens"]))
    out, lse = vt.vt_tree_attention(state["q"], state["cu"], cache, max_tokens=state["max_tokens"], mask=state.get("mask"), scale=state["scale"],
                                    workspace=state["workspace"])
    return {"out": out, "lse": lse}


def _verify_own(state):
    import paper_2603_05210_b200 as vt
    r = vt.vt_verify_tokens(state["probs"], state["tokens"], state["parents"], state["cu"], state["u_accept"], state["u_sample"],
                            max_tokens=state["max_tokens"], draft_probs=state.get("draft_probs"), draft_ids=state.get("draft_ids"), d2t=state.get("d2t"))
    return {"n_accepted": r.n_accepted, "path": r.path, "tokens": r.tokens}


# ---------------------------------------------------------------------------------------------- the plain forms
_BASE, _ORIGINAL = 10000.0, 8192.0                                 # the defaults of the table: base, length of the first training


def _frequencies(case, device):
    """Radians per position of each pair, in 64 bits, and the factor that some scalings put on the result."""
    rot, s = case["rot"], case["factor"]
    i = torch.arange(rot // 2, dtype=torch.float64, device=device)
    base = _BASE * s ** (rot / (rot - 2)) if case["scaling"] == "base" and rot > 2 else _BASE
    w = base ** (-2 * i / rot)
    if case["scaling"] == "linear":
        w = w / s
    elif case["scaling"] == "wavelength":
        turns = _ORIGINAL * w / (2 * math.pi)                      # full turns over the first training's length
        w = w / s + (w - w / s) * ((turns - 1.0) / (4.0 - 1.0)).clamp(0, 1)
    elif case["scaling"] == "ramp":
        pair = lambda turns: rot * math.log(_ORIGINAL / (turns * 2 * math.pi)) / (2 * math.log(_BASE))  # noqa: E731
        lo, hi = max(math.floor(pair(32.0)), 0), min(math.ceil(pair(1.0)), rot - 1)
        w = w + (w / s - w) * ((i - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
    return w, 0.1 * math.log(s) + 1.0 if case["scaling"] == "ramp" else 1.0


def _rotated(x, positions, case, sign):
    w, amplitude = _frequencies(case, x.device)
    angle = positions.double()[:, None] * w                        # in 64 bits: far positions turn often
    c, s = (angle.cos() * amplitude).float()[:, None], (angle.sin() * amplitude * sign).float()[:, None]
    x, rot = x.float(), case["rot"]
    y = x.clone()
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y.bfloat16()


def _rope(state):
    c, at = state["case"], state["positions"]
    return {"q": _rotated(state["q"], at, c, 1), "k": _rotated(state["k"], at, c, 1),
            "grad_q": _rotated(state["grad_q"], at, c, -1), "grad_k": _rotated(state["grad_k"], at, c, -1)}


def _append(state):
    c, at = state["case"], state["positions"]
    where = (state["lens"][state["request"]] + state["within"]).long()
    page = state["table"][state["request"], where // c["page"]].long()
    state["k_cache"][page, where % c["page"]] = _rotated(state["k"], at, c, 1)
    state["v_cache"][page, where % c["page"]] = state["v"]
    return {"q": _rotated(state["q"], at, c, 1), "k_cache": state["k_cache"], "v_cache": state["v_cache"]}


def _laid_out(state):
    """Keys and values [B, Hkv, Lm, D] and queries [B, Hkv, T G, D] in 32 bits, and what attends what [B, T, Lm]."""
    c, cu, lens = state["case"], state["cu"].long(), state["lens"].long()
    B, T, Hq, Hkv, D, page = c["B"], c["T"], c["Hq"], c["Hkv"], c["D"], c["page"]
    count = cu[1:] - cu[:-1]
    Lm = state["table"].shape[1] * page
    i = torch.arange(Lm, device=cu.device)
    at = state["table"].long().clamp(min=0)[:, i // page], i % page
    k, v = (state[n][at].float().transpose(1, 2) for n in ("k_cache", "v_cache"))
    t = torch.arange(T, device=cu.device)
    row = (cu[:-1, None] + t).clamp(max=state["N"] - 1)
    q = state["q"][row].float().view(B, T, Hkv, Hq // Hkv, D).transpose(1, 2).reshape(B, Hkv, T * (Hq // Hkv), D)
    u = i[None] - lens[:, None]
    if c["tree"]:
        words = state["mask"][row].long()
        word = words.gather(2, (u.clamp(0, T - 1) // 32)[:, None].expand(B, T, Lm))
        drafted = (word >> (u.clamp(min=0) % 32)[:, None] & 1) > 0
    else:
        drafted = u[:, None] <= t[None, :, None]
    u, count = u[:, None], count[:, None, None]
    return q, k, v, ((u < 0) | drafted & (u < count)) & (t[None, :, None] < count), row, t[None] < count[:, 0]


def _attend(state):
    c = state["case"]
    G = c["Hq"] // c["Hkv"]
    q, k, v, attends, row, real = _laid_out(state)
    x = (q @ k.transpose(2, 3)) * state["scale"]
    x = x.view(c["B"], c["Hkv"], c["T"], G, -1).masked_fill_(~attends[:, None, :, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)                # a row that attends nothing: every term 0
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(c["B"], c["Hkv"], c["T"] * G, -1) @ v).view(c["B"], c["Hkv"], c["T"], G, -1) / total.clamp(min=1e-38)
    lse = torch.where(total > 0, top + total.log(), -math.inf)[..., 0]
    out = o.permute(0, 2, 1, 3, 4).reshape(c["B"], c["T"], c["Hq"], -1)[real]
    return {"out": out.bfloat16(), "lse": lse.permute(0, 2, 1, 3).reshape(c["B"], c["T"], c["Hq"])[real]}


def _verify(state):
    c, P, cu = state["case"], state["probs"], state["cu"].long()
    B, T, V, N = c["B"], c["T"], c["V"], state["N"]
    device, request, within = P.device, state["request"], state["within"]
    tokens, child = state["tokens"].long(), state["parents"] >= 0
    up = (cu[request] + state["parents"].clamp(min=0)).long()
    siblings = (up[:, None] == up[None, :]) & child[None, :] & child[:, None]
    before = torch.tril(siblings, -1)                              # [n, m]: m is an earlier child of n's parent
    rank = before.sum(1)
    u, p = state["u_accept"].double(), P[up, tokens].double()
    if c["Vd"]:
        # what is left after j rejections is max(p - S q, 0), S the sum of what was left before each of them
        Q = torch.zeros(N, V, device=device)
        Q[:, state["d2t"].long()] = state["draft_probs"]
        q = state["draft_probs"][up, state["draft_ids"].long()].double()
        S, Z = torch.zeros(N, dtype=torch.float64, device=device), torch.ones(N, dtype=torch.float64, device=device)
        accepts = torch.zeros(N, dtype=torch.bool, device=device)
        most = int(rank[child].max()) + 1 if bool(child.any()) else 0
        for j in range(most):                                      # S and Z of each node, after j of its children
            now = child & (rank == j)
            accepts[now] = (u * q * Z[up] < (p - S[up] * q).clamp(min=0))[now]
            has = torch.zeros(N, dtype=torch.bool, device=device)
            has[up[now]] = True
            S = torch.where(has, S + Z, S)
            rows = has.nonzero()[:, 0]
            Z[rows] = (P[rows].double() - S[rows, None] * Q[rows].double()).clamp(min=0).sum(1)
    else:
        again = (before & (tokens[:, None] == tokens[None, :])).any(1)
        p = p.masked_fill(again, 0.0)                              # a token that was turned down once has nothing left
        accepts = child & (p > 0) & (u * (1.0 - (before.double() * p[None]).sum(1)) < p)
    chosen = accepts & ~(before & accepts[None, :]).any(1)         # the first child that is accepted
    on_path = ((chosen | ~child)[None, :] | ~_ancestors(state["parents"], request, cu)).all(1)
    n = torch.zeros(B, dtype=torch.long, device=device).scatter_add_(0, request, (on_path & child).long())
    order = torch.where(on_path & child, within, T).long()
    path = torch.full((B, T), T, device=device)
    path[request, within] = order
    path = path.sort(1).values
    last = cu[:-1] + torch.where(n > 0, path.gather(1, (n - 1).clamp(min=0)[:, None])[:, 0], 0)
    left = P[last].double()
    if c["Vd"]:
        left = (left - S[last, None] * Q[last].double()).clamp(min=0)
    else:
        dead = child & (up == last[request])
        left[request[dead], tokens[dead]] = 0.0
    left = torch.where(left.sum(1, keepdim=True) > 0, left, P[last].double())
    cum = left.cumsum(1)
    y = torch.searchsorted(cum, state["u_sample"].double()[:, None] * cum[:, -1:], right=True)[:, 0].clamp(max=V - 1)
    j = torch.arange(T, device=device)[None]
    taken = tokens[(cu[:-1, None] + path).clamp(max=N - 1)]
    out = torch.where(j < n[:, None], taken, torch.where(j == n[:, None], y[:, None], -1))
    return {"n_accepted": n.int(), "path": torch.where(j < n[:, None], path, -1).int(), "tokens": out.int()}


# ---------------------------------------------------------------------------------------------- exact values
def exact(case, seed):
    if case["op"] == "verify":
        return None                                                # whole numbers: equal or not
    s = prepare(case, seed)
    if case["op"] == "attend":
        return _attend_exact(case, s)
    at = s["positions"]
    if case["op"] == "rope":
        return {"q": _turned(s["q"], at, case, False), "k": _turned(s["k"], at, case, False),
                "grad_q": _turned(s["grad_q"], at, case, True), "grad_k": _turned(s["grad_k"], at, case, True)}
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    flat = s["lens"].long()[s["request"]] + s["within"]
    slot = s["table"].long()[s["request"], flat.div(case["page"], rounding_mode="floor")] * case["page"] + flat.remainder(case["page"])
    k_cache.view(-1, *k_cache.shape[2:])[slot] = _turned(s["k"], at, case, False)
    v_cache.view(-1, *v_cache.shape[2:])[slot] = s["v"].double()
    return {"q": _turned(s["q"], at, case, False), "k_cache": k_cache, "v_cache": v_cache}


def _turned(x, positions, case, back):
    """Pairs as complex numbers, turned by the angle (or back)."""
    rot, s, kind = case["rot"], case["factor"], case["scaling"]
    pairs = torch.arange(0, rot, 2, dtype=torch.float64, device=x.device) / rot
    first = torch.exp(-pairs * math.log(10000.0))
    if kind == "base" and rot > 2:
        w = torch.exp(-pairs * (math.log(10000.0) + math.log(s) * rot / (rot - 2)))
    elif kind == "linear":
        w = first * (1 / s)
    elif kind == "wavelength":
        length = 2 * math.pi / first                               # in positions; long ones are stretched, short ones are not
        share = ((8192.0 / length - 1) / 3).clamp(0, 1)
        w = (1 - share) * first / s + share * first
    elif kind == "ramp":
        edge = [rot / 2 * math.log(8192.0 / (2 * math.pi * t)) / math.log(10000.0) for t in (32, 1)]
        lo, hi = max(int(math.floor(edge[0])), 0), min(int(math.ceil(edge[1])), rot - 1)
        share = ((pairs * rot / 2 - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        w = first * (1 - share) + first / s * share
    else:
        w = first
    size = 1 + math.log(s) / 10 if kind == "ramp" else 1.0
    turn = torch.polar(torch.full_like(w, size).expand(len(positions), -1), (-1.0 if back else 1.0) * positions.double()[:, None] * w)
    y = x.double().clone()
    part = y[..., :rot]
    two = part.unflatten(-1, (rot // 2, 2)) if case["interleaved"] else part.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
    z = torch.view_as_real(torch.complex(two[..., 0], two[..., 1]) * turn[:, None])
    y[..., :rot] = (z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2)
    return y


def _attend_exact(case, s):
    """Request by request, each at its own length."""
    cu, lens, page, G = s["cu"].tolist(), s["lens"].tolist(), case["page"], case["Hq"] // case["Hkv"]
    outs, lses = [], []
    for b in range(case["B"]):
        n, L = cu[b + 1] - cu[b], lens[b]
        i = torch.arange(L + n, device="cuda")
        slot = s["table"][b, i // page].long() * page + i % page
        k = s["k_cache"].flatten(0, 1)[slot].double().repeat_interleave(G, 1)
        v = s["v_cache"].flatten(0, 1)[slot].double().repeat_interleave(G, 1)
        x = torch.einsum("thd,ihd->hti", s["q"][cu[b]:cu[b + 1]].double(), k) * s["scale"]
        if case["tree"]:
            sees = torch.eye(n, dtype=torch.bool, device="cuda")
            for t, p in enumerate(s["parents"][cu[b]:cu[b + 1]].tolist()):
                if p >= 0:
                    sees[t] |= sees[p]
        else:
            sees = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
        x[:, :, L:][:, ~sees] = -math.inf
        lse = torch.logsumexp(x, 2)
        outs.append(torch.einsum("hti,ihd->thd", torch.exp(x - lse[..., None]), v))
        lses.append(lse.T)
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
