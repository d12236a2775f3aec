"""Performance cases of the operators around the adapters' products: token embeddings and their gradient, rows sent to experts (or
adapters) chosen by a router and brought back with weights, with the gradients of both, and the clipped policy loss with its gradient.

`run` computes them in their plain form, elementary torch operations in 32 bits, or, where `own` is true, through the
framework's entry points.  A pass is what a training loop or a server calls at that point of a step.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}
CLIP_LOW, CLIP_HIGH, BETA = 0.2, 0.28, 0.04
PADDING = 0.03  # share of rows that are padding


def listed():
    return [
        # The token that a server has just generated for one request.  Latency.
        dict(name="embedding_one_token", op="embedding", rows=1, vocabulary=32000, d=4096, type="bfloat16", out="bfloat16"),
        # Prompts of a batch, over a vocabulary of an odd size.
        dict(name="embedding_prompts", op="embedding", rows=8001, vocabulary=50001, d=4096, type="bfloat16", out="bfloat16"),
        # One step's tokens: the whole gradient of a table, zeros where no token was.
        dict(name="embedding_backward_vocabulary", op="embedding_backward", rows=32768, vocabulary=50001, d=1024, type="bfloat16",
             grad="float32", accumulate=False),
        # One micro-batch of several, added to the gradient of a large table: only the rows of its tokens are touched.
        dict(name="embedding_backward_micro_batch", op="embedding_backward", rows=8192, vocabulary=131072, d=2048, type="bfloat16",
             grad="float32", accumulate=True),
        # One generated row and its four experts of 64.  Latency.
        dict(name="dispatch_one_row", op="dispatch", rows=1, experts=64, k=4, d=4096, logits="float32", type="bfloat16", normalise=True),
        # A training batch and its eight experts of 128.
        dict(name="dispatch_batch", op="dispatch", rows=8192, experts=128, k=8, d=4096, logits="float32", type="bfloat16", normalise=True),
        # Requests that each generate their next row, back from two experts each.
        dict(name="combine_48_requests", op="combine", rows=48, experts=8, k=2, d=4096, type="bfloat16", out="bfloat16"),
        # That training batch back from its experts.
        dict(name="combine_batch", op="combine", rows=8192, experts=128, k=8, d=4096, type="bfloat16", out="bfloat16"),
        # A training step backward through the return, the router and the dispatch: ragged sizes, weights over all experts.
        dict(name="route_backward_ragged", op="route_backward", rows=1003, experts=23, k=3, d=1023, logits="bfloat16", type="bfloat16",
             normalise=False),
        # The same of a batch with four experts of 64.
        dict(name="route_backward_batch", op="route_backward", rows=8192, experts=64, k=4, d=4096, logits="float32", type="bfloat16",
             normalise=True),
        # The loss of a policy over few actions: many short rows.
        dict(name="policy_128_actions", op="policy", rows=32768, K=128, type="float32", grad="bfloat16", reference=False),
        # The loss of a language model's policy over a large vocabulary, held near a reference.
        dict(name="policy_vocabulary", op="policy", rows=4096, K=50001, type="bfloat16", grad="bfloat16", reference=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["embedding", "embedding_backward", "dispatch", "combine", "route_backward", "policy"])
    kind = ["float32", "bfloat16"]
    if op in ("embedding", "embedding_backward"):
        back = op == "embedding_backward"
        d = _log(rng, 16, 8192)
        if rng.random() < 0.75:
            d = d // 8 * 8  # mostly multiples of eight
        V = _log(rng, 100, min(262144, (50_000_000 if back else 200_000_000) // d))
        case = dict(op=op, rows=_log(rng, 1, min(65536, 32_000_000 // d)), vocabulary=V, d=d, type=rng.choice(kind))
        if back:
            case.update(grad=rng.choice(kind), accumulate=rng.random() < 0.4)
        else:
            case["out"] = rng.choice(kind)
        return case
    if op == "policy":
        K = _log(rng, 2, 131072)
        return dict(op="policy", rows=_log(rng, 1, max(1, min(65536, 4096 * 50001 // K))), K=K, type=rng.choice(kind), grad=rng.choice(kind),
                    reference=rng.random() < 0.5)
    experts = _log(rng, 2, 512)
    k = _log(rng, 1, min(experts, 16))
    d = _log(rng, 16, 8192)
    if rng.random() < 0.75:
        d = d // 8 * 8
    most = 120_000_000 // (d * k) if op != "route_backward" else 60_000_000 // (d * k)
    case = dict(op=op, rows=_log(rng, 1, max(1, min(65536, most, (1 << 24) // experts))), experts=experts, k=k, d=d, type=rng.choice(kind))
    if op == "combine":
        case["out"] = rng.choice(kind)
    else:
        case.update(logits=rng.choice(kind), normalise=rng.random() < 0.5)
    return case


# ------------------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _normal(g, shape, std, dtype):
    return torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float32).mul_(std).to(dtype)


def _law(V):
    """Probabilities of a vocabulary's tokens, the most frequent first."""
    p = 1.0 / (np.arange(V, dtype=np.float64) + 2.7)
    return p / p.sum()


def _tokens(g, T, V):
    """Tokens by that law, frequent ones anywhere in the table, some of them padding."""
    edges = torch.from_numpy(np.cumsum(_law(V))).to(DEVICE)
    u = torch.rand((T,), generator=g, device=DEVICE, dtype=torch.float64)
    at = torch.searchsorted(edges, u).clamp_(max=V - 1)
    tokens = torch.randperm(V, generator=g, device=DEVICE)[at].to(torch.int32)
    tokens[torch.rand((T,), generator=g, device=DEVICE) < PADDING] = -1
    return tokens


def _router_logits(g, T, E, dtype):
    """Logits over experts of unlike popularity; a padding row has all of them masked."""
    l = torch.randn((T, E), generator=g, device=DEVICE).mul_(1.5)
    l += torch.randn((E,), generator=g, device=DEVICE).mul_(0.7)
    l[torch.rand((T,), generator=g, device=DEVICE) < PADDING] = -math.inf
    return l.to(dtype)


def _prepare_embedding(case, seed):
    g = _generator(seed)
    T, V, d = case["rows"], case["vocabulary"], case["d"]
    s = {"tokens": _tokens(g, T, V), "scale": math.sqrt(d)}
    if case["op"] == "embedding":
        s.update(table=_normal(g, (V, d), d ** -0.5, TYPES[case["type"]]), out=TYPES[case["out"]])
        return s
    grad = TYPES[case["grad"]]
    s.update(dy=_normal(g, (T, d), 1e-2, TYPES[case["type"]]), vocabulary=V, grad=grad, accumulate=case["accumulate"])
    s["into"] = _normal(g, (V, d), 0.3, grad) if case["accumulate"] else None  # what earlier micro-batches left
    return s


def _prepare_route(case, seed):
    g = _generator(seed)
    T, E, k, d = (case[n] for n in ("rows", "experts", "k", "d"))
    dtype = TYPES[case["type"]]
    op = case["op"]
    s = {"k": k, "experts": E, "logits": _router_logits(g, T, E, TYPES[case.get("logits", "float32")]), "normalise": case.get("normalise", True)}
    if op == "dispatch":
        s["x"] = _normal(g, (T, d), 1.0, dtype)
    else:
        expert, s["weight"] = _choose(s["logits"], k, s["normalise"])
        _, s["place"], _ = _plan(expert, E)
        s["rows"] = _normal(g, (T * k, d), 1.0, dtype)
        if op == "combine":
            s["out"] = TYPES[case["out"]]
            return s
        s.update(expert=expert, dy=_normal(g, (T, d), 1e-2, dtype), dx_rows=_normal(g, (T * k, d), 1e-2, dtype))
    s["sorted"] = torch.zeros((T * k, d), dtype=dtype, device=DEVICE)  # rows of padding leave its end as it is
    return s


def _prepare_policy(case, seed):
    g = _generator(seed)
    T, K = case["rows"], case["K"]
    logits = torch.randn((T, K), generator=g, device=DEVICE).mul_(2.5)
    noise = torch.rand((T, K), generator=g, device=DEVICE).clamp_(min=1e-30).log_().neg_().log_()
    actions = (logits - noise).argmax(dim=1).to(torch.int32)  # sampled from the distribution of the policy
    del noise
    logits = logits.to(TYPES[case["type"]])
    wide = logits.double()
    logp = (wide.gather(1, actions.long()[:, None]) - torch.logsumexp(wide, dim=1, keepdim=True))[:, 0]
    del wide
    # how far the policy has moved since it sampled; a ratio within a thousandth of a border of the clipping, where 32 bits leave open
    # on which side it is, is moved off it
    moved = torch.randn((T,), generator=g, device=DEVICE, dtype=torch.float64).mul_(0.15)
    for border in (math.log(1.0 - CLIP_LOW), math.log(1.0 + CLIP_HIGH)):
        off = moved - border
        moved = torch.where(off.abs() < 1e-3, border + torch.where(off < 0, -1e-3, 1e-3), moved)
    actions[torch.rand((T,), generator=g, device=DEVICE) < PADDING] = -1
    s = {"logits": logits, "actions": actions, "old": (logp - moved).float(), "scale": 1.0, "grad": TYPES[case["grad"]],
         "advantage": torch.randn((T,), generator=g, device=DEVICE), "reference": None,
         "weight": 1.0 / torch.randint(16, 2048, (T,), generator=g, device=DEVICE).float()}  # one over the length of a row's sequence
    if case["reference"]:
        s["reference"] = (logp + torch.randn((T,), generator=g, device=DEVICE, dtype=torch.float64) * 0.2).float()
    return s


def prepare(case, seed):
    op = case["op"]
    make = _prepare_policy if op == "policy" else _prepare_embedding if op.startswith("embedding") else _prepare_route
    return {"op": op, **make(case, seed)}


# ---------------------------------------------------------------------------------------------------- the plain forms
def _inside(numbers, count):
    return (numbers >= 0) & (numbers < count)


def _embedding(s):
    table, tokens = s["table"], s["tokens"].long()
    rows = table[tokens.clamp(0, table.shape[0] - 1)].float() * s["scale"]
    return torch.where(_inside(tokens, table.shape[0])[:, None], rows, 0.0).to(s["out"])


def _embedding_backward(s):
    tokens, V = s["tokens"].long(), s["vocabulary"]
    # frequent tokens have thousands of rows: sums in 64 bits
    total = torch.zeros((V + 1, s["dy"].shape[1]), dtype=torch.float64, device=DEVICE)
    total.index_add_(0, torch.where(_inside(tokens, V), tokens, V), s["dy"].double())
    total = total[:V] * s["scale"]
    if s["accumulate"]:
        s["into"].copy_(s["into"].double() + total)
        return s["into"]
    return total.to(s["grad"])


def _choose(logits, k, normalise):
    """The k experts of the largest logits (of equal ones the lowest index) and their weights; masked ones are none's: -1, weight 0."""
    l = logits.float()
    order = torch.sort(l, dim=1, descending=True, stable=True)
    top, expert = order.values[:, :k], order.indices[:, :k]
    live = top > -math.inf
    shift = torch.where(live[:, :1], top[:, :1], 0.0)
    e = torch.exp(top - shift)
    total = (e if normalise else torch.exp(l - shift)).sum(dim=1, keepdim=True)
    weight = torch.where(live, e / total, 0.0)
    return torch.where(live, expert, -1).to(torch.int32), weight


def _plan(expert, experts):
    """(row_ptr, place, order): pairs (row, choice) sorted by expert, in their own order within one; pairs without an expert have no place."""
    flat = expert.reshape(-1).long()
    key = torch.where(_inside(flat, experts), flat, experts)
    order = torch.sort(key, stable=True).indices
    counts = (key[:, None] == torch.arange(experts, device=DEVICE)[None, :]).sum(dim=0)
    row_ptr = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEVICE), counts.cumsum(0)])
    at = torch.arange(flat.shape[0], device=DEVICE)
    place = torch.empty_like(at)
    place[order] = at
    place = torch.where(key < experts, place, -1)
    order = torch.where(at < row_ptr[-1], order, -1)
    return row_ptr.to(torch.int32), place.to(torch.int32).view(expert.shape), order.to(torch.int32)


def _dispatch(s):
    expert, weight = _choose(s["logits"], s["k"], s["normalise"])
    row_ptr, place, order = _plan(expert, s["experts"])
    rows = torch.where((order >= 0)[:, None], s["x"][order.clamp(min=0).long() // s["k"]], s["sorted"])
    return {"expert": expert, "weight": weight, "row_ptr": row_ptr, "place": place, "order": order, "rows": rows}


def _gathered(rows, place):
    """[rows][k][d]: a row's own from its experts, zeros where it has none."""
    got = rows[place.clamp(min=0).long()].float()
    return torch.where((place >= 0)[:, :, None], got, 0.0)


def _combine(s):
    return (_gathered(s["rows"], s["place"]) * s["weight"][:, :, None]).sum(dim=1).to(s["out"])


def _route_backward(s):
    place, weight, dy, dtype = s["place"], s["weight"], s["dy"].float(), s["dy"].dtype
    live = place >= 0
    dweight = (_gathered(s["rows"], place) * dy[:, None, :]).sum(dim=2)
    drows = s["sorted"].clone()
    drows[place[live].long()] = (weight[:, :, None] * dy[:, None, :])[live].to(dtype)
    dx = _gathered(s["dx_rows"], place).sum(dim=1).to(dtype)
    mean = (weight * dweight).sum(dim=1, keepdim=True)
    at = torch.where(live, s["expert"].long(), s["experts"])
    dlogits = torch.zeros((place.shape[0], s["experts"] + 1), device=DEVICE)
    if s["normalise"]:
        dlogits.scatter_(1, at, weight * (dweight - mean))
    else:
        l = s["logits"].float()
        top = l.amax(dim=1, keepdim=True)
        e = torch.exp(l - torch.where(top > -math.inf, top, 0.0))
        total = e.sum(dim=1, keepdim=True)
        dlogits[:, :-1] = -(e / torch.where(total > 0, total, 1.0)) * mean
        dlogits.scatter_add_(1, at, weight * dweight)
    return {"drows": drows, "dweight": dweight, "dlogits": dlogits[:, :-1].to(s["logits"].dtype), "dx": dx}


def _policy(s):
    l, actions, advantage = s["logits"].float(), s["actions"].long(), s["advantage"]
    top = l.amax(dim=1, keepdim=True)
    e = torch.exp(l - top)
    total = e.sum(dim=1, keepdim=True)
    counts = _inside(actions, l.shape[1])
    at = actions.clamp(min=0)[:, None]
    logp = (l.gather(1, at) - top - torch.log(total))[:, 0]
    ratio = torch.exp(logp - s["old"])
    free, held = ratio * advantage, ratio.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * advantage
    loss = -torch.minimum(free, held)
    slope = torch.where(free <= held, -free, 0.0)
    if s["reference"] is not None:
        apart = s["reference"] - logp
        loss = loss + BETA * (torch.expm1(apart) - apart)
        slope = slope - BETA * torch.expm1(apart)
    weight = torch.where(counts, s["weight"], 0.0)
    e /= -total
    e.scatter_add_(1, at, torch.ones_like(top))
    e *= (slope * weight * s["scale"])[:, None]
    return {"loss": loss * weight, "grad": e.to(s["grad"]), "logp": torch.where(counts, logp, 0.0)}


def run(s):
    op = s["op"]
    if not own:
        return {"embedding": _embedding, "embedding_backward": _embedding_backward, "dispatch": _dispatch, "combine": _combine,
                "route_backward": _route_backward, "policy": _policy}[op](s)
    import paper_2307_11617_amd as rf
    if op == "embedding":
        return rf.rfast_embedding(s["table"], s["tokens"], scale=s["scale"], out_dtype=s["out"])
    if op == "embedding_backward":
        return rf.rfast_embedding_backward(s["dy"], s["tokens"], s["vocabulary"], scale=s["scale"], grad=s["into"], grad_dtype=s["grad"],
                                           accumulate=s["accumulate"])
    if op == "dispatch":
        r = rf.rfast_route(s["logits"], s["k"], normalise=s["normalise"])
        rows = rf.rfast_route_gather(s["x"], r.place, out=s["sorted"])
        return {"expert": r.expert, "weight": r.weight, "row_ptr": r.row_ptr, "place": r.place, "order": r.order, "rows": rows}
    if op == "combine":
        return rf.rfast_route_combine(s["rows"], s["place"], s["weight"], out_dtype=s["out"])
    if op == "route_backward":
        drows, dweight = rf.rfast_route_combine_backward(s["rows"], s["place"], s["weight"], s["dy"], drows=s["sorted"])
        dlogits = rf.rfast_route_backward(s["logits"], s["expert"], s["weight"], dweight, normalise=s["normalise"])
        dx = rf.rfast_route_combine(s["dx_rows"], s["place"])
        return {"drows": drows, "dweight": dweight, "dlogits": dlogits, "dx": dx}
    logp = torch.empty_like(s["old"])
    loss, grad = rf.rfast_policy_loss(s["logits"], s["actions"], s["old"], s["advantage"], reference=s["reference"], weight=s["weight"],
                                      clip=(CLIP_LOW, CLIP_HIGH), beta=BETA, grad_scale=s["scale"], grad_dtype=s["grad"], logp=logp)
    return {"loss": loss, "grad": grad, "logp": logp}


def _distinct(T, V):
    """How many tokens of a vocabulary T rows have between them, on average."""
    return int(round(float(-np.expm1(T * (1 - PADDING) * np.log1p(-_law(V))).sum()))) if V > 1 else 1


def work(case):
    op, T = case["op"], case["rows"]
    wide = TYPES[case["type"]].itemsize
    if op == "policy":
        K = case["K"]
        return {"bytes": T * K * (wide + TYPES[case["grad"]].itemsize) + (28 if case["reference"] else 24) * T, "flops": 5 * T * K}
    d = case["d"]
    if op == "embedding":
        return {"bytes": _distinct(T, case["vocabulary"]) * d * wide + T * d * TYPES[case["out"]].itemsize + 4 * T, "flops": T * d}
    if op == "embedding_backward":
        V = case["vocabulary"]
        written = (2 * _distinct(T, V) if case["accumulate"] else V) * d * TYPES[case["grad"]].itemsize
        return {"bytes": T * d * wide + written + 4 * T, "flops": T * d}
    P, E = T * case["k"], case["experts"]
    if op == "combine":
        return {"bytes": P * d * wide + T * d * TYPES[case["out"]].itemsize + 8 * P, "flops": 2 * P * d}
    logits = T * E * TYPES[case["logits"]].itemsize
    if op == "dispatch":
        return {"bytes": logits + (T + P) * d * wide + 16 * P + 4 * E, "flops": T * E}
    return {"bytes": (2 if not case["normalise"] else 1) * logits + (3 * P + 2 * T) * d * wide + 16 * P, "flops": 4 * P * d + 4 * T * E}


# ----------------------------------------------------------------------------------------------------- in 64 bits
def _exact_embedding(case, s):
    V = case["vocabulary"]
    tokens = s["tokens"].long()
    real = torch.nonzero((tokens > -1) & (tokens < V))[:, 0]
    if case["op"] == "embedding":
        out = torch.zeros((case["rows"], case["d"]), dtype=torch.float64, device=DEVICE)
        out[real] = torch.index_select(s["table"], 0, tokens[real]).double() * s["scale"]
        return out
    out = torch.zeros((V, case["d"]), dtype=torch.float64, device=DEVICE) if s["into"] is None else s["into"].double()
    return out.index_put_((tokens[real],), s["dy"][real].double() * s["scale"], accumulate=True)


def _exact_choice(logits, k, normalise):
    """Experts and weights from numpy, row for row."""
    l = logits.double().cpu().numpy()
    expert = np.argsort(-l, axis=1, kind="stable")[:, :k]
    chosen = np.take_along_axis(l, expert, axis=1)
    masked = np.isneginf(chosen)
    every = chosen if normalise else l
    top = np.where(masked[:, :1], 0.0, chosen[:, :1])
    total = np.exp(every - top).sum(axis=1, keepdims=True)
    weight = np.exp(chosen - top) / np.where(total > 0, total, 1.0)
    return np.where(masked, -1, expert), weight


def _exact_dispatch(case, s):
    E, k = case["experts"], case["k"]
    expert, weight = _exact_choice(s["logits"], k, case["normalise"])
    flat = expert.ravel()
    pairs = np.nonzero(flat >= 0)[0]
    pairs = pairs[np.argsort(flat[pairs], kind="stable")]
    place, order = np.full(flat.size, -1), np.full(flat.size, -1)
    place[pairs], order[:pairs.size] = np.arange(pairs.size), pairs
    row_ptr = np.concatenate([[0], np.cumsum(np.bincount(flat[pairs], minlength=E))])
    rows = torch.zeros(s["sorted"].shape, dtype=s["x"].dtype, device=DEVICE)
    rows[:pairs.size] = s["x"][torch.from_numpy(pairs // k).to(DEVICE)]

    def whole(a):
        return torch.from_numpy(a.astype(np.int32)).to(DEVICE)

    return {"expert": whole(expert), "weight": torch.from_numpy(weight).to(DEVICE), "row_ptr": whole(row_ptr),
            "place": whole(place.reshape(expert.shape)), "order": whole(order), "rows": rows.double()}


def _exact_route(case, s):
    T, k = s["place"].shape
    place, weight = s["place"].long(), s["weight"].double()
    if case["op"] == "combine":
        y = torch.zeros((T, case["d"]), dtype=torch.float64, device=DEVICE)
        for j in range(k):
            has = torch.nonzero(place[:, j] >= 0)[:, 0]
            y[has] += weight[has, j, None] * s["rows"][place[has, j]].double()
        return y
    dy = s["dy"].double()
    dx = torch.zeros((T, case["d"]), dtype=torch.float64, device=DEVICE)
    drows = torch.zeros(s["rows"].shape, dtype=torch.float64, device=DEVICE)
    dweight = torch.zeros((T, k), dtype=torch.float64, device=DEVICE)
    for j in range(k):
        has = torch.nonzero(place[:, j] >= 0)[:, 0]
        at = place[has, j]
        dx[has] += s["dx_rows"][at].double()
        drows[at] = weight[has, j, None] * dy[has]
        dweight[has, j] = torch.einsum("td,td->t", s["rows"][at].double(), dy[has])
    # dl_e = sum over choices j of dweight_j (d weight_j / d l_e), row by row from the Jacobian of a softmax
    E = case["experts"]
    chosen = (s["expert"].long()[:, :, None] == torch.arange(E, device=DEVICE)).double()  # [T][k][E]
    l = s["logits"].double()
    kept = chosen.sum(dim=1) > 0 if case["normalise"] else l > -math.inf
    p = torch.nan_to_num(torch.softmax(torch.where(kept, l, -math.inf), dim=1), nan=0.0)
    back = (chosen * dweight[:, :, None]).sum(dim=1)
    return {"drows": drows, "dweight": dweight, "dlogits": p * (back - (p * back).sum(dim=1, keepdim=True)), "dx": dx}


def _exact_policy(case, s):
    T, K = s["logits"].shape
    logs = torch.log_softmax(s["logits"].double(), dim=1)
    actions, rows = s["actions"].long(), torch.arange(T, device=DEVICE)
    real = actions >= 0
    at = actions * real
    logp, A = logs[rows, at], s["advantage"].double()
    ratio = (logp - s["old"].double()).exp()
    cut = ((A > 0) & (ratio > 1 + CLIP_HIGH)) | ((A < 0) & (ratio < 1 - CLIP_LOW))
    border = torch.where(A > 0, 1 + CLIP_HIGH, 1 - CLIP_LOW)
    loss, slope = -A * torch.where(cut, border, ratio), -A * torch.where(cut, 0.0, ratio)
    if case["reference"]:
        q = s["reference"].double() - logp
        loss, slope = loss + BETA * (q.exp() - q - 1), slope + BETA * (1 - q.exp())
    share = s["weight"].double() * real
    grad = logs.exp_()
    grad[rows, at] -= 1.0
    return {"loss": loss * share, "grad": grad.mul_((-slope * share * s["scale"])[:, None]), "logp": logp * real}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "policy":
        return _exact_policy(case, s)
    if op.startswith("embedding"):
        return _exact_embedding(case, s)
    return _exact_dispatch(case, s) if op == "dispatch" else _exact_route(case, s)
