"""Performance cases of the operators that train and apply models: low-rank adapters beside a shared projection (forward
and backward), softmax cross-entropy with its gradient, and the AdamW step over many tensors with states in 32 or 8 bits.

`run` computes them in their plain form, elementary torch operations in 32 bits, or, where `own` is true, through the
framework's entry points.  A pass is one call as a training loop or a server makes it.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}
BETA1, BETA2, EPS, GAMMA, DECAY, STEPS_BEFORE = 0.9, 0.999, 1e-8, 1e-3, 0.01, 100
BLOCK = 256        # coordinates that share a scale where states are held in 8 bits
FP8_MOST = 448.0   # largest finite e4m3


def listed():
    return [
        # One request of a server: a single row and its adapter.  Latency, and one read of the projection.
        dict(name="lora_forward_one_row", op="lora_forward", rows=1, segments=1, adapters=8, d=1024, K=4096, rank=16,
             ragged=False, out="bfloat16"),
        # A batch of requests that each generate their next row with an adapter of their own.
        dict(name="lora_forward_48_requests", op="lora_forward", rows=48, segments=48, adapters=64, d=4096, K=8192, rank=16,
             ragged=False, out="bfloat16"),
        # One round of the 128-node softmax workload (d 1024, 128 classes, 256 sampled rows per node) with adapters
        # of rank 8 as the trained vectors: logits in 32 bits.
        dict(name="lora_forward_128_nodes", op="lora_forward", rows=32768, segments=128, adapters=128, d=1024, K=128, rank=8,
             ragged=False, out="float32"),
        # Prompts of very different lengths in one pass through a wide layer.
        dict(name="lora_forward_ragged_wide", op="lora_forward", rows=8001, segments=23, adapters=23, d=4096, K=4096, rank=32,
             ragged=True, out="bfloat16"),
        # The gradient of that round: the adapters' gradients of all 128 nodes.
        dict(name="lora_backward_128_nodes", op="lora_backward", rows=32768, segments=128, adapters=128, d=1024, K=128, rank=8,
             ragged=False, need_dx=False),
        # Training of 16 adapters within a deeper network: the gradient of the rows too.
        dict(name="lora_backward_wide", op="lora_backward", rows=4100, segments=16, adapters=16, d=4096, K=4096, rank=16,
             ragged=True, need_dx=True),
        # The loss of the 128-node round.
        dict(name="xent_128_nodes", op="xent", rows=32768, K=128, type="float32", grad="bfloat16"),
        # A loss over a large vocabulary of an odd size.
        dict(name="xent_vocabulary", op="xent", rows=4096, K=50001, type="bfloat16", grad="bfloat16"),
        # The adapters of 128 nodes (rank 8; d 1024, 128 classes): 256 small tensors in one step.
        dict(name="adamw_256_adapters", op="adamw", tensors=256, size=4608, ragged=True, bits=32, type="float32"),
        # The headline workload's 16 vectors of 11.2 M coordinates.
        dict(name="adamw_16_networks", op="adamw", tensors=16, size=11_200_000, ragged=False, bits=32, type="float32"),
        # The same with moments in 8 bits.
        dict(name="adamw8_16_networks", op="adamw", tensors=16, size=11_200_000, ragged=False, bits=8, type="float32"),
        # The tensors of a network of moderate size held in 16 bits, sizes from a bias to a wide matrix.
        dict(name="adamw8_ragged_bf16", op="adamw", tensors=75, size=200_000, ragged=True, bits=8, type="bfloat16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["lora_forward", "lora_forward", "lora_backward", "lora_backward", "xent", "adamw", "adamw"])
    if op in ("lora_forward", "lora_backward"):
        d = _log(rng, 64, 8192)
        if rng.random() < 0.75:
            d = d // 8 * 8  # feature counts are mostly multiples of eight; class counts and rows are anything
        K = _log(rng, 10, 16384)
        K = min(K, (1 << 26) // d)
        rank = _log(rng, 1, 64)
        adapters = min(_log(rng, 1, 128), 2048 // rank)
        most = max(1, min(32768, 8001 * 4096 * 4096 // (d * K)))
        if op == "lora_backward":
            most = max(1, min(most, 4100 * 4096 * 4096 // (d * K)))
        most = max(1, min(most, (1 << 27) // max(d, K)))
        rows = _log(rng, 1, most)
        case = dict(op=op, rows=rows, segments=max(1, min(adapters, rows)), adapters=adapters, d=d, K=K, rank=rank,
                    ragged=rng.random() < 0.6)
        if op == "lora_forward":
            case["out"] = rng.choice(["float32", "bfloat16"])
        else:
            case["need_dx"] = rng.random() < 0.5
        return case
    if op == "xent":
        K = _log(rng, 2, 131072)
        rows = _log(rng, 1, max(1, min(65536, 4096 * 50001 // K)))
        return dict(op="xent", rows=rows, K=K, type=rng.choice(["float32", "bfloat16"]), grad=rng.choice(["float32", "bfloat16"]))
    tensors = _log(rng, 1, 300)
    size = _log(rng, 100, min(20_000_000, 150_000_000 // tensors))
    return dict(op="adamw", tensors=tensors, size=size, ragged=rng.random() < 0.6, bits=rng.choice([32, 8]),
                type=rng.choice(["float32", "bfloat16"]))


# ------------------------------------------------------------------------------------------------------------- inputs
def _lengths(total, parts, ragged):
    """`total` rows in `parts` lengths: alike, or from none to several times the mean."""
    if not ragged:
        return [total // parts + (i < total % parts) for i in range(parts)]
    w = [((i + 1) * 0.6180339887498949 % 1.0) ** 2 for i in range(parts)]
    got = [int(total * x / sum(w)) for x in w]
    got[-1] += total - sum(got)
    return got


def _sizes(case):
    """Coordinates of each tensor, from a quarter of the mean to nearly twice it."""
    if not case["ragged"]:
        return [case["size"]] * case["tensors"]
    return [max(1, int(case["size"] * (0.25 + 1.5 * ((i + 1) * 0.6180339887498949 % 1.0)))) for i in range(case["tensors"])]


def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _normal(g, shape, std, dtype):
    return torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float32).mul_(std).to(dtype)


def _prepare_lora(case, seed):
    g = _generator(seed)
    T, S, n, d, K, r = (case[k] for k in ("rows", "segments", "adapters", "d", "K", "rank"))
    bf16 = torch.bfloat16
    s = {"x": _normal(g, (T, d), 1.0, bf16), "w": _normal(g, (K, d), d ** -0.5, bf16),
         "a": _normal(g, (n, r, d), d ** -0.5, bf16), "b": _normal(g, (n, K, r), 0.5, bf16), "scale": 2.0 / r}
    ends = torch.tensor(_lengths(T, S, case["ragged"])).cumsum(0)
    s["row_ptr"] = torch.cat([torch.zeros(1, dtype=torch.int64), ends]).to(torch.int32).to(DEVICE)
    if case["op"] == "lora_forward" and S == T:  # requests: any adapter, some of them the same, some rows without one
        s["adapter"] = torch.randint(-1, n, (S,), generator=g, device=DEVICE, dtype=torch.int32)
    else:
        s["adapter"] = torch.arange(S, device=DEVICE, dtype=torch.int32)
    if case["op"] == "lora_backward":  # what a softmax loss sends back: (p - onehot) / rows
        p = torch.softmax(torch.randn((T, K), generator=g, device=DEVICE) * 2.0, dim=1)
        p[torch.arange(T, device=DEVICE), torch.randint(0, K, (T,), generator=g, device=DEVICE)] -= 1.0
        s["dy"] = (p / T).to(bf16)
    return s


def _prepare_xent(case, seed):
    g = _generator(seed)
    T, K = case["rows"], case["K"]
    logits = torch.randn((T, K), generator=g, device=DEVICE).mul_(2.5)
    labels = torch.randint(0, K, (T,), generator=g, device=DEVICE, dtype=torch.int32)
    labels[torch.rand((T,), generator=g, device=DEVICE) < 0.05] = -1  # padding: no loss, no gradient
    return {"logits": logits.to(TYPES[case["type"]]), "labels": labels, "scale": 1.0 / T, "grad": TYPES[case["grad"]]}


def _prepare_adamw(case, seed):
    g = _generator(seed)
    sizes = _sizes(case)
    padded = [-(-c // BLOCK) * BLOCK for c in sizes]  # in the flat buffers every tensor begins at a block
    total = sum(padded)
    size, pad = torch.tensor(sizes, device=DEVICE), torch.tensor(padded, device=DEVICE)
    start = torch.cumsum(pad, 0) - pad
    which = torch.repeat_interleave(torch.arange(len(sizes), device=DEVICE), pad // BLOCK)  # the tensor of each block
    at = torch.arange(total, device=DEVICE).view(-1, BLOCK) - start[which][:, None]
    inside = at < size[which][:, None]
    del at
    dtype = TYPES[case["type"]]

    def values(std, dtype=torch.float32, square=False):
        v = torch.randn((total // BLOCK, BLOCK), generator=g, device=DEVICE).mul_(std)
        v = v.square_() if square else v
        return v.mul_(inside).to(dtype)

    s = {"case": case, "param": values(0.02, dtype), "grad": values(1e-3, dtype), "bits": case["bits"], "which": which,
         "decay": torch.where(torch.arange(len(sizes), device=DEVICE) % 2 == 0, DECAY, 0.0),
         "steps": torch.full((len(sizes),), STEPS_BEFORE, dtype=torch.int32, device=DEVICE)}
    m, v = values(3e-4), values(1e-3, square=True)
    if case["bits"] == 8:
        s["m"], s["m_scale"] = _quantise(m, False)
        s["v"], s["v_scale"] = _quantise(v.sqrt(), True)
    else:
        s["m"], s["v"] = m, v
    if own:
        from paper_2307_11617_amd import RFastAdamW

        def views(t):
            t = t.view(-1)
            return [t[b:b + c] for b, c in zip(start.tolist(), sizes)]

        kw = {}
        if case["bits"] == 8:
            blocks = [(b // BLOCK, -(-c // BLOCK)) for b, c in zip(start.tolist(), sizes)]
            kw = {k: [s[k].view(-1)[b:b + c] for b, c in blocks] for k in ("m_scale", "v_scale")}
        s["optimizer"] = RFastAdamW(views(s["param"]), views(s["grad"]), m=views(s["m"]), v=views(s["v"]), state_bits=case["bits"],
                                    betas=(BETA1, BETA2), eps=EPS, weight_decay=s["decay"].tolist(), steps=STEPS_BEFORE, **kw)
    return s


def prepare(case, seed):
    if case["op"] == "xent":
        return {"op": "xent", **_prepare_xent(case, seed)}
    if case["op"] == "adamw":
        return {"op": "adamw", **_prepare_adamw(case, seed)}
    s = {"op": case["op"], **_prepare_lora(case, seed)}
    if case["op"] == "lora_forward":
        s["out"] = TYPES[case["out"]]
    else:
        s["need_dx"] = case["need_dx"]
    return s


# ---------------------------------------------------------------------------------------------------- the plain forms
def _adapter_columns(s):
    """[rows][adapters * rank]: 1 where the column belongs to the row's adapter.  With it the products of all adapters at
    once, masked, are those of each row's own."""
    T, (n, r, _) = s["x"].shape[0], s["a"].shape
    segment = torch.searchsorted(s["row_ptr"][1:], torch.arange(T, device=DEVICE, dtype=torch.int32), right=True)
    return (s["adapter"][segment][:, None] == torch.arange(n, device=DEVICE).repeat_interleave(r)[None, :]).float()


def _lora_forward(s):
    n, r, d = s["a"].shape
    x = s["x"].float()
    u = (x @ s["a"].float().reshape(n * r, d).t()) * _adapter_columns(s)
    y = x @ s["w"].float().t() + s["scale"] * (u @ s["b"].float().permute(0, 2, 1).reshape(n * r, -1))
    return y.to(s["out"])


def _lora_backward(s):
    n, r, d = s["a"].shape
    K = s["w"].shape[0]
    x, dy, mask = s["x"].float(), s["dy"].float(), _adapter_columns(s)
    a, b = s["a"].float().reshape(n * r, d), s["b"].float().permute(0, 2, 1).reshape(n * r, K)
    u = (x @ a.t()) * mask
    e = s["scale"] * (dy @ b.t()) * mask
    da = (e.t() @ x).view(n, r, d)
    db = (s["scale"] * (u.t() @ dy)).view(n, r, K).permute(0, 2, 1).contiguous()
    dx = (dy @ s["w"].float() + e @ a).to(torch.bfloat16) if s["need_dx"] else None
    return dx, da, db


def _xent(s):
    l, labels = s["logits"].float(), s["labels"].long()
    top = l.amax(dim=1, keepdim=True)
    e = torch.exp(l - top)
    total = e.sum(dim=1, keepdim=True)
    counts = labels >= 0
    at = labels.clamp(min=0)[:, None]
    loss = torch.where(counts, (torch.log(total) + top - l.gather(1, at))[:, 0], 0.0)
    e /= total
    e.scatter_add_(1, at, torch.full_like(top, -1.0))
    return loss, (e * torch.where(counts, s["scale"], 0.0)[:, None]).to(s["grad"])


def _quantise(v, root):
    """Values as e4m3 with the scale that takes a block's largest to 448; a root that is not zero stays so."""
    top = v.abs().amax(dim=1, keepdim=True)
    inverse = torch.where(top > 0, FP8_MOST / top, 0.0)
    q = v * inverse
    if root:
        q = torch.where(v > 0, q.clamp(min=2.0 ** -9), q)
    return q.to(torch.float8_e4m3fn), (top * (1.0 / FP8_MOST))[:, 0]


def _adamw(s):
    t = s["steps"].add_(1).double()
    first = (GAMMA / (1.0 - BETA1 ** t)).float()[s["which"]][:, None]
    second = (1.0 / (1.0 - BETA2 ** t).sqrt()).float()[s["which"]][:, None]
    keep = (1.0 - GAMMA * s["decay"].double()).float()[s["which"]][:, None]
    g, p = s["grad"].float(), s["param"].float()
    m, v = s["m"], s["v"]
    if s["bits"] == 8:
        m, v = m.float() * s["m_scale"][:, None], (v.float() * s["v_scale"][:, None]).square()
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + (g * g) * (1.0 - BETA2)
    root = v.sqrt()
    s["param"].copy_(p * keep - (m * first) / (root * second + EPS))
    if s["bits"] == 8:
        s["m"], s["m_scale"] = _quantise(m, False)
        s["v"], s["v_scale"] = _quantise(root, True)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)


def run(s):
    op = s["op"]
    if own:
        import paper_2307_11617_amd as rf
        if op == "lora_forward":
            return rf.rfast_lora_forward(s["x"], s["w"], s["a"], s["b"], s["row_ptr"], s["adapter"], scale=s["scale"], out_dtype=s["out"])
        if op == "lora_backward":
            return rf.rfast_lora_backward(s["x"], s["w"], s["a"], s["b"], s["row_ptr"], s["adapter"], s["dy"], scale=s["scale"],
                                          need_dx=s["need_dx"])
        if op == "xent":
            return rf.rfast_softmax_xent(s["logits"], s["labels"], grad_scale=s["scale"], grad_dtype=s["grad"])
        s["optimizer"].step(GAMMA)
    elif op == "lora_forward":
        return _lora_forward(s)
    elif op == "lora_backward":
        return _lora_backward(s)
    elif op == "xent":
        return _xent(s)
    else:
        _adamw(s)
    # what is held in 8 bits is an e4m3 number times the scale of its block: both, whole
    return {k: s[k] for k in ("param", "m", "v", "m_scale", "v_scale") if k in s}


def work(case):
    op = case["op"]
    if op == "adamw":
        count = sum(_sizes(case))
        wide = TYPES[case["type"]].itemsize
        state = 16 if case["bits"] == 32 else 4 + 4 * 4 / BLOCK
        return {"bytes": count * (3 * wide + state), "flops": 14 * count}
    if op == "xent":
        T, K = case["rows"], case["K"]
        return {"bytes": T * K * (TYPES[case["type"]].itemsize + TYPES[case["grad"]].itemsize) + 8 * T, "flops": 5 * T * K}
    T, d, K, r = (case[k] for k in ("rows", "d", "K", "rank"))
    used = min(case["adapters"], case["segments"])
    adapters, rows_x, rows_y = 2 * used * r * (d + K), 2 * T * d, T * K
    if op == "lora_forward":
        return {"bytes": rows_x + 2 * K * d + adapters + rows_y * TYPES[case["out"]].itemsize, "flops": 2 * T * (d * K + r * (d + K))}
    dx = case["need_dx"]
    return {"bytes": rows_x * (2 if dx else 1) + 2 * rows_y + adapters + 2 * case["adapters"] * r * 2 * (d + K) + (2 * K * d if dx else 0),
            "flops": 2 * T * (2 * r * (d + K) + ((K + r) * d if dx else 0))}


# ----------------------------------------------------------------------------------------------------- in 64 bits
def _exact_lora(case, s):
    """Segment by segment, from y = (W + s B A) x and its derivatives."""
    bounds, ids = s["row_ptr"].tolist(), s["adapter"].tolist()
    x, w = s["x"].double(), s["w"].double()
    if case["op"] == "lora_forward":
        y = torch.matmul(x, w.t())
        for lo, hi, i in zip(bounds, bounds[1:], ids):
            if i >= 0:
                y[lo:hi] += torch.matmul(torch.matmul(x[lo:hi], s["a"][i].double().t()), s["b"][i].double().t()) * s["scale"]
        return y
    dy = s["dy"].double()
    da, db = (torch.zeros(s[k].shape, dtype=torch.float64, device=DEVICE) for k in ("a", "b"))
    dx = torch.matmul(dy, w) if case["need_dx"] else None
    for lo, hi, i in zip(bounds, bounds[1:], ids):
        a, b, xs, ys = s["a"][i].double(), s["b"][i].double(), x[lo:hi], dy[lo:hi]
        through = torch.matmul(ys, b) * s["scale"]
        da[i] += torch.matmul(through.t(), xs)
        db[i] += torch.matmul(ys.t(), torch.matmul(xs, a.t())) * s["scale"]
        if dx is not None:
            dx[lo:hi] += torch.matmul(through, a)
    return dx, da, db


def _exact_xent(s):
    logs = torch.log_softmax(s["logits"].double(), dim=1)
    rows = torch.arange(logs.shape[0], device=DEVICE)
    valid = s["labels"] >= 0
    at = s["labels"].long() * valid
    loss = -logs[rows, at] * valid
    grad = logs.exp_()
    grad[rows, at] -= 1.0
    return loss, grad * (valid * s["scale"])[:, None]


def _exact_adamw(s):
    t = STEPS_BEFORE + 1
    g = s["grad"].double()
    m, v = s["m"].double(), s["v"].double()
    eight = s["bits"] == 8
    if eight:
        m, v = m * s["m_scale"].double()[:, None], (v * s["v_scale"].double()[:, None]) ** 2
    m = m + (1 - BETA1) * (g - m)
    v = v + (1 - BETA2) * (g ** 2 - v)
    hat_m, hat_v = m / (1 - BETA1 ** t), v / (1 - BETA2 ** t)
    p = s["param"].double()
    p = p - GAMMA * (hat_m / (torch.sqrt(hat_v) + EPS) + s["decay"].double()[s["which"]][:, None] * p)
    if not eight:
        return {"param": p, "m": m, "v": v}
    # an e4m3 code next to a border between two has no value in exact arithmetic that 32 bits have to meet: scales only
    return {"param": p, "m": None, "v": None, "m_scale": m.abs().amax(1) / FP8_MOST, "v_scale": v.sqrt().amax(1) / FP8_MOST}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "xent":
        return _exact_xent(s)
    return _exact_adamw(s) if case["op"] == "adamw" else _exact_lora(case, s)
