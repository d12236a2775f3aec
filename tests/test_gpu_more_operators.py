"""Embeddings, rows to experts and back, and the policy loss against their formulas in 64 bits.

Tolerances are bounds, elementwise, from the roundings on the way: HALF = 2^-24 is half a step of fp32 relative to the value, BF = 2^-8 of
bf16.  A sum of n numbers in fp32 is off by at most n HALF of the sum of their magnitudes in any order; expf, expm1f and a logarithm of the vector
unit by 2 steps (4 HALF) of their value, a hardware exponential of an argument that is itself the product of a rounded difference and a rounded
constant by 3 HALF of that difference more."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2307_11617_amd as rf  # noqa: E402
from paper_2307_11617_amd import RFastAdamW, RFastError  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF, BF = 2.0 ** -24, 2.0 ** -8
F64, BF16, F32, I32 = torch.float64, torch.bfloat16, torch.float32, torch.int32
INF, NAN = float("inf"), float("nan")
TYPES = [F32, BF16]
LEAST = 1e-37  # what falls below the normal numbers of 32 bits on the way


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def normal(g, *shape, std=1.0, dtype=F32):
    return (torch.randn(shape, generator=g) * std).to(dtype)


def last(dtype):
    """The rounding of a result to its type."""
    return BF if dtype == BF16 else HALF


def within(got, want, bound, what):
    got, want = got.detach().cpu().double(), want.double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = (got - want).abs() - bound
    assert over.max() <= 0, f"{what}: off by {(got - want).abs().max():.3g}, {(over > 0).sum()} values beyond their bound, worst by {over.max():.3g}"


def apart(t, ld, offset=0):
    """A copy of matrix t on the GPU whose rows are ld elements apart, `offset` elements into its memory; what lies between is 77."""
    rows, cols = t.shape
    mem = torch.full((offset + rows * ld + 8,), 77.0, dtype=t.dtype, device=DEV)
    v = mem[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    v.copy_(t)
    return v, mem


def untouched(mem, rows, cols, ld, offset=0):
    keep = torch.ones_like(mem, dtype=torch.bool)
    keep[offset:offset + rows * ld].view(rows, ld)[:, :cols] = False
    return bool((mem[keep] == 77.0).all())


# -------------------------------------------------------------------------------------------------------- embeddings
SIZES = [(1, 1, 1), (1, 50, 4096), (3, 7, 5), (70, 33, 64), (65, 100, 65), (129, 1000, 257), (300, 40, 515), (20, 9, 1032), (1000, 300, 8), (5, 3, 2051)]


@pytest.mark.parametrize("T,V,d", SIZES)
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("out", TYPES)
def test_embedding(T, V, d, kind, out):
    g = gen(T + V + d)
    table, tokens = normal(g, V, d, dtype=kind), torch.randint(0, V, (T,), generator=g, dtype=I32)
    tokens[::7] = torch.tensor([-1, V, 2 ** 31 - 1, -2 ** 31])[torch.arange(len(tokens[::7])) % 4].to(I32)
    scale = 1.375
    want = torch.where(((tokens >= 0) & (tokens < V))[:, None], table.double()[tokens.long().clamp(0, V - 1)] * scale, 0.0)
    y = rf.rfast_embedding(table.to(DEV), tokens.to(DEV), scale=scale, out_dtype=out)
    bound = want.abs() * (HALF + (BF * (1 + HALF) if out == BF16 else 0.0))
    within(y, want, bound, "rows")
    a, _ = apart(table, d + 3, 1)
    o, mem = apart(torch.zeros(T, d, dtype=out), d + 5, 3)
    assert rf.rfast_embedding(a, tokens.to(DEV), scale=scale, out=o) is o
    assert torch.equal(o, y) and untouched(mem, T, d, d + 5, 3)


def exact_table(dy, tokens, V, scale, into=None):
    real = (tokens >= 0) & (tokens < V)
    out, size, count = (torch.zeros((V, k), dtype=F64) for k in (dy.shape[1], dy.shape[1], 1))
    at = tokens[real].long()
    out.index_put_((at,), dy[real].double(), accumulate=True)
    size.index_put_((at,), dy[real].double().abs(), accumulate=True)
    count.index_put_((at,), torch.ones((len(at), 1), dtype=F64), accumulate=True)
    want = out * scale
    err = scale * size * (count + 1) * HALF
    if into is not None:
        want = want + into.double()
        err = err + HALF * want.abs() * (1 + HALF)
    return want, err, count[:, 0] > 0


def token_sets(V, g):
    runs = torch.cat([torch.full((n,), i % V) for i, n in enumerate((1, 63, 64, 65, 3, 128, 129, 2, 200, 62, 66, 1, 127, 640))])
    return {"alike": torch.full((1000,), V - 1), "one": torch.tensor([V // 2]), "runs": runs[torch.randperm(len(runs), generator=g)],
            "any": torch.randint(-2, V + 2, (777,), generator=g), "64": torch.randint(0, V, (64,), generator=g),
            "padding": torch.full((130,), -1), "frequent": (torch.rand(5000, generator=g) ** 6 * V).long(), "none": torch.zeros(0, dtype=torch.int64)}


@pytest.mark.parametrize("which", ["alike", "one", "runs", "any", "64", "padding", "frequent", "none"])
@pytest.mark.parametrize("V,d", [(1, 9), (17, 64), (300, 513), (1500, 40), (70001, 3)])
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("accumulate", [False, True])
def test_embedding_backward(which, V, d, kind, accumulate):
    g = gen(V + d)
    tokens = token_sets(V, g)[which].to(I32)
    dy, scale = normal(g, len(tokens), d, dtype=kind), 0.625
    for out in TYPES:
        into = normal(g, V, d, dtype=out) if accumulate else None
        want, err, there = exact_table(dy, tokens, V, scale, into)
        grad = None if into is None else into.to(DEV)
        got = rf.rfast_embedding_backward(dy.to(DEV), tokens.to(DEV), V, scale=scale, grad=grad, grad_dtype=out, accumulate=accumulate)
        assert got.dtype == out and (grad is None or got is grad)
        within(got, want, err + last(out) * (want.abs() + err), "gradient")
        if accumulate:
            assert torch.equal(got.cpu()[~there], into[~there]), "rows without a token"
        else:
            assert not got.cpu()[~there].any(), "rows without a token"


@pytest.mark.parametrize("V", [1 << 10, (1 << 10) - 1, 1 << 16, (1 << 20) + 5, 1 << 21])
def test_embedding_backward_large_vocabularies(V):
    """Numbers of one to three digits, more tokens than one workgroup sorts, and the same bits from every call."""
    g = gen(V)
    T = 30001
    tokens = torch.where(torch.rand(T, generator=g) < 0.3, torch.randint(0, 9, (T,), generator=g) * (V // 9), torch.randint(-5, V + 5, (T,), generator=g)).to(I32)
    dy = normal(g, T, 5)
    want, err, _ = exact_table(dy, tokens, V, 1.0)
    got = rf.rfast_embedding_backward(dy.to(DEV), tokens.to(DEV), V)
    within(got, want, err, "gradient")
    for _ in range(3):
        assert torch.equal(rf.rfast_embedding_backward(dy.to(DEV), tokens.to(DEV), V), got)


def test_embedding_backward_strides():
    g = gen(5)
    T, V, d = 333, 50, 75
    tokens, dy = torch.randint(0, V, (T,), generator=g, dtype=I32).to(DEV), normal(g, T, d, dtype=BF16)
    want = rf.rfast_embedding_backward(dy.to(DEV), tokens, V, scale=2.0)
    y, _ = apart(dy, d + 2, 1)
    grad, mem = apart(torch.zeros(V, d), d + 6, 1)
    rf.rfast_embedding_backward(y, tokens, V, scale=2.0, grad=grad)
    assert torch.equal(grad, want) and untouched(mem, V, d, d + 6, 1)
    rf.rfast_embedding_backward(y, tokens, V, scale=2.0, grad=grad, accumulate=True)
    assert torch.equal(grad, want * 2) and untouched(mem, V, d, d + 6, 1)


def test_embedding_gradient_against_differences():
    """<dy, y(E + h D) - y(E - h D)> / 2h = <gradient, D>: linear, so exact but for roundings of some 600 terms."""
    g = gen(6)
    table, step, tokens = normal(g, 40, 33), normal(g, 40, 33), torch.randint(0, 40, (90,), generator=g, dtype=I32).to(DEV)
    dy = normal(g, 90, 33)
    up, down = (rf.rfast_embedding((table + s * step).to(DEV), tokens, scale=0.5) for s in (0.5, -0.5))
    slope = (dy.double() * (up.cpu().double() - down.cpu().double())).sum()
    grad = rf.rfast_embedding_backward(dy.to(DEV), tokens, 40, scale=0.5).cpu().double()
    # of each difference: three roundings of terms below 6
    assert abs(slope - (grad * step.double()).sum()) <= 90 * 33 * 6 * 6 * 4 * HALF + 40 * 33 * 30 * 20 * HALF


# ---------------------------------------------------------------------------------------------- the order by expert
def exact_plan(expert, n):
    flat = np.asarray(expert).ravel()
    pairs = np.nonzero((flat >= 0) & (flat < n))[0]
    pairs = pairs[np.argsort(flat[pairs], kind="stable")]
    place, order = np.full(flat.size, -1), np.full(flat.size, -1)
    place[pairs], order[:pairs.size] = np.arange(pairs.size), pairs
    return np.searchsorted(flat[pairs], np.arange(n + 1)), place.reshape(np.shape(expert)), order


@pytest.mark.parametrize("pairs", [0, 1, 2, 63, 64, 65, 1000, 4095, 4096, 4097, 70001])
@pytest.mark.parametrize("experts", [1, 2, 7, 63, 64, 128, 255, 256, 1000, 1023, 1024, 5000, 1 << 20, (1 << 20) + 1])
def test_plan(pairs, experts):
    rng = np.random.default_rng(pairs * 31 + experts)
    expert = rng.integers(-1, experts + 1, pairs).astype(np.int32)
    if pairs > 2:
        expert[1], expert[2] = 2 ** 31 - 1, -2 ** 31
    want = exact_plan(expert, experts)
    got = rf.rfast_route_plan(torch.from_numpy(expert).to(DEV), experts)
    for w, t, name in zip(want, got, ("row_ptr", "place", "order")):
        assert np.array_equal(t.cpu().numpy(), w), name


@pytest.mark.parametrize("fill", [0, 6, -1, 7])
def test_plan_of_one_expert(fill):
    expert = torch.full((9001,), fill, dtype=I32)
    for w, t in zip(exact_plan(expert.numpy(), 7), rf.rfast_route_plan(expert.to(DEV), 7)):
        assert np.array_equal(t.cpu().numpy(), w)


def test_plan_of_many_pairs():
    """More than one tile of pairs per workgroup: 3 million pairs, ragged."""
    rng = np.random.default_rng(3)
    expert = (rng.random(3000001) ** 3 * 130).astype(np.int32) - 1
    for n in (128, 5000):
        for w, t in zip(exact_plan(expert, n), rf.rfast_route_plan(torch.from_numpy(expert).to(DEV), n)):
            assert np.array_equal(t.cpu().numpy(), w)


# --------------------------------------------------------------------------------------------------------- the router
def exact_choice(logits, k, normalise):
    """(expert, weight, its bound) of logits without NaN or +infinity."""
    l = logits.double()
    top, expert = torch.sort(l, dim=1, descending=True, stable=True)
    top, expert = top[:, :k], expert[:, :k]
    live = top > -INF
    shift = torch.where(live[:, :1], top[:, :1], 0.0)
    every = top if normalise else l
    e, chosen = torch.exp(every - shift), torch.exp(top - shift)
    total = e.sum(dim=1, keepdim=True)
    weight = torch.where(live, chosen / total.clamp(min=1e-300), 0.0)
    # of each exponential: the rounding of its argument and of the function; of the sum: one per term
    spread = torch.where(every > -INF, (every - shift).abs(), 0.0)
    in_sum = (e * (spread * HALF + 4 * HALF)).sum(dim=1, keepdim=True) / total.clamp(min=1e-300) + e.shape[1] * HALF
    err = weight * (in_sum + torch.where(live, (top - shift).abs(), 0.0) * HALF + 6 * HALF) + LEAST
    return torch.where(live, expert, -1).to(I32), weight, err


ROUTERS = [(1, 1, 1), (1, 64, 4), (5, 2, 2), (33, 8, 8), (100, 9, 3), (65, 17, 5), (64, 33, 2), (70, 64, 8), (31, 100, 20), (40, 129, 33), (9, 256, 64),
           (20, 257, 7), (11, 512, 10), (8, 1000, 6), (3, 1024, 64), (1000, 23, 3)]


@pytest.mark.parametrize("T,E,k", ROUTERS)
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("normalise", [True, False])
def test_route(T, E, k, kind, normalise):
    g = gen(T + E + k)
    logits = normal(g, T, E, std=2.0)
    logits[::3] = (logits[::3] * 2).round() / 2  # many equal ones
    logits[torch.rand((T, E), generator=g) < 0.2] = -INF
    logits[T // 2] = -INF
    logits[T // 3] = torch.where(torch.arange(E) % 2 == 0, 0.0, -0.0)
    logits = logits.to(kind)
    want, weight, err = exact_choice(logits, k, normalise)
    l, _ = apart(logits, E + 3, 1)
    for given in (logits.to(DEV), l):
        r = rf.rfast_route(given, k, normalise=normalise)
        assert torch.equal(r.expert.cpu(), want)
        within(r.weight, weight, err, "weights")
        assert not r.weight.cpu()[want < 0].any()
        for w, t in zip(exact_plan(want.numpy(), E), r[2:]):
            assert np.array_equal(t.cpu().numpy(), w)


@pytest.mark.parametrize("normalise", [True, False])
def test_route_not_finite(normalise):
    l = torch.tensor([[1.0, NAN, 3.0, NAN, 2.0], [1.0, INF, 3.0, 3.0, -INF], [-INF, -INF, 5.0, -INF, -INF], [3e38, -3e38, 0.0, 3e38, 1.0], [-NAN, -INF, -INF, -INF, -INF]])
    r = rf.rfast_route(l.to(DEV), 3, normalise=normalise)
    assert r.expert.cpu().tolist() == [[1, 3, 2], [1, 2, 3], [2, -1, -1], [0, 3, 4], [0, -1, -1]]
    w = r.weight.cpu()
    assert w[0].isnan().all() and w[1].isnan().all() and w[2].tolist() == [1.0, 0.0, 0.0] and w[3].tolist() == [0.5, 0.5, 0.0]
    assert w[4, 0].isnan() and w[4, 1:].tolist() == [0.0, 0.0]


@pytest.mark.parametrize("T,E,k", ROUTERS)
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("normalise", [True, False])
def test_route_backward(T, E, k, kind, normalise):
    g = gen(T + E + k)
    logits = normal(g, T, E, std=2.0)
    logits[torch.rand((T, E), generator=g) < 0.2] = -INF
    logits[T // 2] = -INF
    logits = logits.to(kind)
    expert, weight, _ = exact_choice(logits, k, normalise)
    weight, dweight = weight.float(), normal(g, T, k, std=3.0)
    live = expert >= 0
    w, dw = weight.double(), torch.where(live, dweight.double(), 0.0)
    mean, size = (w * dw).sum(dim=1, keepdim=True), (w * dw).abs().sum(dim=1, keepdim=True)
    at = torch.where(live, expert.long(), E)
    want, err = torch.zeros((T, E + 1), dtype=F64), torch.zeros((T, E + 1), dtype=F64)
    if normalise:
        want.scatter_add_(1, at, w * (dw - mean))
        err.scatter_add_(1, at, HALF * (3 * (w * dw).abs() + w * (k + 4) * size))
    else:
        l = logits.double()
        shift = torch.nan_to_num(l.amax(dim=1, keepdim=True), neginf=0.0)
        e = torch.exp(l - shift)
        total = e.sum(dim=1, keepdim=True).clamp(min=1e-300)
        p, spread = e / total, torch.where(l > -INF, (l - shift).abs(), 0.0)
        p_err = p * ((e * (spread + 4)).sum(dim=1, keepdim=True) / total + E + spread + 6) * HALF
        want[:, :E] = -p * mean
        err[:, :E] = p_err * size + p * HALF * (k + 4) * size
        want.scatter_add_(1, at, w * dw)
        err.scatter_add_(1, at, HALF * 3 * (w * dw).abs())
    want, err = want[:, :E], err[:, :E] + LEAST
    for out in TYPES:
        l, _ = apart(logits, E + 1, 1)
        o, mem = apart(torch.zeros((T, E), dtype=out), E + 2, 1)
        got = rf.rfast_route_backward(l, expert.to(DEV), weight.to(DEV), dweight.to(DEV), normalise=normalise, dlogits=o)
        within(got, want, err + HALF * want.abs() + last(out) * (want.abs() + err), "dlogits")
        assert not got.cpu()[logits == -INF].any() and untouched(mem, T, E, E + 2, 1)
        got = rf.rfast_route_backward(logits.to(DEV), expert.to(DEV), weight.to(DEV), dweight.to(DEV), normalise=normalise, grad_dtype=out)
        assert torch.equal(got, o)


@pytest.mark.parametrize("normalise", [True, False])
def test_route_gradient_against_differences(normalise):
    """Of the weights over logits that stay in order: (w(l + h v) - w(l - h v)) / 2h, h = 2^-7."""
    g = gen(9)
    l = torch.stack([torch.randperm(20, generator=g) for _ in range(30)]) * 0.5 + 0.1 * torch.rand((30, 20), generator=g)
    v, dweight, h = torch.rand((30, 20), generator=g) - 0.5, normal(g, 30, 4), 2.0 ** -7
    r = rf.rfast_route(l.to(DEV), 4, normalise=normalise)
    up, down = (rf.rfast_route((l + s * v).to(DEV), 4, normalise=normalise) for s in (h, -h))
    assert torch.equal(up.expert, r.expert) and torch.equal(down.expert, r.expert)
    slope = (dweight.double() * (up.weight.cpu().double() - down.weight.cpu().double())).sum(dim=1) / (2 * h)
    got = (rf.rfast_route_backward(l.to(DEV), r.expert, r.weight, dweight.to(DEV), normalise=normalise).cpu().double() * v.double()).sum(dim=1)
    # third derivatives of a softmax along |v| <= 1/2 are below 1, so h^2 / 6 of them; roundings: some 40 HALF of weights below 1, over 2h
    assert ((slope - got).abs() <= dweight.double().abs().sum(dim=1) * (h * h / 6 + 40 * HALF / (2 * h) + 40 * HALF)).all()


# ----------------------------------------------------------------------------------------------------------- the rows
class Sent:
    """T rows to k of n experts each, some of them nowhere, `spare` rows behind the last."""

    def __init__(self, T, k, d, n=5, spare=3, kind=BF16, seed=0, drop=0.2):
        g = gen(seed + T + k + d)
        expert = torch.randint(0, n, (T, k), generator=g)
        expert[torch.rand((T, k), generator=g) < drop] = -1
        if T > 2:
            expert[T // 2] = -1
        _, place, order = exact_plan(expert.numpy(), n)
        self.T, self.k, self.d, self.kind = T, k, d, kind
        self.used, self.P = int((order >= 0).sum()), T * k + spare
        self.place, self.order = torch.from_numpy(place).to(I32), torch.from_numpy(order)
        self.place[self.place < 0] = torch.tensor([-1, self.P, 2 ** 31 - 1, -2 ** 31])[torch.arange(int((self.place < 0).sum())) % 4].to(I32)
        self.live = (self.place >= 0) & (self.place < self.P)
        self.x, self.rows, self.dy = (normal(g, n, d, dtype=kind) for n in (T, self.P, T))
        self.rows[self.used:] = NAN  # nobody's: not read
        self.weight = torch.rand((T, k), generator=g)
        self.weight[~self.live] = NAN

    def taken(self, rows):
        """[T][k][d] in 64 bits, zeros where there is no place."""
        got = rows.double()[torch.where(self.live, self.place, 0).long()]
        return torch.where(self.live[:, :, None], got, 0.0)


ROWS = [(1, 1, 1), (1, 4, 4096), (2, 64, 9), (3, 2, 5), (48, 2, 264), (65, 3, 65), (100, 8, 130), (33, 5, 513), (7, 1, 1024), (130, 2, 1025), (20, 6, 2056), (4, 3, 5003)]


@pytest.mark.parametrize("T,k,d", ROWS)
@pytest.mark.parametrize("kind", TYPES)
def test_gather(T, k, d, kind):
    c = Sent(T, k, d, kind=kind)
    want = torch.full((c.P, d), 77.0, dtype=kind)
    want[:c.used] = c.x[c.order[:c.used] // k]
    x, _ = apart(c.x, d + 1, 1)
    for off, extra in ((0, 0), (1, 7)):
        out, mem = apart(torch.full((c.P, d), 77.0, dtype=kind), d + extra, off)
        assert rf.rfast_route_gather(x, c.place.to(DEV), out=out) is out
        assert torch.equal(out.cpu(), want) and untouched(mem, c.P, d, d + extra, off)
    got = rf.rfast_route_gather(c.x.to(DEV), c.place.to(DEV))
    assert got.shape == (T * k, d) and torch.equal(got.cpu()[:c.used], want[:c.used])


@pytest.mark.parametrize("T,k,d", ROWS)
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("weighted", [True, False])
def test_combine(T, k, d, kind, out, weighted):
    c = Sent(T, k, d, kind=kind)
    w = torch.where(c.live, c.weight, 0.0).double() if weighted else torch.ones((T, k), dtype=F64)
    terms = c.taken(c.rows) * w[:, :, None]
    want, err = terms.sum(dim=1), (k + 1) * HALF * terms.abs().sum(dim=1)
    bound = err + (BF * (want.abs() + err) if out == BF16 else 0.0)
    weight = c.weight.to(DEV) if weighted else None
    y = rf.rfast_route_combine(c.rows.to(DEV), c.place.to(DEV), weight, out_dtype=out)
    within(y, want, bound, "rows")
    rows, _ = apart(c.rows, d + 3, 1)
    o, mem = apart(torch.zeros((T, d), dtype=out), d + 1, 1)
    assert rf.rfast_route_combine(rows, c.place.to(DEV), weight, out=o) is o
    assert torch.equal(o, y) and untouched(mem, T, d, d + 1, 1)


@pytest.mark.parametrize("T,k,d", ROWS)
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("weighted", [True, False])
def test_combine_backward(T, k, d, kind, weighted):
    c = Sent(T, k, d, kind=kind)
    products = c.taken(c.rows) * c.dy.double()[:, None, :]
    dw, dw_err = products.sum(dim=2), (d + 1) * HALF * products.abs().sum(dim=2)
    w = c.weight.double() if weighted else torch.ones((T, k), dtype=F64)
    exact = w[:, :, None] * c.dy.double()[:, None, :]
    want = torch.full((c.P, d), 77.0, dtype=F64)
    want[c.place[c.live].long()] = exact[c.live]
    weight = c.weight.to(DEV) if weighted else None
    rows, _ = apart(c.rows, d + 1, 1)
    dy, _ = apart(c.dy, d + 2, 1)
    o, mem = apart(torch.full((c.P, d), 77.0, dtype=kind), d + 3, 1)
    given = (rows, c.place.to(DEV), weight, dy)
    drows, dweight = rf.rfast_route_combine_backward(*given, drows=o)
    assert drows is o and untouched(mem, c.P, d, d + 3, 1)
    within(drows, want, want.abs() * (HALF + (BF * (1 + HALF) if kind == BF16 else 0.0)), "drows")
    assert (drows[c.used:] == 77.0).all()
    within(dweight, dw, dw_err, "dweight")
    assert not dweight.cpu()[~c.live].any()
    none, again = rf.rfast_route_combine_backward(*given, drows=False)
    assert none is None and torch.equal(again, dweight)
    again, none = rf.rfast_route_combine_backward(*given, dweight=False)
    assert none is None and torch.equal(again[:c.used], o[:c.used])


def test_combine_gradient_against_differences():
    """Bilinear, so differences are exact but for roundings."""
    c = Sent(40, 3, 50, kind=F32, drop=0.0)
    g = gen(12)
    rows, weight, place = torch.nan_to_num(c.rows), torch.nan_to_num(c.weight), c.place.to(DEV)
    v, u = normal(g, c.P, 50), normal(g, 40, 3)
    v[c.used:] = 0

    def along(s, t):
        return (c.dy.double() * rf.rfast_route_combine((rows + s * v).to(DEV), place, (weight + t * u).to(DEV)).cpu().double()).sum()

    drows, dweight = rf.rfast_route_combine_backward(rows.to(DEV), place, weight.to(DEV), c.dy.to(DEV))
    for slope, got in ((along(0.5, 0) - along(-0.5, 0), (drows.cpu().double()[:c.used] * v.double()[:c.used]).sum()),
                       (along(0, 0.5) - along(0, -0.5), (dweight.cpu().double() * u.double()).sum())):
        assert abs(slope - got) <= 40 * 50 * 3 * 5 * 5 * 4 * 10 * HALF  # 6000 terms below 100, ten roundings each


def test_rows_of_other_sizes():
    """Sorted rows fewer than the places say, none at all, no rows, no pairs."""
    c = Sent(10, 2, 24, kind=F32, drop=0.0)
    full = rf.rfast_route_gather(c.x.to(DEV), c.place.to(DEV))
    few = torch.full((7, 24), 77.0, device=DEV)
    rf.rfast_route_gather(c.x.to(DEV), c.place.to(DEV), out=few)
    assert torch.equal(few, full[:7])
    y = rf.rfast_route_combine(few, c.place.to(DEV))
    inside = (c.place < 7) & (c.place >= 0)
    assert torch.equal(y.cpu(), torch.where(inside[:, :, None], c.x[:, None, :], 0.0).sum(dim=1))
    none = torch.empty((0, 24), device=DEV)
    assert not rf.rfast_route_combine(none, c.place.to(DEV)).any()
    assert rf.rfast_route_gather(c.x.to(DEV), c.place.to(DEV), out=none) is none
    _, dw = rf.rfast_route_combine_backward(none, c.place.to(DEV), None, c.dy.to(DEV))
    assert not dw.any()
    empty = torch.empty((0, 2), dtype=I32, device=DEV)
    assert rf.rfast_route_gather(none, empty).shape == (0, 24) and rf.rfast_route_combine(full, empty).shape == (0, 24)
    r = rf.rfast_route(torch.empty((0, 8), device=DEV), 2)
    assert r.expert.shape == (0, 2) and r.row_ptr.cpu().tolist() == [0] * 9 and r.order.shape == (0,)
    assert rf.rfast_embedding(c.x.to(DEV), torch.empty(0, dtype=I32, device=DEV)).shape == (0, 24)


# ------------------------------------------------------------------------------------------------------------ policy
LOW, HIGH, BETA = 0.2, 0.28, 0.05


class Policy:
    def __init__(self, T, K, kind, seed=0, std=2.0, reference=True, weighted=True):
        g = gen(seed + T + K)
        logits = normal(g, T, K, std=std)
        if K > 4:
            logits[::5, 1::3] = -INF  # masked classes
        self.actions = torch.randint(0, K, (T,), generator=g)
        if K > 4:
            self.actions[::5] = self.actions[::5] // 3 * 3
        self.logits = logits.to(kind)
        self.T, self.K, self.kind = T, K, kind
        logs = torch.log_softmax(self.logits.double(), dim=1)
        self.logp = logs[torch.arange(T), self.actions]
        # ratios on both sides of both borders, none within a hundredth of one
        moved = torch.tensor([-0.5, -0.25, -0.1, 0.0, 0.1, 0.2, 0.3, 0.6], dtype=F64)[torch.randint(0, 8, (T,), generator=g)]
        self.old = (self.logp - moved).float()
        self.advantage = normal(g, T)
        self.advantage[::11] = 0.0
        self.reference = (self.logp + 0.3 * torch.randn(T, generator=g, dtype=F64)).float() if reference else None
        self.weight = torch.rand(T, generator=g) if weighted else None
        if weighted:
            self.weight[3::13] = 0.0
        self.actions = self.actions.to(I32)
        self.actions[2::9] = torch.tensor([-1, K, 2 ** 31 - 1, -2 ** 31])[torch.arange(len(self.actions[2::9])) % 4].to(I32)

    def exact(self, scale, low=LOW, high=HIGH, beta=BETA):
        """loss, grad, logp and bounds on the errors of each before a last rounding."""
        T, K = self.T, self.K
        l, rows = self.logits.double(), torch.arange(T)
        real = (self.actions >= 0) & (self.actions < K)
        at = torch.where(real, self.actions.long(), 0)
        shift = l.amax(dim=1, keepdim=True)
        p = torch.softmax(l, dim=1)
        spread = torch.where(l > -INF, shift - l, 0.0)
        log_sum = torch.logsumexp(l - shift, dim=1)
        # a row's sum: per lane at most 128 terms, one in 1024 of a longer row; 16 lanes and 16 wavefronts by trees
        in_sum = (p * (3 * spread + 4)).sum(dim=1) * HALF + (min(K, 144) + K / 1024) * HALF
        logp, own = torch.log_softmax(l, dim=1)[rows, at], l[rows, at] - shift[:, 0]
        logp_err = HALF * own.abs() + in_sum + 6 * HALF * log_sum.abs() + 2 * HALF * logp.abs() + HALF
        old, A = self.old.double(), self.advantage.double()
        ratio = torch.exp(logp - old)
        ratio_err = ratio * (logp_err + HALF * (logp - old).abs() + 4 * HALF)
        cut = ((A > 0) & (ratio > 1 + high)) | ((A < 0) & (ratio < 1 - low))
        gain = A * torch.where(cut, torch.where(A > 0, 1 + high, 1 - low).double(), ratio)
        gain_err = A.abs() * torch.where(cut, 4 * HALF, ratio_err) + 2 * HALF * gain.abs()
        loss, loss_err = -gain, gain_err
        slope, slope_err = torch.where(cut, 0.0, -gain), torch.where(cut, 0.0, gain_err)
        if self.reference is not None:
            q = self.reference.double() - logp
            q_err, m = logp_err + HALF * q.abs(), torch.expm1(q)
            m_err = torch.exp(q) * q_err + 4 * HALF * m.abs()
            loss = loss + beta * (m - q)
            loss_err = loss_err + beta * (m.abs() * q_err + 4 * HALF * m.abs() + 4 * HALF * (m.abs() + q.abs())) + HALF * loss.abs()
            slope, slope_err = slope - beta * m, slope_err + beta * (m_err + 3 * HALF * m.abs()) + HALF * (slope - beta * m).abs()
        w = (self.weight.double() if self.weight is not None else torch.ones(T, dtype=F64)) * real
        loss, loss_err = w * loss, w * loss_err + HALF * (w * loss).abs()
        c, c_err = w * slope * scale, (w * slope_err + 2 * HALF * (w * slope).abs()) * scale
        hot = torch.zeros((T, K), dtype=F64)
        hot[rows, at] = 1.0
        p_err = p * (3 * spread * HALF + (in_sum + 10 * HALF)[:, None])
        grad = c[:, None] * (hot - p)
        grad_err = c_err[:, None] * (hot - p).abs() + c.abs()[:, None] * (p_err + 2 * HALF * (hot + p)) + LEAST
        tiny = LEAST
        return (loss, loss_err + tiny), (grad, grad_err), (torch.where(real, logp, 0.0), torch.where(real, logp_err, 0.0))

    def dev(self):
        return [None if t is None else t.to(DEV) for t in (self.logits, self.actions, self.old, self.advantage, self.reference, self.weight)]


POLICIES = [(1, 2), (1, 7), (3, 1), (70, 4), (33, 9), (64, 64), (50, 65), (40, 128), (30, 200), (20, 513), (17, 1025), (9, 4100), (5, 20011), (3, 50001), (2, 36285), (2, 44000), (2, 60000), (2, 70003), (2, 89855), (2, 97003), (2, 120001),
            (2, 131065), (2, 131072)]


@pytest.mark.parametrize("T,K", POLICIES)
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("extras", [True, False])
def test_policy(T, K, kind, extras):
    c = Policy(T, K, kind, reference=extras, weighted=extras)
    l, a, old, adv, ref, weight = c.dev()
    scale = 0.75
    (loss, loss_err), (grad, grad_err), (logp, logp_err) = c.exact(scale)
    for out in TYPES:
        got = torch.full((T,), 77.0, device=DEV)
        y, g = rf.rfast_policy_loss(l, a, old, adv, reference=ref, weight=weight, clip=(LOW, HIGH), beta=BETA, grad_scale=scale, grad_dtype=out, logp=got)
        within(y, loss, loss_err, "loss")
        within(got, logp, logp_err, "logp")
        within(g, grad, grad_err + last(out) * (grad.abs() + grad_err), "gradient")
        assert not g.cpu()[c.logits == -INF].any()
    # in the logits' place, with rows apart, without a gradient
    m, mem = apart(c.logits, K + 3, 1)
    y2, g2 = rf.rfast_policy_loss(m, a, old, adv, reference=ref, weight=weight, clip=(LOW, HIGH), beta=BETA, grad_scale=scale, grad=m)
    within(g2, grad, grad_err + last(kind) * (grad.abs() + grad_err), "gradient in place")
    assert untouched(mem, T, K, K + 3, 1)
    y3, none = rf.rfast_policy_loss(l, a, old, adv, reference=ref, weight=weight, clip=(LOW, HIGH), beta=BETA, grad=False)
    assert none is None and torch.equal(y3, y)


def test_policy_without_clipping_is_cross_entropy():
    """old = logp and advantage 1: the loss is -1 and its gradient that of the cross-entropy."""
    c = Policy(200, 300, F32, reference=False, weighted=False)
    l, a, _, adv, _, _ = c.dev()
    loss, grad = rf.rfast_softmax_xent(l, a)
    got, g = rf.rfast_policy_loss(l, a, -loss, torch.ones_like(adv))
    real = ((c.actions >= 0) & (c.actions < 300)).to(DEV)
    # the ratio is exp of the difference of two roundings of the same number: off by two half steps of a number below 32 and those of expf
    off = 64 * HALF + 4 * HALF
    assert ((got[real] + 1).abs() <= off).all() and not got[~real].any()
    assert ((g - grad).abs() <= grad.abs() * (off + 4 * HALF) + 2 * HALF).all()


@pytest.mark.parametrize("K", [5, 100, 3000, 70000])
def test_policy_rows_at_the_edges(K):
    """Masked rows and actions, values that are not finite, weights of zero, ratios that overflow."""
    T = 12
    l = torch.randn((T, K), generator=gen(K))
    a = torch.full((T,), 1, dtype=I32)
    old, adv, ref, w = torch.full((T,), -2.0), torch.ones(T), torch.full((T,), -2.0), torch.ones(T)
    l[0] = -INF                        # masked out entirely
    l[1, 1] = -INF                     # the action is masked
    l[2, 1], old[2] = -INF, -INF       # and was
    l[3, 0] = NAN
    l[4, 2] = INF
    l[5, 0], w[5] = NAN, 0.0           # weight zero
    old[6], w[6] = NAN, 0.0
    old[7], adv[7] = -1e30, 1.0        # a ratio beyond 32 bits, clipped
    old[8], adv[8] = -1e30, 0.0        # of no advantage
    old[9], adv[9] = -1e30, -1.0       # that counts
    a[10], l[10, 0], old[10] = -1, NAN, NAN
    l[11] = 1e38                       # all alike and large
    given = [t.to(DEV) for t in (l, a, old, adv)]
    logp = torch.full((T,), 5.0, device=DEV)
    loss, grad = rf.rfast_policy_loss(*given, weight=w.to(DEV), logp=logp)
    loss, grad, logp = loss.cpu(), grad.cpu(), logp.cpu()
    assert loss[0] == 0 and not grad[0].any() and logp[0] == 0
    assert loss[1] == 0 and not grad[1].any() and logp[1] == -INF
    assert loss[2] == 0 and not grad[2].any() and logp[2] == -INF
    for t in (3, 4):
        assert loss[t].isnan() and grad[t].isnan().all() and logp[t].isnan()
    assert loss[5] == 0 and not grad[5].any() and loss[6] == 0 and not grad[6].any()
    assert abs(loss[7] + 1.2) <= 4 * HALF and not grad[7].any()
    assert loss[8] == 0 and not grad[8].any()
    assert loss[9] == INF and not grad[9].isfinite().all()
    assert loss[10] == 0 and not grad[10].any() and logp[10] == 0
    assert abs(logp[11] + np.log(K)) <= 200 * HALF * np.log(K) and grad[11].isfinite().all()
    loss, grad = (t.cpu() for t in rf.rfast_policy_loss(*given, reference=ref.to(DEV), weight=w.to(DEV), beta=0.5))
    assert loss[1] == INF and not grad[1].any() and loss[0] == 0 and not grad[0].any() and loss[10] == 0 and not grad[10].any()
    assert grad[11].isfinite().all() and grad[7].isfinite().all() and grad[7].any()


def test_policy_fewer_rows():
    c = Policy(40, 30, F32)
    l, a, old, adv, ref, w = c.dev()
    whole = rf.rfast_policy_loss(l, a, old, adv, reference=ref, weight=w, beta=0.1)
    for n in (0, 1, 17, 40, 99, -3):
        loss, grad, logp = torch.full((40,), 77.0, device=DEV), torch.full((40, 30), 77.0, device=DEV), torch.full((40,), 77.0, device=DEV)
        rf.rfast_policy_loss(l, a, old, adv, reference=ref, weight=w, beta=0.1, loss=loss, grad=grad, logp=logp, rows=torch.tensor([n], dtype=I32, device=DEV))
        m = min(max(n, 0), 40)
        assert torch.equal(loss[:m], whole[0][:m]) and torch.equal(grad[:m], whole[1][:m])
        assert (loss[m:] == 77).all() and (grad[m:] == 77).all() and (logp[m:] == 77).all()


def test_policy_gradient_against_differences():
    """Central differences along a direction, h = 2^-6, in logits of 32 bits; no ratio comes near a border on the way."""
    c = Policy(60, 40, F32, std=1.0)
    l, a, old, adv, ref, w = c.dev()
    v, h = (torch.rand((60, 40), generator=gen(3)) - 0.5) * 0.2, 2.0 ** -4

    def at(s):
        kw = dict(reference=ref, weight=w, clip=(LOW, HIGH), beta=BETA)
        return rf.rfast_policy_loss(l + s * v.to(DEV), a, old, adv, **kw)

    up, down = at(h)[0].cpu().double(), at(-h)[0].cpu().double()
    got = torch.nan_to_num((at(0.0)[1].cpu().double() * v.double())).sum(dim=1)
    # along v logp moves by at most 0.2 per unit, so third derivatives of r A and of the second term (r, exp(q) < 4) stay below (0.2)^3 * 8 * (|A| + beta) each;
    # roundings of a loss below 5 (|A| + 1): some 100 HALF with the sums of 40 terms, over 2h
    size = adv.cpu().double().abs() + 1
    assert ((up - down) / (2 * h) - got).abs().max() > 0
    assert (((up - down) / (2 * h) - got).abs() <= size * (h * h / 6 * 0.2 ** 3 * 8 * 4 + 5 * 100 * HALF / (2 * h))).all()


# ------------------------------------------------------------------------------------------------- refusals on tensors
def test_refusals_on_tensors():
    x, i = torch.zeros((4, 8), device=DEV), torch.zeros(4, dtype=I32, device=DEV)
    place, w = torch.zeros((4, 2), dtype=I32, device=DEV), torch.zeros((4, 2), device=DEV)
    f = torch.zeros(4, device=DEV)
    bad = [lambda: rf.rfast_embedding(x[0], i), lambda: rf.rfast_embedding(x, i.long()), lambda: rf.rfast_embedding(x.half(), i),
           lambda: rf.rfast_embedding(x.t(), i), lambda: rf.rfast_embedding(x, i, out=torch.zeros((4, 7), device=DEV)),
           lambda: rf.rfast_embedding(x, i.cpu()), lambda: rf.rfast_embedding(x, i, out=x), lambda: rf.rfast_embedding(x, i, out=x.clone(), out_dtype=BF16),
           lambda: rf.rfast_embedding_backward(x, i[:3], 5), lambda: rf.rfast_embedding_backward(x, i, 0), lambda: rf.rfast_embedding_backward(x, i, 5, accumulate=True),
           lambda: rf.rfast_embedding_backward(x, i, 5, grad=x), lambda: rf.rfast_embedding_backward(x, i, 4, grad=x), lambda: rf.rfast_embedding_backward(x, i, 5, grad_dtype=F64),
           lambda: rf.rfast_route(x, 0), lambda: rf.rfast_route(x, 9), lambda: rf.rfast_route(x.double(), 2), lambda: rf.rfast_route(torch.zeros((2, 1025), device=DEV), 2),
           lambda: rf.rfast_route(x[0], 1), lambda: rf.rfast_route_plan(i, 0), lambda: rf.rfast_route_plan(i.long(), 3), lambda: rf.rfast_route_plan(place.t(), 3),
           lambda: rf.rfast_route_gather(x, place[:3]), lambda: rf.rfast_route_gather(x, i), lambda: rf.rfast_route_gather(x, place, out=torch.zeros((8, 7), device=DEV)),
           lambda: rf.rfast_route_gather(x, place, out=torch.zeros((8, 8), device=DEV, dtype=BF16)), lambda: rf.rfast_route_gather(x, place, out=x),
           lambda: rf.rfast_route_gather(x, place.long()), lambda: rf.rfast_route_combine(x, place, w[:3]), lambda: rf.rfast_route_combine(x, place, w.double()),
           lambda: rf.rfast_route_combine(x, place, w, out=x), lambda: rf.rfast_route_combine_backward(x, place, w, x.bfloat16()),
           lambda: rf.rfast_route_combine_backward(x, place, w, x.clone(), drows=x), lambda: rf.rfast_route_backward(x, place, w, w[:3]),
           lambda: rf.rfast_route_backward(x, place.long(), w, w), lambda: rf.rfast_route_backward(x, place, w, w, normalise=False, dlogits=x),
           lambda: rf.rfast_policy_loss(x, i, f, f[:3]), lambda: rf.rfast_policy_loss(x, i.long(), f, f), lambda: rf.rfast_policy_loss(x, i, f, f, clip=(1.5, 0.2)),
           lambda: rf.rfast_policy_loss(x, i, f, f, beta=-1.0), lambda: rf.rfast_policy_loss(x, i, f, f.clone(), loss=f), lambda: rf.rfast_policy_loss(x.half(), i, f, f),
           lambda: rf.rfast_policy_loss(x, i, f, f, weight=f.double()), lambda: rf.rfast_policy_loss(x, i, f, f, reference=f.cpu())]
    for k, call in enumerate(bad):
        with pytest.raises(RFastError):
            call()
            print("accepted:", k)


# ----------------------------------------------------------------------------------------------- all of them together
class Step:
    """A training step of a policy whose tokens go through adapters chosen by a router: embedding, router, dispatch, adapters, return, head,
    policy loss, and back to the gradients of the table, the router's projection and the adapters.  Projections that are not adapters are the
    program's own products, in 32 bits."""

    def __init__(self, T=300, V=500, d=64, E=6, k=2, K=130, rank=4, seed=0):
        g = gen(seed)
        self.sizes = (T, V, d, E, k, K)
        self.table, self.gate = normal(g, V, d, std=0.5), normal(g, E, d, std=0.3)
        self.w, self.a, self.b = normal(g, d, d, std=d ** -0.5, dtype=BF16), normal(g, E, rank, d, std=d ** -0.5, dtype=BF16), normal(g, E, d, rank, std=0.5, dtype=BF16)
        self.head = normal(g, K, d, std=d ** -0.5)
        self.tokens = torch.randint(0, V, (T,), generator=g, dtype=I32)
        self.tokens[5::50] = -1
        self.actions = torch.randint(0, K, (T,), generator=g, dtype=I32)
        self.actions[5::50] = -1
        # (far from the borders of the clipping, on either side: logp is about -5)
        self.old, self.adv, self.ref = torch.where(torch.arange(T) % 2 == 0, -8.0, -2.0), normal(g, T), normal(g, T, std=0.1) - 5.0

    def to_device(self):
        for n, t in list(vars(self).items()):
            if isinstance(t, torch.Tensor):
                setattr(self, n, t.to(DEV))
        return self

    def run(self):
        T, V, d, E, k, K = self.sizes
        x = rf.rfast_embedding(self.table, self.tokens)
        choice = (x @ self.gate.t()).masked_fill_((self.tokens < 0)[:, None], -INF)  # padding goes to no expert
        r = rf.rfast_route(choice, k)
        xb = x.to(BF16)
        rows = rf.rfast_route_gather(xb, r.place, out=torch.full((T * k, d), NAN, dtype=BF16, device=DEV))
        out = rf.rfast_lora_forward(rows, self.w, self.a, self.b, r.row_ptr, scale=0.5, out=torch.full_like(rows, NAN))
        y = rf.rfast_route_combine(out, r.place, r.weight, out_dtype=F32)
        logits = y @ self.head.t()
        logp = torch.empty_like(self.old)
        loss, dl = rf.rfast_policy_loss(logits, self.actions, self.old, self.adv, reference=self.ref, beta=0.1, grad_scale=1.0 / T, logp=logp)
        dy = (dl @ self.head).to(BF16)
        dout, dweight = rf.rfast_route_combine_backward(out, r.place, r.weight, dy, drows=torch.full_like(out, NAN))
        drows, da, db = rf.rfast_lora_backward(rows, self.w, self.a, self.b, r.row_ptr, None, dout, scale=0.5)
        dgate_logits = rf.rfast_route_backward(choice, r.expert, r.weight, dweight)
        dx = rf.rfast_route_combine(drows, r.place, out_dtype=F32) + dgate_logits @ self.gate
        dtable = rf.rfast_embedding_backward(dx, self.tokens, V)
        return dict(expert=r.expert, loss=loss, logp=logp, head=dl.t() @ y, a=da, b=db, gate=dgate_logits.t() @ x, table=dtable)

    def exact(self, expert):
        """The same by autograd in 64 bits on the CPU, roundings to bf16 where the step has them (passed over by the gradient)."""
        T, V, d, E, k, K = self.sizes

        def rounded(t):
            return t + (t.to(BF16).to(F64) - t).detach()

        p = {n: getattr(self, n).double().requires_grad_() for n in ("table", "gate", "a", "b", "head")}
        real = (self.tokens >= 0).double()[:, None]
        x = p["table"][self.tokens.clamp(min=0).long()] * real
        chosen = torch.gather(x @ p["gate"].t(), 1, expert.clamp(min=0).long())
        weight = torch.softmax(chosen, dim=1)
        xb = rounded(x)
        y = 0
        for j in range(k):
            e = expert[:, j].clamp(min=0).long()
            u = torch.matmul(p["a"][e], xb[:, :, None])
            out = rounded(xb @ self.w.double().t() + 0.5 * torch.matmul(p["b"][e], u)[:, :, 0])
            y = y + weight[:, j:j + 1] * out * real
        logs = torch.log_softmax(y @ p["head"].t(), dim=1)
        counts = self.actions >= 0
        logp = logs[torch.arange(T), self.actions.clamp(min=0).long()]
        ratio, A = torch.exp(logp - self.old.double()), self.adv.double()
        q = self.ref.double() - logp
        loss = -torch.minimum(ratio * A, ratio.clamp(0.8, 1.2) * A) + 0.1 * (torch.exp(q) - q - 1)
        loss = loss * counts
        (loss.sum() / T).backward()
        return dict(loss=loss.detach(), logp=(logp * counts).detach(), **{n: t.grad for n, t in p.items()}), ratio.detach()


def test_a_step_of_all():
    s = Step()
    got = {n: t.cpu() for n, t in s.to_device().run().items()}
    s = Step()
    x = torch.where((s.tokens >= 0)[:, None], s.table[s.tokens.clamp(min=0).long()], 0.0).double()
    near = torch.sort(x @ s.gate.double().t(), dim=1, descending=True)
    assert torch.equal(got["expert"][s.tokens >= 0].long(), near.indices[:, :2][s.tokens >= 0])
    assert (got["expert"][s.tokens < 0] == -1).all() and (s.tokens < 0).any()
    want, ratio = s.exact(got["expert"])
    clear = ((ratio - 0.8).abs() > 1e-3) & ((ratio - 1.2).abs() > 1e-3) | (s.actions < 0)
    assert clear.all()
    for name in ("loss", "logp", "head", "a", "b", "gate", "table"):
        w = want[name]
        off = (got[name].double() - w).norm() / w.norm()
        # forward the roundings are the same but for numbers next to a border of two bf16; backward dy, dout and drows are rounded
        # to bf16 once each, and dout's product with the weights once more: four roundings of 2^-8, in norm
        assert off <= 4 * BF, (name, float(off))


def test_a_step_captured_and_replayed():
    """Every replay is the eager step, with the program's own work between, and while an eager run of the same tensors lives."""
    s = Step(seed=4).to_device()
    s.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = s.run()
    for turn in range(5):
        s.tokens.copy_((s.tokens + 7 * turn) % s.sizes[1])
        s.adv.mul_(0.9)
        want = s.run()
        for t in out.values():
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        for n in out:
            assert torch.equal(out[n], want[n]), (turn, n)


def test_two_graphs_and_two_streams_share_nothing():
    steps = [Step(seed=5).to_device(), Step(T=517, V=90, d=128, E=9, k=3, K=70, rank=8, seed=6).to_device()]
    alone = [s.run() for s in steps]
    torch.cuda.synchronize()
    streams, graphs, outs = [torch.cuda.Stream(), torch.cuda.Stream()], [], []
    for s in steps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(s.run())
        graphs.append(g)
    for _ in range(4):
        eager = []
        for k in (0, 1):
            with torch.cuda.stream(streams[k]):
                graphs[k].replay()
                eager.append(steps[k].run())
        torch.cuda.synchronize()
        for k in (0, 1):
            for n in alone[k]:
                assert torch.equal(outs[k][n], alone[k][n]) and torch.equal(eager[k][n], alone[k][n]), n


def test_updates_by_adamw():
    """The step's gradients as the optimizer's: parameters move, and gradients stay where the optimizer reads them."""
    s = Step(seed=7).to_device()
    grads = {n: t for n, t in s.run().items() if n in ("table", "head", "gate")}
    params = {n: getattr(s, n) for n in grads}
    before = {n: p.clone() for n, p in params.items()}
    opt = RFastAdamW(list(params.values()), list(grads.values()))
    opt.step(1e-2)
    for n, p in params.items():
        # the first step of AdamW moves every coordinate with a gradient well above eps by gamma
        moved, large = (p - before[n]).abs(), grads[n].abs() > 1e-5
        assert large.any() and ((moved[large] - 1e-2).abs() <= 1e-2 * 2e-3 + 4 * HALF).all() and not moved[grads[n] == 0].any()
