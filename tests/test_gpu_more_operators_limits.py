"""Embeddings, rows to experts and back, and the policy loss where their range ends: offsets that pass 32 bits, lengths around those where the
sort changes its form, masks of the type's lowest value, memory that is handed on.

What a call computes of rows far behind is compared with the same call on those rows alone, bit for bit: neither the arithmetic nor its
order depends on where rows are."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import paper_2307_11617_amd as rf  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32
INF = float("inf")


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def tiled(rows, d, dtype, seed=0):
    """A large matrix of few random rows repeated."""
    few = torch.randn((997, d), generator=gen(seed)).to(dtype).to(DEV)
    out = torch.empty((rows, d), dtype=dtype, device=DEV)
    for i in range(0, rows, 997):
        out[i:i + 997] = few[:min(997, rows - i)]
    return out


def test_embedding_offsets_pass_32_bits():
    V, d = 560001, 8192  # 4.6e9 elements
    table = tiled(V, d, BF16)
    tokens = torch.tensor([V - 1, 0, 524287, 524288, 262144, V - 3, -1, V], dtype=I32)
    out = rf.rfast_embedding(table, tokens.to(DEV), scale=0.5)
    want = table[tokens[:6].long().to(DEV)] * 0.5
    assert torch.equal(out[:6], want) and not out[6:].any()
    dy = torch.randn((8, d), generator=gen(1)).to(BF16).to(DEV)
    grad = table  # written whole: zeros but for the tokens' rows
    rf.rfast_embedding_backward(dy, tokens.to(DEV), V, scale=2.0, grad=grad)
    assert torch.equal(grad[tokens[:6].long().to(DEV)], dy[:6] * 2.0)
    grad[tokens[:6].long().to(DEV)] = 0
    assert all(not grad[i:i + 40000].any() for i in range(0, V, 40000))
    rf.rfast_embedding_backward(dy, tokens.to(DEV), V, scale=2.0, grad=grad, accumulate=True)
    assert torch.equal(grad[tokens[:6].long().to(DEV)], dy[:6] * 2.0)


def test_embedding_rows_pass_32_bits():
    T, d, V = 530001, 8192, 4096
    dy = tiled(T, d, BF16)
    tokens = torch.full((T,), -1, dtype=I32)
    at = torch.tensor([0, 5, 262143, 524287, 524288, T - 2, T - 1])
    tokens[at] = torch.tensor([7, 9, 7, 4095, 7, 9, 7], dtype=I32)
    got = rf.rfast_embedding_backward(dy, tokens.to(DEV), V)
    want = rf.rfast_embedding_backward(dy[at.to(DEV)], tokens[at].to(DEV), V)
    assert torch.equal(got, want) and got.any()
    table = torch.randn((V, d), generator=gen(2)).to(BF16).to(DEV)
    out = rf.rfast_embedding(table, tokens.to(DEV), out=dy)
    assert torch.equal(out[at.to(DEV)], table[tokens[at].long().to(DEV)]) and not out[1:5].any() and not out[524289:T - 2].any()


def test_rows_pass_32_bits():
    T, k, d = 280001, 2, 8192
    x = tiled(T, d, BF16)
    place = torch.randperm(T * k, generator=gen(3)).to(I32).view(T, k)
    place[5, 1] = -1
    place, weight = place.to(DEV), torch.rand((T, k), generator=gen(4)).to(DEV)
    rows = rf.rfast_route_gather(x, place)
    for t in (0, 5, 131071, 262143, 262144, T - 1):
        for j in range(k):
            if place[t, j] >= 0:
                assert torch.equal(rows[place[t, j].long()], x[t])
    y = rf.rfast_route_combine(rows, place, weight, out=torch.empty_like(x))
    far = [0, 5, 262143, 262144, T - 2, T - 1]
    at = torch.where(place[far] >= 0, torch.arange(len(far) * k, device=DEV, dtype=I32).view(-1, k), -1)
    few = rows[place[far].clamp(min=0).long().view(-1)]
    assert torch.equal(y[far], rf.rfast_route_combine(few, at, weight[far]))
    drows, dweight = rf.rfast_route_combine_backward(rows, place, weight, x, drows=torch.zeros_like(rows))
    want, want_weight = rf.rfast_route_combine_backward(few, at, weight[far], x[far], drows=torch.zeros_like(few))
    assert torch.equal(dweight[far], want_weight)
    live = at.view(-1) >= 0
    assert torch.equal(drows[place[far].view(-1)[live].long()], want[live])


def test_policy_offsets_pass_32_bits():
    T, K = 70001, 65537
    logits = tiled(T, K, BF16)
    actions = torch.randint(0, K, (T,), generator=gen(5), dtype=I32).to(DEV)
    old, adv = torch.randn(T, generator=gen(6)).to(DEV) - 11.0, torch.randn(T, generator=gen(7)).to(DEV)
    far = [0, 1, 32767, 32768, 65535, 65536, T - 1]
    want_loss, want = rf.rfast_policy_loss(logits[far], actions[far], old[far], adv[far])
    loss, grad = rf.rfast_policy_loss(logits, actions, old, adv, grad=logits)
    assert torch.equal(loss[far], want_loss) and torch.equal(grad[far], want)


@pytest.mark.parametrize("kind,out", [(BF16, BF16), (F32, F32)])
def test_losses_past_the_caches(kind, out):
    """A gradient of more than 256 MB takes another way out than one of a few rows.

    Rows of an odd number of classes begin at different places behind a multiple of 16 bytes, from which groups of logits are counted, so the order of
    a row's sum differs between the two calls.  Its terms are positive and the longest chain of additions has at most 144 of them (128 of a
    lane, 6 + 4 of trees, and some), so two orders differ by 288 half steps of 32 bits relative, and with them e / sum; a logarithm by as much
    absolutely, and by 8 half steps of itself for its function, product and sums.  The gradient then rounds three times, and to its type."""
    T, K = 3001, 50001
    half = 2.0 ** -24
    logits = tiled(T, K, kind)
    actions = torch.randint(-1, K, (T,), generator=gen(8), dtype=I32).to(DEV)
    old, adv = torch.randn(T, generator=gen(9)).to(DEV) - 11.0, torch.randn(T, generator=gen(10)).to(DEV)
    some = [0, 1, 1500, T - 2, T - 1]
    xent = rf.rfast_softmax_xent(logits[some], actions[some])
    policy = rf.rfast_policy_loss(logits[some], actions[some], old[some], adv[some])
    hot = torch.nn.functional.one_hot(actions[some].clamp(min=0).long(), K) * (actions[some] >= 0)[:, None]

    def alike(loss, grad, want, factor, more):
        """factor: what multiplies softmax - onehot; more: its relative error."""
        off = 288 * half + 8 * half * (want[0].abs() + 12)
        assert ((loss[some] - want[0]).abs() <= factor * off + 8 * half * want[0].abs()).all()
        g, w = grad[some].double(), want[1].double()
        bound = (w.abs() + factor[:, None] * hot) * (288 + 8 + more[:, None]) * half + 2 * (2.0 ** -8 if out == BF16 else half) * w.abs()
        assert ((g - w).abs() <= bound).all()

    loss, grad = rf.rfast_softmax_xent(logits, actions, grad_dtype=out)
    alike(loss, grad, xent, torch.ones(5, device=DEV), torch.zeros(5, device=DEV))
    # the ratio's error is that of logp (below 24): 288 half steps and 8 of 24, and it is at most the loss over the advantage where it is not clipped
    loss, grad = rf.rfast_policy_loss(logits, actions, old, adv, grad=logits)
    alike(loss, grad, policy, torch.maximum(policy[0].abs(), torch.ones(5, device=DEV)), torch.full((5,), 288.0 + 8 * 24 + 8, device=DEV))


@pytest.mark.parametrize("T,k,d", [(70000, 3, 1000), (9000, 9, 2048)])
def test_rows_past_the_caches(T, k, d):
    """So do more than 256 MB of rows."""
    place = torch.randperm(T * k, generator=gen(11)).to(I32).view(T, k)
    place[7, 0] = -1
    place, weight, x = place.to(DEV), torch.rand((T, k), generator=gen(12)).to(DEV), tiled(T, d, BF16)
    rows = rf.rfast_route_gather(x, place, out=torch.zeros((T * k, d), dtype=BF16, device=DEV))
    want = torch.zeros_like(rows)
    for j in range(k):
        live = place[:, j] >= 0
        want[place[live, j].long()] = x[live]
    assert torch.equal(rows, want)
    some = [0, 7, T // 2, T - 1]
    at = torch.where(place[some] >= 0, torch.arange(len(some) * k, device=DEV, dtype=I32).view(-1, k), -1)
    few = rows[place[some].clamp(min=0).long().view(-1)]
    assert torch.equal(rf.rfast_route_combine(rows, place, weight)[some], rf.rfast_route_combine(few, at, weight[some]))
    drows, dweight = rf.rfast_route_combine_backward(rows, place, weight, x, drows=want)
    want, want_weight = rf.rfast_route_combine_backward(few, at, weight[some], x[some])
    live = at.view(-1) >= 0
    assert torch.equal(dweight[some], want_weight) and torch.equal(drows[place[some].view(-1)[live].long()], want[live])


@pytest.mark.parametrize("pairs", [255, 256, 257, 1023, 1024, 1025, 2047, 2048, 2049, 3073, 8192, 32767, 32768, 32769, 262144, 262145])
@pytest.mark.parametrize("experts", [40, 200, 400, 900, 60000, 300000])
def test_sort_where_its_form_changes(pairs, experts):
    rng = np.random.default_rng(pairs + experts)
    expert = (rng.random(pairs) ** 2 * (experts + 2)).astype(np.int32) - 1
    inside = np.nonzero((expert >= 0) & (expert < experts))[0]
    inside = inside[np.argsort(expert[inside], kind="stable")]
    place, order = np.full(pairs, -1), np.full(pairs, -1)
    place[inside], order[:inside.size] = np.arange(inside.size), inside
    row_ptr, p, o = rf.rfast_route_plan(torch.from_numpy(expert).to(DEV), experts)
    assert np.array_equal(row_ptr.cpu().numpy(), np.searchsorted(expert[inside], np.arange(experts + 1)))
    assert np.array_equal(p.cpu().numpy(), place) and np.array_equal(o.cpu().numpy(), order)


@pytest.mark.parametrize("T", [16, 17, 63, 64, 65, 255, 256, 257, 4096, 4097, 8192, 8193])
@pytest.mark.parametrize("V,d,gap", [(70, 8, 0), (70, 8, 3), (3000, 20, 0), (5, 1500, 1), (900, 256, 0), (900, 264, 0), (12, 7, 0)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embedding_gradient_where_its_form_changes(T, V, d, gap, accumulate):
    """Small whole numbers, whose sums are exact in 32 bits, so that every order gives the same bits; rows of padding hold NaN."""
    g = gen(T + V + d)
    tokens = torch.randint(-1, V + 1, (T,), generator=g, dtype=I32)
    tokens[torch.rand(T, generator=g) < 0.3] = V // 2
    dy = torch.randint(-8, 9, (T, d), generator=g).float()
    real = (tokens >= 0) & (tokens < V)
    grad = torch.randint(-8, 9, (V, d + gap), generator=g).float()
    want = grad.clone()
    if not accumulate:
        want[:, :d] = 0
    want[:, :d].index_put_((tokens[real].long(),), dy[real] * 2, accumulate=True)
    dy[~real] = float("nan")
    grad = grad.to(DEV)
    rf.rfast_embedding_backward(dy.to(DEV), tokens.to(DEV), V, scale=2.0, grad=grad[:, :d], accumulate=accumulate)
    assert torch.equal(grad.cpu(), want)
    grad = grad.to(BF16) * 0 + 1
    half = dy.to(BF16).to(DEV)
    rf.rfast_embedding_backward(half, tokens.to(DEV), V, scale=2.0, grad=grad[:, :d], accumulate=accumulate)
    total = torch.zeros((V, d)).index_put_((tokens[real].long(),), dy[real] * 2, accumulate=True) + (1 if accumulate else 0)
    assert torch.equal(grad[:, :d].cpu(), total.to(BF16)) and (grad[:, d:] == 1).all()


@pytest.mark.parametrize("rows", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 128, 129, 256, 257])
@pytest.mark.parametrize("experts,k", [(5, 3), (64, 4), (65, 8), (300, 1)])
def test_router_where_one_workgroup_ends(rows, experts, k):
    """The same rows in a longer batch, and the order of their choices made apart."""
    logits = torch.randn((rows, experts), generator=gen(rows + experts)).to(DEV)
    r = rf.rfast_route(logits, k)
    long = rf.rfast_route(torch.cat([logits, torch.randn((2000, experts), generator=gen(9)).to(DEV)]), k)
    assert torch.equal(r.expert, long.expert[:rows]) and torch.equal(r.weight, long.weight[:rows])
    for a, b in zip(r[2:], rf.rfast_route_plan(r.expert, experts)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masks_of_the_lowest_value(dtype):
    """Not masked out, but of no weight beside any other; alone, all alike."""
    low = torch.finfo(dtype).min
    l = torch.full((3, 70), low)
    l[0, 5], l[0, 9] = 1.0, 2.0
    l[2, 3] = -INF
    l = l.to(dtype).to(DEV)
    for normalise in (True, False):
        r = rf.rfast_route(l, 4, normalise=normalise)
        assert r.expert.tolist() == [[9, 5, 0, 1], [0, 1, 2, 3], [0, 1, 2, 4]]
        assert r.weight[0, 2:].tolist() == [0.0, 0.0] and abs(float(r.weight[0].sum()) - 1) < 1e-6
        share = 0.25 if normalise else 1 / 70
        # one division of whole numbers, or of 70 ones by their sum
        assert (r.weight[1] - share).abs().max() <= 2.0 ** -23 * share
        d = rf.rfast_route_backward(l, r.expert, r.weight, torch.ones_like(r.weight), normalise=normalise)
        assert torch.isfinite(d).all()
    a = torch.tensor([9, 3, 4], dtype=I32, device=DEV)
    old, adv = torch.tensor([-0.5, -4.0, -4.0], device=DEV), torch.ones(3, device=DEV)
    logp = torch.empty(3, device=DEV)
    loss, grad = rf.rfast_policy_loss(l, a, old, adv, reference=old, beta=0.1, logp=logp)
    assert torch.isfinite(loss).all() and torch.isfinite(grad).all() and torch.isfinite(logp).all()
    assert not grad[0, :5].any() and grad[2, 3] == 0 and abs(float(logp[1]) + np.log(70)) < 1e-5


def test_memory_is_handed_on_in_order():
    """Workspaces and results of many calls in a row come out of the same memory, and no call sees another's."""
    tokens = [torch.randint(-1, 3000, (n,), generator=gen(n), dtype=I32).to(DEV) for n in (5000, 40, 9000, 70, 3000)]
    dys = [torch.randn((len(t), 96), generator=gen(1)).to(DEV) for t in tokens]
    want = [rf.rfast_embedding_backward(dy, t, 3000).clone() for dy, t in zip(dys, tokens)]
    torch.cuda.synchronize()
    for _ in range(20):
        got = [rf.rfast_embedding_backward(dy, t, 3000) for dy, t in zip(dys, tokens)]
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        del got
