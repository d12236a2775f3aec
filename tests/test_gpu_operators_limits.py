"""The operators on tensors where their range ends: moments that fade, memory that is handed on, extents of 32 bits.

Tolerances as in test_gpu_operators.py: bounds from the roundings on the way."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
import harness  # noqa: E402
from paper_2307_11617_amd import RFastAdamW, RFastError, rfast_lora_backward, rfast_lora_forward, rfast_softmax_xent  # noqa: E402
from test_gpu_adapters import quad  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
LEAST = 448 * 2.0 ** -126  # a block whose largest magnitude is below this is held as zeros


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def test_adamw_eight_bits_after_the_last_gradient():
    """Gradients that end, as an adapter's without rows: its moments fade to nothing over a thousand steps, and no parameter is lost."""
    p = torch.randn(700, generator=gen(1)).to(DEV)
    g = torch.zeros(700, device=DEV)
    g[::3] = torch.randn(234, generator=gen(2)).to(DEV) * 1e-3
    start, touched = p.clone(), g != 0
    o = RFastAdamW([p], [g], state_bits=8)
    for _ in range(3):
        o.step(1e-3)
    g.zero_()
    for _ in range(500):
        o.step(1e-3)
    after = p.clone()  # from here a step is 0.9^500 of the first ones, nothing beside a parameter
    for _ in range(500):
        o.step(1e-3)
    assert torch.isfinite(p).all() and torch.equal(p, after)
    assert torch.equal(p[~touched], start[~touched]) and (p[touched] != start[touched]).all()
    m, v = o.m[0].view(F8).float(), o.v[0].view(F8).float()
    assert torch.isfinite(v).all() and (v[touched] > 0).all()
    assert (m == 0).all() and (o.m_scale[0] == 0).all() and (o.steps() == 1003).all()


@pytest.mark.parametrize("top", [1e-44, 1e-40, 1e-38, 1.2e-36, 5e-36, 5.9e-36, 1e-34, 1e-30])
def test_adamw_eight_bits_tiny_moments(top):
    """A block of moments of every size around what a scale can hold, without a gradient: one step makes 0.9 of them, or zeros."""
    p = torch.randn(256, generator=gen(3)).to(DEV)
    start = p.clone()
    codes = torch.linspace(-448, 448, 257)[:256].to(F8)
    codes[100:140] = 0
    scale = torch.tensor([top / 448], dtype=F32)
    m, s = codes.to(DEV), scale.to(DEV)
    m0 = (codes.float() * scale).double()
    o = RFastAdamW([p], [torch.zeros(256, device=DEV)], m=[m], v=[torch.zeros(256, dtype=F8, device=DEV)], m_scale=[s],
                   v_scale=[torch.zeros(1, device=DEV)], state_bits=8, steps=100)
    o.step(1e-3)
    assert torch.equal(p, start)  # at most 1e-3 * 1e-30 / 1e-8
    want = 0.9 * m0
    got = (m.float().cpu() * s.cpu()).double()
    assert torch.isfinite(m.float()).all()
    if 0.9 * top < LEAST:
        assert (got == 0).all() and s.item() == 0
    else:
        assert abs(s.item() - 0.9 * top / 448) <= 2.0 ** -21 * top / 448
        # half a step of a code, of the smallest codes half their distance 2^-9; the roundings of 0.9, the products and the scale
        bound = (2.0 ** -4 + 2.0 ** -20) * want.abs() + 2.0 ** -10 * s.item() * (1 + 2.0 ** -20) + 2.0 ** -148
        assert ((got - want).abs() <= bound).all()


def test_adamw_rounds_eight_bits_tiny_moments():
    """The same of the rounds' variant: nodes whose moments have faded go on as if they had none."""
    w = quad(5, 300, 31)
    gpu = harness.make_gpu(w)
    gpu.set_adamw(state_bits=8)
    gpu.init(np.random.default_rng(4).standard_normal((w.n, w.p)).astype(np.float32), None)
    codes = np.arange(w.n * w.p, dtype=np.int64).reshape(w.n, w.p) % 120  # finite codes, zero among them
    gpu.write("ADAMW_M", codes.astype(np.uint8))
    gpu.write("ADAMW_M_SCALE", np.full((w.n, 2), 2e-39, np.float32))
    gpu.write("Z", np.zeros((w.n, w.p), np.float32))
    x = gpu.read("X")
    everyone = torch.ones((1, w.n), dtype=torch.uint8, device=DEV)
    st, dev = harness.upload_chunk(gpu, w, 0, 1)
    gpu.run(1, everyone, dev["delay_R"], dev["delay_C"], dev["drop_R"], dev["drop_C"], w.gamma, None)
    gpu.check()
    assert (gpu.read("ADAMW_M") == 0).all() and (gpu.read("ADAMW_M_SCALE") == 0).all()
    st, dev = harness.upload_chunk(gpu, w, 1, 20)
    gpu.run(19, dev["active"], dev["delay_R"], dev["delay_C"], dev["drop_R"], dev["drop_C"], w.gamma, None)
    gpu.check()
    assert np.isfinite(gpu.read("X")).all() and (gpu.read("X") != x).any()
    assert ((gpu.read("ADAMW_M") & 0x7F) != 0x7F).all() and ((gpu.read("ADAMW_V") & 0x7F) != 0x7F).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_memory_of_its_own_outlives_the_object(bits):
    """Moments, scales and workspace that the object made are not handed on while steps on other streams still use them."""
    g = gen(5)
    first = [torch.randn(700001, generator=g).to(DEV) for _ in range(6)]
    grads = [torch.randn(700001, generator=g).to(DEV) for _ in range(6)]
    want = [p.clone() for p in first]
    plain = RFastAdamW(want, grads, state_bits=bits)
    for _ in range(40):
        plain.step(1e-2)
    torch.cuda.synchronize()
    for streams in (1, 2):
        params = [p.clone() for p in first]
        opt = RFastAdamW(params, grads, state_bits=bits)
        sizes = [t.numel() * t.element_size() for t in [*opt.m, *opt.v, *(s for s in opt.m_scale + opt.v_scale if s is not None), opt.workspace]]
        torch.cuda.synchronize()
        sides = [torch.cuda.Stream() for _ in range(streams)]
        for k in range(streams):
            sides[k].wait_stream(sides[k - 1])
            with torch.cuda.stream(sides[k]):
                for _ in range(40 // streams):
                    opt.step(1e-2)
        del opt
        taken = [torch.full((b,), 255, dtype=torch.uint8, device=DEV) for b in sizes for _ in (0, 1)]
        torch.cuda.synchronize()
        for t in taken:
            assert (t == 255).all()
        for p, q in zip(params, want):
            assert torch.equal(p, q)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_smallest_eps(bits):
    """The smallest eps that is taken leaves what never had a gradient alone; smaller ones are refused, by the rounds' variant too."""
    p = torch.ones(300, device=DEV)
    g = torch.zeros(300, device=DEV)
    g[::2] = 1e-3
    o = RFastAdamW([p], [g], state_bits=bits, eps=2.0 ** -126)
    for _ in range(3):
        o.step(1e-2)
    assert torch.equal(p[1::2], torch.ones(150, device=DEV)) and torch.isfinite(p).all() and (p[::2] < 1).all()
    w = quad(3, 40, 33)
    gpu = harness.make_gpu(w)
    for eps in (2.0 ** -127, 1e-60):
        with pytest.raises(RFastError, match="eps"):
            RFastAdamW([p], [g], state_bits=bits, eps=eps)
        with pytest.raises(RFastError, match="eps"):
            gpu.set_adamw(eps=eps, state_bits=bits)
    gpu.set_adamw(eps=2.0 ** -126, state_bits=bits)
    gpu.init(None, None)
    gpu.write("Z", np.zeros((w.n, w.p), np.float32))
    st, dev = harness.upload_chunk(gpu, w, 0, 1)
    gpu.run(1, torch.ones((1, w.n), dtype=torch.uint8, device=DEV), dev["delay_R"], dev["delay_C"], dev["drop_R"], dev["drop_C"], w.gamma, None)
    gpu.check()
    assert np.isfinite(gpu.read("X")).all()


@pytest.mark.parametrize("left", [0, 7, 900])
def test_xent_longest_rows(left):
    """Rows of nearly 2^31 classes: offsets within a row pass 32 bits.  One that counts, padding, one that is masked out entirely."""
    K = 2 ** 31 - 1 - left
    logits = torch.zeros((1, K), dtype=BF16, device=DEV)
    label = torch.tensor([K - 3], dtype=torch.int32, device=DEV)
    loss, grad = rfast_softmax_xent(logits, label, grad_scale=2.0 ** 40, grad=logits)
    # K equal logits: sums of ones are exact in each of 1024 lanes (2^21) and off by 2^-24 of the sum at each of ten joins; log and the division
    # by four steps; the gradient is rounded to bf16
    assert abs(loss.item() - np.log(K)) <= 2.0 ** -19 * np.log(K)
    p = 2.0 ** 40 / K
    assert abs(grad[0, K - 3].item() - (p - 2.0 ** 40)) <= 2.0 ** -8 * 2.0 ** 40
    grad[0, K - 3] = grad[0, 0]
    assert abs(grad[0, 0].item() - p) <= 2.0 ** -7 * p and (grad == grad[0, 0]).all()
    for lse in (None, torch.zeros(1, device=DEV)):
        logits.fill_(1.0)
        loss, grad = rfast_softmax_xent(logits, torch.full_like(label, -1), grad=logits, lse=lse)
        assert loss.item() == 0 and not grad.any()
    logits.fill_(float("-inf"))
    loss, grad = rfast_softmax_xent(logits, label, grad=logits)
    assert loss.item() == 0 and not grad.any()


def test_extents_that_32_bits_do_not_hold_are_refused():
    """Sizes of 2^32 and a little more are not taken for that little."""
    wide = torch.empty((1, 2 ** 32 + 8), dtype=BF16, device=DEV)
    label = torch.zeros(1, dtype=torch.int32, device=DEV)
    with pytest.raises(RFastError, match="range"):
        rfast_softmax_xent(wide, label, grad=False)
    x = wide.view(-1, 1)  # rows of one feature
    w, a, b = (torch.zeros(s, dtype=BF16, device=DEV) for s in ((1, 1), (1, 2, 1), (1, 1, 2)))
    ptr = torch.tensor([0, 8], dtype=torch.int32, device=DEV)
    with pytest.raises(RFastError, match="range"):
        rfast_lora_forward(x, w, a, b, ptr, out=x)
    with pytest.raises(RFastError, match="range"):
        rfast_lora_backward(x, w, a, b, ptr, None, x, dx=x)


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("K", [7, 300, 5000])
def test_xent_gradient_in_other_columns_of_the_logits_rows(types, K):
    """A buffer whose rows hold logits and gradient side by side is no overlap; columns that both have are one."""
    T, (lt, gt) = 9, types
    narrow = 4 // gt.itemsize if lt == F32 else 1  # gradient elements per logit's width
    logits = torch.randn((T, K), generator=gen(8)).to(lt).to(DEV)
    label = torch.arange(T, dtype=torch.int32, device=DEV) % K
    both = torch.full((T, 3 * K + 4), 7.0, dtype=lt, device=DEV)
    for at in (0, 2 * K, 2 * K + 1):
        both.fill_(7.0)
        both[:, K:2 * K] = logits
        want_loss, want = rfast_softmax_xent(both[:, K:2 * K], label, grad_dtype=gt)  # (the order of a sum goes by the rows' addresses)
        grad = both.view(gt)[:, at * narrow:at * narrow + K]
        loss, got = rfast_softmax_xent(both[:, K:2 * K], label, grad=grad)
        assert torch.equal(got, want) and torch.equal(loss, want_loss) and torch.equal(both[:, K:2 * K], logits)
    for at in (2 * K - 1, K + 1):
        with pytest.raises(RFastError, match="overlaps"):
            rfast_softmax_xent(both[:, K:2 * K], label, grad=both.view(gt)[:, at * narrow:at * narrow + K])


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_counters_stay_at_their_largest(bits):
    """Steps behind the 2^31st are like it: both corrections have been one for long."""
    most, p, g = 2 ** 31 - 1, torch.zeros(100, device=DEV), torch.full((100,), 1e-3, device=DEV)
    o = RFastAdamW([p], [g], state_bits=bits, steps=most - 1)
    for _ in range(4):
        o.step(1e-2)
    assert list(o.steps()) == [most] and torch.isfinite(p).all() and (p < 0).all()
    o.set_steps([most])
    q, h = torch.zeros(100, device=DEV), g.clone()
    r = RFastAdamW([q], [h], state_bits=bits, steps=most)
    for _ in range(4):
        r.step(1e-2)
    assert torch.equal(p, q)


def test_adamw_counters_out_of_range_are_refused():
    p, g = torch.zeros(10, device=DEV), torch.zeros(10, device=DEV)
    o = RFastAdamW([p], [g], steps=7)
    for bad in (2 ** 32, 2 ** 32 + 5, 2 ** 31, -1, 2 ** 64 + 5):
        with pytest.raises(RFastError, match="range"):
            o.set_steps([bad])
        with pytest.raises(RFastError, match="range"):
            RFastAdamW([p], [g], steps=bad)
    with pytest.raises(RFastError, match="range"):
        o.set_steps(np.array([2 ** 32 + 5]))
    assert list(o.steps()) == [7]
    o.set_steps(np.array([9]))
    assert list(o.steps()) == [9]


@pytest.mark.parametrize("K", [48, 264])
def test_lora_offsets_that_pass_32_bits(K):
    """Rows and outputs 40000 elements apart, 70000 of them: the last lie 2.8e9 elements behind the first, and are what the same rows alone give."""
    T, d, r, apart, scale = 70000, 64, 8, 40000, 0.5
    g = gen(9)
    x, w, a, b, dy = ((torch.randn(s, generator=g) * std).to(BF16).to(DEV) for s, std in
                      (((T, d), 1), ((K, d), 0.1), ((2, r, d), 0.1), ((2, K, r), 0.5), ((T, K), 0.1)))
    wide = torch.zeros((T, apart), dtype=BF16, device=DEV)
    xs, ys, dxs = wide[:, :d], wide[:, 1024:1024 + K], wide[:, 2048:2048 + d]
    dys = torch.zeros((T, apart), dtype=BF16, device=DEV)[:, 512:512 + K]
    xs.copy_(x)
    dys.copy_(dy)
    ptr = torch.tensor([0, 35001, T], dtype=torch.int32, device=DEV)
    y = rfast_lora_forward(xs, w, a, b, ptr, scale=scale, out=ys)
    dx, da, db = rfast_lora_backward(xs, w, a, b, ptr, None, dys, scale=scale, dx=dxs)
    want = rfast_lora_forward(x, w, a, b, ptr, scale=scale)
    back = rfast_lora_backward(x, w, a, b, ptr, None, dy, scale=scale)
    for got, other in ((y, want), (dx, back[0]), (da, back[1]), (db, back[2])):
        assert torch.isfinite(other).all() and torch.equal(got, other)
    low = 69900  # and the last rows against the formula: a sum of n exact products of bf16 is off by 2^-23 n of their magnitudes, rounded to bf16
    x64, w64, a64, b64, dy64 = x[low:].double(), w.double(), a[1].double(), b[1].double(), dy[low:].double()
    y64 = x64 @ w64.t() + scale * (x64 @ a64.t()) @ b64.t()
    size = x64.abs() @ w64.abs().t() + scale * (x64.abs() @ a64.abs().t()) @ b64.abs().t()
    assert ((y[low:].double() - y64).abs() <= 2.0 ** -23 * 2 * (d + 2 * r + 8) * size + 2.0 ** -8 * y64.abs() * 1.01).all()
    assert not wide[:, 3000:].any()


def test_training_step_captured_whole():
    """Forward, loss, backward and step of adapters in one graph: every replay is the eager step from the same state."""
    T, d, K, r = 300, 72, 40, 6
    g = gen(10)
    w = (torch.randn((K, d), generator=g) * 0.1).to(BF16).to(DEV)
    ptr = torch.tensor([0, 100, 100, 250], dtype=torch.int32, device=DEV)  # (rows behind the last segment too)
    start = [torch.randn((3, r, d), generator=g) * 0.1, torch.randn((3, K, r), generator=g) * 0.3]
    data = [((torch.randn((T, d), generator=g)).to(BF16), torch.randint(-1, K, (T,), generator=g).to(torch.int32)) for _ in range(5)]

    def make():
        x, label = torch.zeros((T, d), dtype=BF16, device=DEV), torch.zeros(T, dtype=torch.int32, device=DEV)
        master = [t.to(DEV) for t in start]
        held = [t.to(BF16) for t in master]
        grads = [torch.zeros_like(t) for t in master]
        logits, dy = torch.zeros((T, K), device=DEV), torch.zeros((T, K), dtype=BF16, device=DEV)
        loss, opt = torch.zeros(T, device=DEV), RFastAdamW(master, grads, copies=held, state_bits=8, weight_decay=0.01)

        def step():
            rfast_lora_forward(x, w, *held, ptr, scale=0.5, out=logits)
            rfast_softmax_xent(logits, label, grad_scale=1 / T, grad=dy, loss=loss, rows=ptr[3:])
            rfast_lora_backward(x, w, *held, ptr, None, dy, scale=0.5, need_dx=False, da=grads[0], db=grads[1])
            opt.step(1e-2)
        return x, label, step, [*master, *held, *grads, loss, logits, dy], opt

    (x, label, step, state, opt), (x2, label2, step2, state2, opt2) = make(), make()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k, (rows, classes) in enumerate(data):
        for to, frm in ((x, rows), (x2, rows), (label, classes), (label2, classes)):
            to.copy_(frm)
        graph.replay()
        step2()
        torch.cuda.synchronize()
        for p, q in zip(state, state2):
            assert torch.equal(p, q) and torch.isfinite(p).all()
        assert (opt.steps() == k + 1).all() and (opt2.steps() == k + 1).all()
    assert (state[0][1] != start[0][1].to(DEV)).any() and not state[4][1].any()  # the second adapter has no rows: decay alone


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_tensor_of_more_than_2_to_the_31(bits):
    """One tensor of 2^31 + 513 coordinates, all alike but for its last ones: offsets pass 32 bits, the last block is short."""
    count = 2 ** 31 + 513
    p, g = torch.zeros(count, dtype=BF16, device=DEV), torch.ones(count, dtype=BF16, device=DEV)
    g[-700:] = -1.0
    g[-1] = 0.0
    o = RFastAdamW([p], [g], state_bits=bits)
    o.step(0.5)  # the first step is gamma times the gradient's sign, to eps
    assert (p[:-700] == -0.5).all() and (p[-700:-1] == 0.5).all() and p[-1].item() == 0
    m = o.m[0].view(F8) if bits == 8 else o.m[0]
    assert (m[-700:-1].float() < 0).all() and m[-1].float().item() == 0 and (o.steps() == 1).all()
    if bits == 8:
        scale = o.m_scale[0]  # (the last block is the last coordinate alone)
        assert scale.numel() == 2 ** 23 + 3 and (scale[:-1] == scale[0]).all() and scale[0] > 0 and scale[-1] == 0
