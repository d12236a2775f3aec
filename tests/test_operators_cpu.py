"""What the operators that take tensors refuse before any device work, and how they size their workspaces: no GPU needed."""
import ctypes as C

import pytest

import paper_2307_11617_amd as rf
from paper_2307_11617_amd.binding import RfastAdamwOptions, RfastAdamwTensor, RfastLoraShape

DEV = 1 << 20  # never dereferenced: every call below is refused first


def shape(**kw):
    d = dict(rows=10, segments=2, adapters=2, d=64, K=48, rank=4, ld_x=64, ld_y=48, y_type=1, scale=1.0)
    d.update(kw)
    return RfastLoraShape(*[d[f[0]] for f in RfastLoraShape._fields_])


def test_lora_workspace_is_pure_and_checks_ranges():
    sizes = [rf.rfast_lora_workspace_bytes(shape(), k) for k in range(3)]
    assert 0 < sizes[0] < sizes[1] < sizes[2] and sizes == [rf.rfast_lora_workspace_bytes(shape(), k) for k in range(3)]
    assert rf.rfast_lora_workspace_bytes(shape(rows=0), 0) >= 0
    for kw in (dict(rows=-1), dict(segments=0), dict(adapters=0), dict(adapters=65536), dict(d=0), dict(K=0), dict(rank=0), dict(rank=65),
               dict(rows=1 << 28), dict(d=1 << 23), dict(rows=1 << 27, K=1 << 22)):
        assert rf.rfast_lora_workspace_bytes(shape(**kw), 0) == 0, kw
    assert rf.rfast_lora_workspace_bytes(shape(), 3) == 0 and rf.rfast_lora_workspace_bytes(shape(), -1) == 0


def test_lora_workspace_for_many_rows_does_for_few():
    for d, K, rank in ((1024, 128, 8), (4096, 4096, 16), (512, 33000, 64), (100, 70, 1), (8192, 8, 3)):
        for k in (0, 1, 2):
            last = 0
            for rows in (1, 64, 65, 128, 129, 300, 512, 1000, 2048, 4100, 8001, 16384, 16385, 40000):
                now = rf.rfast_lora_workspace_bytes(shape(rows=rows, d=d, K=K, rank=rank, ld_x=d, ld_y=K), k)
                assert now >= last > -1, (d, K, rows, k)
                last = now


def forward(s, x=DEV, w=DEV, a=DEV, b=DEV, ptr=DEV, ad=None, y=DEV, ws=DEV, nbytes=1 << 40):
    code = rf.lib().rfast_lora_forward(C.byref(s) if s is not None else None, x, w, a, b, ptr, ad, y, ws, nbytes, None)
    return code, rf.rfast_last_error(None)


def backward(s, dy=DEV, dx=None, da=DEV, db=DEV, ws=DEV, nbytes=1 << 40):
    code = rf.lib().rfast_lora_backward(C.byref(s), DEV, DEV, DEV, DEV, DEV, None, dy, dx, da, db, ws, nbytes, None)
    return code, rf.rfast_last_error(None)


def test_lora_refusals():
    assert forward(None)[0] == -1
    for kw in (dict(rank=0), dict(rank=65), dict(rows=-1), dict(segments=0), dict(ld_x=63), dict(ld_y=47), dict(y_type=2)):
        assert forward(shape(**kw))[0] == -1, kw
    for scale in (float("nan"), float("inf")):
        assert forward(shape(scale=scale))[0] == -4
    for kw in (dict(x=None), dict(w=None), dict(a=None), dict(b=None), dict(ptr=None), dict(y=None), dict(ws=None), dict(ws=DEV + 8), dict(x=DEV + 1),
               dict(ptr=DEV + 2), dict(ad=DEV + 2), dict(y=DEV + 1)):
        assert forward(shape(), **kw)[0] == -1, kw
    assert forward(shape(y_type=0), y=DEV + 2)[0] == -1
    code, msg = forward(shape(), nbytes=100)
    assert code == -5 and "workspace" in msg
    for kw in (dict(dy=None), dict(da=None), dict(db=None), dict(dx=DEV + 1), dict(da=DEV + 2)):
        assert backward(shape(), **kw)[0] == -1, kw
    assert backward(shape(y_type=0))[0] == -1
    need = rf.rfast_lora_workspace_bytes(shape(), 2)
    assert backward(shape(), dx=DEV, nbytes=need - 1)[0] == -5


def xent(rows=4, K=8, logits=DEV, lt=0, ldl=8, labels=DEV, loss=DEV, lse=None, grad=DEV + 4096, gt=0, ldg=8, d_rows=None):
    return rf.lib().rfast_softmax_xent(rows, K, logits, lt, ldl, labels, 1.0, loss, lse, grad, gt, ldg, d_rows, None)


def test_xent_refusals():
    for kw in (dict(rows=-1), dict(K=0), dict(logits=None), dict(labels=None), dict(lt=2), dict(gt=-1), dict(ldl=7), dict(ldg=7), dict(logits=DEV + 2),
               dict(labels=DEV + 1), dict(loss=DEV + 2), dict(lse=DEV + 2), dict(grad=DEV + 4098), dict(d_rows=DEV + 1), dict(grad=DEV + 8),
               dict(grad=DEV, gt=1), dict(grad=DEV, ldg=9)):
        assert xent(**kw) == -1, kw
    assert xent(rows=0) == 0


def tensors(n=2, **kw):
    t = (RfastAdamwTensor * n)()
    for i in range(n):
        d = dict(param=DEV + 65536 * (8 * i), grad=DEV + 65536 * (8 * i + 1), m=DEV + 65536 * (8 * i + 2), v=DEV + 65536 * (8 * i + 3), m_scale=None,
                 v_scale=None, copy=None, count=1000, weight_decay=0.0, steps=0)
        d.update(kw if i == n - 1 else {})
        t[i] = RfastAdamwTensor(*[d[f[0]] for f in RfastAdamwTensor._fields_])
    return t


def create(t, ws=DEV + (1 << 30), nbytes=1 << 40, **kw):
    d = dict(param_type=0, grad_type=0, state_bits=32, beta1=0.9, beta2=0.999, eps=1e-8)
    d.update(kw)
    h = C.c_void_p()
    code = rf.lib().rfast_adamw_create(C.byref(h), len(t), t, C.byref(RfastAdamwOptions(*d.values())), ws, nbytes, None)
    assert not h.value
    return code, rf.rfast_last_error(None)


def test_adamw_refusals():
    t = tensors()
    need = rf.rfast_adamw_workspace_bytes(t)
    assert need > 0 and rf.rfast_adamw_workspace_bytes(tensors(count=-1)) == 0 and rf.rfast_adamw_workspace_bytes(tensors(count=1 << 47)) == 0
    assert rf.lib().rfast_adamw_workspace_bytes(0, t) == 0
    assert create(t, nbytes=need - 1)[0] == -5
    assert create(t, ws=DEV + (1 << 30) + 4)[0] == -1
    for kw in (dict(param_type=2), dict(grad_type=-1), dict(state_bits=4)):
        assert create(t, **kw)[0] == -1, kw
    for kw in (dict(beta1=1.0), dict(beta2=-0.1), dict(beta1=float("nan")), dict(eps=0.0), dict(eps=float("inf"))):
        assert create(t, **kw)[0] == -4, kw
    for kw in (dict(count=-1), dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(m_scale=DEV + 65536 * 13), dict(param=DEV + 65536 * 8 + 2),
               dict(copy=DEV + 65536 * 13 + 1)):
        assert create(tensors(**kw))[0] == -1, kw
    for kw in (dict(weight_decay=-1.0), dict(weight_decay=float("nan")), dict(steps=-1), dict(steps=1 << 31)):
        assert create(tensors(**kw))[0] == -4, kw
    # what a step writes overlaps the other tensor's memory, or its own gradient
    for kw in (dict(param=DEV), dict(m=DEV + 65536 + 100), dict(v=DEV + 65536 * 10 + 8), dict(grad=DEV + 65536 * 8), dict(copy=DEV + 65536 * 9), dict(m=DEV + (1 << 30))):
        code, msg = create(tensors(**kw))
        assert code == -1 and "overlap" in msg, kw
    assert create(tensors(), state_bits=8)[0] == -1  # no scales
    L = rf.lib()
    assert L.rfast_adamw_step(None, 1.0, None, None) == -1 and L.rfast_adamw_steps(None, None, None) == -1
    assert L.rfast_adamw_create(None, 1, t, None, DEV, 1, None) == -1
    L.rfast_adamw_destroy(None)


@pytest.mark.parametrize("bad", ["x", "row_ptr"])
def test_tensors_on_the_host_are_refused(bad):
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(rf.RFastError):
        rf.rfast_lora_forward(x, torch.zeros(6, 8, dtype=torch.bfloat16), torch.zeros(1, 2, 8, dtype=torch.bfloat16),
                              torch.zeros(1, 6, 2, dtype=torch.bfloat16), torch.tensor([0, 4], dtype=torch.int32))
    with pytest.raises(rf.RFastError):
        rf.rfast_softmax_xent(x, torch.zeros(4, dtype=torch.int32))
    with pytest.raises(rf.RFastError):
        rf.RFastAdamW([torch.zeros(4)], [torch.zeros(4)])


@pytest.mark.parametrize("eps", [2.0 ** -127, 1e-40, 1e-60, 5e-324])
def test_adamw_refuses_an_eps_that_32_bits_do_not_hold(eps):
    """A coordinate that never had a gradient is divided by eps alone: 0 / 0, or by the infinite reciprocal of a denormal."""
    code, msg = create(tensors(), eps=eps)
    assert code == -4 and "eps" in msg


def test_lora_most_segments_beside_most_tiles():
    """Blocks of rows and tiles of matrices turned over, in one launch, are fewer than 2^32 lanes together."""
    def lanes(s):
        tiles = s.adapters * ((s.K + 63) // 64 + (s.d + 63) // 64) + (s.K + 63) // 64 * ((s.d + 63) // 64)
        rows = 16 if s.rows <= 1024 else 32
        waves = 8 if s.rows <= 1024 else 4
        return (s.rows // rows + s.segments + 2 + (tiles + waves - 1) // waves) * 64 * waves
    taken = 0
    for rows in (1, 1000, 1024, 1025, 1 << 16):
        for K in range(32704 - 64 * 4, 32704 + 1):
            s = shape(rows=rows, segments=1 << 22, adapters=65535, d=64, K=K, rank=1, ld_x=64, ld_y=K)
            if rf.rfast_lora_workspace_bytes(s, 2) > 0:
                taken += 1
                assert lanes(s) < 1 << 32, (rows, K)
    assert taken > 0
    s = shape(rows=1000, segments=1, adapters=65535, d=64, K=32704 - 64, rank=1, ld_x=64, ld_y=32704)  # few segments beside nearly as many tiles
    assert rf.rfast_lora_workspace_bytes(s, 2) > 0 and lanes(s) < 1 << 32
