"""What the operators around the adapters' products (embeddings, rows to experts and back, policy loss) refuse before any device work, and how
they size their workspaces: no GPU needed."""
import numpy as np
import pytest

import paper_2307_11617_amd as rf

MB = 1 << 20
DEV = [MB * 64 * (i + 1) for i in range(16)]  # addresses far apart, never dereferenced: every call below is refused first
INF, NAN = float("inf"), float("nan")


def call(name, order, defaults, kw):
    d = dict(defaults)
    assert set(kw) <= set(d), kw
    d.update(kw)
    return getattr(rf.lib(), name)(*[d[k] for k in order.split()], None)


def policy(**kw):
    return call("rfast_policy_loss", "rows K logits lt ldl actions old adv ref weight low high beta scale loss logp grad gt ldg d_rows",
                dict(rows=4, K=8, logits=DEV[0], lt=0, ldl=8, actions=DEV[1], old=DEV[2], adv=DEV[3], ref=DEV[4], weight=DEV[5], low=0.2, high=0.2,
                     beta=0.1, scale=1.0, loss=DEV[6], logp=DEV[7], grad=DEV[8], gt=0, ldg=8, d_rows=DEV[9]), kw)


def test_policy_refusals():
    for kw in (dict(rows=-1), dict(K=0), dict(logits=None), dict(actions=None), dict(old=None), dict(adv=None), dict(lt=2), dict(gt=-1), dict(ldl=7),
               dict(ldg=7), dict(logits=DEV[0] + 2), dict(actions=DEV[1] + 1), dict(old=DEV[2] + 2), dict(adv=DEV[3] + 1), dict(ref=DEV[4] + 2),
               dict(weight=DEV[5] + 3), dict(loss=DEV[6] + 2), dict(logp=DEV[7] + 1), dict(grad=DEV[8] + 2), dict(d_rows=DEV[9] + 2),
               dict(grad=DEV[0] + 8), dict(grad=DEV[0], gt=1), dict(grad=DEV[2]), dict(loss=DEV[2]), dict(logp=DEV[3] + 4), dict(loss=DEV[7]),
               dict(logp=DEV[0] + 16), dict(loss=DEV[8]), dict(loss=DEV[9])):
        assert policy(**kw) == -1, kw
    for kw in (dict(low=-0.1), dict(low=1.5), dict(low=NAN), dict(high=-0.1), dict(high=INF), dict(high=NAN), dict(beta=-1.0), dict(beta=INF), dict(beta=NAN), dict(scale=INF), dict(scale=NAN)):
        assert policy(**kw) == -4, kw
        assert policy(rows=0, **kw) == -4, kw
    assert policy(rows=0) == 0


def embedding(**kw):
    return call("rfast_embedding", "rows V d table tt ldt tokens scale out ot ldo",
                dict(rows=4, V=10, d=8, table=DEV[0], tt=0, ldt=8, tokens=DEV[1], scale=1.0, out=DEV[2], ot=0, ldo=8), kw)


def test_embedding_refusals():
    for kw in (dict(rows=-1), dict(V=0), dict(d=0), dict(d=2 ** 31 - 1), dict(table=None), dict(tokens=None), dict(out=None), dict(tt=2), dict(ot=-1),
               dict(ldt=7), dict(ldo=7), dict(table=DEV[0] + 2), dict(tokens=DEV[1] + 2), dict(out=DEV[2] + 1), dict(ot=1, out=DEV[2] + 1),
               dict(out=DEV[0]), dict(out=DEV[0] + 9 * 32), dict(out=DEV[1])):
        assert embedding(**kw) == -1, kw
    assert embedding(rows=0) == 0
    for scale in (INF, -INF, NAN):
        assert embedding(scale=scale) == -4 and back(scale=scale) == -4


def back(**kw):
    return call("rfast_embedding_backward", "rows V d dy yt ldy tokens scale grad gt ldg acc ws nbytes",
                dict(rows=4, V=10, d=8, dy=DEV[0], yt=0, ldy=8, tokens=DEV[1], scale=1.0, grad=DEV[2], gt=0, ldg=8, acc=0, ws=DEV[3], nbytes=MB), kw)


def test_embedding_backward_refusals_and_workspace():
    for kw in (dict(rows=-1), dict(V=0), dict(d=0), dict(dy=None), dict(tokens=None), dict(grad=None), dict(yt=2), dict(gt=2), dict(ldy=7), dict(ldg=7),
               dict(acc=2), dict(acc=-1), dict(dy=DEV[0] + 2), dict(tokens=DEV[1] + 1), dict(grad=DEV[2] + 2), dict(ws=None), dict(ws=DEV[3] + 128),
               dict(grad=DEV[0]), dict(grad=DEV[1]), dict(ws=DEV[0]), dict(ws=DEV[1] - 256), dict(ws=DEV[2])):
        assert back(**kw) == -1, kw
    need = rf.rfast_embedding_backward_workspace_bytes(4, 10, 8)
    assert back(nbytes=need - 1) == -5 and "workspace" in rf.rfast_last_error(None)
    assert back(rows=0, dy=None, tokens=None, acc=1) == 0
    for bad in ((-1, 10, 8), (4, 0, 8), (4, 10, 0), (4, 10, 2 ** 31 - 1)):
        assert rf.lib().rfast_embedding_backward_workspace_bytes(*bad) == 0
    for V in (10, 1000, 50001, 1 << 21):
        sizes = [rf.rfast_embedding_backward_workspace_bytes(n, V, 64) for n in (0, 1, 64, 65, 4096, 4097, 70000)]
        assert sizes == sorted(sizes) and sizes[0] > 0
    assert rf.rfast_embedding_backward_workspace_bytes(2 ** 31 - 1, 2 ** 31 - 1, 1) > 2 ** 35


def route(**kw):
    return call("rfast_route", "rows E k logits lt ld norm expert weight row_ptr place order ws nbytes",
                dict(rows=4, E=8, k=2, logits=DEV[0], lt=0, ld=8, norm=1, expert=DEV[1], weight=DEV[2], row_ptr=DEV[3], place=DEV[4], order=DEV[5],
                     ws=DEV[6], nbytes=MB), kw)


def plan(**kw):
    return call("rfast_route_plan", "pairs E expert row_ptr place order ws nbytes",
                dict(pairs=8, E=8, expert=DEV[1], row_ptr=DEV[3], place=DEV[4], order=DEV[5], ws=DEV[6], nbytes=MB), kw)


def test_route_refusals():
    for kw in (dict(rows=-1), dict(E=0, k=0), dict(E=1025, ld=1025), dict(k=0), dict(k=9), dict(E=100, ld=100, k=65), dict(rows=1 << 30, k=2), dict(lt=2),
               dict(norm=2), dict(logits=None), dict(expert=None), dict(weight=None), dict(row_ptr=None), dict(place=None), dict(order=None), dict(ld=7),
               dict(logits=DEV[0] + 1), dict(expert=DEV[1] + 2), dict(weight=DEV[2] + 1), dict(row_ptr=DEV[3] + 2), dict(place=DEV[4] + 1),
               dict(order=DEV[5] + 2), dict(ws=None), dict(ws=DEV[6] + 8), dict(expert=DEV[0]), dict(weight=DEV[1] + 4), dict(place=DEV[5]),
               dict(ws=DEV[0]), dict(row_ptr=DEV[6])):
        assert route(**kw) == -1, kw
    need = rf.rfast_route_workspace_bytes(8, 8)
    assert route(nbytes=need - 1) == -5 and plan(nbytes=need - 1) == -5
    for kw in (dict(pairs=-1), dict(E=0), dict(expert=None), dict(row_ptr=None), dict(place=None), dict(order=None), dict(expert=DEV[1] + 1),
               dict(row_ptr=DEV[3] + 1), dict(place=DEV[4] + 2), dict(order=DEV[5] + 1), dict(ws=None), dict(ws=DEV[6] + 4), dict(place=DEV[1]),
               dict(order=DEV[4] + 28), dict(row_ptr=DEV[5] + 28), dict(ws=DEV[3])):
        assert plan(**kw) == -1, kw
    assert rf.lib().rfast_route_workspace_bytes(-1, 4) == 0 and rf.lib().rfast_route_workspace_bytes(4, 0) == 0
    for E in (1, 64, 1024, 70000, 2 ** 31 - 1):
        sizes = [rf.rfast_route_workspace_bytes(n, E) for n in (0, 1, 4096, 4097, 1 << 20, 2 ** 31 - 1)]
        assert sizes == sorted(sizes) and sizes[0] > 0


def route_back(**kw):
    return call("rfast_route_backward", "rows E k logits lt ld norm expert weight dweight out ot ldo",
                dict(rows=4, E=8, k=2, logits=DEV[0], lt=0, ld=8, norm=0, expert=DEV[1], weight=DEV[2], dweight=DEV[3], out=DEV[4], ot=0, ldo=8), kw)


def test_route_backward_refusals():
    for kw in (dict(rows=-1), dict(E=0), dict(E=1025, ld=2000, ldo=2000), dict(k=0), dict(k=9), dict(lt=2), dict(ot=2), dict(norm=-1), dict(logits=None),
               dict(expert=None), dict(weight=None), dict(dweight=None), dict(out=None), dict(ld=7), dict(ldo=7), dict(logits=DEV[0] + 2),
               dict(expert=DEV[1] + 1), dict(weight=DEV[2] + 2), dict(dweight=DEV[3] + 1), dict(out=DEV[4] + 2), dict(out=DEV[0]), dict(out=DEV[3])):
        assert route_back(**kw) == -1, kw
    assert route_back(rows=0) == 0


def gather(**kw):
    return call("rfast_route_gather", "rows k d x t ldx place out P ldo",
                dict(rows=4, k=2, d=8, x=DEV[0], t=0, ldx=8, place=DEV[1], out=DEV[2], P=8, ldo=8), kw)


def combine(**kw):
    return call("rfast_route_combine", "rows k d s t P lds place weight y yt ldy",
                dict(rows=4, k=2, d=8, s=DEV[0], t=0, P=8, lds=8, place=DEV[1], weight=DEV[2], y=DEV[3], yt=0, ldy=8), kw)


def combine_back(**kw):
    return call("rfast_route_combine_backward", "rows k d s t P lds place weight dy lddy ds ldds dw",
                dict(rows=4, k=2, d=8, s=DEV[0], t=0, P=8, lds=8, place=DEV[1], weight=DEV[2], dy=DEV[3], lddy=8, ds=DEV[4], ldds=8, dw=DEV[5]), kw)


def test_rows_refusals():
    sizes = (dict(rows=-1), dict(k=0), dict(k=65), dict(d=0), dict(d=2 ** 31 - 1), dict(P=-1), dict(rows=1 << 30), dict(t=2), dict(place=None),
             dict(place=DEV[1] + 2))
    for kw in sizes + (dict(x=None), dict(out=None), dict(ldx=7), dict(ldo=7), dict(x=DEV[0] + 2), dict(out=DEV[2] + 2), dict(out=DEV[0]), dict(out=DEV[1]),
                       dict(d=2 ** 30, ldx=2 ** 30, ldo=2 ** 30)):
        assert gather(**kw) == -1, kw
    for kw in sizes + (dict(s=None), dict(y=None), dict(lds=7), dict(ldy=7), dict(yt=-1), dict(s=DEV[0] + 2), dict(weight=DEV[2] + 1), dict(y=DEV[3] + 2),
                       dict(y=DEV[0] + 32), dict(y=DEV[1]), dict(y=DEV[2])):
        assert combine(**kw) == -1, kw
    for kw in sizes + (dict(s=None), dict(dy=None), dict(lds=7), dict(lddy=7), dict(ldds=7), dict(s=DEV[0] + 1), dict(weight=DEV[2] + 2), dict(dy=DEV[3] + 1),
                       dict(ds=DEV[4] + 2), dict(dw=DEV[5] + 1), dict(ds=DEV[0]), dict(ds=DEV[3]), dict(dw=DEV[2]), dict(dw=DEV[4] + 4)):
        assert combine_back(**kw) == -1, kw
    assert gather(rows=0) == 0 and gather(P=0, out=None) == 0 and combine(rows=0) == 0 and combine_back(rows=0) == 0
    assert combine_back(ds=None, dw=None) == 0


def test_tensors_on_the_host_are_refused():
    torch = pytest.importorskip("torch")
    x, i = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32)
    place = torch.zeros((4, 1), dtype=torch.int32)
    for call in (lambda: rf.rfast_embedding(x, i), lambda: rf.rfast_embedding_backward(x, i, 5), lambda: rf.rfast_route(x, 2),
                 lambda: rf.rfast_route_plan(i, 4), lambda: rf.rfast_route_gather(x, place), lambda: rf.rfast_route_combine(x, place),
                 lambda: rf.rfast_route_combine_backward(x, place, None, x), lambda: rf.rfast_policy_loss(x, i, x[:, 0], x[:, 0]),
                 lambda: rf.rfast_route_backward(x, place, None, None)):
        with pytest.raises(rf.RFastError):
            call()


def test_sizes_beyond_32_bits_are_refused():
    for call in (lambda: rf.rfast_route_workspace_bytes(1 << 32, 4), lambda: rf.rfast_route_workspace_bytes(4, 1 << 31),
                 lambda: rf.rfast_embedding_backward_workspace_bytes(1, 1 << 33, 4)):
        with pytest.raises(rf.RFastError):
            call()
    assert np.iinfo(np.int32).max == 2 ** 31 - 1
