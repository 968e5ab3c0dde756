"""A network chained with group normalisation, with whole activations and with 8-bit checkpoints, against the same composition of the
oracle's functions. What the CUDA path stores in bf16 or in 8 bits is rounded at the same places on the oracle's side."""
import numpy as np
import pytest
import torch

import oracle
from paper_1901_09290_b200 import binding as B
from paper_1901_09290_b200 import harness
from paper_1901_09290_b200 import workloads as W
from tests import helpers as Hh

gpu = pytest.mark.gpu
GROUPS = 4


def _r(a):
    return oracle.round_bf16(np.asarray(a, np.float32)).astype(np.float64)


def _stored(a):
    return oracle.act_unpack(*oracle.act_pack(a))


def _rel(got, ref):
    return np.linalg.norm((got - ref).ravel()) / max(np.linalg.norm(ref.ravel()), 1e-300)


def _network():
    """A stem with pooling, a bottleneck with a projection and one without; ragged channels."""
    net = W.resnet50(32)
    return W.with_sizes(net, W.uniform_keep(net, 0.2))


class _Oracle:
    def __init__(self, step, checkpoints):
        self.s, self.ck = step, checkpoints
        self.L = step.net.layers
        self.w = [oracle.round_bf16(w.numpy()) for w in step.model.w]
        f = lambda t: t.cpu().numpy().astype(np.float64)
        self.gamma, self.beta = ({i: f(t) for i, t in d.items()} for d in (step.gamma, step.beta))
        self.keep = _stored if checkpoints else (lambda a: a)

    def begin(self, i):
        return W.group_begin(self.L[i].K, GROUPS)

    def act(self, i):
        return 0 if any(ds == i for _, ds, _ in self.s.blocks) else 1

    def layer(self, i, x, res=None):
        l = self.L[i]
        y = _r(oracle.conv_fwd(x.astype(np.float32), self.w[i], l.stride, l.pad))
        a, mean, rstd = oracle.gn_act_fwd(y, self.gamma[i], self.beta[i], self.begin(i), 1e-5, res, self.act(i))
        self.y[i], self.stats[i] = self.keep(y), (mean.astype(np.float32), rstd.astype(np.float32))
        return _r(a)

    def norm_bwd(self, i, dy, res=None):
        mean, rstd = self.stats[i]
        dx, dres, self.dg[i], self.db[i], a = oracle.gn_act_bwd(self.y[i], dy, self.gamma[i], self.beta[i], mean, rstd, self.begin(i), res, self.act(i))
        return _r(dx), _r(dres), _r(a)

    def filters(self, i, x, dy):
        l = self.L[i]
        self.dw[i] = oracle.conv_wgrad(x.astype(np.float32), dy.astype(np.float32), l.R, l.R, l.stride, l.pad)

    def run(self, x0, g):
        s, L = self.s, self.L
        self.y, self.stats, self.dg, self.db, self.dw, a = {}, {}, {}, {}, {}, {}
        a[0] = self.layer(0, x0)
        cur, sel = oracle.maxpool_fwd(a[0], 3, 2, 1)
        saved = []
        for main, ds, _ in s.blocks:
            sc = self.layer(ds, cur) if ds is not None else cur
            t = cur
            for i in main[:-1]:
                a[i] = t = self.layer(i, t)
            saved.append((self.keep(cur), self.keep(sc) if ds is not None else self.keep(cur)))
            cur = self.layer(main[-1], t, sc)
        out, d = cur, g
        for (main, ds, _), (x_in, sc) in zip(reversed(s.blocks), reversed(saved)):
            dy, dres, _ = self.norm_bwd(main[-1], d, sc)
            for k in range(len(main) - 1, -1, -1):
                i, l = main[k], L[main[k]]
                d_t = _r(oracle.conv_dgrad(dy.astype(np.float32), self.w[i], l.H, l.H, l.stride, l.pad))
                x, mine = x_in, dy
                if k:
                    dy, _, again = self.norm_bwd(main[k - 1], d_t)
                    x = again if self.ck else a[main[k - 1]]
                self.filters(i, x, mine)
            back = dres
            if ds is not None:
                l = L[ds]
                dy, _, _ = self.norm_bwd(ds, dres)
                self.filters(ds, x_in, dy)
                back = _r(oracle.conv_dgrad(dy.astype(np.float32), self.w[ds], l.H, l.H, l.stride, l.pad))
            d = _r(d_t + back)
        dy, _, _ = self.norm_bwd(0, _r(oracle.maxpool_bwd(d, sel, L[0].P, L[0].P)))
        self.filters(0, x0, dy)
        return out


# Bounds as for the chained batch-norm block: a value whose last bf16 bit rounds the other way, a code that takes the other neighbour and a
# ReLU decided differently at an isolated element compound along the chain. (A code's step is 2^-7 of its block's largest value, and the
# few values that change theirs do it where a bf16 rounding changed.)
@gpu
@pytest.mark.parametrize("checkpoints", [False, True])
def test_chain_with_group_norm(checkpoints):
    net, N, seed = _network(), 3, W.BASE_SEED + 7300
    kw = dict(groups=GROUPS, max_blocks=2)
    s = harness.CheckpointedStep(Hh.ctx(), net, N, seed, **kw) if checkpoints else harness.ChainedStep(Hh.ctx(), net, N, seed, norm="group", **kw)
    out = s.forward().clone()
    s.backward()
    torch.cuda.synchronize()
    Hh.ctx().poll()
    f = lambda t, C: t.float().cpu().numpy()[..., :C].astype(np.float64)
    C = net.layers[s.out_index].K
    o = _Oracle(s, checkpoints)
    ref = o.run(f(s.x0, net.layers[0].C), f(s.g_last, C))
    assert _rel(f(out, C), ref) < 5e-3
    for i in s.used:
        assert _rel(s.dm.g[i].cpu().numpy().astype(np.float64), o.dw[i]) < 2e-2, net.layers[i].name
        assert _rel(s.dg[i].cpu().numpy().astype(np.float64), o.dg[i]) < 2e-2, net.layers[i].name
        assert _rel(s.db[i].cpu().numpy().astype(np.float64), o.db[i]) < 2e-2, net.layers[i].name
    # the step as a whole, twice: the same gradients, and from a captured graph too
    first = [s.dm.g[i].clone() for i in s.used]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.forward()
        s.backward()
    for i in s.used:
        s.dm.g[i].zero_()
    g.replay()
    torch.cuda.synchronize()
    Hh.ctx().poll()
    assert all(torch.equal(a, s.dm.g[i]) for a, i in zip(first, s.used))


@gpu
def test_checkpoints_cost_the_gradients_little_and_save_most_of_the_memory():
    """The same step with and without checkpoints. A restored value is off by at most amax/127 of its block, 0.02 of a standard deviation where
    amax is 2.5 of them. That changes the sums a layer takes by a per cent or two, and decides ReLUs the other way: only those with
    |z| <= 0.02, at a density of at most 0.4 a fraction of 0.016 of the elements, against the half that passes its gradient on: a relative change of at
    most sqrt(0.016 / 0.5) = 0.18 in the gradient behind a ReLU. Behind D of them, independent, it is sqrt(D) times that."""
    net, N, seed = _network(), 3, W.BASE_SEED + 7301
    a = harness.ChainedStep(Hh.ctx(), net, N, seed, norm="group", groups=GROUPS, max_blocks=2)
    b = harness.CheckpointedStep(Hh.ctx(), net, N, seed, groups=GROUPS, max_blocks=2)
    for s in (a, b):
        s.step()
    torch.cuda.synchronize()
    depth = {0: 7}                                                # ReLUs between a convolution and the end: its own, and those behind it
    for n, (main, ds, _) in enumerate(a.blocks):
        after = 3 * (len(a.blocks) - 1 - n)
        depth.update({i: after + 3 - k for k, i in enumerate(main)})
        if ds is not None:
            depth[ds] = after + 1
    for i in a.used:
        u, v = a.dm.g[i].double(), b.dm.g[i].double()
        assert float((u - v).norm() / u.norm()) < 0.18 * depth[i] ** 0.5, net.layers[i].name
    whole = sum(t.numel() * 2 for d in (a.y, a.a) for t in d.values())
    assert b.saved_bytes() < 0.5 * whole


def test_groups_of_pruned_layers():
    assert W.group_begin(12, 4) == [0, 3, 6, 9, 12] and W.group_begin(3, 8) == [0, 1, 2, 3]
    assert W.group_begin(371, 32)[-1] == 371 and len(W.group_begin(371, 32)) == 33
    # channels 0-3, 4-7, 8-11: two of the first group stay, none of the second, all of the third
    assert W.pruned_group_begin([1, 3, 8, 9, 10, 11], [0, 4, 8, 12]) == [0, 2, 6]
    d = B.make_gn_desc(1, 4, 4, 6, 2, group_begin=W.pruned_group_begin([1, 3, 8, 9, 10, 11], [0, 4, 8, 12]))
    assert [d.group_begin[k] for k in range(3)] == [0, 2, 6]


def test_struct_layouts():
    import ctypes
    assert ctypes.sizeof(B.pt_gn_desc) == 48 and B.pt_gn_desc.group_begin.offset == 40
    assert ctypes.sizeof(B.pt_pack_desc) == 24
    B.lib()
    assert B.pt_act_scale_bytes(10, 33) == 32 and B.pt_act_scale_bytes(0, 5) == 0 and B.pt_act_scale_bytes(-1, 5) == 0 and B.pt_act_scale_bytes(3, 0) == 0


def test_chain_refuses_other_norms():
    with pytest.raises(ValueError):
        harness.ChainedStep(None, None, 1, 0, norm="layer")
