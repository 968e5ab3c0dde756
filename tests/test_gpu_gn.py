"""Parity of the group-normalisation kernels and of the 8-bit activation checkpoints (through the C ABI) with the fp64 oracle.

Tolerances. A bf16 output is off by its rounding, 2^-8 of the value at most, and by what the fp32 arithmetic before it leaves: a few
roundings (2^-24 each) of terms whose magnitudes are known, 2 ulp and |z| * 2^-24 from the exponential of a sigmoid (|z| stays below 16
here: 2e-6), less than 1e-5 of the sum of the terms' magnitudes in all. Sums over an image are fp32 over the few pixels of a thread and
wider after that: 1e-5 of the sum of the magnitudes is generous. Statistics: a thread's fp32 sums of k values are off by k/2 * 2^-24 of
the magnitudes' sum at most, k <= 64 here: 2e-6."""
import numpy as np
import pytest
import torch

import oracle
from paper_1901_09290_b200 import binding as B
from paper_1901_09290_b200 import workloads as W
from tests import helpers as Hh

pytestmark = pytest.mark.gpu

CANARY = 7680.0


def _bf(t):
    return W.bf16_round(t)


def _inputs(N, H, Wd, C, seed, with_res):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen)
    u = lambda n: torch.rand(n, generator=gen)
    x = _bf(r(N, H, Wd, C) * (u(C) * 1.5 + 0.25) + u(C) - 0.25)
    res = _bf(r(N, H, Wd, C)) if with_res else None
    dy = _bf(r(N, H, Wd, C))
    return x, res, dy, u(C) + 0.5, u(C) - 0.5


def _out(N, H, Wd, C, ld):
    return Hh.out_buffer((N, H, Wd), C, ld, False, CANARY)


def _take(t, C):
    """The values, once the pad lanes are seen to be zeros."""
    a = t.float().cpu().numpy().astype(np.float64)
    assert np.all(a[..., C:] == 0), "pad lanes of an output are zeros"
    return a[..., :C]


def _close(got, ref, slack, what, bf16=True):
    tol = slack + (np.abs(ref) * 2.0 ** -8 if bf16 else np.abs(ref) * 2.0 ** -24)
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off, the worst by {np.nanmax(np.abs(got - ref) / np.maximum(tol, 1e-30)):.2f} of the bound"


def _spread(v, begin):
    return np.repeat(np.asarray(v, np.float64), np.diff(begin), axis=1)[:, None, None, :]


def _pack(c, xd, npix, C, ld, ldq=None):
    d = B.make_pack_desc(npix, C, ld, ldq)
    codes, scales = B.checkpoint_buffers(npix, C, ldq)
    codes.fill_(77)
    scales.fill_(88)
    B.pt_act_pack(c, d, xd, codes, scales)
    return d, codes, scales


def _ws(c, d):
    return torch.empty(B.pt_gn_workspace_bytes(c, d), dtype=torch.uint8, device="cuda")


def check_forward(N, H, Wd, C, groups, act, with_res, ld=None, begin=None, pack=False, seed=1):
    c, ld = Hh.ctx(), ld or W.pad8(C)
    table = begin is not None or C % groups != 0
    begin = begin or oracle.group_begin(C, groups)
    x, res, _, g, b = _inputs(N, H, Wd, C, seed, with_res)
    d = B.make_gn_desc(N, H, Wd, C, groups, ld, 1e-5, act, begin if table else None)
    xd, rd, y = Hh.to_dev_padded(x, ld), Hh.to_dev_padded(res, ld) if with_res else None, _out(N, H, Wd, C, ld)
    mean, rstd = (torch.full((N, groups), CANARY, device="cuda") for _ in range(2))
    codes, scales = B.checkpoint_buffers(N * H * Wd, C) if pack else (None, None)
    if pack:
        codes.fill_(77)
        scales.fill_(88)
    B.pt_gn_act_fwd(c, d, xd, rd, g.cuda(), b.cuda(), mean, rstd, y, codes, scales)
    torch.cuda.synchronize()
    c.poll()
    ry, rmean, rrstd = oracle.gn_act_fwd(x.numpy(), g.numpy(), b.numpy(), begin, float(np.float32(1e-5)), res.numpy() if with_res else None, act)
    mag = _spread(1 / rrstd, begin)
    assert np.all(np.abs(mean.cpu().numpy() - rmean) <= 2e-6 * (np.abs(rmean) + 1 / rrstd))
    assert np.all(np.abs(rstd.cpu().numpy() / rrstd - 1) <= 4e-6)
    xhat = (x.numpy() - _spread(rmean, begin)) / mag
    terms = np.abs(xhat * g.numpy()) + np.abs(b.numpy()) + (np.abs(res.numpy()) if with_res else 0)
    _close(_take(y, C), ry, 1e-5 * (terms + np.abs(g.numpy())), "y")
    if pack:
        _, want, wants = _pack(c, xd, N * H * Wd, C, ld)
        assert torch.equal(codes, want) and torch.equal(scales, wants), "the checkpoint is pt_act_pack's, bit for bit"


def check_backward(N, H, Wd, C, groups, act, with_res, ld=None, begin=None, packed=False, want_y=True, seed=2, in_place=False):
    c, ld = Hh.ctx(), ld or W.pad8(C)
    table = begin is not None or C % groups != 0
    begin = begin or oracle.group_begin(C, groups)
    x, res, dy, g, b = _inputs(N, H, Wd, C, seed, with_res)
    d = B.make_gn_desc(N, H, Wd, C, groups, ld, 1e-5, act, begin if table else None)
    _, mean, rstd = oracle.gn_act_fwd(x.numpy(), g.numpy(), b.numpy(), begin, 1e-5, None, act)
    mean, rstd = mean.astype(np.float32), rstd.astype(np.float32)
    xd, rd, dyd = Hh.to_dev_padded(x, ld), Hh.to_dev_padded(res, ld) if with_res else None, Hh.to_dev_padded(dy, ld)
    dx, dres = _out(N, H, Wd, C, ld), _out(N, H, Wd, C, ld) if with_res else None
    if in_place:
        dx, dres = xd if not packed else dyd, rd
    dg, db = (torch.full((C,), CANARY, device="cuda") for _ in range(2))
    md, sd, y = torch.from_numpy(mean).cuda(), torch.from_numpy(rstd).cuda(), None
    if packed:
        _, codes, scales = _pack(c, xd, N * H * Wd, C, ld)
        y = _out(N, H, Wd, C, ld) if want_y else None
        B.pt_gn_act_bwd_packed(c, d, codes, scales, rd, dyd, g.cuda(), b.cuda(), md, sd, dx, dres, dg, db, y, _ws(c, d))
        x = torch.from_numpy(oracle.act_unpack(*oracle.act_pack(x.numpy())))
    else:
        B.pt_gn_act_bwd(c, d, xd, rd, dyd, g.cuda(), b.cuda(), md, sd, dx, dres, dg, db, _ws(c, d))
    torch.cuda.synchronize()
    c.poll()
    rdx, rdz, rdg, rdb, ry = oracle.gn_act_bwd(x.numpy(), dy.numpy(), g.numpy(), b.numpy(), mean, rstd, begin,
                                               res.numpy() if with_res else None, act)
    xhat = (x.double().numpy() - _spread(mean, begin)) * _spread(rstd, begin)
    ady, ag = np.abs(dy.double().numpy()), np.abs(g.double().numpy())
    means = np.stack([(ady * ag)[..., s:e].mean((1, 2, 3)) for s, e in zip(begin[:-1], begin[1:])], 1)
    meanx = np.stack([(ady * ag * np.abs(xhat))[..., s:e].mean((1, 2, 3)) for s, e in zip(begin[:-1], begin[1:])], 1)
    terms = _spread(rstd, begin) * (ag * ady + _spread(means, begin) + np.abs(xhat) * _spread(meanx, begin))
    _close(_take(dx, C), rdx, 1e-5 * terms, "dx")
    _close(dg.cpu().numpy(), rdg, 1e-5 * (ady * np.abs(xhat)).sum((0, 1, 2)), "dgamma", bf16=False)
    _close(db.cpu().numpy(), rdb, 1e-5 * ady.sum((0, 1, 2)), "dbeta", bf16=False)
    if with_res:
        _close(_take(dres, C), rdz, 1e-5 * ady * (act == 2), "dresidual")
    if y is not None:
        _close(_take(y, C), ry, 1e-5 * (np.abs(xhat) * ag + np.abs(b.numpy()) + (np.abs(res.numpy()) if with_res else 0)), "y again")


# one channel; one pixel; groups that end inside a vector of 8 channels; one group; a group per channel; many pixels per thread; few wide
# pixels; more than one vector of pad lanes; the widest pitch
SHAPES = [(2, 5, 7, 1, 1), (3, 1, 1, 16, 2), (3, 8, 8, 11, 3), (2, 14, 14, 93, 5), (4, 7, 7, 64, 1), (2, 6, 5, 40, 40), (1, 33, 31, 24, 3),
          (2, 3, 2, 371, 32), (5, 9, 9, 16, 4), (1, 2, 2, 2041, 16)]


@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("with_res", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, with_res, act):
    check_forward(*shape, act, with_res, pack=act == 2 or with_res)


@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("with_res", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(shape, with_res, act):
    check_backward(*shape, act, with_res)


@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("with_res", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward_from_a_checkpoint(shape, with_res, act):
    check_backward(*shape, act, with_res, packed=True, want_y=act != 0)


# images larger than what a few blocks keep on chip, and batches beyond the device's blocks
@pytest.mark.parametrize("shape", [(2, 64, 64, 96, 8), (1, 112, 112, 24, 3), (300, 4, 4, 32, 4), (37, 14, 15, 160, 7)])
@pytest.mark.parametrize("with_res", [False, True])
def test_large_images_and_many_images(shape, with_res):
    check_forward(*shape, 2, with_res, pack=True)
    check_backward(*shape, 1, with_res)
    check_backward(*shape, 2, with_res, packed=True)


@pytest.mark.parametrize("C,ld", [(8, 64), (13, 48), (93, 96), (64, 200), (41, 2048)])
def test_pitches(C, ld):
    check_forward(2, 6, 5, C, 1, 1, True, ld=ld, pack=True)
    check_backward(2, 6, 5, C, 1, 1, True, ld=ld)
    check_backward(2, 6, 5, C, 1, 1, True, ld=ld, packed=True)


@pytest.mark.parametrize("begin", [[0, 1, 2, 20], [0, 19, 20], [0, 3, 11, 12, 20]])
def test_tables_of_groups(begin):
    check_forward(3, 5, 5, 20, len(begin) - 1, 2, True, begin=begin)
    check_backward(3, 5, 5, 20, len(begin) - 1, 2, True, begin=begin)
    check_backward(3, 5, 5, 20, len(begin) - 1, 2, True, begin=begin, packed=True)


def test_many_groups():
    check_forward(2, 3, 3, 1500, 256, 1, False)                  # the largest table
    check_backward(2, 3, 3, 1500, 256, 1, False)
    check_forward(2, 3, 3, 1024, 1024, 0, False)                 # a group per channel
    check_backward(2, 3, 3, 1024, 512, 2, True, packed=True)


@pytest.mark.parametrize("packed", [False, True])
def test_backward_in_place(packed):
    check_backward(3, 9, 7, 27, 3, 1, True, packed=packed, in_place=True)
    check_backward(2, 40, 40, 64, 4, 2, True, packed=packed, in_place=True)


def test_forward_in_place():
    c = Hh.ctx()
    N, H, C, G = 5, 30, 48, 6
    x, res, _, g, b = _inputs(N, H, H, C, 3, True)
    d = B.make_gn_desc(N, H, H, C, G, act=B.PT_ACT_SILU)
    mean, rstd = (torch.empty((N, G), device="cuda") for _ in range(2))
    y = _out(N, H, H, C, C)
    B.pt_gn_act_fwd(c, d, x.bfloat16().cuda(), res.bfloat16().cuda(), g.cuda(), b.cuda(), mean, rstd, y)
    for over in (0, 1):
        xd, rd = x.bfloat16().cuda(), res.bfloat16().cuda()
        out = rd if over else xd
        B.pt_gn_act_fwd(c, d, xd, rd, g.cuda(), b.cuda(), mean, rstd, out)
        assert torch.equal(out, y)


def test_a_large_mean_costs_the_statistics_nothing():
    """Values about 1000 with steps of 8 (bf16): the variance comes from differences, not from sums of squares."""
    c = Hh.ctx()
    N, H, C, G = 2, 24, 32, 2
    gen = torch.Generator().manual_seed(5)
    x = _bf(1000 + 8 * torch.randint(-1, 2, (N, H, H, C), generator=gen).float())
    d = B.make_gn_desc(N, H, H, C, G, act=0)
    mean, rstd = (torch.empty((N, G), device="cuda") for _ in range(2))
    y = _out(N, H, H, C, C)
    one, zero = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    B.pt_gn_act_fwd(c, d, x.bfloat16().cuda(), None, one, zero, mean, rstd, y)
    ry, rmean, rrstd = oracle.gn_act_fwd(x.numpy(), np.ones(C), np.zeros(C), oracle.group_begin(C, G), 1e-5, act=0)
    assert np.all(np.abs(mean.cpu().numpy() / rmean - 1) <= 2.0 ** -23)
    assert np.all(np.abs(rstd.cpu().numpy() / rrstd - 1) <= 4e-6)


def test_infinities_and_nan_stay_in_their_group():
    c = Hh.ctx()
    N, H, C, G = 3, 6, 40, 4
    x, res, dy, g, b = _inputs(N, H, H, C, 6, False)
    clean = x.clone()
    x[0, 1, 2, 3], x[2, 5, 5, 39] = float("nan"), float("inf")
    d = B.make_gn_desc(N, H, H, C, G, act=B.PT_ACT_RELU)
    outs = []
    for v in (clean, x):
        mean, rstd = (torch.empty((N, G), device="cuda") for _ in range(2))
        y, dx = _out(N, H, H, C, C), _out(N, H, H, C, C)
        dg, db = (torch.empty(C, device="cuda") for _ in range(2))
        B.pt_gn_act_fwd(c, d, v.bfloat16().cuda(), None, g.cuda(), b.cuda(), mean, rstd, y)
        B.pt_gn_act_bwd(c, d, v.bfloat16().cuda(), None, dy.bfloat16().cuda(), g.cuda(), b.cuda(), mean, rstd, dx, None, dg, db, _ws(c, d))
        outs.append((y.cpu(), dx.cpu(), dg.cpu()))
    hit = torch.zeros((N, H, H, C), dtype=torch.bool)
    hit[0, ..., :10] = True
    hit[2, ..., 30:] = True
    for k in (0, 1):
        assert torch.isnan(outs[1][k][hit]).all() and torch.equal(outs[1][k][~hit], outs[0][k][~hit])
    assert torch.isnan(outs[1][2][:10]).all() and torch.equal(outs[1][2][10:30], outs[0][2][10:30])


@pytest.mark.parametrize("act", [1, 2])
def test_residuals_of_the_lowest_value_and_nan(act):
    """A residual of the type's lowest value leaves nothing of its element, forward and backward; a NaN in the residual stays in its element.
    "Nothing" of a SiLU is |z| * sigmoid(z) at the least values the kernel takes for them, 2^20 and 2^-60: 2^-40, a per cent more for what
    x adds to z (below 10 of 2^20) and the rounding to bf16; times |dy| for the gradient."""
    nothing = 1.01 * 2.0 ** -40
    c = Hh.ctx()
    N, H, C, G = 2, 5, 24, 3
    x, res, dy, g, b = _inputs(N, H, H, C, 9, True)
    low = torch.finfo(torch.bfloat16).min
    hit = torch.zeros((N, H, H, C), dtype=torch.bool)
    hit[0, 1, 2, 3:12], hit[1, 4, 4, 23], hit[1, 0, 0, 0] = True, True, True
    res[hit] = low
    d = B.make_gn_desc(N, H, H, C, G, act=act)
    gd, bd = g.cuda(), b.cuda()
    mean, rstd = (torch.empty((N, G), device="cuda") for _ in range(2))
    y = _out(N, H, H, C, C)
    xd = x.bfloat16().cuda()
    B.pt_gn_act_fwd(c, d, xd, res.bfloat16().cuda(), gd, bd, mean, rstd, y)
    assert float(y.cpu()[hit].abs().max()) <= nothing
    dx, dres = _out(N, H, H, C, C), _out(N, H, H, C, C)
    dg, db = (torch.empty(C, device="cuda") for _ in range(2))
    B.pt_gn_act_bwd(c, d, xd, res.bfloat16().cuda(), dy.bfloat16().cuda(), gd, bd, mean, rstd, dx, dres, dg, db, _ws(c, d))
    m, s = mean.cpu().numpy(), rstd.cpu().numpy()
    rdx, rdz, rdg, rdb, _ = oracle.gn_act_bwd(x.numpy(), dy.numpy(), g.numpy(), b.numpy(), m, s, oracle.group_begin(C, G), res.numpy(), act)
    assert bool((dres.cpu()[hit].abs() <= nothing * dy[hit].abs()).all()) and torch.isfinite(dx).all()
    ady = np.abs(dy.double().numpy())
    _close(_take(dres, C), rdz, 1e-5 * ady, "dresidual")
    _close(db.cpu().numpy(), rdb, 1e-5 * ady.sum((0, 1, 2)), "dbeta", bf16=False)
    # |dx| is rstd * a few |dy| here: all of its terms are below 40
    _close(_take(dx, C), rdx, 1e-5 * 40 * s.max() * np.ones_like(rdx), "dx")
    # a NaN
    clean, y2 = res.clone(), _out(N, H, H, C, C)
    res[0, 2, 2, 5] = float("nan")
    B.pt_gn_act_fwd(c, d, xd, res.bfloat16().cuda(), gd, bd, mean, rstd, y2)
    bad = torch.isnan(y2.cpu())
    assert bad[0, 2, 2, 5] and int(bad.sum()) == 1 and torch.equal(y2.cpu()[~bad], y.cpu()[~bad]) and not torch.isnan(clean).any()


@pytest.mark.parametrize("act", [0, 1, 2])
def test_groups_without_variance(act):
    """A group of equal values far from 0 is its beta: x - mean is 0, however large 1/sqrt(eps) is. (The fp32 mean of equal bf16 values is exact.)"""
    c = Hh.ctx()
    N, H, C, G = 2, 6, 16, 2
    x = torch.full((N, H, H, C), 1000.0)
    x[..., 8:] = -0.0078125
    _, res, dy, g, b = _inputs(N, H, H, C, 10, True)
    d = B.make_gn_desc(N, H, H, C, G, act=act)
    mean, rstd = (torch.empty((N, G), device="cuda") for _ in range(2))
    for r in (None, res):
        y = _out(N, H, H, C, C)
        B.pt_gn_act_fwd(c, d, x.bfloat16().cuda(), None if r is None else r.bfloat16().cuda(), g.cuda(), b.cuda(), mean, rstd, y)
        z = b.double().numpy() + (0.0 if r is None else r.double().numpy()) + np.zeros((N, H, H, C))
        _close(_take(y, C), oracle._act(z, act), 1e-5 * (np.abs(z) + 1), "y")
    assert torch.equal(mean.cpu(), torch.tensor([[1000.0, -0.0078125]] * N))
    # the gradients at such values, against the formula's
    dx, dg, db = _out(N, H, H, C, C), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    B.pt_gn_act_bwd(c, d, x.bfloat16().cuda(), None, dy.bfloat16().cuda(), g.cuda(), b.cuda(), mean, rstd, dx, None, dg, db, _ws(c, d))
    s = rstd.cpu().numpy()
    rdx, _, rdg, rdb, _ = oracle.gn_act_bwd(x.numpy(), dy.numpy(), g.numpy(), b.numpy(), mean.cpu().numpy(), s, oracle.group_begin(C, G), None, act)
    _close(_take(dx, C), rdx, 1e-5 * 10 * s.max() * np.ones_like(rdx), "dx")      # (terms: |gamma * dy| < 8 and its mean, times rstd)
    _close(db.cpu().numpy(), rdb, 1e-5 * np.abs(dy.numpy()).sum((0, 1, 2)), "dbeta", bf16=False)
    assert float(dg.abs().max()) == 0.0


def test_relu_is_decided_exactly_at_zero():
    """Values whose z is 0 or the smallest step beside it: gradients pass where z > 0 in exact arithmetic."""
    c = Hh.ctx()
    N, H, C = 1, 16, 8
    vals = torch.tensor([-1.0, -0.0, 0.0, 1.0])
    x = vals[torch.arange(H * H * C) % 4].reshape(N, H, H, C)
    mean, rstd = torch.zeros((1, 1), device="cuda"), torch.full((1, 1), 2.0 / 3.0, device="cuda")
    g = torch.full((C,), 0.75)
    for beta in (0.0, 2.0 ** -40, -2.0 ** -40, float(np.float32(-0.75) * np.float32(2.0 / 3.0))):
        b = torch.full((C,), beta)
        d = B.make_gn_desc(N, H, H, C, 1, act=B.PT_ACT_RELU)
        dy, dx, dres = torch.ones((N, H, H, C), dtype=torch.bfloat16, device="cuda"), _out(N, H, H, C, C), _out(N, H, H, C, C)
        dg, db = (torch.empty(C, device="cuda") for _ in range(2))
        zero = torch.zeros((N, H, H, C), dtype=torch.bfloat16, device="cuda")
        z = x.double() * float(np.float32(2.0 / 3.0)) * 0.75 + float(np.float32(beta))
        want = (z > 0).double().sum((0, 1, 2))
        for res in (None, zero):
            B.pt_gn_act_bwd(c, d, x.bfloat16().cuda(), res, dy, g.cuda(), b.cuda(), mean, rstd, dx, dres, dg, db, _ws(c, d))
            assert torch.equal(db.cpu().double(), want) and torch.equal(dres.cpu() > 0, z > 0)


@pytest.mark.parametrize("nan_at", [(0,), (1,), (0, 1), (6, 7)])
def test_relu_is_decided_exactly_beside_a_nan(nan_at):
    """A NaN in the residual, or in its pad lanes, which are never used, leaves the decisions of the other values alone. gamma * rstd =
    0.75 * fl(2/3) = 0.5 + 2^-26, which fp32 rounds to 0.5, so that z = 256 * gamma * rstd - 128 = 2^-18 is 0 in fp32 and positive."""
    c = Hh.ctx()
    N, H, C, ld = 1, 8, 6, 8
    x, r = torch.full((N, H, H, ld), 256.0), torch.full((N, H, H, ld), -128.0)
    r[..., list(nan_at)] = float("nan")
    mean, rstd = torch.zeros((1, 1), device="cuda"), torch.full((1, 1), 2.0 / 3.0, device="cuda")
    g, b = torch.full((C,), 0.75, device="cuda"), torch.zeros(C, device="cuda")
    d = B.make_gn_desc(N, H, H, C, 1, ld, act=B.PT_ACT_RELU)
    dy, dx, dres = torch.ones((N, H, H, ld), dtype=torch.bfloat16, device="cuda"), _out(N, H, H, C, ld), _out(N, H, H, C, ld)
    dg, db = (torch.empty(C, device="cuda") for _ in range(2))
    B.pt_gn_act_bwd(c, d, x.bfloat16().cuda(), r.bfloat16().cuda(), dy, g, b, mean, rstd, dx, dres, dg, db, _ws(c, d))
    want = np.array([0.0 if k in nan_at else 1.0 for k in range(C)])
    assert np.array_equal(_take(dres, C), np.broadcast_to(want, (N, H, H, C)))
    assert np.array_equal(db.cpu().numpy(), want * H * H)


# units in several rounds over the device's blocks, whose pixels a ring does not hold, and in slabs of channels with ragged groups
@pytest.mark.parametrize("shape", [(310, 18, 18, 64, 4), (333, 5, 6, 264, 11), (700, 5, 3, 72, 9), (160, 23, 17, 130, 6)])
def test_many_units_of_a_cluster(shape):
    check_forward(*shape, 2, True)
    check_forward(*shape, 1, False)
    check_backward(*shape, 1, True)
    check_backward(*shape, 2, False)


@pytest.mark.parametrize("shape", [(610, 3, 3, 64, 4), (333, 4, 3, 264, 11), (700, 2, 3, 72, 9), (6, 23, 17, 130, 6)])
def test_many_units_of_a_cluster_with_checkpoints(shape):
    check_forward(*shape, 2, True, pack=True)
    check_backward(*shape, 1, True, packed=True)
    check_backward(*shape, 2, False, packed=True)


def test_graphs_of_their_own_and_an_eager_call_between():
    """Two captured passes, a workspace each, replayed in turn and at once beside an eager one: the same bits throughout."""
    c = Hh.ctx()
    N, H, C, G = 40, 12, 48, 6
    x, res, dy, g, b = _inputs(N, H, H, C, 11, True)
    d = B.make_gn_desc(N, H, H, C, G, C, act=B.PT_ACT_RELU)
    xd, rd, dyd, gd, bd = Hh.to_dev_padded(x, C), Hh.to_dev_padded(res, C), Hh.to_dev_padded(dy, C), g.cuda(), b.cuda()
    mean, rstd = (torch.zeros((N, G), device="cuda") for _ in range(2))
    B.pt_gn_act_fwd(c, d, xd, rd, gd, bd, mean, rstd, _out(N, H, H, C, C))

    def bufs():
        return [_out(N, H, H, C, C), _out(N, H, H, C, C), torch.zeros(C, device="cuda"), torch.zeros(C, device="cuda"), _ws(c, d)]

    go = lambda o, stream=None: B.pt_gn_act_bwd(c, d, xd, rd, dyd, gd, bd, mean, rstd, *o, stream)
    eager = bufs()
    go(eager)
    torch.cuda.synchronize()
    graphs, outs, sides = [], [bufs(), bufs()], [torch.cuda.Stream(), torch.cuda.Stream()]
    for o in outs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            go(o)
        graphs.append(graph)
    later = bufs()
    torch.cuda.synchronize()
    for _ in range(4):
        for graph, side in zip(graphs, sides):
            with torch.cuda.stream(side):
                graph.replay()
        go(later)
    torch.cuda.synchronize()
    c.poll()
    for o in outs + [later]:
        assert all(torch.equal(p, q) for p, q in zip(eager[:4], o[:4]))


def test_identical_runs_streams_and_graphs():
    c = Hh.ctx()
    N, H, C, G = 24, 20, 77, 7
    x, res, dy, g, b = _inputs(N, H, H, C, 7, True)
    ld = W.pad16(C)
    d = B.make_gn_desc(N, H, H, C, G, ld, act=B.PT_ACT_SILU, group_begin=oracle.group_begin(C, G))
    xd, rd, dyd = (Hh.to_dev_padded(t, ld) for t in (x, res, dy))
    gd, bd = g.cuda(), b.cuda()

    def bufs():
        o = {k: _out(N, H, H, C, ld) for k in ("y", "dx", "dres", "again")}
        o.update({k: torch.zeros((N, G), device="cuda") for k in ("mean", "rstd")}, **{k: torch.zeros(C, device="cuda") for k in ("dg", "db")})
        o["codes"], o["scales"] = B.checkpoint_buffers(N * H * H, C)
        o["scales"].zero_()
        o["ws"] = _ws(c, d)
        return o

    def go(o, stream=None):
        B.pt_gn_act_fwd(c, d, xd, rd, gd, bd, o["mean"], o["rstd"], o["y"], o["codes"], o["scales"], stream)
        B.pt_gn_act_bwd_packed(c, d, o["codes"], o["scales"], rd, dyd, gd, bd, o["mean"], o["rstd"], o["dx"], o["dres"], o["dg"], o["db"],
                               o["again"], o["ws"], stream)

    first, second, graphed = bufs(), bufs(), bufs()
    go(first)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    third = bufs()
    torch.cuda.synchronize()
    go(second)
    go(third, side)                                              # two calls at once, a workspace each
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(graphed)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    c.poll()
    for o in (second, third, graphed):
        assert all(torch.equal(first[k], o[k]) for k in first if k != "ws")


def test_offsets_beyond_32_bits():
    """A tensor of more than 2^31 elements: its last image is what it is by itself."""
    c = Hh.ctx()
    H, C, G = 64, 256, 8
    N = (1 << 31) // (H * H * C) + 2
    gen = torch.Generator(device="cuda").manual_seed(8)
    x = torch.empty((N, H, H, C), dtype=torch.bfloat16, device="cuda")
    x.normal_(generator=gen)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    gam, bet = torch.rand(C, generator=gen, device="cuda") + 0.5, torch.rand(C, generator=gen, device="cuda")

    def run(n, x, y, dx):
        d = B.make_gn_desc(n, H, H, C, G, act=B.PT_ACT_RELU)
        mean, rstd = (torch.empty((n, G), device="cuda") for _ in range(2))
        dg, db = (torch.empty(C, device="cuda") for _ in range(2))
        codes, scales = B.checkpoint_buffers(n * H * H, C)
        B.pt_gn_act_fwd(c, d, x, None, gam, bet, mean, rstd, y, codes, scales)
        B.pt_gn_act_bwd_packed(c, d, codes, scales, None, y, gam, bet, mean, rstd, dx, None, dg, db, None, _ws(c, d))
        back = torch.empty((H, H, C), dtype=torch.bfloat16, device="cuda")
        m = (n - 1) * H * H
        B.pt_act_unpack(c, B.make_pack_desc(H * H, C), codes[m:], scales[m * (C // 32):], back)
        return mean[-1], rstd[-1], y[-1], dx[-1], back

    whole = [t.clone() for t in run(N, x, y, dx)]
    last = run(1, x[-1:].clone(), torch.empty_like(x[-1:]), torch.empty_like(x[-1:]))
    torch.cuda.synchronize()
    c.poll()
    names = ("mean", "rstd", "y", "dx", "checkpoint")
    # The sums of one image may be split over more blocks than those of many: the statistics differ by what each may be off (above). That
    # is 2e-6 of |mean| + the standard deviation for a mean (each value's rounding is relative to the value, and they are about 1, while
    # the means here are about 1 / sqrt(131072)), twice that between two of them, and 4e-6 twice for rstd. A bf16 result then differs by a
    # step at most.
    for k, a, b in zip(names, whole, last):
        off = (a.double() - b.double()).abs().max()
        if k == "checkpoint":
            assert torch.equal(a, b)
        elif k == "mean":
            assert float(off) <= 4e-6 * float(b.abs().max() + 1 / last[1].min())
        else:
            assert float(off) <= (8e-6 if k == "rstd" else 2.0 ** -7) * float(b.abs().max()), k


# ------------------------------------------------------------------------------------------------ checkpoints by themselves
@pytest.mark.parametrize("npix,C,ld,ldq", [(1, 1, 8, 8), (70, 8, 8, 8), (33, 16, 16, 24), (129, 20, 24, 24), (50, 33, 48, 40), (64, 64, 64, 64),
                                           (37, 93, 96, 96), (3, 371, 376, 400), (5, 2041, 2048, 2048), (1000, 41, 48, 48)])
def test_pack_and_unpack(npix, C, ld, ldq):
    c = Hh.ctx()
    rng = np.random.default_rng(npix + C)
    x = rng.standard_normal((npix, C)) * np.exp2(rng.integers(-8, 8, (npix, 1)))
    x[0] = 0
    if npix > 30:
        x[1:20] *= np.exp2(np.linspace(-140, 118, 19))[:, None]          # every scale byte's neighbourhood, subnormals among them
        x[20, 0], x[21, -1], x[22, C // 2] = np.inf, np.nan, -np.inf
        x[23] = np.resize([127.5, 127.0, -127.5, 0.5, -1.5, 126.5, 63.75], C)
        x[24] = 3.3895e38
    x = torch.from_numpy(oracle.round_bf16(x.astype(np.float32)))
    want, wants = oracle.act_pack(x.numpy())
    d, codes, scales = _pack(c, Hh.to_dev_padded(x, ld), npix, C, ld, ldq)
    n, p8 = wants.size, W.pad8(C)
    assert np.array_equal(codes[:, :C].cpu().numpy(), want)
    assert np.array_equal(scales[:n].cpu().numpy().reshape(wants.shape), wants)
    assert (codes[:, C:p8] == 0).all() and (codes[:, p8:] == 77).all() and (scales[n:] == 88).all()
    back = torch.full((npix, ld), CANARY, dtype=torch.bfloat16, device="cuda")
    B.pt_act_unpack(c, d, codes, scales, back)
    ref = oracle.act_unpack(want, wants)
    got = back.float().cpu().numpy().astype(np.float64)
    assert np.array_equal(got[:, :C], ref, equal_nan=True) and np.all(got[:, C:] == 0)


def test_empty_checkpoint_and_refusals():
    c = Hh.ctx()
    t = torch.zeros(4096, dtype=torch.bfloat16, device="cuda")
    codes, scales = B.checkpoint_buffers(16, 32)
    B.pt_act_pack(c, B.make_pack_desc(0, 32), t, codes, scales)          # nothing to do
    B.pt_act_unpack(c, B.make_pack_desc(0, 32), codes, scales, t)

    def refused(call, status):
        with pytest.raises(B.PtError) as e:
            call()
        assert e.value.status == status

    pd = lambda **k: B.pt_pack_desc(*[k.get(n, v) for n, v in (("npix", 16), ("C", 32), ("ld", 32), ("ldq", 32))])
    for bad in (pd(npix=-1), pd(C=0), pd(ld=31), pd(ld=36), pd(ldq=24), pd(ldq=36)):
        refused(lambda: B.pt_act_pack(c, bad, t, codes, scales), 1)
        refused(lambda: B.pt_act_unpack(c, bad, codes, scales, t), 1)
    refused(lambda: B.pt_act_pack(c, pd(C=2049, ld=2056, ldq=2056), t, codes, scales), 2)
    refused(lambda: B.pt_act_pack(c, pd(), t, None, scales), 1)
    refused(lambda: B.pt_act_pack(c, pd(), t[1:], codes, scales), 1)
    x, y = torch.zeros((2, 4, 4, 32), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 4, 4, 32), dtype=torch.bfloat16, device="cuda")
    v, s = torch.zeros(32, device="cuda"), torch.zeros((2, 4), device="cuda")
    good = B.make_gn_desc(2, 4, 4, 32, 4)
    ws = _ws(c, good)
    fwd = lambda d, **k: B.pt_gn_act_fwd(c, d, k.get("x", x), None, k.get("gamma", v), v, s, s.clone(), k.get("y", y), k.get("codes"), k.get("scales"))
    bwd = lambda d, **k: B.pt_gn_act_bwd(c, d, x, None, k.get("dy", x), v, v, s, s, y, None, v.clone(), v.clone(), k.get("ws", ws))
    gd = lambda **k: B.make_gn_desc(*[k.get(n, w) for n, w in (("N", 2), ("H", 4), ("W", 4), ("C", 32), ("groups", 4), ("ld", 32), ("eps", 1e-5), ("act", 1),
                                                              ("begin", None), ("ldq", None))])
    for bad in (gd(N=0), gd(H=0), gd(C=33), gd(C=0), gd(groups=0), gd(groups=33), gd(groups=5), gd(ld=36), gd(eps=-1.0), gd(eps=float("nan")),
                gd(act=3), gd(act=-1), gd(groups=2, begin=[0, 32, 32]), gd(groups=2, begin=[1, 16, 32]), gd(groups=2, begin=[0, 16, 31]),
                gd(groups=3, begin=[0, 20, 10, 32]), gd(groups=2, begin=[0, -4, 32])):
        refused(lambda: fwd(bad), 1)
        refused(lambda: bwd(bad), 1)
        assert B.pt_gn_workspace_bytes(c, bad) == 0
    refused(lambda: fwd(gd(H=1 << 16, W=1 << 15)), 2)
    refused(lambda: fwd(gd(C=2049, ld=2056, groups=3)), 2)
    refused(lambda: fwd(gd(C=2048, ld=2048, groups=300, begin=oracle.group_begin(2048, 300))), 2)
    refused(lambda: fwd(good, x=None), 1)
    refused(lambda: fwd(good, gamma=None), 1)
    refused(lambda: fwd(good, codes=codes), 1)                           # codes without scales
    refused(lambda: fwd(gd(ldq=36), codes=codes, scales=scales), 1)
    refused(lambda: fwd(good, x=x.view(-1)[1:]), 1)
    refused(lambda: bwd(good, dy=None), 1)
    refused(lambda: bwd(good, ws=None), 3)
    refused(lambda: bwd(good, ws=ws[:ws.numel() - 16]), 3)
    with pytest.raises(ValueError):
        gd(groups=3, begin=[0, 32])


def test_more_images_than_units_are_counted_in_are_refused():
    c = Hh.ctx()
    t, v, s = torch.zeros(64, dtype=torch.bfloat16, device="cuda"), torch.zeros(8, device="cuda"), torch.zeros(8, device="cuda")
    for N in ((1 << 24) + 1, 2 ** 31 - 1):
        d = B.make_gn_desc(N, 1, 1, 8, 1, 8)
        assert B.pt_gn_workspace_bytes(c, d) == 0
        with pytest.raises(B.PtError) as e:
            B.pt_gn_act_fwd(c, d, t, None, v, v, s, s.clone(), t.clone(), None, None)
        assert e.value.status == 2
    assert B.pt_gn_workspace_bytes(c, B.make_gn_desc(1 << 24, 1, 1, 8, 1, 8)) > 0
