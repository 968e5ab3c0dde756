"""Group norm and 8-bit checkpoints at the ends of their range, against 64-bit references. Tolerances are derived at the tests."""
import os
import subprocess
import sys
import threading

import numpy as np
import pytest
import torch

import oracle
from paper_1901_09290_b200 import binding as B
from paper_1901_09290_b200 import harness
from paper_1901_09290_b200 import workloads as W
from tests import helpers as Hh

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ------------------------------------------------------------------------------------------------ checkpoints
@pytest.mark.parametrize("npix,ldq", [(257, (1 << 24) + (1 << 17)), (5, (1 << 31) - 8)])
def test_codes_of_a_pitch_that_passes_32_bits_within_a_block(npix, ldq):
    """Pixels whose codes lie 4 GB apart while one thread block covers them all: each is where its pitch says, and nothing else is written."""
    c, C = Hh.ctx(), 8
    gen = torch.Generator().manual_seed(21)
    x = W.bf16_round(torch.randn((npix, C), generator=gen)).bfloat16().cuda()
    dense, scales = B.checkpoint_buffers(npix, C)
    B.pt_act_pack(c, B.make_pack_desc(npix, C), x, dense, scales)
    wide = torch.zeros((npix, ldq), dtype=torch.int8, device="cuda")
    d, wide_scales, back = B.make_pack_desc(npix, C, C, ldq), torch.zeros_like(scales), torch.zeros_like(x)
    B.pt_act_pack(c, d, x, wide, wide_scales)
    B.pt_act_unpack(c, d, wide, wide_scales, back)
    torch.cuda.synchronize()
    c.poll()
    assert torch.equal(wide[:, :C], dense) and torch.equal(wide_scales[:npix], scales[:npix])
    assert int(torch.count_nonzero(wide)) == int(torch.count_nonzero(dense))
    want = oracle.act_unpack(dense.cpu().numpy(), scales[:npix].cpu().numpy().reshape(npix, 1))
    assert np.array_equal(back.float().cpu().numpy().astype(np.float64), want)


# ------------------------------------------------------------------------------------------------ statistics of the forward pass
# A thread takes its pixels in runs and joins them. The k-th addition of a run is off by 2^-24 of the sum so far at most. The first run,
# at most 16 pixels, is about the first of them: if that one is d away from equal others, the sum of squares grows by d^2 a step, so that
# it is off by (1 + 2 + .. + 15) * 2^-24 d^2 = 7.2e-6 d^2, and the run's sum of squares about its mean is 15/16 d^2: 7.6e-6 of the
# variance, 3.8e-6 of rstd = var^-1/2. (A first pixel that is no further away than others loses less: 16 * 2^-24.) The next run is about
# the mean of the first, d/16 away: 48 * (d/16)^2 = 0.19 d^2 in 48 steps, 3e-7 of the variance; later ones less. 4e-6 holds rstd. A mean is
# off by half of that at most, of the pixels' distances from the pivot: 4e-6 of the deviation, and a rounding of the mean to fp32.
def _stats(x, G, copies, eps=1e-5, pack=False):
    """rstd and mean of an image [H][W][C] of `copies` equal ones by the kernel, and in 64 bits; y of the last copy."""
    c = Hh.ctx()
    H, Wd, C = x.shape
    xb = W.bf16_round(x)
    xd = torch.zeros((copies, H, Wd, W.pad8(C)), dtype=torch.bfloat16, device="cuda")
    xd[..., :C] = xb.bfloat16().cuda()
    d = B.make_gn_desc(copies, H, Wd, C, G, eps=eps, act=B.PT_ACT_NONE)
    mean, rstd = (torch.full((copies, G), 7.0, device="cuda") for _ in range(2))
    y, one, zero = torch.empty_like(xd), torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    codes, scales = B.checkpoint_buffers(copies * H * Wd, C) if pack else (None, None)
    B.pt_gn_act_fwd(c, d, xd, None, one, zero, mean, rstd, y, codes, scales)
    torch.cuda.synchronize()
    c.poll()
    v = xb.double().reshape(H * Wd, G, C // G).permute(1, 0, 2).reshape(G, -1)
    m = v.mean(1)
    var = ((v - m[:, None]) ** 2).mean(1)
    return mean.double().cpu(), rstd.double().cpu(), m, (var + eps).rsqrt(), var.sqrt(), y[-1, ..., :C].double().cpu(), xb.double()


@pytest.mark.parametrize("base,odd", [(0.0, 100.0), (0.0, 1000.0), (10.0, 0.0), (1000.0, 0.0)])
@pytest.mark.parametrize("H,C,G,copies", [(224, 8, 1, 300), (56, 64, 8, 2), (56, 1040, 4, 150), (112, 16, 2, 3)])
def test_statistics_of_images_whose_first_pixels_are_unlike_the_rest(H, C, G, copies, base, odd):
    """A border or a mask: one block per image and many, many pixels per thread and one."""
    gen = torch.Generator().manual_seed(22)
    x = base + torch.randn((H, H, C), generator=gen)
    x.view(H * H, C)[:4] = odd
    mean, rstd, m, r, dev, _, _ = _stats(x, G, copies, pack=base == 0.0)
    assert float((rstd / r - 1).abs().max()) <= 4e-6
    assert bool(((mean - m).abs() <= 4e-6 * dev + 2.0 ** -24 * m.abs()).all())


@pytest.mark.parametrize("H,C,G,copies", [(30, 8, 1, 2), (30, 32, 2, 400), (5, 2040, 3, 2)])
@pytest.mark.parametrize("at", [0, 1, 24])
def test_one_step_in_a_constant_group_is_its_variance(H, C, G, copies, at):
    """Every value 1000 but one, which is 1004, the next bf16: the variance is all in one thread's sums, or between its mean and the others'."""
    x = torch.full((H, H, C), 1000.0)
    x.view(H * H, G, C // G)[at, :, 0] = 1004.0
    mean, rstd, m, r, dev, _, _ = _stats(x, G, copies, eps=0.0)
    assert float((rstd / r - 1).abs().max()) <= 4e-6
    assert bool(((mean - m).abs() <= 4e-6 * dev + 2.0 ** -24 * m.abs()).all())


@pytest.mark.parametrize("H,C,G,copies", [(20, 24, 3, 2), (20, 24, 3, 400), (3, 8, 1, 1)])
@pytest.mark.parametrize("scale", [2.0 ** -50, 2.0 ** 49, 2.0 ** 64, 2.0 ** 80, 2.0 ** 125])
def test_squares_at_the_ends_of_fp32(H, C, G, copies, scale):
    """The largest and the smallest values that the header admits (|x| < 2^52: normal values below 8 times 2^49; a variance of 2^-100), as
    they are; and larger ones: NaN where squares overflow, in the scaled group only, and nothing finite and wrong."""
    gen = torch.Generator().manual_seed(23)
    x = torch.randn((H, H, C), generator=gen)
    x[..., :C // G] *= scale
    mean, rstd, m, r, dev, y, xb = _stats(x, G, copies, eps=0.0)
    over = torch.isnan(rstd)                       # (threads of one pixel have no squares of their own: 2^64 is right at 3x3)
    assert not over[:, 1:].any() and not (scale < 2.0 ** 64 and over.any()) and (scale < 2.0 ** 80 or over[:, 0].all())
    assert bool((over | ((rstd / r - 1).abs() <= 4e-6)).all())
    assert bool((over | ((mean - m).abs() <= 4e-6 * dev + 2.0 ** -24 * m.abs())).all())
    # y: its rounding to bf16, and 1e-5 of its terms, which are below 8
    want = ((xb.reshape(H, H, G, -1) - m[:, None]) * r[:, None]).reshape(H, H, C)
    gone = over[-1].repeat_interleave(C // G)
    assert torch.isnan(y[..., gone]).all()
    assert bool(((y - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5 * 8)[..., ~gone].all())


# ------------------------------------------------------------------------------------------------ gradients
def _backward(x, dy, g, b, mean, rstd, begin, act, res=None, packed=False, want_dres=True):
    """dx, dresidual, dgamma, dbeta of x [N][H][W][C] (C a multiple of 8) by the kernel, as fp64."""
    c = Hh.ctx()
    N, H, Wd, C = x.shape
    G = len(begin) - 1
    d = B.make_gn_desc(N, H, Wd, C, G, C, act=act, group_begin=begin)
    f = lambda a: torch.as_tensor(np.asarray(a), dtype=torch.float32).cuda()
    xd, dyd, rd = x.bfloat16().cuda(), dy.bfloat16().cuda(), res.bfloat16().cuda() if res is not None else None
    dx, dres = torch.empty_like(xd), torch.empty_like(xd) if want_dres else None
    dg, db = (torch.full((C,), 7.0, device="cuda") for _ in range(2))
    ws = torch.empty(B.pt_gn_workspace_bytes(c, d), dtype=torch.uint8, device="cuda")
    if packed:
        codes, scales = B.checkpoint_buffers(N * H * Wd, C)
        B.pt_act_pack(c, B.make_pack_desc(N * H * Wd, C), xd, codes, scales)
        B.pt_gn_act_bwd_packed(c, d, codes, scales, rd, dyd, f(g), f(b), f(mean), f(rstd), dx, dres, dg, db, None, ws)
    else:
        B.pt_gn_act_bwd(c, d, xd, rd, dyd, f(g), f(b), f(mean), f(rstd), dx, dres, dg, db, ws)
    torch.cuda.synchronize()
    c.poll()
    h = lambda t: t.double().cpu().numpy() if t is not None else None
    return h(dx), h(dres), h(dg), h(db)


@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("rstd", [2.0 ** -60, 2.0 ** -50, 1e-13, 1e13, 2.0 ** 50, 2.0 ** 60])
def test_gradients_at_small_and_large_deviations(rstd, packed, act):
    """dx keeps its term in xhat where rstd^3 is not an fp32 number. The bound is that of ordinary values: a rounding to bf16 and 1e-5 of the
    terms' magnitudes."""
    gen = torch.Generator().manual_seed(24)
    N, H, C, begin = 2, 9, 24, [0, 11, 24]
    x = W.bf16_round(torch.randn((N, H, H, C), generator=gen) / rstd)
    dy, g, b = W.bf16_round(torch.randn((N, H, H, C), generator=gen)), torch.rand(C, generator=gen) + 0.5, torch.rand(C, generator=gen) - 0.5
    _, mean, _ = oracle.gn_act_fwd(x.numpy(), g.numpy(), b.numpy(), begin, 0.0)
    mean, rs = mean.astype(np.float32), np.full((N, 2), rstd, np.float32)
    dx, _, dg, db = _backward(x, dy, g, b, mean, rs, begin, act, packed=packed)
    xv = oracle.act_unpack(*oracle.act_pack(x.numpy())) if packed else x.double().numpy()
    rdx, _, rdg, rdb, _ = oracle.gn_act_bwd(xv, dy.numpy(), g.numpy(), b.numpy(), mean, rs, begin, None, act)
    sp = lambda v: np.repeat(np.asarray(v, np.float64), np.diff(begin), axis=1)[:, None, None, :]
    xhat, w = np.abs(xv - sp(mean)) * sp(rs), np.abs(dy.double().numpy() * g.double().numpy()) * (1.1 if act == 2 else 1.0)
    # (SiLU's slope is 1.1 at most)
    means = lambda v: sp(np.stack([v[..., s:e].mean((1, 2, 3)) for s, e in zip(begin[:-1], begin[1:])], 1))
    terms = sp(rs) * (w + means(w) + xhat * means(w * xhat))
    assert np.all(np.abs(dx - rdx) <= 2.0 ** -8 * np.abs(rdx) + 1e-5 * terms)
    ady = np.abs(dy.double().numpy()) * 1.1
    assert np.all(np.abs(dg - rdg) <= 1e-5 * (ady * xhat).sum((0, 1, 2))) and np.all(np.abs(db - rdb) <= 1e-5 * ady.sum((0, 1, 2)))


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("N", [33 * 296 + 5, 1 << 20, 1 << 24])
def test_parameter_gradients_over_many_small_images(N, packed):
    """Images of one pixel with equal gradients of one sign: chains of equal additions, which fp32 rounds the same way every time. 32 units are
    added in fp32, off by 2^-24 of their sum so far each, (1 + .. + 32)/32 * 2^-24 = 1e-6 of the sum; a product of rounded factors before
    them adds 3 * 2^-24, the rounding of a block's sum 2^-24; the sums of at most 320 blocks are added ten in a row, (1 + .. + 9)/10 * 2^-24,
    and those in five steps, 5 * 2^-24: 1.9e-6 in all."""
    C, begin = 8, [0, 3, 8]
    x, dy = torch.full((N, 1, 1, C), 1.5), torch.full((N, 1, 1, C), 0.69921875)
    mean, rstd = np.full((N, 2), 0.3, np.float32), np.full((N, 2), 0.9, np.float32)
    _, _, dg, db = _backward(x, dy, np.ones(C), np.ones(C), mean, rstd, begin, 1, packed=packed, want_dres=False)
    xhat = (1.5 - float(np.float32(0.3))) * float(np.float32(0.9))
    assert np.abs(db / (N * 0.69921875) - 1).max() <= 1.9e-6
    assert np.abs(dg / (N * 0.69921875 * xhat) - 1).max() <= 1.9e-6


def test_one_call_for_many_images_is_many_calls():
    """dgamma and dbeta of a batch whose blocks take dozens of images each are the sums of the batch's parts, which take a few."""
    gen = torch.Generator().manual_seed(25)
    N, H, C, begin = 24000, 2, 16, [0, 5, 16]
    x, dy = W.bf16_round(torch.randn((N, H, H, C), generator=gen)), W.bf16_round(torch.randn((N, H, H, C), generator=gen).abs())
    g, b = torch.rand(C, generator=gen) + 0.5, torch.rand(C, generator=gen) - 0.5
    mean, rstd = np.zeros((N, 2), np.float32), np.ones((N, 2), np.float32)
    dx, _, dg, db = _backward(x, dy, g, b, mean, rstd, begin, 2)
    parts = [_backward(x[s:s + 2000], dy[s:s + 2000], g, b, mean[s:s + 2000], rstd[s:s + 2000], begin, 2) for s in range(0, N, 2000)]
    assert np.array_equal(dx, np.concatenate([q[0] for q in parts]))
    ady = dy.double().numpy() * 1.1                             # (SiLU's slope is 1.1 at most)
    # both sides: 1.9e-6 of the magnitudes as above, and SiLU's slope, off the same way on both
    assert np.all(np.abs(dg - sum(q[2] for q in parts)) <= 3.8e-6 * (ady * np.abs(x.double().numpy())).sum((0, 1, 2)))
    assert np.all(np.abs(db - sum(q[3] for q in parts)) <= 3.8e-6 * ady.sum((0, 1, 2)))


@pytest.mark.parametrize("with_res", [False, True])
@pytest.mark.parametrize("packed", [False, True])
def test_relu_where_beta_is_lost_beside_the_mean(packed, with_res):
    """A group of equal values is its beta: of either sign, however small beside the mean, with either sign of gamma and without one, z > 0
    exactly where beta > 0."""
    N, H, C = 2, 4, 32
    gen = torch.Generator().manual_seed(26)
    beta = torch.tensor([1e-12, -1e-12, 1e-4, -1e-4, 2.0 ** -100, -(2.0 ** -100), 0.0, -0.0]).repeat(4)
    gamma = torch.tensor([1.0, -1.0, 0.75, 0.0]).repeat_interleave(8)
    for value in (1000.0, -0.5, 0.0):
        x, dy = torch.full((N, H, H, C), value), W.bf16_round(torch.rand((N, H, H, C), generator=gen) + 0.5)
        res = torch.zeros_like(x) if with_res else None
        dx, dres, dg, db = _backward(x, dy, gamma, beta, np.full((N, 1), value, np.float32), np.full((N, 1), 1e-5 ** -0.5, np.float32), [0, C], 1, res, packed)
        want = dy.double().numpy() * (beta.numpy() > 0)
        assert np.array_equal(dres, want), value
        assert np.all(np.abs(db - want.sum((0, 1, 2))) <= 1e-6 * want.sum((0, 1, 2)))


@pytest.mark.parametrize("with_res", [False, True])
def test_relu_next_to_its_limit(with_res):
    """beta is minus gamma * xhat of a value, rounded to fp32: z there is its rounding, 2^-25 of beta or less, and the next bf16 values lie on
    either side. Against the formula in 64 bits, which is off by 2^-52 of beta."""
    gen = torch.Generator().manual_seed(27)
    N, H, C = 1, 3, 2048
    for mean, scale in ((0.0, 1.0), (3.14159, 1.0), (100.3, 0.01), (-7.7, 1e-6), (1e-3, 1e4)):
        mean, rstd = np.full((N, 1), mean, np.float32), np.full((N, 1), 1.37 / scale, np.float32)
        gamma = torch.where(torch.rand(C, generator=gen) < 0.5, -1.0, 1.0) * (torch.rand(C, generator=gen) + 0.1)
        at = W.bf16_round(torch.from_numpy(mean.astype(np.float32))[0] + scale * torch.randn(C, generator=gen))
        xhat = (at.double() - float(mean[0, 0])) * float(rstd[0, 0])
        beta = -(xhat * gamma.double()).float()
        bits = at.bfloat16().view(torch.int16).to(torch.int32)
        x = torch.stack([(bits + k).to(torch.int16).view(torch.bfloat16).float() for k in (-2, -1, -1, 0, 0, 0, 1, 1, 2)]).view(N, H, H, C)
        dy = torch.ones((N, H, H, C))
        res = torch.zeros_like(x) if with_res else None
        _, dres, _, db = _backward(x, dy, gamma, beta, mean, rstd, [0, C], 1, res)
        z = (x.double() - float(mean[0, 0])) * float(rstd[0, 0]) * gamma.double() + beta.double()
        assert np.array_equal(dres > 0, (z > 0).numpy())
        assert np.array_equal(db, (z > 0).sum((0, 1, 2)).double().numpy())


@pytest.mark.parametrize("with_res", [False, True])
@pytest.mark.parametrize("packed", [False, True])
def test_relu_where_gamma_times_rstd_is_no_fp32_number(packed, with_res):
    """z = gamma * xhat, of the sign of x - mean, where gamma * rstd underflows to 0 in fp32; a gamma of 0 passes nothing."""
    gen = torch.Generator().manual_seed(28)
    N, H, C = 2, 5, 16
    x = W.bf16_round(torch.randn((N, H, H, C), generator=gen) * 2.0 ** 50)
    dy, gamma = torch.ones((N, H, H, C)), torch.tensor([1e-38, -1e-38, 1e-40, 0.0]).repeat(4)
    mean, rstd = np.zeros((N, 1), np.float32), np.full((N, 1), 2.0 ** -50, np.float32)
    _, dres, _, db = _backward(x, dy, gamma, np.zeros(C), mean, rstd, [0, C], 1, torch.zeros_like(x) if with_res else None, packed)
    xv = oracle.act_unpack(*oracle.act_pack(x.numpy())) if packed else x.double().numpy()
    want = xv * np.sign(gamma.double().numpy()) > 0
    assert np.array_equal(dres > 0, want) and np.array_equal(db, want.sum((0, 1, 2)))


# ------------------------------------------------------------------------------------------------ refusals
def test_sizes_whose_products_pass_64_bits_are_refused():
    c = Hh.ctx()
    t, v, s = torch.zeros(64, dtype=torch.bfloat16, device="cuda"), torch.zeros(8, device="cuda"), torch.zeros(8, device="cuda")
    most = (1 << 31) - 1
    for H, Wd in ((most, most), (most, 1 << 30), (1 << 30, 1 << 30), (1 << 16, 1 << 15)):
        d = B.make_gn_desc(1, H, Wd, 8, 1, 8)
        assert B.pt_gn_workspace_bytes(c, d) == 0, (H, Wd)
        with pytest.raises(B.PtError) as e:
            B.pt_gn_act_fwd(c, d, t, None, v, v, s, s.clone(), t.clone())
        assert e.value.status == 2
    codes, scales = B.checkpoint_buffers(4, 8)
    for npix in ((1 << 40) + 1, (1 << 63) - 1):
        for call in (lambda d: B.pt_act_pack(c, d, t, codes, scales), lambda d: B.pt_act_unpack(c, d, codes, scales, t)):
            with pytest.raises(B.PtError) as e:
                call(B.make_pack_desc(npix, 8))
            assert e.value.status == 2


# ------------------------------------------------------------------------------------------------ the chained step
def _network():
    net = W.resnet50(32)
    return W.with_sizes(net, W.uniform_keep(net, 0.2))


def test_saved_bytes_count_what_the_backward_pass_reads():
    """From the shapes: a code per channel, padded to 8, and a scale byte per 32 of every convolution's output, every block's input and every
    projection; two statistics per image and group; a byte per value of the pooled stem."""
    net, N, groups = _network(), 3, 4
    s = harness.CheckpointedStep(Hh.ctx(), net, N, W.BASE_SEED + 7400, groups=groups, max_blocks=2)
    ck = lambda P, K: N * P * P * W.pad8(K) + (N * P * P * ((K + 31) // 32) + 15) // 16 * 16
    L = net.layers
    want = sum(ck(L[i].P, L[i].K) + 2 * 4 * N * min(groups, L[i].K) for i in s.used)
    want += sum(ck(L[m[0]].H, L[m[0]].C) for m, _, _ in s.blocks) + sum(ck(L[d].P, L[d].K) for _, d, _ in s.blocks if d is not None)
    assert s.pool
    want += N * s.pool_index.shape[1] ** 2 * W.pad16(L[0].K)
    assert s.saved_bytes() == want
    s.step()
    torch.cuda.synchronize()
    Hh.ctx().poll()
    assert s.saved_bytes() == want


def test_group_norm_chain_is_the_same_on_side_streams():
    """A pruned ResNet-50 chained with group norm, with the weight gradients and the projection shortcuts (their norms too, with a workspace
    of their own) on side streams: every result is what it is on one stream, bit for bit where the launches are the same; weight gradients,
    whose sums are split differently, to the rounding of fp32 sums over up to 200 K pixels, and bit for bit from run to run."""
    c = Hh.ctx()
    net, seed = W.resnet50(), W.BASE_SEED + 7500
    netp = W.with_sizes(net, W.staged_keep_to_flops(net, seed, 0.60))
    model = W.gen_model(netp, seed)
    runs = []
    for streams in (0, 2, 2):
        s = harness.ChainedStep(c, netp, 16, seed, model=model, norm="group", wgrad_streams=streams)
        for _ in range(2):                                       # the second step's launches meet the first one's
            out = s.forward()
            s.backward()
        torch.cuda.synchronize()
        c.poll()
        runs.append(dict(out=[out.clone(), s.dy[0].clone()] + [t.clone() for i in s.used for t in (s.sm[i], s.si[i], s.dg[i], s.db[i])],
                         dw=[s.dm.g[i].clone() for i in s.used]))
        del s
        torch.cuda.empty_cache()
    c.set_wgrad_cta_limit(0)
    one, a, b = runs
    for r in (a, b):
        assert all(torch.equal(x, y) for x, y in zip(r["out"], one["out"]))
        assert all(float((x - y).abs().max()) <= 2e-4 * float(y.abs().max()) for x, y in zip(r["dw"], one["dw"]))
    assert all(torch.equal(x, y) for x, y in zip(a["dw"], b["dw"]))


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("large", [30.0, 1e3, 1e5, 1e7, 1e12, 2.0 ** 100])
def test_silu_gradients_at_large_values(large, packed):
    """SiLU's slope is 1 for large z, and 0 for -z, whatever the neighbouring channels hold. dresidual: a rounding to bf16, 2^-8 of the slope, and
    1e-5 of |dy| (what the header states for z below -41: |z| * 2^-60 at most, |z| taken as 2^20 at most)."""
    gen = torch.Generator().manual_seed(29)
    N, H, C, begin = 2, 7, 16, [0, 16]
    x, dy = (W.bf16_round(torch.randn((N, H, H, C), generator=gen)) for _ in range(2))
    r = W.bf16_round(torch.randn((N, H, H, C), generator=gen))
    at = torch.rand((N, H, H, C), generator=gen)
    r = torch.where(at < 0.25, W.bf16_round(torch.tensor(large)), torch.where(at < 0.4, -W.bf16_round(torch.tensor(large)), r))
    g, b = torch.rand(C, generator=gen) + 0.5, torch.rand(C, generator=gen) - 0.5
    mean, rstd = np.full((N, 1), 0.1, np.float32), np.full((N, 1), 1.1, np.float32)
    dx, dres, dg, db = _backward(x, dy, g, b, mean, rstd, begin, 2, r, packed)
    xv = oracle.act_unpack(*oracle.act_pack(x.numpy())) if packed else x.double().numpy()
    with np.errstate(over="ignore", invalid="ignore"):
        xhat = (xv - float(mean[0, 0])) * float(rstd[0, 0])
        z = xhat * g.double().numpy() + b.double().numpy() + r.double().numpy()
        e = np.exp(-np.abs(z))
        s = np.where(z >= 0, 1.0, e) / (1.0 + e)
        slope = s + np.where(np.abs(z) < 700, z, 0.0) * s * (np.where(z >= 0, e, 1.0) / (1.0 + e))
    ady = np.abs(dy.double().numpy())
    want = dy.double().numpy() * slope
    assert np.all(np.abs(dres - want) <= 2.0 ** -8 * np.abs(want) + 1e-5 * ady)
    assert np.all(np.abs(db - want.sum((0, 1, 2))) <= 1e-5 * 1.1 * ady.sum((0, 1, 2)))
    assert np.all(np.abs(dg - (want * xhat).sum((0, 1, 2))) <= 1e-5 * 1.1 * (ady * np.abs(xhat)).sum((0, 1, 2)))


_FIRST = '''
import torch
from paper_1901_09290_b200 import binding as B
c, N, H, C, G = B.Context(0), 6, 9, 24, 3
g = torch.Generator(device="cuda").manual_seed(1)
x, dy = (torch.randn((N, H, H, C), generator=g, device="cuda").bfloat16() for _ in range(2))
gam, bet = torch.rand(C, device="cuda"), torch.rand(C, device="cuda")
d, pd = B.make_gn_desc(N, H, H, C, G, act=B.PT_ACT_SILU), B.make_pack_desc(N * H * H, C)
def bufs():
    o = [torch.zeros((N, G), device="cuda") for _ in range(2)] + [torch.zeros_like(x) for _ in range(3)] + [torch.zeros(C, device="cuda") for _ in range(2)]
    return o + list(B.checkpoint_buffers(N * H * H, C)) + [torch.empty(B.pt_gn_workspace_bytes(c, d), dtype=torch.uint8, device="cuda")]
def go(mean, rstd, y, dx, back, dg, db, codes, scales, ws):
    B.pt_gn_act_fwd(c, d, x, None, gam, bet, mean, rstd, y, codes, scales)
    B.pt_gn_act_bwd_packed(c, d, codes, scales, None, dy, gam, bet, mean, rstd, dx, None, dg, db, None, ws)
    B.pt_act_unpack(c, pd, codes, scales, back)
    B.pt_act_pack(c, pd, back, codes, scales)
a, b = bufs(), bufs()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    go(*a)
graph.replay()
go(*b)
torch.cuda.synchronize()
c.poll()
assert all(torch.equal(p, q) for p, q in zip(a[:8], b[:8])) and a[3].abs().max() > 0
print("same")
'''


def test_the_first_calls_of_a_process_may_be_captured():
    """Nothing is left to a first call that a capture does not allow."""
    r = subprocess.run([sys.executable, "-c", _FIRST], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stderr[-2000:]


def test_two_threads_of_a_context():
    """Calls of one context from two threads at once, on streams of their own, first ones of their shapes: as one by one."""
    c, C, G = Hh.ctx(), 40, 5
    gen = torch.Generator(device="cuda").manual_seed(30)
    one, zero = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    shapes = [(n, h) for n in (3, 7, 11) for h in (5, 13, 17, 23)]
    xs = {s: torch.randn((s[0], s[1], s[1], C), generator=gen, device="cuda").bfloat16() for s in shapes}

    def run(out, stream):
        torch.cuda.set_device(0)
        for N, H in shapes:
            d = B.make_gn_desc(N, H, H, C, G, act=B.PT_ACT_NONE, eps=2e-5)
            o = [torch.empty_like(xs[N, H]), torch.empty((N, G), device="cuda"), torch.empty((N, G), device="cuda")]
            stream.wait_stream(torch.cuda.current_stream())
            B.pt_gn_act_fwd(c, d, xs[N, H], None, one, zero, o[1], o[2], o[0], stream=stream)
            out.append(o)

    torch.cuda.synchronize()
    outs, streams = [[], []], [torch.cuda.Stream(), torch.cuda.Stream()]
    threads = [threading.Thread(target=run, args=a) for a in zip(outs, streams)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    last = []
    run(last, torch.cuda.current_stream())
    torch.cuda.synchronize()
    c.poll()
    assert len(outs[0]) == len(outs[1]) == len(shapes)
    for a, b, e in zip(outs[0], outs[1], last):
        assert all(torch.equal(p, r) and torch.equal(q, r) for p, q, r in zip(a, b, e))
