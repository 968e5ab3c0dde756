"""Pins of the oracle's group normalisation and of its 8-bit activation checkpoints, independent of their own formulas."""
import numpy as np
import pytest
import torch

import oracle


def _rand(shape, seed):
    return np.random.default_rng(seed).standard_normal(shape)


@pytest.mark.parametrize("C,groups", [(12, 3), (12, 12), (12, 1)])
def test_forward_is_the_library_routine(C, groups):
    x, g, b = _rand((3, 4, 5, C), 1) * 2 + 1, _rand(C, 2), _rand(C, 3)
    y, mean, rstd = oracle.gn_act_fwd(x, g, b, oracle.group_begin(C, groups), 1e-3, act=0)
    t = torch.from_numpy(x).permute(0, 3, 1, 2)
    want = torch.nn.functional.group_norm(t, groups, torch.from_numpy(g), torch.from_numpy(b), 1e-3).permute(0, 2, 3, 1).numpy()
    assert np.allclose(y, want, rtol=0, atol=1e-12)
    r = _rand(x.shape, 4)
    assert np.allclose(oracle.gn_act_fwd(x, g, b, oracle.group_begin(C, groups), 1e-3, r, 1)[0], np.maximum(want + r, 0), atol=1e-12)
    z = torch.from_numpy(want)
    assert np.allclose(oracle.gn_act_fwd(x, g, b, oracle.group_begin(C, groups), 1e-3, act=2)[0], torch.nn.functional.silu(z).numpy(), atol=1e-12)


def test_groups_of_unequal_sizes_are_normalised_by_themselves():
    x, g, b = _rand((2, 3, 3, 10), 5), _rand(10, 6), _rand(10, 7)
    y, mean, rstd = oracle.gn_act_fwd(x, g, b, [0, 1, 7, 10], act=0)
    for s, e in ((0, 1), (1, 7), (7, 10)):
        part = oracle.gn_act_fwd(x[..., s:e], g[s:e], b[s:e], [0, e - s], act=0)[0]
        assert np.allclose(y[..., s:e], part, atol=1e-13)
    assert mean.shape == rstd.shape == (2, 3)


@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("with_res", [False, True])
def test_backward_against_finite_differences(act, with_res):
    begin = [0, 2, 5]
    x, G = _rand((2, 2, 3, 5), 8), _rand((2, 2, 3, 5), 9)
    g, b = np.random.default_rng(10).uniform(0.5, 1.5, 5), np.random.default_rng(11).uniform(0.2, 0.6, 5)
    r = _rand(x.shape, 12) if with_res else None
    eps, h = 1e-3, 1e-6

    def loss(x_, g_, b_, r_):
        return float((oracle.gn_act_fwd(x_, g_, b_, begin, eps, r_, act)[0] * G).sum())

    y, mean, rstd = oracle.gn_act_fwd(x, g, b, begin, eps, r, act)
    assert np.abs(y[y != 0]).min() > 10 * h                     # no value within a step of the ReLU's kink
    dx, dres, dg, db, again = oracle.gn_act_bwd(x, G, g, b, mean, rstd, begin, r, act)
    assert np.allclose(again, y, atol=1e-13)
    for which, grad in ((0, dx), (1, dg), (2, db)) + (((3, dres),) if with_res else ()):
        args = [x, g, b, r]
        for at in np.ndindex(grad.shape):
            d = np.zeros_like(args[which])
            d[at] = h
            up, down = list(args), list(args)
            up[which], down[which] = args[which] + d, args[which] - d
            assert abs((loss(*up) - loss(*down)) / (2 * h) - grad[at]) < 1e-6


def test_checkpoint_by_hand():
    x = np.zeros((1, 40))
    x[0, :4] = [127.0, -1.0, 0.5, 1.5]                           # step 1: 0.5 and 1.5 go to the even neighbour
    x[0, 32:36] = [127.5, 1.0, 3.0, -127.5]                      # rint(127.5) = 128 is too large: step 2
    codes, scales = oracle.act_pack(x)
    assert scales.tolist() == [[127, 128]]
    assert codes[0, :4].tolist() == [127, -1, 0, 2] and codes[0, 32:36].tolist() == [64, 0, 2, -64]
    assert oracle.act_unpack(codes, scales)[0, 32] == 128.0


def test_checkpoint_error_and_special_values():
    rng = np.random.default_rng(13)
    x = oracle.round_bf16(rng.standard_normal((50, 70)) * np.exp2(rng.integers(-140, 120, (50, 1)).astype(float))).astype(np.float64)
    x[3, 40], x[4, 65] = np.inf, np.nan
    x[5] = 0
    x[6] = (2 - 2.0 ** -7) * 2.0 ** 127                            # the largest bf16
    codes, scales = oracle.act_pack(x)
    back = oracle.act_unpack(codes, scales)
    assert scales[3].tolist()[1] == 255 and scales[4].tolist()[2] == 255 and scales[5].tolist() == [0, 0, 0]
    for n in range(50):
        for k in range(3):
            v, w = x[n, 32 * k:32 * k + 32], back[n, 32 * k:32 * k + 32]
            if not np.all(np.isfinite(v)):
                assert np.all(np.isnan(w))
                continue
            assert np.abs(v - w).max() <= max(np.abs(v).max() / 127, 2.0 ** -128)
            assert np.array_equal(oracle.round_bf16(w), w), "a restored value is exact in bf16"
            again = oracle.act_pack(w[None])                        # a checkpoint of restored values restores them
            assert np.array_equal(oracle.act_unpack(*again)[0], w)
