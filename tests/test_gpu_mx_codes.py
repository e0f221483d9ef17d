"""Codes of the microscaled formats where little is left of a value: the sign of zero, numbers below the normal ones."""
import numpy as np
import pytest
import torch

import mx_helpers as mx
import paper_1711_04713_amd as lp
from test_gpu_mx import ROUNDINGS, TYPES, ckpt8_buffers, mx4_buffers, philox_draws

pytestmark = pytest.mark.gpu


def mx4_codes(x, mode, seed):
    """Whole code bytes: the sign is that of the value, also where the magnitude rounds to zero; NaN is 0."""
    v = x.double().numpy()
    codes, scales, zeros, clipped = mx.mx4_quantize(v, mode, philox_draws(v.size, seed) if mode == "stochastic" else None)
    sign = np.zeros((v.shape[0], codes.shape[1] * 2), np.uint8)
    sign[:, :v.shape[1]] = np.signbit(v) & ~np.isnan(v)
    return (codes & 0x77) | sign[:, 0::2] << 3 | sign[:, 1::2] << 7, scales, zeros, clipped


def check_mx4(x, mode, seed=0x123456789abcdef):
    want = mx4_codes(x, mode, seed)
    codes, scales = mx4_buffers(*x.shape)
    counts = [torch.zeros(1, dtype=torch.int64, device="cuda") for _ in range(2)]
    lp.lp_mx4_quantize(x.cuda(), codes, scales, ROUNDINGS[mode], seed, *counts)
    assert np.array_equal(scales.cpu().numpy(), want[1])
    assert np.array_equal(codes.cpu().numpy(), want[0])
    assert tuple(c.item() for c in counts) == want[2:]
    again = mx4_buffers(*x.shape)
    lp.lp_mx4_quantize(x.cuda(), *again, ROUNDINGS[mode], seed)      # without counters
    assert torch.equal(again[0], codes) and torch.equal(again[1], scales)


@pytest.mark.parametrize("mode", list(ROUNDINGS))
@pytest.mark.parametrize("dtype", TYPES)
def test_the_sign_of_zero(dtype, mode):
    g = torch.Generator().manual_seed(1)
    x = torch.randn((9, 300), generator=g)
    little = torch.tensor([0.0, -0.0, 0.01, -0.01, 0.12, -0.12, float("nan"), -float("nan"), 4.0, -4.0, float("inf"), -float("inf")])
    x = torch.where(torch.rand(x.shape, generator=g) < 0.6, little[torch.randint(0, len(little), x.shape, generator=g)], x).to(dtype)
    x[2], x[3, 32:64] = 0.0, -0.0
    x[4, :32] = torch.tensor([-0.0, float("nan")]).repeat(16).to(dtype)
    check_mx4(x, mode)


def below_normal(dtype):
    """Blocks whose largest magnitude lies around the smallest normal number of the type, and of 32 bits."""
    g = torch.Generator().manual_seed(2)
    tiny = torch.finfo(dtype).tiny
    x = torch.rand((40, 256), generator=g, dtype=torch.double) * torch.tensor([2.0 ** (k / 4) for k in range(-16, 24)], dtype=torch.double)[:, None] * tiny
    x = (x * torch.sign(torch.randn(x.shape, generator=g))).to(dtype)
    # halves of the least code's magnitudes of 32 bits, exactly: 2^-127 and 3 * 2^-127
    if dtype != torch.float16:
        x[0, :4] = torch.tensor([2.0 ** -127, -(2.0 ** -127), 3 * 2.0 ** -127, -3 * 2.0 ** -127], dtype=torch.double).to(dtype)
    return x


@pytest.mark.parametrize("mode", list(ROUNDINGS))
@pytest.mark.parametrize("dtype", TYPES)
def test_numbers_below_the_normal_ones(dtype, mode):
    x = below_normal(dtype)
    check_mx4(x, mode)
    seed = 77
    want = mx.ckpt8_quantize(x.double().numpy(), mode, philox_draws(x.numel(), seed) if mode == "stochastic" else None)
    codes, scales = ckpt8_buffers(*x.shape)
    lp.lp_ckpt8_save(x.cuda(), codes, scales, r=ROUNDINGS[mode], seed=seed)
    assert np.array_equal(scales.cpu().numpy(), want[1])
    assert np.array_equal(codes.cpu().numpy(), want[0])


def test_relu_gradient_of_values_that_are_kept_as_zero():
    """The slope is that of the kept value: half a step of the block (2^-5 here) and less is 0, a little more is not."""
    x = torch.zeros((1, 64))
    x[0, 0], x[0, 1:7] = 4.0, torch.tensor([2.0 ** -5, 2.0 ** -5 * 1.01, 2.0 ** -9, -1.0, 1.0, -(2.0 ** -5) * 1.01])
    x[0, 32:40] = torch.tensor([2.0 ** -5, 2.0 ** -7, 2.0 ** -9, 2.0 ** -13, 2.0 ** -12 * 1.01, -0.0, 0.0, -1e-9])    # largest: 2^-5
    codes, scales = ckpt8_buffers(1, 64)
    y, dx = torch.empty((1, 64), device="cuda"), torch.empty((1, 64), device="cuda")
    lp.lp_ckpt8_save(x.cuda(), codes, scales, act=lp.LP_ACT_RELU, y=y)
    lp.lp_ckpt8_act_bwd(codes, scales, torch.full((1, 64), 3.0, device="cuda"), dx, lp.LP_ACT_RELU)
    want = torch.zeros((1, 64))
    want[0, [0, 2, 5]] = 3.0
    want[0, [32, 33, 34, 36]] = 3.0
    assert torch.equal(dx.cpu(), want)
    assert torch.equal(y.cpu() > 0, x > 0)
