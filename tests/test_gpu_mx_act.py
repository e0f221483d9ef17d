"""SiLU and GELU of 32-bit tensors, and their slopes, against 64 bits: errors of a few half steps over the whole range.

With h = 2^-24, half a step: the hardware's 2^x and reciprocal are off by one step (2 h), every other operation by h.
 * a = exp(-|z|): the argument times log2 e is held in two numbers, the second's share is added to 2^x: 2 h + h, 3 h.
 * s(|z|) = 1 / (1 + a): a's share 1.5 h at most, the sum h, the reciprocal after a Newton step h: below 4 h.  s(-|z|) = a times
   that: 3 h of a (its share of the sum is of the opposite sign), h + h, the product h: 6 h.
 * SiLU: 7 h.  Its slope s (1 + g t), t = s(-g): 6 h of s and of t, h for the sum, h for the product.
 * GELU: z = g (c + c A g^2) is off by 3 h of itself (two constants and a square, one rounding of the sum; the product with g is
   held in two numbers), which is 3 h |z| of a.  dz / dg = c (1 + 3 A g^2): 4 h.
 * Results of 16 bits: the argument is in one number, its constant and its product are h |z| each: 2 h |z|, GELU 4 h |z|.
Where a is below the smallest normal number, beyond |z| = 87, it may be taken as 0."""
import numpy as np
import pytest
import torch

import mx_helpers as mx
import paper_1711_04713_amd as lp
from test_gpu_mx import ACTS, ckpt8_buffers

pytestmark = pytest.mark.gpu

H = 2.0 ** -24
C, A = 2 * np.sqrt(2 / np.pi), 0.044715


def arguments(cols, seed):
    """Every size of argument from 2^-20 to 200, both signs; the last columns far out."""
    g = torch.Generator().manual_seed(seed)
    x = torch.exp(torch.empty(cols, dtype=torch.double).uniform_(np.log(2.0 ** -20), np.log(200.0), generator=g))
    x = torch.where(torch.rand(cols, generator=g) < 0.5, torch.empty(cols, dtype=torch.double).uniform_(0.0, 100.0, generator=g), x)
    x = (x * torch.sign(torch.randn(cols, generator=g))).float()
    x[-8:] = torch.tensor([0.0, -0.0, 3e38, -3e38, 1e5, -1e5, float("inf"), -float("inf")])
    return x


def parts(x, act):
    """In 64 bits: s(z), s(-z), |z| and dz / dx."""
    z = x if act == "silu" else C * (x + A * x ** 3)
    a = np.exp(-np.abs(z))
    big, small = 1 / (1 + a), a / (1 + a)
    dz = np.ones_like(x) if act == "silu" else C * (1 + 3 * A * x * x)
    return np.where(z < 0, small, big), np.where(z < 0, big, small), np.minimum(np.abs(z), 200.0), dz


def check_values(y, x, act):
    x = x.double().numpy()
    finite = np.clip(x, -1e30, 3.5e38)
    s, _, z, _ = parts(np.clip(finite, -1e4, 1e4), act)
    want = np.where(x == np.inf, np.inf, finite * s)
    got = y.cpu().double().numpy()
    off = np.abs(np.where(np.isinf(want), 0, got - np.where(np.isinf(want), 0, want)))
    bound = np.abs(np.where(np.isinf(want), 0, want)) * H * (8 + (3 * z if act == "gelu" else 0)) + 1.2e-36
    assert np.array_equal(np.isinf(got), np.isinf(want)) and not np.isnan(got).any()
    worst = int(np.argmax(off / bound))
    assert off[worst] <= bound[worst], (act, x[worst], got[worst], want[worst], off[worst] / bound[worst])


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_values_beside_the_checkpoint(act):
    x = arguments(1 << 16, 1)
    y = torch.empty((1, len(x)), device="cuda")
    codes, scales = ckpt8_buffers(1, len(x))
    lp.lp_ckpt8_save(x.cuda().view(1, -1), codes, scales, act=ACTS[act], y=y)
    check_values(y[0], x, act)


# few rows, tiles, parts that are joined
@pytest.mark.parametrize("m,k", [(1, 512), (70, 512), (40, 8192)])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_values_of_a_product(act, m, k):
    """Inputs of 0: the function of the bias alone."""
    n = 2000
    bias = arguments(n, 2)
    w = [torch.zeros(b, dtype=torch.uint8, device="cuda") for b in lp.lp_mx4_bytes(n, k)]
    w[1].fill_(127)
    y = torch.empty((m, n), device="cuda")
    ws = torch.empty(max(lp.lp_mx4_fc_workspace_bytes(m, k, n), 16), dtype=torch.uint8, device="cuda")
    lp.lp_mx4_fc_fwd(m, k, n, torch.zeros((m, k), device="cuda"), w[0], w[1], y, bias=bias.cuda(), act=ACTS[act], workspace=ws)
    for row in {0, m // 2, m - 1}:
        check_values(y[row], bias, act)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_slopes(act):
    x = arguments(1 << 16, 3)[None, :-8]
    codes, scales = mx.ckpt8_quantize(x.double().numpy())
    kept = mx.ckpt8_values(codes, scales, x.shape[1])
    dx = torch.empty_like(x, device="cuda")
    lp.lp_ckpt8_act_bwd(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), torch.ones_like(x, device="cuda"), dx, ACTS[act])
    s, t, z, dz = parts(kept, act)
    z = 3 * z if act == "gelu" else np.zeros_like(z)
    turn = kept * t * dz
    want = s * (1 + turn)
    off = np.abs(dx.cpu().double().numpy() - want)
    bound = H * (s * np.abs(turn) * (s * z + 13) + s * np.abs(1 + turn) + np.abs(want) * (t * z + 9)) + 1.2e-36
    worst = np.unravel_index(int(np.argmax(off / bound)), off.shape)
    assert off[worst] <= bound[worst], (act, kept[worst], want[worst], off[worst] / bound[worst])


@pytest.mark.parametrize("act,grows", [("silu", 2), ("gelu", 4)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_every_number_of_16_bits(dtype, act, grows):
    x = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(dtype).view(1, -1)
    y = torch.empty_like(x, device="cuda")
    codes, scales = ckpt8_buffers(*x.shape)
    lp.lp_ckpt8_save(x.cuda(), codes, scales, act=ACTS[act], y=y)
    known = torch.isfinite(x)
    h = x[known].double().numpy()
    s, _, z, _ = parts(np.clip(h, -1e4, 1e4), act)
    mx.close(y.cpu()[known], h * s, np.abs(h * s) * H * (grows * z + 7) + 1.2e-36, dtype)
    nan = torch.isnan(x)
    assert bool(y.cpu()[nan].isnan().all())
    assert bool((y.cpu()[x == float("inf")] == float("inf")).all()) and bool((y.cpu()[x == -float("inf")] == 0).all())
