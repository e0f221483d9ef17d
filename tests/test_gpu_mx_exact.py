"""The microscaled products with operands whose sums are exact in 32 bits: small whole numbers, one scale.  Every result is equal to
the product in 64 bits, so that not one element of a stage can be missing or counted twice."""
import pytest
import torch

import mx_helpers as mx
import paper_1711_04713_amd as lp

pytestmark = pytest.mark.gpu


def whole_numbers(shape, most, seed, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda").to(dtype)


def strided(t, extra):
    """t inside rows that are `extra` elements longer and full of NaN."""
    wide = torch.full((t.shape[0], t.shape[1] + extra), float("nan"), dtype=t.dtype, device="cuda")
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def mx4(rows, cols, seed):
    """An mx4 tensor with scales of 1, and its values: multiples of 1/2 up to 6."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    blocks = mx.mx4_blocks(cols)
    code = torch.randint(0, 16, (rows, blocks * 32), generator=g, device="cuda")
    code[:, cols:] = 0
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.double, device="cuda")
    values = table[code & 7] * (1 - 2.0 * (code >> 3))
    return (code[:, 0::2] | code[:, 1::2] << 4).to(torch.uint8), torch.full((rows, blocks), 127, dtype=torch.uint8, device="cuda"), values[:, :cols].contiguous()


def ckpt8(rows, cols, seed):
    """A ckpt8 tensor with scales of 1, and its values: whole numbers up to 127."""
    blocks = mx.ckpt8_blocks(cols)
    codes = whole_numbers((rows, blocks * 32), 127, seed, torch.int8)
    codes[:, cols:] = 0
    return codes, torch.full((rows, blocks), 133, dtype=torch.uint8, device="cuda"), codes[:, :cols].double().contiguous()


def workspace(size):
    return torch.full((size,), 0xA5, dtype=torch.uint8, device="cuda") if size else None


# dY in whole words, a reduction that ends inside a stage of 64: one stage and less, a few, many; parts, cut last rounds; the three tiles
@pytest.mark.parametrize("size", [(3, 300, 30), (70, 96, 62), (64, 128, 66), (70, 96, 130), (130, 257, 190), (200, 4096, 1002), (1000, 2000, 1030),
                                  (513, 500, 4098), (40, 4096, 8200), (2300, 2400, 62), (2048, 4096, 4110), (4104, 1031, 1030), (4096, 4096, 1090)])
@pytest.mark.parametrize("extra", [0, 2, 8])
def test_input_gradient_of_ragged_reductions(size, extra):
    m, k, n = size
    codes, scales, w = mx4(n, k, 1)
    dy = whole_numbers((m, n), 8, 2, torch.bfloat16)              # sums below 48 n < 2^23 in steps of 1/2
    want = torch.mm(dy.double(), w)
    d, ws = strided(dy, extra), workspace(lp.lp_mx4_fc_dgrad_workspace_bytes(m, k, n))
    for dtype in (torch.float32, torch.bfloat16, torch.float32):
        dx = torch.full((m, k), float("nan"), dtype=dtype, device="cuda")
        lp.lp_mx4_fc_dgrad(m, k, n, d, codes, scales, dx, workspace=ws)
        assert torch.equal(dx, want.to(dtype))


# the same, and weight tiles that reach past the last output where the reduction is in whole stages
@pytest.mark.parametrize("size", [(30, 300, 66), (62, 96, 64), (66, 128, 64), (64, 300, 66), (128, 200, 70), (255, 4096, 1002), (256, 4096, 1002), (1030, 2000, 1000),
                                  (1024, 640, 1000), (8200, 512, 130), (2050, 300, 64), (4000, 200, 136), (2080, 2560, 2560), (1090, 4096, 4100), (1088, 4096, 4100),
                                  (4110, 4096, 2048)])
@pytest.mark.parametrize("extra", [0, 2, 8])
def test_weight_gradient_of_ragged_reductions_and_tiles(size, extra):
    m, k, n = size
    codes, scales, x = ckpt8(m, k, 3)
    dy = whole_numbers((m, n), 8, 4, torch.bfloat16)              # sums below 1016 m < 2^24
    want, sums = torch.mm(dy.double().t().contiguous(), x), dy.double().sum(0)
    d, ws = strided(dy, extra), workspace(lp.lp_ckpt8_fc_wgrad_workspace_bytes(m, k, n))
    for dtype in (torch.float32, torch.bfloat16, torch.float32):
        dw, db = torch.full((n, k), float("nan"), dtype=dtype, device="cuda"), torch.full((n,), float("nan"), device="cuda")
        lp.lp_ckpt8_fc_wgrad(m, k, n, d, codes, scales, dw, dbias=db, workspace=ws)
        assert torch.equal(dw, want.to(dtype))
        assert torch.equal(db, sums.float())


def mx4_of_blocks(rows, cols, seed, spread):
    """mx4 with a 6 in every block, so that its floats are quantized back to it, and scales of 2^-spread .. 2^spread; values."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes, scales, values = mx4(rows, cols, seed)
    codes[:, ::16] = codes[:, ::16] & 0xF0 | 7
    values[:, ::32] = 6.0
    codes[:, (cols + 31) // 32 * 16:] = 0
    if spread:
        scales += torch.randint(-spread, spread + 1, scales.shape, generator=g, device="cuda").to(torch.uint8)       # (wraps round)
        values *= torch.exp2(scales.double() - 127).repeat_interleave(32, 1)[:, :cols]
    return codes, scales, values


# few rows, tiles of 64, 128 and 256 rows, parts, cut last rounds, reductions of one stage of 256 to 98 and any remainder; sums below
# 36 K in steps of 1/4, with scales 144 K in steps of 1/16: below 2^24 of them
@pytest.mark.parametrize("size", [(1, 4096, 640), (3, 25088, 65), (16, 1500, 300), (16, 25088, 256), (20, 25088, 4096), (40, 25088, 300), (64, 4096, 4096),
                                  (256, 25088, 4096), (600, 25088, 1000), (130, 255, 190), (700, 257, 700), (1030, 4000, 4100), (2048, 4096, 2050),
                                  (4328, 2048, 197), (4100, 4096, 4100), (4090, 4096, 8200), (4000, 8100, 4090)])
def test_forward_of_deep_and_ragged_products(size):
    m, k, n = size
    spread = 1 if k <= 4096 else 0
    x, w = mx4_of_blocks(m, k, 5, spread), mx4_of_blocks(n, k, 6, spread)
    want = torch.mm(x[2], w[2].t().contiguous())
    ws = workspace(lp.lp_mx4_fc_workspace_bytes(m, k, n))
    for dtype in (torch.float32, torch.bfloat16):
        for codes in (True, False):
            y = torch.full((m, n), float("nan"), dtype=dtype, device="cuda")
            if codes:
                lp.lp_mx4_fc_fwd(m, k, n, x[0], w[0], w[1], y, x_scales=x[1], workspace=ws)
            else:
                lp.lp_mx4_fc_fwd(m, k, n, x[2].to(dtype), w[0], w[1], y, workspace=ws)                                # (exact in both types)
            assert torch.equal(y, want.to(dtype))
