"""CPU-only checks of the microscaled calls: sizes, and the refusal of every bad argument before anything is launched (the
addresses below are never followed)."""
import ctypes

import pytest
import torch

import paper_1711_04713_amd as lp

OK, EINVAL, EUNSUPPORTED, EWORKSPACE = 0, 1, 2, 3
A = 0x10000        # an aligned address
BIG = 1 << 40      # a workspace large enough for anything


def test_sizes():
    assert lp.lp_mx4_bytes(3, 1) == (3 * 128, 3 * 8)
    assert lp.lp_mx4_bytes(3, 256) == (3 * 128, 3 * 8)
    assert lp.lp_mx4_bytes(3, 257) == (3 * 256, 3 * 16)
    assert lp.lp_ckpt8_bytes(5, 33) == (5 * 64, 5 * 2)
    assert lp.lp_mx4_bytes(0, 7) == (0, 0) and lp.lp_ckpt8_bytes(0, 7) == (0, 0)
    for f in (lp.lp_mx4_bytes, lp.lp_ckpt8_bytes):
        for rows, cols in ((1 << 26, 256), (1 << 31, 1), (1, 1 << 31), (1 << 62, 1 << 62)):   # 2^34 padded elements, or sizes of 32 bits
            with pytest.raises(lp.LpError) as e:
                f(rows, cols)
            assert e.value.status == EUNSUPPORTED
    f(1 << 25, 256)


def test_workspaces():
    sizes = (lp.lp_mx4_fc_workspace_bytes, lp.lp_mx4_fc_dgrad_workspace_bytes, lp.lp_ckpt8_fc_wgrad_workspace_bytes)
    for f in sizes:
        for bad in ((-1, 5, 5), (5, 0, 5), (5, 5, 0), (5, -1, 5), (5, 5, -7)):
            with pytest.raises(lp.LpError) as e:
                f(*bad)
            assert e.value.status == EINVAL
        for big in ((1 << 24) + 1, 5, 5), (5, (1 << 24) + 1, 5), (5, 5, (1 << 24) + 1):
            with pytest.raises(lp.LpError) as e:
                f(*big)
            assert e.value.status == EUNSUPPORTED
        assert f(0, 5, 5) >= 0 and f(1, 1, 1) >= 0


def quantize(x=A, xt=1, rows=4, cols=40, ld=40, codes=A, scales=A, r=1):
    return lp.load().lp_mx4_quantize(x, xt, rows, cols, ld, codes, scales, r, 0, None, None, None)


def dequantize(codes=A, scales=A, rows=4, cols=40, y=A, yt=1, ld=40):
    return lp.load().lp_mx4_dequantize(codes, scales, rows, cols, y, yt, ld, None)


def save(x=A, xt=1, rows=4, cols=40, ld=40, codes=A, scales=A, r=1, act=1, y=A + 4096, ldy=40):
    return lp.load().lp_ckpt8_save(x, xt, rows, cols, ld, codes, scales, r, 0, act, y, ldy, None)


def restore(codes=A, scales=A, rows=4, cols=40, y=A, yt=1, ld=40):
    return lp.load().lp_ckpt8_load(codes, scales, rows, cols, y, yt, ld, None)


def act_bwd(codes=A, scales=A, rows=4, cols=40, dy=A, t=1, lddy=40, act=2, dx=A + 4096, lddx=40):
    return lp.load().lp_ckpt8_act_bwd(codes, scales, rows, cols, dy, t, lddy, act, dx, lddx, None)


def fwd(M=4, K=40, N=24, x=A, xt=1, ldx=40, xs=None, wc=A, ws=A, bias=A, y=A, yt=1, ldy=24, act=0, work=A, size=BIG):
    return lp.load().lp_mx4_fc_fwd(M, K, N, x, xt, ldx, xs, wc, ws, bias, y, yt, ldy, act, work, size, None)


def dgrad(M=4, K=40, N=24, dy=A, lddy=24, wc=A, ws=A, dx=A, dxt=1, lddx=40, work=A, size=BIG):
    return lp.load().lp_mx4_fc_dgrad(M, K, N, dy, lddy, wc, ws, dx, dxt, lddx, work, size, None)


def wgrad(M=4, K=40, N=24, dy=A, lddy=24, xc=A, xs=A, dw=A, dwt=0, lddw=40, db=A, work=A, size=BIG):
    return lp.load().lp_ckpt8_fc_wgrad(M, K, N, dy, lddy, xc, xs, dw, dwt, lddw, db, 0, work, size, None)


INVALID = [
    (quantize, [dict(xt=3), dict(xt=-1), dict(r=3), dict(r=-1), dict(x=None), dict(codes=None), dict(scales=None), dict(ld=39), dict(codes=A + 8),
                dict(scales=A + 4), dict(x=A + 1), dict(xt=0, x=A + 2)]),
    (dequantize, [dict(yt=3), dict(y=None), dict(codes=None), dict(scales=None), dict(ld=39), dict(codes=A + 8), dict(scales=A + 1), dict(y=A + 1)]),
    (save, [dict(xt=3), dict(r=3), dict(act=4), dict(act=-1), dict(x=None), dict(codes=None), dict(scales=None), dict(ld=39), dict(ldy=39),
            dict(codes=A + 8), dict(x=A + 1), dict(y=A + 1), dict(y=A, ldy=48)]),
    (restore, [dict(yt=3), dict(y=None), dict(codes=None), dict(scales=None), dict(ld=39), dict(codes=A + 4), dict(yt=0, y=A + 2)]),
    (act_bwd, [dict(t=3), dict(act=4), dict(dy=None), dict(dx=None), dict(codes=None), dict(scales=None), dict(lddy=39), dict(lddx=39),
               dict(dx=A, lddx=41), dict(codes=A + 8), dict(dy=A + 1)]),
    (fwd, [dict(M=-1), dict(K=0), dict(N=0), dict(xt=3), dict(yt=-1), dict(act=4), dict(x=None), dict(wc=None), dict(ws=None), dict(y=None), dict(ldx=39),
           dict(ldy=23), dict(wc=A + 8), dict(ws=A + 4), dict(x=A + 1), dict(xs=A + 4), dict(xs=A, x=A + 8), dict(bias=A + 2), dict(yt=0, y=A + 2)]),
    (dgrad, [dict(M=-1), dict(K=0), dict(N=0), dict(dxt=3), dict(dy=None), dict(wc=None), dict(ws=None), dict(dx=None), dict(lddy=23), dict(lddx=39),
             dict(wc=A + 8), dict(ws=A + 4), dict(dy=A + 1), dict(dxt=0, dx=A + 2)]),
    (wgrad, [dict(M=-1), dict(K=0), dict(N=0), dict(dwt=3), dict(dy=None), dict(xc=None), dict(xs=None), dict(dw=None), dict(lddy=23), dict(lddw=39),
             dict(xc=A + 8), dict(dy=A + 1), dict(dw=A + 2), dict(db=A + 2)]),
]


@pytest.mark.parametrize("call,bad", [(c, b) for c, bs in INVALID for b in bs])
def test_invalid_arguments(call, bad):
    assert call(**bad) == EINVAL


def test_unsupported_calls():
    for call in (quantize, dequantize, save, restore):
        assert call(rows=1 << 26, cols=256, ld=256, **({"ldy": 256} if call is save else {})) == EUNSUPPORTED
    assert act_bwd(rows=1 << 31, cols=1) == EUNSUPPORTED
    assert dgrad(dxt=2) == EUNSUPPORTED and wgrad(dwt=2) == EUNSUPPORTED
    for call in (fwd, dgrad, wgrad):
        for big in (dict(M=(1 << 24) + 1), dict(K=(1 << 24) + 1), dict(N=(1 << 24) + 1)):
            assert call(**big) == EUNSUPPORTED


def test_workspaces_that_are_missing_or_small():
    for call, size, dims in ((fwd, lp.lp_mx4_fc_workspace_bytes, [(300, 4096, 256), (100, 25088, 64)]), (dgrad, lp.lp_mx4_fc_dgrad_workspace_bytes, [(4, 64, 25088)]),
                             (wgrad, lp.lp_ckpt8_fc_wgrad_workspace_bytes, [(25088, 64, 40)])):
        for m, k, n in dims:
            need = size(m, k, n)
            if need == 0:
                continue
            lds = dict(ldx=k, ldy=n) if call is fwd else dict(lddy=n, lddx=k) if call is dgrad else dict(lddy=n, lddw=k)
            assert call(M=m, K=k, N=n, work=None, size=0, **lds) == EWORKSPACE
            assert call(M=m, K=k, N=n, work=A, size=need - 1, **lds) == EWORKSPACE
            assert call(M=m, K=k, N=n, work=A + 8, size=need, **lds) == EINVAL


def test_calls_without_rows_do_nothing():
    nothing = dict(rows=0)
    for call in (quantize, dequantize, save, restore, act_bwd):
        assert call(**nothing) == OK and call(cols=0) == OK
    assert fwd(M=0, x=None, y=None, work=None, size=0) == OK and dgrad(M=0, dy=None, dx=None, work=None, size=0) == OK


def test_binding_refuses_tensors_that_do_not_fit():
    x, c, s = torch.zeros((4, 40)), torch.zeros((4, 128), dtype=torch.uint8), torch.zeros((4, 8), dtype=torch.uint8)
    wc, ws = torch.zeros((24, 128), dtype=torch.uint8), torch.zeros((24, 8), dtype=torch.uint8)
    dy, y = torch.zeros((4, 24), dtype=torch.bfloat16), torch.zeros((4, 24))
    calls = [
        lambda: lp.lp_mx4_quantize(x, c, s),                                   # not on the GPU
        lambda: lp.lp_mx4_quantize(x.t(), c, s),                               # column stride
        lambda: lp.lp_mx4_quantize(x, c[:3], s),
        lambda: lp.lp_mx4_quantize(x, c, s[:, :4]),
        lambda: lp.lp_mx4_dequantize(c, s, x[:, :7].t()),
        lambda: lp.lp_ckpt8_save(x, torch.zeros((4, 64), dtype=torch.int8), torch.zeros((4, 2), dtype=torch.uint8), y=x.half()),
        lambda: lp.lp_ckpt8_act_bwd(torch.zeros((4, 64), dtype=torch.int8), torch.zeros((4, 2), dtype=torch.uint8), x, x.half(), lp.LP_ACT_RELU),
        lambda: lp.lp_mx4_fc_fwd(4, 40, 24, x, wc[:23], ws, y),
        lambda: lp.lp_mx4_fc_fwd(4, 41, 24, x, wc, ws, y),
        lambda: lp.lp_mx4_fc_fwd(4, 40, 24, x, wc, ws, y, bias=torch.zeros(24).half()),
        lambda: lp.lp_mx4_fc_fwd(4, 40, 24, c, wc, ws, y, x_scales=s[:3]),
        lambda: lp.lp_mx4_fc_dgrad(4, 40, 24, y, wc, ws, x),                   # dy is not bfloat16
        lambda: lp.lp_mx4_fc_dgrad(4, 40, 24, dy, wc, ws, x[:3]),
        lambda: lp.lp_ckpt8_fc_wgrad(4, 40, 24, dy, c, s, torch.zeros((24, 40))),
    ]
    for k, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail("call %d was taken" % k)
    assert ctypes.sizeof(ctypes.c_size_t) == 8
