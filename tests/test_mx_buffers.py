"""CPU-only checks of the memory that the microscaled calls write beside their results: counters and workspaces."""
import pytest
import torch

import paper_1711_04713_amd as lp
from paper_1711_04713_amd import binding
from test_mx_host import A, EINVAL


def test_counters_that_begin_inside_a_word():
    """An addition of 64 bits there would touch what lies behind the counter (the addresses are never followed)."""
    for zeros, sats in ((A + 4, None), (None, A + 4), (A + 1, A), (A, A + 2)):
        assert lp.load().lp_mx4_quantize(A, 1, 4, 40, 40, A, A, 1, 0, zeros, sats, None) == EINVAL


class Reached(Exception):
    pass


@pytest.fixture
def on_the_cpu(monkeypatch):
    """The binding's own checks for tensors of the CPU: where all are passed, Reached instead of the call."""
    def reached():
        raise Reached

    monkeypatch.setattr(binding, "_device", lambda: torch.empty(0).get_device())
    monkeypatch.setattr(binding, "load", reached)
    binding._dtypes.update({torch.float32: lp.LP_F32, torch.bfloat16: lp.LP_BF16, torch.float16: lp.LP_F16})


def quantize(**counters):
    lp.lp_mx4_quantize(torch.zeros((4, 40)), torch.zeros((4, 128), dtype=torch.uint8), torch.zeros((4, 8), dtype=torch.uint8), **counters)


def test_counters_are_integers_of_64_bits(on_the_cpu):
    for name in ("zero_count", "sat_count"):
        for good in (None, torch.zeros(1, dtype=torch.int64), torch.zeros((), dtype=torch.int64), torch.zeros(5, dtype=torch.int64)[3:], torch.zeros(1, dtype=torch.uint64)):
            with pytest.raises(Reached):
                quantize(**{name: good})
        for bad in (torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(8, dtype=torch.uint8), torch.zeros(1, dtype=torch.double),
                    torch.zeros(0, dtype=torch.int64)):
            with pytest.raises(ValueError):
                quantize(**{name: bad})


def test_workspaces_are_dense(on_the_cpu):
    x, y, dy = torch.zeros((4, 40)), torch.zeros((4, 24)), torch.zeros((4, 24), dtype=torch.bfloat16)
    w = torch.zeros((24, 128), dtype=torch.uint8), torch.zeros((24, 8), dtype=torch.uint8)
    kept = torch.zeros((4, 64), dtype=torch.int8), torch.zeros((4, 2), dtype=torch.uint8)
    calls = (lambda ws: lp.lp_mx4_fc_fwd(4, 40, 24, x, *w, y, workspace=ws), lambda ws: lp.lp_mx4_fc_dgrad(4, 40, 24, dy, *w, x, workspace=ws),
             lambda ws: lp.lp_ckpt8_fc_wgrad(4, 40, 24, dy, *kept, torch.zeros((24, 40)), workspace=ws))
    for call in calls:
        for good in (None, torch.zeros(4096, dtype=torch.uint8), torch.zeros((4, 8)), torch.zeros(4096)[16:]):
            with pytest.raises(Reached):
                call(good)
        for bad in (torch.zeros((4096, 2))[:, 0], torch.zeros(1, dtype=torch.uint8).expand(4096), torch.zeros((8, 8)).t()[1:]):
            with pytest.raises(ValueError):
                call(bad)


EUNSUPPORTED = 2
LONG = (1 << 32) + 4      # rows that an int of 32 bits holds as 4


def test_sizes_that_an_int_does_not_hold_are_refused():
    for f in (lp.lp_mx4_fc_workspace_bytes, lp.lp_mx4_fc_dgrad_workspace_bytes, lp.lp_ckpt8_fc_wgrad_workspace_bytes):
        for dims in ((LONG, 40, 24), (4, LONG, 24), (4, 40, LONG), (1 << 64, 40, 24)):
            with pytest.raises(lp.LpError) as e:
                f(*dims)
            assert e.value.status == EUNSUPPORTED
        for dims in ((-LONG, 40, 24), (-(1 << 33) + 4, 40, 24), (4, -(1 << 32) + 40, 24)):
            with pytest.raises(lp.LpError) as e:
                f(*dims)
            assert e.value.status == EINVAL
    for f in (lp.lp_mx4_bytes, lp.lp_ckpt8_bytes):
        for dims in (((1 << 64) + 4, 40), (4, (1 << 64) + 40), (-(1 << 64) + 4, 40), (-4, 40)):
            with pytest.raises(lp.LpError) as e:
                f(*dims)
            assert e.value.status == EUNSUPPORTED


def test_products_of_more_rows_than_an_int_holds_are_refused(monkeypatch, on_the_cpu):
    """Tensors without memory (the calls return before they would follow an address)."""
    seen = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: seen.append((name, args)) or 0

    monkeypatch.setattr(binding, "load", Library)
    monkeypatch.setattr(binding, "_stream", lambda: None)

    def meta(rows, cols, dtype=torch.bfloat16):
        return torch.empty((rows, cols), dtype=dtype, device="meta")

    monkeypatch.setattr(binding, "_device", lambda: meta(1, 1).get_device())
    w = meta(1, 128, torch.uint8), meta(1, 8, torch.uint8)
    lp.lp_mx4_fc_fwd(LONG, 1, 1, meta(LONG, 1), *w, meta(LONG, 1))
    lp.lp_mx4_fc_dgrad(LONG, 1, 1, meta(LONG, 1), *w, meta(LONG, 1))
    lp.lp_ckpt8_fc_wgrad(LONG, 1, 1, meta(LONG, 1), meta(LONG, 32, torch.int8), meta(LONG, 1, torch.uint8), meta(1, 1))
    assert [name for name, _ in seen] == ["lp_mx4_fc_fwd", "lp_mx4_fc_dgrad", "lp_ckpt8_fc_wgrad"]
    assert all(1 << 24 < args[0] < 1 << 31 and args[1:3] == (1, 1) for _, args in seen)        # above the calls' limit, and held by an int
