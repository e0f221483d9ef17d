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
