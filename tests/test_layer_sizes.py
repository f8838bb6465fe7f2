"""Sizes and numbers that do not fit the C structures are refused, not wrapped around."""
import pytest
import torch

from layer_util import PlanWithoutDevice
from paper_2503_22796_amd import binding as B

BIG = 2 ** 32


def refused(call):
    with pytest.raises(B.DifaError) as e:
        call()
    assert e.value.status == B.DIFA_ERR_INVALID_ARG


@pytest.mark.parametrize("at", range(4))
def test_workspace_of_sizes_beyond_32_bits(at):
    sizes = [1, 40, 64, 4096]
    with PlanWithoutDevice() as plan:
        assert B.difa_linear_workspace(plan, *sizes) > 0
        for more in (BIG, -BIG, 2 ** 31):
            wrong = list(sizes)
            wrong[at] += more
            refused(lambda: B.difa_linear_workspace(plan, *wrong))


def test_norm_workspace_of_sizes_beyond_32_bits():
    with PlanWithoutDevice(max_tokens=10) as plan:
        assert B.difa_qk_norm_rotate_workspace(plan, 4, 5) > 0
        for n in ((BIG + 4, 5), (4, BIG + 5), (BIG - 4, 5)):
            refused(lambda: B.difa_qk_norm_rotate_workspace(plan, *n))


def test_linear_of_more_rows_than_31_bits(monkeypatch):
    with PlanWithoutDevice(dtype=torch.float32) as plan:
        monkeypatch.setattr(B, "_on_device", lambda *_: None)
        x, out = torch.zeros(1, 4).expand(2 ** 31 + 7, 4), torch.zeros(1, 8).expand(2 ** 31 + 7, 8)
        refused(lambda: B.difa_linear(plan, x, torch.zeros(8, 4), out, stream=0))
        refused(lambda: B.difa_linear(plan, x[:3], torch.zeros(8, 4), torch.zeros(3, 8), activation=2 ** 31, stream=0))


@pytest.mark.parametrize("dims,theta", [((2 ** 31,), 1e4), ((2 ** 32 + 64,), 1e4), ((64,), 1e39)])
def test_table_of_numbers_that_do_not_fit(dims, theta, monkeypatch):
    with PlanWithoutDevice(head_dim=64) as plan:
        monkeypatch.setattr(torch.Tensor, "get_device", lambda _: 0)          # past the check of devices, with host tensors
        refused(lambda: B.difa_rope_table(plan, torch.zeros(4, 1), dims, theta, torch.zeros(4, 32, 2), stream=0))


def test_flags_beyond_32_bits(monkeypatch):
    with PlanWithoutDevice(max_tokens=4) as plan:
        monkeypatch.setattr(torch.Tensor, "get_device", lambda _: 0)
        q, x = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16), torch.zeros(1, 4, 1, 64, dtype=torch.bfloat16)
        s = (x, x, None, None, None)
        for flags in (BIG, -1):
            refused(lambda: B.difa_rotate(plan, q, None, q, None, torch.zeros(4, 32, 2), 4, flags, stream=0))
            refused(lambda: B.difa_qk_norm_rotate(plan, None, s, q, q.clone(), None, flags=flags, stream=0))
            refused(lambda: B.difa_qk_norm_rotate_backward(plan, None, s, q, q, None, None, s, flags=flags, stream=0))
