"""Sizes whose grids have 2^32 work-items and more, which no single launch takes."""
import pytest
import torch

from layer_util import Plan, PlanWithoutDevice
from paper_2503_22796_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_linear_of_one_feature_and_2_to_30_rows(dtype):
    """Tiles of 64 rows: 2^24 workgroups of 256 threads, and one more."""
    m = (1 << 30) + 33
    print(f"linear {m} x 1 -> 1, {dtype}", flush=True)
    x = (torch.arange(m, device="cuda", dtype=torch.int32) % 127 - 63).to(dtype).view(m, 1)
    out = torch.zeros(m, 1, dtype=dtype, device="cuda")
    with Plan(dtype=dtype) as plan:
        B.difa_linear(plan, x, torch.full((1, 1), 2.0, dtype=dtype, device="cuda"), out)
        torch.cuda.synchronize()
    x *= 2                                       # whole numbers: exact in both types
    assert torch.equal(out, x)


def test_linear_by_way_of_copies_of_2_to_26_rows():
    """Four rows are copied by a workgroup of 256 threads: 2^24 of them and some more."""
    m, k, n = (1 << 26) + 77, 9, 8
    print(f"linear {m} x {k} -> {n} with copies", flush=True)
    x = (torch.arange(m * k, device="cuda", dtype=torch.int32) % 11 - 5).to(torch.bfloat16).view(m, k)
    w = (torch.arange(n * k, device="cuda", dtype=torch.int32) % 7 - 3).to(torch.bfloat16).view(n, k)
    out = torch.zeros(m, n, dtype=torch.bfloat16, device="cuda")
    with Plan() as plan:
        size = B.difa_linear_workspace(plan, 1, m, n, k)
        assert size > m * k * 2                  # there is room for the copies
        B.difa_linear(plan, x, w, out, workspace=torch.zeros(size, dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
    for i in range(0, m, 1 << 23):               # sums of whole numbers below 2^8: exact
        want = sum(x[i:i + (1 << 23), j:j + 1].float() * w[:, j].float() for j in range(k))
        assert torch.equal(out[i:i + (1 << 23)].float(), want), i


def test_linear_of_a_row_and_2_to_26_features():
    """The kernel for few rows takes 16 features a workgroup: more of them than go in one launch."""
    n, k = (1 << 26) + 40, 8
    print(f"linear 1 x {k} -> {n}", flush=True)
    w = (torch.arange(n * k, device="cuda", dtype=torch.int32) % 13 - 6).to(torch.bfloat16).view(n, k)
    x = torch.arange(-3, 5, device="cuda").to(torch.bfloat16).view(1, k)
    out = torch.zeros(1, n, dtype=torch.bfloat16, device="cuda")
    with Plan() as plan:
        B.difa_linear(plan, x, w, out)
        torch.cuda.synchronize()
    assert torch.equal(out[0].float(), (w.float() * x.float()).sum(1))        # whole numbers below 2^8


def test_rotate_and_norm_of_2_to_24_batch_entries():
    """A workgroup of 256 threads for every entry's one token."""
    batch, D = (1 << 24) + 5, 64
    print(f"rotate and norm, {batch} entries", flush=True)
    x = (torch.arange(batch * D, device="cuda", dtype=torch.int64) % 251).to(torch.int16).sub_(125).to(torch.bfloat16).view(batch, 1, 1, D)
    table = torch.tensor([[0.0, 1.0], [1.0, 0.0]], device="cuda").repeat(D // 4, 1).view(1, D // 2, 2).contiguous()
    out = torch.zeros_like(x)
    # (a plan object of this size would set aside gigabytes for the attention's schedules; these calls need its description only)
    with PlanWithoutDevice(batch, 1, D) as plan:
        B.difa_rotate(plan, x, None, out, None, table, 1)
        torch.cuda.synchronize()
        pairs, got = x.view(-1, D // 4, 4), out.view(-1, D // 4, 4)
        assert torch.equal(got[:, :, 0], -pairs[:, :, 1]) and torch.equal(got[:, :, 1], pairs[:, :, 0]) and torch.equal(got[:, :, 2:], pairs[:, :, 2:])
        ones = x.sign_().masked_fill_(x == 0, 1.0)
        out.zero_()
        k = torch.zeros_like(out)
        # rows of one size: the root mean square is 1 + 5e-7, which rounds away
        B.difa_qk_norm_rotate(plan, None, (ones, ones, None, None, None), out, k, None, eps=1e-6)
        torch.cuda.synchronize()
        assert torch.equal(out, ones) and torch.equal(k, ones)
