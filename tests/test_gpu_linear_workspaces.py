"""difa_linear with workspaces of every useful size, and rows that only copies make fast: whole numbers, which come out exact."""
import pytest
import torch

from layer_util import Plan
from oracle import layer_oracle as O
from paper_2503_22796_amd import binding as B

pytestmark = pytest.mark.gpu

TICKETS = 16384                                  # bytes at a workspace's beginning
GUARD = 4096


def whole(*shape, seed, most=3, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g).to(dtype)


def copies(m, n, k):
    """Bytes that copies of bf16's x and w take, as the header gives them."""
    return TICKETS + 2 * (m + n) * ((k + 63) // 64 * 64)


def product(plan, x, w, sizes):
    """The product with a workspace of each of `sizes`, twice; what lies behind it stays."""
    want = O.linear(x.cpu(), w.cpu()).float().to(x.dtype)
    out = torch.zeros(want.shape, dtype=x.dtype, device="cuda")
    for size in sizes:
        space = torch.full((size + GUARD,), 0xa5, dtype=torch.uint8, device="cuda")
        space[:size] = 0
        for turn in range(2):
            out.fill_(float("nan"))
            B.difa_linear(plan, x, w, out, workspace=space[:size])
            assert torch.equal(out.cpu(), want), (size, turn)
            assert bool((space[size:] == 0xa5).all()), size
            assert bool((space[:min(size, TICKETS)] == 0).all()), size         # ready for the next call


@pytest.mark.parametrize("dtype,rows,k,n", [(torch.bfloat16, 333, 6144, 256), (torch.bfloat16, 100, 4096, 128), (torch.float32, 120, 4096, 136),
                                            (torch.float32, 64, 2051, 100)])
def test_fewer_parts_than_asked_for(dtype, rows, k, n):
    x, w = whole(1, rows, k, seed=1, dtype=dtype).cuda(), whole(n, k, seed=2, dtype=dtype).cuda()
    with Plan(dtype=dtype) as plan:
        full = B.difa_linear_workspace(plan, 1, rows, n, k)
        side = 128 if dtype == torch.bfloat16 else 64
        part = -(-rows // side) * -(-n // side) * side * side * 4
        parts, rest = divmod(full - TICKETS, part)
        assert parts >= 3 and rest == 0
        print(f"{rows} x {k} -> {n} in up to {parts} parts", flush=True)
        product(plan, x, w, [0, 16, TICKETS] + [TICKETS + p * part + d for p in range(1, parts + 1) for d in (-16, 0)] + [full + 16])


def test_room_for_copies_but_not_for_parts():
    rows, k, n = 300, 2999, 500
    x, w = whole(1, rows, k, seed=3).cuda(), whole(n, k, seed=4).cuda()
    with Plan() as plan:
        full, least = B.difa_linear_workspace(plan, 1, rows, n, k), copies(rows, n, k)
        assert least < full
        print(f"{rows} x {k} -> {n} with {least} to {full} bytes", flush=True)
        product(plan, x, w, [0, least - 16, least, (least + full) // 32 * 16, full - 16, full])


@pytest.mark.parametrize("rows", [20, 300, 3000])
@pytest.mark.parametrize("at,step", [(1, 0), (0, 1), (3, 5), (8, 4)])
def test_rows_of_a_wider_tensor(rows, at, step):
    """k is a multiple of eight, but rows do not start at multiples of 16 bytes: x, w, or both."""
    k, n = 1024, 264
    wide_x, wide_w = whole(rows, k + 8 + step, seed=5).cuda(), whole(n, k + 8 + step, seed=6).cuda()
    x, w = wide_x[None, :, at:at + k], wide_w[:, at:at + k]
    with Plan() as plan:
        print(f"{rows} rows {k + 8 + step} apart from {at} on", flush=True)
        least = copies(rows, n, k)
        for a, b in ((x, w), (x.contiguous(), w), (x, w.contiguous())):
            product(plan, a, b, [0, B.difa_linear_workspace(plan, 1, rows, n, k), least - 16, least, 2 * least])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [20, 77])
def test_batch_entries_anywhere(rows, dtype):
    """Entries far apart (text rows of a joint tensor with many image tokens), one x for all, rows of the entries in turn."""
    k, n, behind = 1536, 136, 30_000
    joint = torch.zeros(2, rows + behind, k, dtype=dtype, device="cuda")
    joint[:, :rows] = whole(2, rows, k, seed=7, dtype=dtype).cuda()
    w = whole(n, k, seed=8, dtype=dtype).cuda()
    with Plan(dtype=dtype) as plan:
        print(f"2 x {rows} rows", flush=True)
        for x in (joint[:, :rows], joint[:1, :rows].expand(2, rows, k), joint[:, :rows].transpose(0, 1).contiguous().transpose(0, 1)):
            product(plan, x, w, [0, copies(2 * rows, n, k)])
