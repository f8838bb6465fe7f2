"""difa_rope_table and difa_rotate on the GPU against the 64-bit forms."""
import pytest
import torch

from layer_util import F32, Plan, check, half_step, randn, seen, stored, turned_size
from oracle import layer_oracle as O
from paper_2503_22796_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,D,dims,theta,far", [
    (1, 64, (64,), 1e4, 0), (7, 64, (8, 28, 28), 1e4, 0), (333, 128, (16, 56, 56), 1e4, 0), (5000, 128, (128,), 5e5, 0),
    (65, 128, (2, 2, 2, 2), 256.0, 0),                 # most pairs are not turned
    (1000, 64, (32, 32), 1e4, 16_000_000),             # far positions: integers near 2^24
    (40, 128, (64, 64), 1.5, -3_000_000), (40_001, 64, (20, 20, 20), 1e4, 0)])
def test_table(rows, D, dims, theta, far):
    g = torch.Generator().manual_seed(rows)
    pos = torch.randint(-50, 20_000, (rows, len(dims)), generator=g).float() + far
    pos[rows // 2] += 0.25
    pos[0] = 0
    got = torch.full((rows, D // 2, 2), float("nan"), device="cuda")
    with Plan(head_dim=D) as plan:
        print(f"table {rows} {D} {dims}", flush=True)
        B.difa_rope_table(plan, pos.cuda(), dims, theta, got)
        torch.cuda.synchronize()
    ref = O.rope_table(pos, dims, theta, D)
    # half a step of the value, and the angle's own error in 64 bits: both sides form it with a frequency that is off by some
    # 2^-50 relative (a power with an exponent of up to 25 in base 2), times an angle below 2^24 + 2^15
    check(got, ref, F32 * ref.abs() + 2.0 ** -50 * 2.0 * pos.abs().max().double() + 1e-15, "table")
    assert torch.equal(got[0].cpu(), torch.tensor([1.0, 0.0]).expand(D // 2, 2))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("batch,heads,D,tokens,layout,halves,inverse,per_batch,queries_only", [
    (1, 1, 64, 1, "bhnd", False, False, False, False), (2, 3, 64, 17, "bnhd", True, False, True, False),
    (1, 5, 128, 130, "bhnd", True, True, False, False), (2, 24, 128, 77, "bnhd", False, True, False, True),
    (3, 7, 64, 333, "bhnd", False, False, True, False), (1, 2, 128, 5000, "bhnd", False, False, False, False)])
def test_rotate(dtype, batch, heads, D, tokens, layout, halves, inverse, per_batch, queries_only):
    q, k = (randn(batch, heads, tokens, D, seed=i, dtype=dtype) for i in (1, 2))
    pos = torch.arange((batch if per_batch else 1) * tokens * 2).reshape(-1, 2).float() % 517
    table = O.rope_table(pos, (D // 4, D // 2), 1e4, D).float()
    table = table.reshape(batch, tokens, D // 2, 2) if per_batch else table
    flags = (B.DIFA_ROPE_HALVES if halves else 0) | (B.DIFA_ROPE_INVERSE if inverse else 0)
    with Plan(batch, heads, D, dtype, layout, tokens + 3) as plan:
        print(f"rotate {batch} {heads} {D} {tokens}", flush=True)
        ins = [stored(x, layout) for x in (q, k)]
        outs = [torch.full_like(x, float("nan")) for x in ins]
        t = table.cuda()
        if queries_only:
            B.difa_rotate(plan, ins[0], None, outs[0], None, t, tokens, flags)
            outs, ins, xs = outs[:1], ins[:1], (q,)
        else:
            B.difa_rotate(plan, ins[0], ins[1], outs[0], outs[1], t, tokens, flags)
            xs = (q, k)
        for x, got in zip(xs, outs):
            ref = O.rotate(x, table, halves, inverse)
            # two products and a sum in fp32, one rounding to the type
            check(seen(got, layout), ref, half_step(dtype) * ref.abs() * 1.01 + 3 * F32 * turned_size(x.double(), table.double(), halves), "rotated")
        kept = [o.clone() for o in outs]
        B.difa_rotate(plan, ins[0], None, ins[0], None, t, tokens, flags)         # in place
        assert torch.equal(ins[0], kept[0])


def test_rotate_leaves_what_lies_behind_and_takes_another_stream():
    D, tokens = 64, 19
    buf = torch.full((2, 2, tokens + 5, D), 3.0, dtype=torch.bfloat16, device="cuda")
    x = randn(1, 2, tokens, D, seed=5).cuda()
    out = buf.view(-1)[:x.numel()].view_as(x)
    table = O.rope_table(torch.arange(tokens).float()[:, None], (D,), 1e4, D).float().cuda()
    side = torch.cuda.Stream()
    with Plan(1, 2, D, max_tokens=tokens) as plan:
        B.difa_rotate(plan, x, None, out, None, table, tokens, stream=side)
        side.synchronize()
        assert bool((buf.view(-1)[x.numel():] == 3.0).all())
        want = torch.empty_like(x)
        B.difa_rotate(plan, x, None, want, None, table, tokens)
        assert torch.equal(out, want)


def test_infinities_and_nan_stay_in_their_pairs():
    D = 64
    x = randn(1, 1, 4, D, seed=6)
    x[0, 0, 1, 10], x[0, 0, 2, 33] = float("inf"), float("nan")
    table = O.rope_table(torch.arange(1.0, 5.0)[:, None], (D,), 1e4, D).float()
    out = torch.empty(1, 1, 4, D, dtype=torch.bfloat16, device="cuda")
    with Plan(1, 1, D, max_tokens=4) as plan:
        B.difa_rotate(plan, x.cuda(), None, out, None, table.cuda(), 4)
        got = out.cpu()[0, 0]
    bad = ~torch.isfinite(got)
    assert bad[1, 10:12].all() and bad[2, 32:34].all() and int(bad.sum()) == 4
