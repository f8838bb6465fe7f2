"""Tensors of more than 2^31 values: every offset of the operators around the attention in 64 bits."""
import pytest
import torch

from layer_util import F32, NORM, Plan, check, half_step, turned_size
from oracle import layer_oracle as O
from paper_2503_22796_amd import binding as B

pytestmark = pytest.mark.gpu

ROWS = (0, 1, 12345, 349_524, 349_525, 349_526, 699_050, 699_051, 699_999, 700_000 - 1)     # 2^31 values are 699 050.7 token rows


def _fill(*shape):
    x = torch.empty(*shape, dtype=torch.bfloat16, device="cuda")
    flat, step = x.view(-1), 1 << 28
    for i in range(0, flat.numel(), step):
        part = flat[i:i + step]
        part.copy_(((torch.arange(part.numel(), device="cuda", dtype=torch.int32) * 7919 + i // step) % 4093 - 2046).float() / 512)
    return x


@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
def test_rotate_and_norm(layout):
    H, D, n = 24, 128, 700_000
    rows = torch.tensor(sorted(set(ROWS)))
    pos = torch.arange(n, device="cuda").float()[:, None] % 8191
    with Plan(1, H, D, torch.bfloat16, layout, n) as plan:
        print(f"2.15 G values, {layout}", flush=True)
        table = torch.empty(n, D // 2, 2, device="cuda")
        B.difa_rope_table(plan, pos, (D,), 1e4, table)
        joint = (1, H, n, D) if layout == "bhnd" else (1, n, H, D)
        t = table[rows.cuda()].cpu()

        def picked(x):                                   # [1, H, rows, D]
            return (x[:, :, rows.cuda()] if layout == "bhnd" else x[:, rows.cuda()].transpose(1, 2)).cpu()

        q, out = _fill(*joint), torch.zeros(joint, dtype=torch.bfloat16, device="cuda")
        B.difa_rotate(plan, q, None, out, None, table, n)
        x = picked(q)
        ref = O.rotate(x, t)
        check(picked(out), ref, half_step(torch.bfloat16) * 1.01 * ref.abs() + 3 * F32 * turned_size(x.double(), t.double(), False), "rotated")
        # a stream of 2^31 values and more, q = k, gathered and normed; then its gradients
        s = q if layout == "bnhd" else q.transpose(1, 2)
        k, v = torch.zeros_like(out), torch.zeros_like(out)
        B.difa_qk_norm_rotate(plan, None, (s, s, s, None, None), out, k, v, table=table)
        normed = O.norm(picked(q), None, 1e-6)
        ref = O.rotate(normed, t)
        bound = half_step(torch.bfloat16) * 1.01 * ref.abs() + (NORM + 3 * F32) * turned_size(normed, t.double(), False)
        check(picked(out), ref, bound, "normed")
        check(picked(k), ref, bound, "normed keys")
        assert torch.equal(picked(v), picked(q))
        dq = torch.empty_like(v)
        g = dq if layout == "bnhd" else dq.transpose(1, 2)
        dk = torch.empty_like(v)
        h = dk if layout == "bnhd" else dk.transpose(1, 2)
        B.difa_qk_norm_rotate_backward(plan, None, (s, s, None, None, None), v, v, None, None, (g, h, None, None, None), table=table)
        xs = picked(q).double()
        turned = O.rotate(xs, t, inverse=True)
        r = 1 / torch.sqrt((xs * xs).mean(-1, keepdim=True) + 1e-6)
        nn = xs * r
        want = r * (turned - nn * (turned * nn).mean(-1, keepdim=True))
        size = turned_size(xs, t.double(), False)
        bound = half_step(torch.bfloat16) * 1.01 * want.abs() + 4 * NORM * r * (size + nn.abs() * (size * nn.abs()).mean(-1, keepdim=True))
        check(picked(dq), want, bound, "dq")
        check(picked(dk), want, bound, "dk")


def test_linear():
    """Results, inputs and batch entries behind 2^31 values."""
    m, n, k = 532_481, 4096, 64
    x = _fill(1, m, k)
    w = _fill(n, k)
    rows = torch.tensor([0, 1, 255, 256, 262_143, 524_287, 524_288, m - 1])
    with Plan() as plan:
        out = torch.zeros(1, m, n, dtype=torch.bfloat16, device="cuda")
        B.difa_linear(plan, x, w, out)
        xs = x[:, rows.cuda()].cpu()
        ref, size = O.linear(xs, w.cpu()), O.linear(xs.abs(), w.cpu().abs())
        check(out[:, rows.cuda()], ref, half_step(torch.bfloat16) * 1.01 * ref.abs() + (k + 2) * F32 * size, "many rows")
        # the result as x, in two batch entries far apart: read where it is, and by way of copies
        w2 = _fill(136, n)
        view = out.view(-1).as_strided((2, 300, n), (2_179_000_000, n, 1))
        v = view.cpu()
        ref, size = O.linear(v, w2.cpu()), O.linear(v.abs(), w2.cpu().abs())
        for space in (None, torch.zeros(16 << 20, dtype=torch.uint8, device="cuda")):
            two = torch.zeros(2, 300, 136, dtype=torch.bfloat16, device="cuda")
            B.difa_linear(plan, view, w2, two, workspace=space)
            check(two, ref, half_step(torch.bfloat16) * 1.01 * ref.abs() + (n + 2) * F32 * size, "entries far apart")
