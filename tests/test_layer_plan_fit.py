"""Tensors that fit each other but not the plan object are refused before their addresses are used: the plan gives the element
size and the extents that the kernels go by."""
import ctypes

import pytest
import torch

from layer_util import PlanWithoutDevice
from paper_2503_22796_amd import binding as B

z = torch.zeros
BF16, F32 = torch.bfloat16, torch.float32
DEVICE = "the plan's device"                      # what a call is refused for whose tensors fit in everything else


def refused(call, why):
    with pytest.raises(B.DifaError, match=why) as e:
        call()
    assert e.value.status == B.DIFA_ERR_INVALID_ARG


def test_describe():
    with PlanWithoutDevice(3, 5, 128, F32, "bnhd", 77, True) as plan:
        d = B.difa_plan_describe(plan)
        assert (d.batch, d.heads, d.head_dim, d.dtype, d.layout, d.max_tokens, d.flags) == (3, 5, 128, B.DIFA_DTYPE_F32, B.DIFA_LAYOUT_BNHD, 77, B.DIFA_FLAG_IMAGE_FIRST)
        assert B.lib.difa_plan_describe(plan, None) == B.DIFA_ERR_INVALID_ARG
    assert B.lib.difa_plan_describe(None, ctypes.byref(d)) == B.DIFA_ERR_INVALID_ARG
    with pytest.raises(B.DifaError):
        B.difa_linear(None, z(2, 8), z(4, 8), z(2, 4), stream=0)


def test_a_handle_that_is_used_again_is_looked_at_again():
    """The object behind a handle that did not come from difa_plan_create may be another one at the next call."""
    with PlanWithoutDevice(dtype=F32) as a, PlanWithoutDevice(dtype=BF16) as b:
        args = z(2, 8), z(4, 8), z(2, 4)
        refused(lambda: B.difa_linear(a, *args, stream=0), DEVICE)
        a.value, kept = b.value, a.value
        refused(lambda: B.difa_linear(a, *args, stream=0), "element type")
        a.value = kept


@pytest.mark.parametrize("head_dim,width", [(128, 32), (64, 64), (64, 31)])
def test_table(head_dim, width):
    with PlanWithoutDevice(head_dim=head_dim) as plan:
        pos = z(4, 1)
        refused(lambda: B.difa_rope_table(plan, pos, (8,), 1e4, z(4, head_dim // 2, 2), stream=0), DEVICE)
        refused(lambda: B.difa_rope_table(plan, pos, (8,), 1e4, z(4, width, 2), stream=0), "head_dim / 2")


WRONG = [(1, 3, 10, 64, BF16), (2, 2, 10, 64, BF16), (2, 4, 10, 64, BF16), (2, 3, 10, 128, BF16), (2, 3, 10, 64, F32), (4, 3, 10, 64, BF16)]


def joint(layout, B_, H, n, D, dtype):
    return z(B_, H, n, D, dtype=dtype) if layout == "bhnd" else z(B_, n, H, D, dtype=dtype)


@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
def test_rotate(layout):
    with PlanWithoutDevice(2, 3, 64, BF16, layout, 10) as plan:
        def call(B_, H, n, D, dtype, layout=layout):
            q = joint(layout, B_, H, n, D, dtype)
            return lambda: B.difa_rotate(plan, q, q.clone(), q, q.clone(), z(n, D // 2, 2), n, stream=0)

        refused(call(2, 3, 10, 64, BF16), DEVICE)
        for w in WRONG:
            refused(call(*w), "joint tensors|table")
        refused(call(2, 3, 10, 64, BF16, "bnhd" if layout == "bhnd" else "bhnd"), "joint tensors")


@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
def test_norm_and_its_gradients(layout):
    with PlanWithoutDevice(2, 3, 64, BF16, layout, 10) as plan:
        def call(B_, H, n, D, dtype, layout=layout, grads=False, rows=None):
            q = joint(layout, B_, H, n, D, dtype)
            x = z(B_, n, 3, H, D, dtype=dtype)
            s = (x[:, :, 0], x[:, :, 1], x[:, :, 2], None, None)
            t = z(rows, D // 2, 2) if rows else None
            if grads:
                return lambda: B.difa_qk_norm_rotate_backward(plan, None, s, q, q, q, None, s, table=t, stream=0)
            return lambda: B.difa_qk_norm_rotate(plan, None, s, q, q, q, table=t, stream=0)

        for grads in (False, True):
            refused(call(2, 3, 10, 64, BF16, grads=grads), DEVICE)
            refused(call(2, 3, 10, 64, BF16, grads=grads, rows=10), DEVICE)
            refused(call(2, 3, 10, 64, BF16, grads=grads, rows=9), "table")
            for w in WRONG:
                refused(call(*w, grads=grads), "plan's")
            refused(call(2, 3, 10, 64, BF16, "bnhd" if layout == "bhnd" else "bhnd", grads=grads), "joint tensors")


def test_gradients_of_other_tokens_or_types():
    with PlanWithoutDevice(2, 3, 64, BF16, "bhnd", 10) as plan:
        q, x = z(2, 3, 10, 64, dtype=BF16), z(2, 10, 3, 3, 64, dtype=BF16)
        s = (x[:, :, 0], x[:, :, 1], x[:, :, 2], None, None)

        def call(g):
            return lambda: B.difa_qk_norm_rotate_backward(plan, None, s, q, q, q, None, g, stream=0)

        refused(call(s), DEVICE)
        refused(call(tuple(t if t is None else t[:, :9] for t in s)), "tokens")
        refused(call(tuple(t if t is None else t[:1] for t in s)), "plan's")
        refused(call(tuple(t if t is None else t.float() for t in s)), "plan's")


@pytest.mark.parametrize("plan_type,tensors", [(F32, BF16), (BF16, F32)])
def test_linear(plan_type, tensors):
    with PlanWithoutDevice(dtype=plan_type) as plan:
        def call(t, **more):
            more = {k: v.to(t) for k, v in more.items()}
            return lambda: B.difa_linear(plan, z(2, 5, 8, dtype=t), z(16, 8, dtype=t), z(2, 5, 16, dtype=t), stream=0, **more)

        refused(call(plan_type), DEVICE)
        refused(call(plan_type, bias=z(16), gate=z(2, 16), residual=z(2, 5, 16)), DEVICE)
        refused(call(tensors), "plan's element type")


def test_workspaces_with_gaps():
    """A view whose bytes reach further than their number."""
    with PlanWithoutDevice(dtype=F32) as plan:
        space = z(1 << 16, dtype=torch.uint8)
        call = lambda ws: lambda: B.difa_linear(plan, z(2, 8), z(4, 8), z(2, 4), workspace=ws, stream=0)  # noqa: E731
        refused(call(space), DEVICE)
        refused(call(space[::2]), "contiguous")
        refused(call(space[:1].expand(1 << 16)), "contiguous")
    with PlanWithoutDevice(max_tokens=4) as plan:
        q, x = z(1, 1, 4, 64, dtype=BF16), z(1, 4, 1, 64, dtype=BF16)
        s = (x, x, x, None, None)
        refused(lambda: B.difa_qk_norm_rotate_backward(plan, None, s, q, q, q, None, s, workspace=space[::2], stream=0), "contiguous")


@pytest.mark.gpu
def test_one_tensor_on_the_host():
    from layer_util import Plan
    with Plan(1, 2, 64, F32, "bhnd", 4) as plan:
        c = lambda *s: z(*s, device="cuda")  # noqa: E731
        x, w, out, bias, gate, res, ws = c(4, 8), c(16, 8), c(4, 16), c(16), c(16), c(4, 16), c(64).view(torch.uint8)
        ops = dict(bias=bias, gate=gate, residual=res, workspace=ws)
        B.difa_linear(plan, x, w, out, **ops)
        for name in ops:
            refused(lambda: B.difa_linear(plan, x, w, out, **{**ops, name: ops[name].cpu()}), DEVICE)
        for args in ((x.cpu(), w, out), (x, w.cpu(), out), (x, w, out.cpu())):
            refused(lambda: B.difa_linear(plan, *args, stream=torch.cuda.current_stream()), DEVICE)
        j, t, n, g = c(1, 2, 4, 64), c(4, 32, 2), c(64), c(64)
        s = (c(1, 4, 2, 64), c(1, 4, 2, 64), c(1, 4, 2, 64), n, n)
        refused(lambda: B.difa_rotate(plan, j, None, j, None, t.cpu(), 4), DEVICE)
        refused(lambda: B.difa_rope_table(plan, c(4, 1).cpu(), (64,), 1e4, t, stream=0), DEVICE)
        refused(lambda: B.difa_qk_norm_rotate(plan, None, s[:4] + (n.cpu(),), j, j.clone(), j.clone(), table=t), DEVICE)
        refused(lambda: B.difa_qk_norm_rotate_backward(plan, None, s, j, j, j, None, tuple(x.clone() for x in s[:3]) + (g, g.cpu()), table=t), DEVICE)
