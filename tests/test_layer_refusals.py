"""Calls that the operators around the attention refuse: on the host, before anything looks at a device."""
import ctypes

import pytest
import torch

from layer_util import PlanWithoutDevice
from paper_2503_22796_amd import binding as B

BAD = B.DIFA_ERR_INVALID_ARG
P = 1 << 20                                     # stands for an aligned device address; no refused call looks behind it


def status(call, plan, *args):
    st = getattr(B.lib, call)(plan, *args)
    if st != B.DIFA_OK and plan is not None:
        assert B.difa_last_error(plan) != ""
    return st


def test_without_a_plan():
    n = ctypes.c_int64(0)
    assert B.lib.difa_rope_table(None, None, None, 1, None, None) == BAD
    assert B.lib.difa_rotate(None, P, None, P, None, P, 1, 1, 0, None) == BAD
    assert B.lib.difa_qk_norm_rotate(None, None, None, None, 1, 1e-6, 0, P, P, P, None) == BAD
    assert B.lib.difa_qk_norm_rotate_backward(None, None, None, None, 1, 1e-6, 0, P, P, P, None, None, None, 0, None) == BAD
    assert B.lib.difa_qk_norm_rotate_workspace(None, 1, 1, ctypes.byref(n)) == BAD
    assert B.lib.difa_linear_workspace(None, 1, 1, 1, 1, ctypes.byref(n)) == BAD
    assert B.lib.difa_linear(None, None, P, P, None, None, None, P, None, 0, None) == BAD


@pytest.mark.parametrize("axes,dims,theta,rows,positions,table", [
    (0, (0, 0, 0, 0), 1e4, 4, P, P), (5, (2, 2, 2, 2), 1e4, 4, P, P), (1, (3, 0, 0, 0), 1e4, 4, P, P), (1, (0, 0, 0, 0), 1e4, 4, P, P),
    (2, (64, 2, 0, 0), 1e4, 4, P, P), (2, (2147483646, 2, 0, 0), 1e4, 4, P, P), (1, (64, 0, 0, 0), 1.0, 4, P, P),
    (1, (64, 0, 0, 0), float("nan"), 4, P, P), (1, (64, 0, 0, 0), float("inf"), 4, P, P), (1, (64, 0, 0, 0), 1e4, 0, P, P),
    (1, (64, 0, 0, 0), 1e4, 4, None, P), (1, (64, 0, 0, 0), 1e4, 4, P, None), (1, (64, 0, 0, 0), 1e4, 4, P + 2, P),
    (1, (64, 0, 0, 0), 1e4, 4, P, P + 8)])
def test_rope_table(axes, dims, theta, rows, positions, table):
    with PlanWithoutDevice(head_dim=64) as plan:
        d = B.difa_rope_desc_t(axes, (ctypes.c_int32 * 4)(*dims), theta)
        assert status("difa_rope_table", plan, ctypes.addressof(d), positions, rows, table, None) == BAD
        assert status("difa_rope_table", plan, None, P, 4, P, None) == BAD


BYTES = 2 * 3 * 10 * 64 * 2                     # the joint tensors of the plan below


@pytest.mark.parametrize("q,k,qo,ko,table,tb,n,flags", [
    (None, P, P, P, P, 1, 10, 0), (P, None, P, 2 * P, P, 1, 10, 0), (P, 2 * P, 3 * P, None, P, 1, 10, 0), (P, None, None, None, P, 1, 10, 0),
    (P, None, P, None, None, 1, 10, 0), (P, None, P, None, P, 1, 0, 0), (P, None, P, None, P, 1, 11, 0), (P, None, P, None, P, 3, 10, 0),
    (P, None, P, None, P, 0, 10, 0), (P, None, P, None, P, 1, 10, 4), (P + 2, None, 2 * P, None, P, 1, 10, 0),
    (P, None, 2 * P + 8, None, P, 1, 10, 0), (P, None, P, None, P + 4, 1, 10, 0), (P, None, P + 16, None, 9 * P, 1, 10, 0),
    (P, None, P + BYTES - 16, None, 9 * P, 1, 10, 0), (P, 2 * P, 2 * P, P, 9 * P, 1, 10, 0), (P, 2 * P, 3 * P, 3 * P, 9 * P, 1, 10, 0)])
def test_rotate(q, k, qo, ko, table, tb, n, flags):
    with PlanWithoutDevice(batch=2, heads=3, max_tokens=10) as plan:
        assert status("difa_rotate", plan, q, k, qo, ko, table, tb, n, flags, None) == BAD


def _stream(n=5, **more):
    s = dict(q=P, k=2 * P, v=3 * P, stride_b=5 * 192, stride_n=192, stride_h=64, q_weight=4 * P, k_weight=5 * P, n_tokens=n)
    s.update(more)
    return B.difa_qkv_t(**s)


def _grad(**more):
    s = dict(q=11 * P, k=12 * P, v=13 * P, stride_b=5 * 192, stride_n=192, stride_h=64, q_weight=14 * P, k_weight=15 * P)
    s.update(more)
    return B.difa_qkv_grad_t(**s)


BAD_STREAMS = [dict(q=None), dict(k=None), dict(q=P + 2), dict(v=P + 8), dict(stride_n=-192), dict(stride_n=191), dict(stride_b=4),
               dict(stride_h=63), dict(q_weight=P + 1), dict(n_tokens=-1), dict(n_tokens=6), dict(n_tokens=2 ** 31 - 1)]


@pytest.mark.parametrize("bad", range(len(BAD_STREAMS) + 11))
def test_qk_norm_rotate(bad):
    text, image, call = _stream(), _stream(), dict(table=6 * P, tb=1, eps=1e-6, flags=0, q=7 * P, k=8 * P, v=9 * P)
    if bad < len(BAD_STREAMS):
        text = _stream(**BAD_STREAMS[bad])
    else:
        i = bad - len(BAD_STREAMS)
        call.update([dict(table=P + 4), dict(tb=3), dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(flags=2),
                     dict(q=None), dict(k=7 * P + 2), dict(v=None), dict(k=7 * P), dict(q=P)][i])
    with PlanWithoutDevice(batch=2, heads=3, max_tokens=10) as plan:
        for a, b in ((text, image), (image, text)):
            args = (ctypes.addressof(a), ctypes.addressof(b), call["table"], call["tb"], call["eps"], call["flags"], call["q"], call["k"], call["v"], None)
            assert status("difa_qk_norm_rotate", plan, *args) == BAD
        assert status("difa_qk_norm_rotate", plan, None, None, None, 1, 1e-6, 0, P, 2 * P, None, None) == BAD


@pytest.mark.parametrize("bad", range(len(BAD_STREAMS) + 18))
def test_qk_norm_rotate_backward(bad):
    text, grad = _stream(), _grad()
    call = dict(table=6 * P, tb=1, eps=1e-6, flags=0, dq=7 * P, dk=8 * P, dv=9 * P, ws=16 * P, size=1 << 20)
    if bad < len(BAD_STREAMS):
        text = _stream(**BAD_STREAMS[bad])
    elif bad < len(BAD_STREAMS) + 10:
        grad = _grad(**[dict(q=None), dict(v=None), dict(k=P + 4), dict(stride_n=3), dict(q_weight=P + 2), dict(q=12 * P),
                        dict(q=7 * P), dict(stride_b=0), dict(stride_n=56), dict(stride_h=0)][bad - len(BAD_STREAMS)])
    else:
        i = bad - len(BAD_STREAMS) - 10
        call.update([dict(dq=None), dict(dk=8 * P + 2), dict(ws=None), dict(ws=16 * P + 4), dict(size=0), dict(eps=-1.0), dict(flags=4),
                     dict(tb=5)][i])
    image, none = _stream(), _grad(q_weight=None, k_weight=None)
    with PlanWithoutDevice(batch=2, heads=3, max_tokens=10) as plan:
        for a, b, ga, gb in ((text, image, grad, none), (image, text, none, grad)):
            args = (ctypes.addressof(a), ctypes.addressof(b), call["table"], call["tb"], call["eps"], call["flags"], call["dq"], call["dk"],
                    call["dv"], ctypes.addressof(ga), ctypes.addressof(gb), call["ws"], call["size"], None)
            assert status("difa_qk_norm_rotate_backward", plan, *args) == BAD
        # a stream with tokens and no place for its gradients
        assert status("difa_qk_norm_rotate_backward", plan, ctypes.addressof(image), None, None, 1, 1e-6, 0, P, 2 * P, None, None, None,
                      None, 0, None) == BAD


def test_workspaces():
    n = ctypes.c_int64(-1)
    with PlanWithoutDevice(batch=2, heads=3, max_tokens=10) as plan:
        for a, b in ((-1, 5), (5, -1), (0, 0), (6, 5), (2 ** 31 - 1, 2 ** 31 - 1)):
            assert status("difa_qk_norm_rotate_workspace", plan, a, b, ctypes.byref(n)) == BAD
        assert status("difa_qk_norm_rotate_workspace", plan, 5, 5, None) == BAD
        assert status("difa_qk_norm_rotate_workspace", plan, 0, 10, ctypes.byref(n)) == B.DIFA_OK and n.value > 0
        for sizes in ((0, 1, 1, 1), (1, 0, 1, 1), (1, 1, 0, 1), (1, 1, 1, 0), (2 ** 16, 2 ** 15, 1, 1)):
            assert status("difa_linear_workspace", plan, *sizes, ctypes.byref(n)) == BAD
        assert status("difa_linear_workspace", plan, 1, 1, 1, 1, None) == BAD
        most = 2 ** 31 - 513
        for sizes in ((2, 100, 64, 4096), (1, most, most, most), (1, most, 1, most), (1, 5, most, 7), (1, most, most, 1)):
            assert status("difa_linear_workspace", plan, *sizes, ctypes.byref(n)) == B.DIFA_OK and 0 <= n.value < 2 ** 50, sizes
        for sizes in ((1, most + 1, 1, 1), (1, 1, most + 1, 1), (1, 1, 1, most + 1)):
            assert status("difa_linear_workspace", plan, *sizes, ctypes.byref(n)) == BAD


LINEAR = dict(batch=2, rows=5, n=16, k=24, activation=0, x_stride_b=120, x_stride_n=24, w_stride=24, out_stride_b=80, out_stride_n=16,
              residual_stride_b=80, residual_stride_n=16, gate_stride_b=16)


@pytest.mark.parametrize("desc,ptrs", [
    (dict(batch=0), {}), (dict(rows=0), {}), (dict(n=0), {}), (dict(k=0), {}), (dict(k=-8), {}), (dict(batch=2 ** 16, rows=2 ** 15), {}),
    (dict(activation=-1), {}), (dict(activation=4), {}), (dict(x_stride_n=-1), {}), (dict(x_stride_b=-1), {}), (dict(gate_stride_b=-1), {}),
    (dict(residual_stride_n=-1), {}), (dict(w_stride=23), {}), (dict(out_stride_n=15), {}), (dict(out_stride_b=0), {}),
    ({}, dict(x=None)), ({}, dict(w=None)), ({}, dict(out=None)), ({}, dict(x=P + 1)), ({}, dict(out=6 * P + 1)), ({}, dict(bias=P + 1)),
    ({}, dict(ws=P + 8)), ({}, dict(size=-1)), ({}, dict(out=P)), ({}, dict(out=2 * P)), ({}, dict(out=3 * P)), ({}, dict(out=4 * P)),
    (dict(residual_stride_n=32), dict(residual=6 * P)), (dict(residual_stride_b=160), dict(residual=6 * P))])
def test_linear(desc, ptrs):
    p = dict(x=P, w=2 * P, bias=3 * P, gate=4 * P, residual=5 * P, out=6 * P, ws=7 * P, size=1 << 20)
    p.update(ptrs)
    d = B.difa_linear_desc_t(**{**LINEAR, **desc})
    with PlanWithoutDevice() as plan:
        assert status("difa_linear", plan, ctypes.addressof(d), p["x"], p["w"], p["bias"], p["gate"], p["residual"], p["out"], p["ws"], p["size"], None) == BAD
        assert status("difa_linear", plan, None, P, 2 * P, None, None, None, 3 * P, None, 0, None) == BAD


def test_binding_refuses_shapes_and_types():
    z = torch.zeros
    with PlanWithoutDevice(heads=2, dtype=torch.float32, max_tokens=4) as plan:
        s = 0                                                                      # a raw stream: no device is asked for one
        x, w = z(1, 4, 8), z(16, 8)
        bad = [lambda: B.difa_rope_table(plan, z(4, 5), (2,) * 5, 1e4, z(4, 32, 2), stream=s),
               lambda: B.difa_rope_table(plan, z(4, 2), (2,), 1e4, z(4, 32, 2), stream=s),
               lambda: B.difa_rope_table(plan, z(4, 1).double(), (64,), 1e4, z(4, 32, 2), stream=s),
               lambda: B.difa_rope_table(plan, z(4, 1), (64,), 1e4, z(3, 32, 2), stream=s),
               lambda: B.difa_rotate(plan, x, None, x, None, z(3, 32, 2), 4, stream=s),
               lambda: B.difa_rotate(plan, x, None, x, None, z(4, 32, 2).double(), 4, stream=s),
               lambda: B.difa_qk_norm_rotate(plan, None, (z(1, 4, 2, 64), z(1, 4, 2, 64).transpose(1, 2), None, None, None), x, x, None, stream=s),
               lambda: B.difa_qk_norm_rotate(plan, None, (z(1, 4, 2, 64), z(1, 4, 2, 64), None, z(32), None), x, x, None, stream=s),
               lambda: B.difa_linear(plan, x, z(16, 9), z(1, 4, 16), stream=s),
               lambda: B.difa_linear(plan, x, w, z(1, 4, 15), stream=s),
               lambda: B.difa_linear(plan, x, z(1, 8).expand(16, 8), z(1, 4, 16), stream=s),
               lambda: B.difa_linear(plan, x, w, z(4, 16), stream=s),
               lambda: B.difa_linear(plan, z(8), w, z(16), stream=s),
               lambda: B.difa_linear(plan, z(2, 1, 4, 8), w, z(2, 1, 4, 16), stream=s),
               lambda: B.difa_linear(plan, x, w, z(1, 4, 16), gate=z(1, 1, 16), stream=s),
               lambda: B.difa_linear(plan, x, w, z(1, 4, 16).bfloat16(), stream=s),
               lambda: B.difa_linear(plan, x, w, z(1, 4, 16), bias=z(15), stream=s),
               lambda: B.difa_linear(plan, x, w, z(1, 4, 16), gate=z(2, 16), stream=s),
               lambda: B.difa_linear(plan, x, w, z(1, 4, 16), residual=z(1, 3, 16), stream=s),
               lambda: B.difa_linear(plan, x.transpose(1, 2).contiguous().transpose(1, 2), w, z(1, 4, 16), stream=s)]
        j, tab, st = z(1, 2, 4, 64), z(4, 32, 2), (z(1, 4, 2, 64), z(1, 4, 2, 64), z(1, 4, 2, 64), z(64), z(64))
        h = z(1, 2, 4, 64).bfloat16()
        bad += [lambda: B.difa_rotate(plan, j[:, :, :, ::2], None, j, None, tab, 4, stream=s),
                lambda: B.difa_rotate(plan, j.transpose(1, 2), None, j, None, tab, 4, stream=s),
                lambda: B.difa_rotate(plan, j, None, h, None, tab, 4, stream=s),
                lambda: B.difa_rotate(plan, j, None, j, None, z(4, 16, 2), 4, stream=s),
                lambda: B.difa_rotate(plan, z(1, 2, 5, 64), None, j, None, tab, 4, stream=s),
                lambda: B.difa_qk_norm_rotate(plan, None, None, j, j, None, stream=s),
                lambda: B.difa_qk_norm_rotate(plan, None, st, z(1, 2, 5, 64), j, j, stream=s),
                lambda: B.difa_qk_norm_rotate(plan, None, st, j, h, j, stream=s),
                lambda: B.difa_qk_norm_rotate(plan, None, st, z(1, 3, 4, 64), z(1, 3, 4, 64), z(1, 3, 4, 64), stream=s),
                lambda: B.difa_qk_norm_rotate(plan, None, st[:3] + (z(64).bfloat16(), None), j, j, j, stream=s),
                lambda: B.difa_qk_norm_rotate(plan, tuple(t[:, :2, :1] if t.dim() == 4 else t for t in st), tuple(t[:, :2] if t.dim() == 4 else t for t in st), j, j, j, stream=s),
                lambda: B.difa_qk_norm_rotate(plan, None, st, j, j, j, table=z(4, 16, 2), stream=s),
                lambda: B.difa_qk_norm_rotate_backward(plan, None, st, j, j, j, None, tuple(t.bfloat16() for t in st[:3]) + (None, None), stream=s),
                lambda: B.difa_qk_norm_rotate_backward(plan, None, st, j, j, j, None, st[:3] + (z(64).bfloat16(), None), stream=s)]
        for call in bad:
            with pytest.raises(B.DifaError) as e:
                call()
            assert e.value.status == BAD
