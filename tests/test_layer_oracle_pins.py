"""The plain 64-bit forms of the operators around the attention, pinned by their definitions, by torch's own operators and by
differences."""
import math

import pytest
import torch

from layer_util import randn
from oracle import layer_oracle as O


def test_table_by_hand():
    t = O.rope_table(torch.tensor([[3.0, 5.0]]), (4, 2), 100.0, 8)
    want = [3.0, 3.0 / 10.0, 5.0, 0.0]                                   # 100^(-2/4) = 1/10; the last pair is not turned
    for p, angle in enumerate(want):
        assert abs(float(t[0, p, 0]) - math.cos(angle)) < 1e-15 and abs(float(t[0, p, 1]) - math.sin(angle)) < 1e-15


@pytest.mark.parametrize("halves", [False, True])
def test_rotation_by_hand_and_back(halves):
    x = randn(2, 3, 5, 8, seed=1, dtype=torch.float64)
    table = O.rope_table(randn(5, 1, seed=2, scale=9.0, dtype=torch.float32), (8,), 50.0, 8)
    y = O.rotate(x, table, halves)
    a, b = (1, 5) if halves else (2, 3)                                  # pair 1
    c, s = table[4, 1]
    assert torch.allclose(y[1, 2, 4, a], x[1, 2, 4, a] * c - x[1, 2, 4, b] * s, atol=1e-15)
    assert torch.allclose(y[1, 2, 4, b], x[1, 2, 4, a] * s + x[1, 2, 4, b] * c, atol=1e-15)
    assert torch.allclose(y.norm(dim=-1), x.norm(dim=-1), atol=1e-13)
    assert torch.allclose(O.rotate(y, table, halves, inverse=True), x, atol=1e-14)


def test_products_of_rotated_rows_depend_on_distances_only():
    q, k = randn(1, 1, 1, 16, seed=3, dtype=torch.float64), randn(1, 1, 1, 16, seed=4, dtype=torch.float64)

    def score(i, j):
        at = lambda p: O.rope_table(torch.tensor([p]), (8, 8), 1e4, 16)  # noqa: E731
        return float((O.rotate(q, at(i)) * O.rotate(k, at(j))).sum())

    assert abs(score([5.0, 2.0], [1.0, 9.0]) - score([105.0, 32.0], [101.0, 39.0])) < 1e-12


def test_norm_is_torchs():
    x, w = randn(2, 7, 3, 64, seed=5, dtype=torch.float64), randn(64, seed=6, dtype=torch.float64)
    assert torch.allclose(O.norm(x, w, 1e-6), torch.nn.functional.rms_norm(x, (64,), w, 1e-6), atol=1e-14)


@pytest.mark.parametrize("image_first", [False, True])
def test_joint_order(image_first):
    text, image = randn(1, 2, 3, 4, seed=7), randn(1, 5, 3, 4, seed=8)
    j = O.joined(text, image, image_first)
    at = 5 if image_first else 0
    assert torch.equal(j[0, 1, at + 1], text[0, 1, 1]) and torch.equal(j[0, 2, (0 if image_first else 2) + 4], image[0, 4, 2])


@pytest.mark.parametrize("image_first,halves,with_table", [(False, False, True), (True, True, True), (False, False, False)])
def test_gradients_against_differences_and_autograd(image_first, halves, with_table):
    B, H, D, eps = 2, 2, 8, 1e-3
    streams = [[randn(B, t, H, D, seed=10 + 5 * i + j, dtype=torch.float64).requires_grad_() for j in range(3)] +
               [randn(D, seed=30 + 5 * i + j, about=1.0, dtype=torch.float64).requires_grad_() for j in range(2)]
               for i, t in enumerate((3, 4))]
    table = O.rope_table(randn(7, 2, seed=50, scale=5.0, dtype=torch.float32), (4, 4), 100.0, D) if with_table else None
    d = [randn(B, H, 7, D, seed=60 + i, dtype=torch.float64) for i in range(3)]

    def loss():
        return sum((o * g).sum() for o, g in zip(O.qk_norm_rotate(*streams, table, eps, image_first, halves), d))

    loss().backward()
    with torch.no_grad():
        got = O.qk_norm_rotate_backward(*streams, table, eps, *d, image_first, halves)
        for s, g in zip(streams, got):
            for leaf, grad in zip(s, g):
                assert torch.allclose(leaf.grad, grad, atol=1e-12)
                flat, at = leaf.data.view(-1), leaf.numel() // 3
                old, h = float(flat[at]), 1e-5
                flat[at] = old + h
                up = float(loss())
                flat[at] = old - h
                down = float(loss())
                flat[at] = old
                assert abs((up - down) / (2 * h) - float(grad.reshape(-1)[at])) < 1e-7


@pytest.mark.parametrize("act", ["none", "gelu_tanh", "gelu_erf", "silu"])
def test_linear_is_torchs(act):
    F = torch.nn.functional
    x, w, b = (randn(*s, seed=70 + i, dtype=torch.float64) for i, s in enumerate(((2, 3, 5), (4, 5), (4,))))
    gate, res = randn(2, 4, seed=80, dtype=torch.float64), randn(2, 3, 4, seed=81, dtype=torch.float64)
    f = {"none": lambda y: y, "gelu_tanh": lambda y: F.gelu(y, approximate="tanh"), "gelu_erf": F.gelu, "silu": F.silu}[act]
    assert torch.allclose(O.linear(x, w, b, act, gate, res), res + gate[:, None] * f(F.linear(x, w, b)), atol=1e-13)
    assert torch.allclose(O.linear(x, w, act=act), f(F.linear(x, w)), atol=1e-13)
