"""Features that nothing turns: an infinity or NaN stays where it is."""
import pytest
import torch

from layer_util import Plan, randn
from oracle import layer_oracle as O
from paper_2503_22796_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_rotate_behind_the_last_axis(value, halves, dtype):
    D, n = 64, 3
    flags = B.DIFA_ROPE_HALVES if halves else 0
    x = randn(1, 1, n, D, seed=1, dtype=dtype)
    first, second = O.pair_features(D, halves)
    x[0, 0, 1, first[20]] = value                # pairs 4 .. 31 are not turned
    x[0, 0, 2, second[31]] = value
    xc, out, table = x.cuda(), torch.zeros(1, 1, n, D, dtype=dtype, device="cuda"), torch.empty(n, D // 2, 2, device="cuda")
    with Plan(1, 1, D, dtype, max_tokens=n) as plan:
        B.difa_rope_table(plan, torch.arange(1.0, n + 1, device="cuda")[:, None].contiguous(), (8,), 1e4, table)
        for f in (flags, flags | B.DIFA_ROPE_INVERSE):
            B.difa_rotate(plan, xc, None, out, None, table, n, f)
            got = out.cpu()
            for still in (first[4:], second[4:]):
                torch.testing.assert_close(got[..., still], x[..., still], rtol=0, atol=0, equal_nan=True)
            assert torch.isfinite(got[..., first[:4]]).all() and torch.isfinite(got[..., second[:4]]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("halves", [False, True])
def test_norm_without_a_table(halves, dtype):
    """x / sqrt(mean(x^2) + eps) with one infinity: zeros, and NaN for the infinity alone."""
    D, n = 128, 4
    x = randn(1, n, 1, D, seed=2, dtype=dtype)
    x[0, 1, 0, 5], x[0, 2, 0, 70] = float("inf"), float("-inf")
    xc = x.cuda()
    q, k = (torch.zeros(1, 1, n, D, dtype=dtype, device="cuda") for _ in range(2))
    with Plan(1, 1, D, dtype, max_tokens=n) as plan:
        B.difa_qk_norm_rotate(plan, None, (xc, xc, None, None, None), q, k, None, eps=1e-6, flags=B.DIFA_ROPE_HALVES if halves else 0)
        for got in (q.cpu()[0, 0], k.cpu()[0, 0]):
            bad = torch.isnan(got)
            assert bad[1, 5] and bad[2, 70] and int(bad.sum()) == 2
            assert int((got[1:3] == 0).sum()) == 2 * (D - 1) and torch.isfinite(got[[0, 3]]).all()


@pytest.mark.parametrize("halves", [False, True])
def test_weight_gradients_without_a_table(halves):
    """sum of g n: an infinite g is in its own feature's sum."""
    D, n = 64, 9
    x, d = randn(1, n, 1, D, seed=3).cuda(), randn(1, 1, n, D, seed=4)
    d[0, 0, 4, 33] = float("inf")
    d = d.cuda()
    gx, gw = torch.empty(1, n, 2, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, D, device="cuda")
    with Plan(1, 1, D, max_tokens=n) as plan:
        space = torch.empty(B.difa_qk_norm_rotate_workspace(plan, 0, n), dtype=torch.uint8, device="cuda")
        B.difa_qk_norm_rotate_backward(plan, None, (x, x, None, None, None), d, d, None, None,
                                       (gx[:, :, :1], gx[:, :, 1:], None, gw[0], gw[1]), workspace=space, flags=B.DIFA_ROPE_HALVES if halves else 0)
        bad = ~torch.isfinite(gw.cpu())
        assert bad[:, 33].all() and int(bad.sum()) == 2
