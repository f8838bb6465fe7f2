"""Inputs and derived tolerances of the tests of the operators around a layer's attention."""
import ctypes

import torch

from oracle import layer_oracle as O
from paper_2503_22796_amd import binding as B

F32 = 2.0 ** -24                                     # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def randn(*shape, seed, scale=1.0, about=0.0, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale + about).to(dtype)


def dtype_code(dtype):
    return B.DIFA_DTYPE_BF16 if dtype == torch.bfloat16 else B.DIFA_DTYPE_F32


class Plan:
    def __init__(self, batch=1, heads=1, head_dim=64, dtype=torch.bfloat16, layout="bhnd", max_tokens=1, image_first=False):
        self.args = (batch, heads, head_dim, dtype_code(dtype), B.DIFA_LAYOUT_BHND if layout == "bhnd" else B.DIFA_LAYOUT_BNHD,
                     max_tokens, 0.0, 0, B.DIFA_FLAG_IMAGE_FIRST if image_first else 0)

    def __enter__(self):
        self.handle = B.difa_plan_create(*self.args)
        return self.handle

    def __exit__(self, *_):
        torch.cuda.synchronize()
        B.difa_plan_destroy(self.handle)


class PlanWithoutDevice(Plan):
    """A plan object that refuses like any other and can run nothing."""

    def __enter__(self):
        B.lib.difa_testing_plan_without_device.restype = ctypes.c_void_p
        B.lib.difa_testing_plan_without_device.argtypes = [ctypes.c_void_p]
        desc = B.difa_plan_desc_t(*self.args)
        self.handle = ctypes.c_void_p(B.lib.difa_testing_plan_without_device(ctypes.addressof(desc)))
        assert self.handle.value
        return self.handle

    def __exit__(self, *_):
        B.lib.difa_testing_free_plan_without_device.restype = None
        B.lib.difa_testing_free_plan_without_device.argtypes = [ctypes.c_void_p]
        B.lib.difa_testing_free_plan_without_device(self.handle)


def stored(x, layout):
    """A joint [B, H, N, D] tensor on the GPU as the layout holds it."""
    return (x if layout == "bhnd" else x.transpose(1, 2)).contiguous().cuda()


def seen(x, layout):
    x = x.cpu()
    return x if layout == "bhnd" else x.transpose(1, 2)


def check(got, ref, bound, what):
    """Every element within its bound, and finite where the reference is."""
    got, ref = got.double().cpu(), ref.double()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert torch.isfinite(got).all(), f"{what}: values that are not finite"
    excess = (got - ref).abs() - bound
    assert float(excess.max()) <= 0, f"{what}: {int((excess > 0).sum())} of {ref.numel()} outside, worst by {float(excess.max()):.3e}"


def turned_size(x, table, halves):
    """|x| |cos| + |y| |sin| of every feature: what a rotation's roundings are relative to."""
    if table is None:
        return x.abs()
    a = O.rotate(x.abs(), torch.stack([table[..., 0].abs(), -table[..., 1].abs()], -1), halves)
    b = O.rotate(x.abs(), table.abs(), halves)
    first, second = O.pair_features(x.shape[-1], halves)
    out = torch.empty_like(a)
    out[..., first], out[..., second] = a[..., first], b[..., second]
    return out


# x r w: the sum of squares takes 12 roundings on the way to any lane (all terms positive: 12 half steps relative, half of
# that in r), then the mean, eps, the reciprocal root (4 half steps) and the three products: below 16 half steps = 2^-20.
NORM = 2.0 ** -20


def norm_bound(x, w, table, eps, halves, dtype, ref):
    """x: joint [B, H, N, D] normed already (64 bits)."""
    size = turned_size(x, table, halves)
    return half_step(dtype) * ref.abs() * (1 + 2.0 ** -7) + (NORM + 3 * F32) * size
