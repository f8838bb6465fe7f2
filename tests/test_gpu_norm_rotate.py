"""difa_qk_norm_rotate and its gradients on the GPU against the 64-bit forms."""
import pytest
import torch

from layer_util import F32, NORM, Plan, check, half_step, norm_bound, randn, seen, stored, turned_size
from oracle import layer_oracle as O
from paper_2503_22796_amd import binding as B

pytestmark = pytest.mark.gpu

EPS = 1e-6


def packed(batch, tokens, heads, D, seed, dtype, scale=2.0):
    """A stream's projection [batch, tokens, 3, heads, D] on the CPU, or None."""
    return randn(batch, tokens, 3, heads, D, seed=seed, scale=scale, dtype=dtype) if tokens else None


def weights(D, seed, dtype):
    return [randn(D, seed=seed + i, scale=0.3, about=1.0, dtype=dtype) for i in (0, 1)]


def stream_of(x, w, cuda):
    if x is None:
        return None
    x = x.cuda() if cuda else x
    return (x[:, :, 0], x[:, :, 1], x[:, :, 2], *[None if t is None else (t.cuda() if cuda else t) for t in w])


CASES = [  # batch, heads, D, n_text, n_img, layout, image_first, halves, table (0 none, 1 shared, 2 per entry), weights
    (1, 4, 64, 16, 64, "bhnd", False, False, 1, True),
    (1, 1, 128, 0, 1, "bhnd", False, False, 1, True),
    (2, 3, 64, 1, 0, "bnhd", True, True, 1, True),
    (2, 5, 128, 77, 130, "bnhd", False, False, 2, True),
    (1, 24, 128, 333, 500, "bhnd", True, False, 1, True),
    (3, 7, 64, 13, 257, "bhnd", False, True, 0, False),
    (1, 2, 64, 512, 4097, "bnhd", True, False, 2, True)]


def make(case, dtype):
    batch, heads, D, n_text, n_img, layout, image_first, halves, tab, weighted = case
    n = n_text + n_img
    xs = [packed(batch, n_text, heads, D, 1, dtype), packed(batch, n_img, heads, D, 2, dtype)]
    ws = [weights(D, 10 + 5 * i, dtype) if weighted else [None, None] for i in (0, 1)]
    table = None
    if tab:
        rows = n * (batch if tab == 2 else 1)
        table = O.rope_table(torch.arange(2 * rows).reshape(-1, 2).float() % 311, (D // 2, D // 2), 1e4, D).float()
        table = table.reshape(batch, n, D // 2, 2) if tab == 2 else table
    return xs, ws, table, n


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("case", CASES)
def test_forward(case, dtype):
    batch, heads, D, n_text, n_img, layout, image_first, halves, _, _ = case
    xs, ws, table, n = make(case, dtype)
    with Plan(batch, heads, D, dtype, layout, n + 1, image_first) as plan:
        print(f"norm {case}", flush=True)
        shape = (batch, heads, n, D) if layout == "bhnd" else (batch, n, heads, D)
        outs = [torch.full(shape, float("nan"), dtype=dtype, device="cuda") for _ in range(3)]
        args = [stream_of(x, w, True) for x, w in zip(xs, ws)]
        t = None if table is None else table.cuda()
        B.difa_qk_norm_rotate(plan, *args, *outs, table=t, eps=EPS, flags=B.DIFA_ROPE_HALVES if halves else 0)
        got = [seen(o, layout) for o in outs]
        again = [torch.full_like(o, float("nan")) for o in outs[:2]]              # without v
        B.difa_qk_norm_rotate(plan, *[a and (a[0], a[1], None, *a[3:]) for a in args], *again, None, table=t, eps=EPS,
                              flags=B.DIFA_ROPE_HALVES if halves else 0)
        assert torch.equal(again[0], outs[0]) and torch.equal(again[1], outs[1])
    text, image = (stream_of(x, w, False) for x, w in zip(xs, ws))
    ref = O.qk_norm_rotate(text, image, table, EPS, image_first, halves)
    for i in (0, 1):
        normed = O.joined(*(None if s is None else O.norm(s[i], s[3 + i], EPS) for s in (text, image)), image_first)
        check(got[i], ref[i], norm_bound(normed, None, None if table is None else table.double(), EPS, halves, dtype, ref[i]), "qk"[i])
    assert torch.equal(got[2].double(), ref[2])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("case", CASES)
def test_backward(case, dtype):
    batch, heads, D, n_text, n_img, layout, image_first, halves, _, weighted = case
    xs, ws, table, n = make(case, dtype)
    d = [randn(batch, heads, n, D, seed=40 + i, dtype=dtype) for i in range(3)]
    flags = B.DIFA_ROPE_HALVES if halves else 0
    with Plan(batch, heads, D, dtype, layout, n, image_first) as plan:
        print(f"norm backward {case}", flush=True)
        args = [stream_of(x, w, True) for x, w in zip(xs, ws)]
        dd = [stored(g, layout) for g in d]
        t = None if table is None else table.cuda()
        ws_bytes = B.difa_qk_norm_rotate_workspace(plan, n_text, n_img)

        def call(wanted=True):
            grads, dws = [], []
            for x in xs:
                g = None if x is None else torch.full(x.shape, float("nan"), dtype=dtype, device="cuda")
                w = torch.full((2, D), float("nan"), device="cuda")
                grads.append(g)
                dws.append(w)
            outs = [None if g is None else (g[:, :, 0], g[:, :, 1], g[:, :, 2], w[0] if wanted else None, w[1] if wanted else None)
                    for g, w in zip(grads, dws)]
            space = torch.full((ws_bytes,), 0xff, dtype=torch.uint8, device="cuda") if wanted else None      # NaN in every float
            B.difa_qk_norm_rotate_backward(plan, *args, *dd, *outs, workspace=space, table=t, eps=EPS, flags=flags)
            torch.cuda.synchronize()
            return grads, dws

        grads, dws = call()
        again, dws2 = call()
        plain, _ = call(wanted=False)
    text, image = (stream_of(x, w, False) for x, w in zip(xs, ws))
    ref = O.qk_norm_rotate_backward(text, image, table, EPS, *d, image_first, halves)
    tt = None if table is None else table.double()
    for s, g, g2, g3, w, w2, r, begin in zip((text, image), grads, again, plain, dws, dws2, ref, (n_img if image_first else 0, 0 if image_first else n_text)):
        if s is None:
            continue
        assert torch.equal(g, g2) and torch.equal(g, g3) and torch.equal(w, w2), "the same call gives the same bits"
        count = s[0].shape[1]
        for i in (0, 1):
            x = s[i].double()
            rr = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
            nn = (x * rr).abs()
            size = turned_size(d[i].double(), tt, halves)[:, :, begin:begin + count].transpose(1, 2)   # of the turned-back gradient
            gw = size if s[3 + i] is None else size * s[3 + i].double().abs()
            # every factor carries at most NORM; the mean's sum of products 12 roundings more: 2^-18 in all
            bound = half_step(dtype) * r[i].abs() * 1.01 + 4 * NORM * rr * (gw + nn * (gw * nn).mean(-1, keepdim=True))
            check(g[:, :, i], r[i], bound, f"d{'qk'[i]}")
            # each product NORM and 3 half steps; a lane adds at most (tokens / groups of a block) * heads of them, then 32 groups, 64
            # slices' workgroups and 16 slices: with fewer than 2^11 sums in a row, 2^11 half steps = 2^-13 of the sizes' sum
            terms = (size * nn).sum(dim=(0, 1, 2))
            check(w[i], r[3 + i], (2.0 ** -13 + 2 * NORM) * terms, f"d{'qk'[i]}_weight")
        assert torch.equal(g[:, :, 2].double().cpu(), r[2])


def _one(x, eps, dtype=torch.bfloat16, w=None):
    """The normed queries of one head per row of x [rows, D]."""
    rows, D = x.shape
    with Plan(1, 1, D, dtype, "bhnd", rows) as plan:
        xs = x.to(dtype).cuda()[None, :, None]
        q, k = torch.empty(1, 1, rows, D, dtype=dtype, device="cuda"), torch.empty(1, 1, rows, D, dtype=dtype, device="cuda")
        B.difa_qk_norm_rotate(plan, None, (xs, xs, None, w, w), q, k, None, eps=eps)
        bits = torch.int16 if dtype == torch.bfloat16 else torch.int32
        assert torch.equal(q.view(bits), k.view(bits))
        return q[0, 0].cpu()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_zeros_and_extreme_values(dtype):
    x = randn(6, 64, seed=7, dtype=torch.float32)
    x[0] = 0
    x[1] *= 1e30                                # squares beyond fp32
    x[2] *= 1e-30                               # ... and below it: eps is all that counts
    x[3] = torch.finfo(torch.bfloat16).max
    x[4, 1:] = 0
    x = x.to(dtype)
    got, ref = _one(x, EPS, dtype), O.norm(x.float(), None, EPS)
    assert bool((got[0] == 0).all())
    # below: the normed row is in the range of fp32's small numbers, off by its smallest step besides
    check(got, ref, half_step(dtype) * ref.abs() * 1.01 + NORM * ref.abs() + 2.0 ** -133, "extreme rows")


def test_a_value_that_is_not_finite_stays_in_its_head():
    x = randn(5, 128, seed=8, dtype=torch.float32)
    x[1, 3], x[3, 100] = float("nan"), float("inf")
    got = _one(x, EPS)
    assert torch.isfinite(got[[0, 2, 4]].float()).all() and torch.isnan(got[1].float()).all() and torch.isnan(got[3, 100].float())


def test_strides_and_rows_behind():
    """Streams whose heads lie outside their tokens, and joint tensors with room behind that stays as it was."""
    heads, D, nt, ni = 3, 64, 5, 21
    text = randn(2, heads, nt, 3, D, seed=9).cuda()
    image = randn(2, heads, ni + 2, 3, D, seed=10).cuda()
    views = [tuple(x[:, :, :m, i].transpose(1, 2) for i in range(3)) + (None, None) for x, m in ((text, nt), (image, ni))]
    n = nt + ni
    with Plan(2, heads, D, max_tokens=n) as plan:
        bufs = [torch.full((2 * heads * n * D + 64,), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
        outs = [b[:-64].view(2, heads, n, D) for b in bufs]
        B.difa_qk_norm_rotate(plan, *views, *outs, eps=EPS)
        assert all(bool((b[-64:] == 7.0).all()) for b in bufs)
        ref = O.qk_norm_rotate(*[tuple(t if t is None else t.cpu() for t in v) for v in views], None, EPS)
        for got, r in zip(outs, ref):
            check(got, r, (half_step(torch.bfloat16) * 1.01 + NORM) * r.abs(), "strided")
        # gradients into such views: what lies between the rows stays
        gt, gi = torch.full_like(text, 5.0), torch.full_like(image, 5.0)
        gviews = [tuple(x[:, :, :m, i].transpose(1, 2) for i in range(3)) + (None, None) for x, m in ((gt, nt), (gi, ni))]
        B.difa_qk_norm_rotate_backward(plan, *views, *outs, *gviews, eps=EPS)
        assert bool((gi[:, :, ni:] == 5.0).all())
        rb = O.qk_norm_rotate_backward(*[tuple(t if t is None else t.cpu() for t in v) for v in views], None, EPS, *[o.cpu() for o in outs])
        for v, r in zip(gviews, rb):
            assert torch.equal(v[2].double().cpu(), r[2])
            scale = (r[0].abs() + 1).max()
            check(v[0], r[0], (half_step(torch.bfloat16) * 1.01) * r[0].abs() + 8 * NORM * scale, "strided gradient")


def test_gradient_against_differences():
    """The backward call's answer against the forward call's own differences, fp32."""
    heads, D, ni = 2, 64, 3
    x, w = randn(1, ni, 3, heads, D, seed=11, dtype=torch.float32), randn(D, seed=12, about=1.0, dtype=torch.float32)
    d = [randn(1, heads, ni, D, seed=13 + i, dtype=torch.float32).cuda() for i in range(3)]
    table = O.rope_table(torch.arange(3.0)[:, None], (D,), 1e4, D).float().cuda()
    with Plan(1, heads, D, torch.float32, "bhnd", ni) as plan:
        def loss(x, w):
            outs = [torch.empty(1, heads, ni, D, device="cuda") for _ in range(3)]
            xc, wc = x.cuda(), w.cuda()
            B.difa_qk_norm_rotate(plan, None, (xc[:, :, 0], xc[:, :, 1], xc[:, :, 2], wc, wc), *outs, table=table, eps=EPS)
            return float(sum((o.double() * g.double()).sum() for o, g in zip(outs, d)))

        xc, wc = x.cuda(), w.cuda()
        gx, gw = torch.empty_like(xc), torch.empty(2, D, device="cuda")
        space = torch.empty(B.difa_qk_norm_rotate_workspace(plan, 0, ni), dtype=torch.uint8, device="cuda")
        B.difa_qk_norm_rotate_backward(plan, None, (xc[:, :, 0], xc[:, :, 1], xc[:, :, 2], wc, wc), *d, None,
                                       (gx[:, :, 0], gx[:, :, 1], gx[:, :, 2], gw[0], gw[1]), workspace=space, table=table, eps=EPS)
        h = 2.0 ** -6
        for at in ((0, 1, 0, 1, 5), (0, 2, 1, 0, 63), (0, 0, 2, 1, 9)):
            up, down = x.clone(), x.clone()
            up[at] += h
            down[at] -= h
            # third derivatives of order 1 times h^2 / 6, and 128 features' half steps over 2 h
            assert abs((loss(up, w) - loss(down, w)) / (2 * h) - float(gx[at])) < 1e-3
        up, down = w.clone(), w.clone()
        up[7] += h
        down[7] -= h
        assert abs((loss(x, up) - loss(x, down)) / (2 * h) - float(gw[0, 7] + gw[1, 7])) < 1e-3
