"""difa_linear on the GPU against the 64-bit form."""
import pytest
import torch

from layer_util import F32, Plan, check, half_step, randn
from oracle import layer_oracle as O
from paper_2503_22796_amd import binding as B

pytestmark = pytest.mark.gpu

ACTS = {"none": B.DIFA_ACT_NONE, "gelu_tanh": B.DIFA_ACT_GELU_TANH, "gelu_erf": B.DIFA_ACT_GELU_ERF, "silu": B.DIFA_ACT_SILU}


def run(x, w, bias=None, act="none", gate=None, residual=None, workspace="full", out=None):
    batch, rows, k = x.shape
    n = w.shape[0]
    with Plan(dtype=x.dtype) as plan:
        print(f"linear {batch} x {rows}, {k} -> {n}, {x.dtype}, {act}", flush=True)
        dev = [None if t is None else t.cuda() for t in (x, w, bias, gate, residual)]
        out = torch.full((batch, rows, n), float("nan"), dtype=x.dtype, device="cuda") if out is None else out
        size = B.difa_linear_workspace(plan, batch, rows, n, k) if workspace == "full" else 0
        ws = torch.zeros(size, dtype=torch.uint8, device="cuda") if size else None
        got = []
        for _ in range(2):                       # the second call finds the workspace as the first left it
            B.difa_linear(plan, dev[0], dev[1], out, bias=dev[2], activation=ACTS[act], gate=dev[3], residual=dev[4], workspace=ws)
            torch.cuda.synchronize()
            got.append(out.clone())
        assert torch.equal(got[0].view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32),
                           got[1].view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32)), "the same call gives the same bits"
        return got[0].cpu()


def whole(*shape, seed, most, dtype):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g).to(dtype)


SIZES = [  # batch, rows, k, n
    (1, 1, 1, 1), (1, 1, 64, 64), (2, 1, 1536, 9216), (1, 3, 7, 5), (2, 5, 24, 16), (1, 16, 256, 100), (3, 11, 520, 136), (1, 17, 96, 48),
    (1, 33, 33, 65), (1, 64, 2048, 200), (2, 77, 1000, 320), (2, 333, 6144, 1536), (1, 129, 40, 2000), (1, 500, 776, 77),
    (1, 1025, 512, 1032), (1, 640, 3001, 515), (2, 333, 1001, 1536), (2, 20, 2047, 900), (1, 50, 1000, 640), (2, 1024, 1536, 640), (1, 4099, 136, 264), (1, 8192, 64, 512), (2, 2500, 320, 1544), (1, 300, 4104, 264)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("batch,rows,k,n", SIZES)
def test_whole_numbers_are_exact(batch, rows, k, n, dtype):
    """Whole numbers whose products and sums fp32 holds exactly: the result is the exact one, rounded once.  Any mix-up of
    rows, features or parts of k shows."""
    x, w = whole(batch, rows, k, seed=1, most=4, dtype=dtype), whole(n, k, seed=2, most=4, dtype=dtype)
    bias, gate = whole(n, seed=3, most=9, dtype=dtype), whole(batch, n, seed=4, most=3, dtype=dtype)
    res = whole(batch, rows, n, seed=5, most=99, dtype=dtype)
    assert k * 16 + 9 < 2 ** 20                  # times the gate, plus the residual: below 2^24
    for b, g, r in ((None, None, None), (bias, gate, res)):
        ref = O.linear(x, w, b, "none", g, r)
        got = run(x, w, b, "none", g, r)
        assert torch.equal(got, ref.float().to(dtype))
    if k >= 256:
        assert torch.equal(run(x, w, workspace=None), O.linear(x, w).float().to(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("batch,rows,k,n", [(2, 1, 640, 384), (1, 40, 1536, 264), (2, 333, 520, 192), (1, 2048, 192, 1024), (1, 61, 77, 33)])
def test_values(batch, rows, k, n, act, dtype):
    x, w = randn(batch, rows, k, seed=1, dtype=dtype), randn(n, k, seed=2, scale=2 * k ** -0.5, dtype=dtype)
    bias, gate, res = randn(n, seed=3, dtype=dtype), randn(batch, n, seed=4, dtype=dtype), randn(batch, rows, n, seed=5, dtype=dtype)
    got = run(x, w, bias, act, gate, res)
    ref = O.linear(x, w, bias, act, gate, res)
    y = O.linear(x, w, bias)
    size = O.linear(x.abs(), w.abs(), bias.abs())
    # k roundings of sums (all below `size`), the activation's slope below 1.13 and its own arithmetic 2^-20 of its argument,
    # the gate, the residual
    bound = half_step(dtype) * ref.abs() * 1.01 + gate.double().abs()[:, None] * (1.13 * (k + 2) * F32 * size + 2.0 ** -20 * y.abs()) + \
        4 * F32 * (res.double().abs() + ref.abs())
    check(got, ref, bound, f"{act}")
    # the roundings are independent: their root mean square stays well below that.  bf16 and fp32 steps: 1 / sqrt(3) of half a
    # step at most; sums: sqrt(k) half steps of a partial sum no larger than sqrt(k) |x| |w|, gate and slope below 1.13 on average
    err, rms = float((got.double() - ref).pow(2).mean().sqrt()), float(ref.pow(2).mean().sqrt())
    typical = float(O.linear(x.double() ** 2, w.double() ** 2).mean().sqrt())
    assert err <= half_step(dtype) / 3 ** 0.5 * rms * 1.05 + 2 * F32 * k ** 0.5 * typical + 2.0 ** -20 * float(y.pow(2).mean().sqrt())


@pytest.mark.parametrize("act", list(ACTS))
def test_activations_over_their_range(act):
    """One input feature, weight 1: the activation of every value, far tails and infinities among them."""
    v = torch.cat([torch.linspace(-30, 30, 4001), torch.tensor([0.0, 1e-30, -1e-30, 1e4, -1e4, 1e30, -1e30, 3e38, -3e38])])
    x = v.reshape(1, -1, 1)
    got = run(x, torch.ones(1, 1), act=act)
    ref = O.linear(x, torch.ones(1, 1), act=act)
    if act != "none":                            # cubes beyond 64 bits: the limits
        ref = torch.where(x.abs() > 1e12, x.clamp(min=0.0).double(), ref)
    # relative to the argument, as the slopes are of order 1
    check(got, ref, 2.0 ** -20 * torch.minimum(x.double().abs(), ref.abs() + 1.0) + F32 * ref.abs(), act)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_in_place_and_rows_behind(dtype):
    """Image rows of a joint tensor as x, a padded weight, a residual stream updated in place inside a larger buffer."""
    batch, n_text, rows, k, n = 2, 13, 150, 128, 96
    joint = whole(batch, n_text + rows, k, seed=1, most=4, dtype=dtype).cuda()
    w = whole(n, k + 16, seed=2, most=4, dtype=dtype).cuda()
    stream = whole(batch, rows + 3, n + 8, seed=3, most=50, dtype=dtype).cuda()
    gate = whole(n, seed=4, most=2, dtype=dtype).cuda()
    before = stream.clone()
    x, out = joint[:, n_text:], stream[:, 1:rows + 1, 4:4 + n]
    with Plan(dtype=dtype) as plan:
        ws = torch.zeros(max(B.difa_linear_workspace(plan, batch, rows, n, k), 16), dtype=torch.uint8, device="cuda")
        B.difa_linear(plan, x, w[:, :k], out, gate=gate, residual=out, workspace=ws)
    want = before.cpu().clone()
    want[:, 1:rows + 1, 4:4 + n] = O.linear(x.cpu(), w[:, :k].cpu(), gate=gate.cpu().expand(batch, n), residual=before[:, 1:rows + 1, 4:4 + n].cpu()).float().to(dtype)
    assert torch.equal(stream.cpu(), want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [3, 40, 700])
def test_alignments(rows, dtype):
    """Rows that start at every offset from 16 bytes on."""
    k, n = 96, 80
    for at in range(8):
        xb, wb = whole(rows * (k + 1) + 8, seed=at, most=4, dtype=dtype).cuda(), whole(n * (k + 8) + 8, seed=20 + at, most=4, dtype=dtype).cuda()
        ob = torch.zeros(rows * n + 8, dtype=dtype, device="cuda")
        x = xb[at:at + rows * k].view(rows, k) if at % 2 else xb[at:].as_strided((rows, k), (k + 1, 1))
        w = wb[(at * 3) % 8:].as_strided((n, k), (k + (8 if at < 4 else 3), 1))
        out = ob[at:at + rows * n].view(rows, n)
        with Plan(dtype=dtype) as plan:
            B.difa_linear(plan, x, w, out)
        assert torch.equal(out.cpu(), O.linear(x.cpu()[None], w.cpu())[0].float().to(dtype)), at
        assert bool((ob[:at] == 0).all()) and bool((ob[at + rows * n:] == 0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_that_nothing_is_multiplied_by(dtype):
    """One batch entry, one row: any stride."""
    k, n = 72, 40
    buf, w = whole(3_000_000, seed=1, most=4, dtype=dtype).cuda(), whole(n, k, seed=2, most=4, dtype=dtype).cuda()
    for shape, strides in (((1, 1, k), (1, 7)), ((1, 5, k), (3, k)), ((2, 1, k), (2_900_000, 5)), ((1, 40, k), (9, 70_001)), ((40, 1, k), (70_008, 3))):
        x = buf.as_strided(shape, strides + (1,))
        out = torch.zeros(shape[:2] + (n,), dtype=dtype, device="cuda")
        with Plan(dtype=dtype) as plan:
            B.difa_linear(plan, x, w, out)
            assert torch.equal(out.cpu(), O.linear(x.cpu(), w.cpu()).float().to(dtype)), (shape, strides)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [50, 700])
def test_rows_of_x_that_overlap_or_repeat(rows, dtype):
    """A window that slides over a signal, and one row for all: x is only read."""
    k, n = 256, 136
    signal, w = whole(rows * 8 + k, seed=1, most=4, dtype=dtype).cuda(), whole(n, k, seed=2, most=4, dtype=dtype).cuda()
    for step in (8, 0):
        x = signal.as_strided((1, rows, k), (0, step, 1))
        out = torch.zeros(1, rows, n, dtype=dtype, device="cuda")
        with Plan(dtype=dtype) as plan:
            B.difa_linear(plan, x, w, out)
        assert torch.equal(out.cpu(), O.linear(x.cpu(), w.cpu()).float().to(dtype)), step


@pytest.mark.parametrize("rows", [1, 60, 600])
def test_values_that_are_not_finite_stay_in_their_rows_and_features(rows):
    k, n = 264, 136
    x, w = randn(1, rows, k, seed=1), randn(n, k, seed=2)
    x[0, rows // 2, 5], w[7, 263] = float("inf"), float("nan")
    bad = ~torch.isfinite(run(x, w).float()[0])
    assert bad[rows // 2].all() and bad[:, 7].all() and int(bad.sum()) == rows + n - 1


def test_one_workspace_for_calls_of_many_shapes():
    shapes = [(1, 333, 6144, 256), (1, 40, 4096, 128), (1, 100, 2048, 64), (2, 333, 6144, 1536), (1, 300, 2999, 500),
              (1, 20, 6144, 64)]
    with Plan() as plan:
        ws = torch.zeros(max(B.difa_linear_workspace(plan, b, r, n, k) for b, r, k, n in shapes) or 16, dtype=torch.uint8, device="cuda")
        for turn in range(2):
            for b, r, k, n in shapes:
                x, w = whole(b, r, k, seed=r, most=3, dtype=torch.bfloat16), whole(n, k, seed=k, most=3, dtype=torch.bfloat16)
                out = torch.empty(b, r, n, dtype=torch.bfloat16, device="cuda")
                xc, wc = x.cuda(), w.cuda()
                B.difa_linear(plan, xc, wc, out, workspace=ws)
                small = torch.empty_like(out)
                B.difa_linear(plan, xc, wc, small, workspace=ws[:64])            # too small to be of use
                want = O.linear(x, w).float().bfloat16()
                assert torch.equal(out.cpu(), want) and torch.equal(small.cpu(), want), (turn, b, r, k, n)


def test_captured_calls_on_two_streams():
    """A product in parts of k and one by way of copies, captured with a workspace each and replayed side by side, eager calls with a
    third workspace in between."""
    shapes = ((2, 333, 6144, 256), (1, 300, 2999, 500))
    with Plan() as plan:
        runs = []
        for b, r, k, n in shapes:
            x, w = whole(b, r, k, seed=r, most=3, dtype=torch.bfloat16), whole(n, k, seed=k, most=3, dtype=torch.bfloat16)
            size = B.difa_linear_workspace(plan, b, r, n, k)
            assert size > 0
            stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
            dev = (x.cuda(), w.cuda(), torch.empty(b, r, n, dtype=torch.bfloat16, device="cuda"),
                   *(torch.zeros(size, dtype=torch.uint8, device="cuda") for _ in range(2)))
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                B.difa_linear(plan, dev[0], dev[1], dev[2], workspace=dev[3])
                stream.synchronize()
                with torch.cuda.graph(graph, stream=stream):
                    B.difa_linear(plan, dev[0], dev[1], dev[2], workspace=dev[3])
            runs.append((stream, graph, dev, O.linear(x, w).float().bfloat16().cuda()))
        print("two captured products", flush=True)
        for turn in range(4):
            for stream, _, dev, _ in runs:
                with torch.cuda.stream(stream):
                    dev[2].fill_(float("nan"))
            for _ in range(5):
                for stream, graph, _, _ in runs:
                    with torch.cuda.stream(stream):
                        graph.replay()
            torch.cuda.synchronize()
            for stream, _, dev, want in runs:
                assert torch.equal(dev[2], want), turn
                eager = torch.empty_like(want)
                B.difa_linear(plan, dev[0], dev[1], eager, workspace=dev[4])
                assert torch.equal(eager, want), turn
            torch.cuda.synchronize()
        for run in runs:
            run[1].reset()


@pytest.mark.parametrize("workspace", ["full", None])
@pytest.mark.parametrize("rows,k,n", [(1, 16384, 40), (20, 16385, 33), (40, 16384, 264), (300, 8193, 520), (1000, 8192, 1536), (6000, 8192, 520)])
def test_fp32_sums_of_many_products(rows, k, n, workspace):
    """Values of one sign, whose sums grow: what is rounded is no chain of k sums."""
    x, w = randn(1, rows, k, seed=1, dtype=torch.float32).abs(), randn(n, k, seed=2, dtype=torch.float32).abs()
    got, ref = run(x, w, workspace=workspace), O.linear(x, w)
    err = float((got.double() / ref - 1).pow(2).mean().sqrt())
    # A rounding is at most half a step of its sum, 1 / sqrt(3) of that as root mean square; the i-th of c equal sums is i / c of
    # the last, so that a chain of c of them has sqrt(c / 3) roundings of the last.  k / c chains of c = 512, each k / c of the
    # whole, a chain of k / c sums of them, and the result's own: 0.58 * (sqrt(171 * 512 / k) + sqrt(k / 1536) + 1) half steps;
    # one chain of 8192 has 30, of 2048 (eight wavefronts of 16384) 15, their sums 1.5 more.  Half as much again for chance.
    assert err <= 1.5 * F32 / 3 ** 0.5 * ((512 * 512 / 3 / k) ** 0.5 + (k / 512 / 3) ** 0.5 + 1), err / F32


def test_fp32_gelu_erf_where_little_is_left():
    """Relative to the result, on the negative side too, where it is v times what a normal variable has below v."""
    v = torch.linspace(-12, 6, 5003).reshape(1, -1, 1)
    ref = O.linear(v, torch.ones(1, 1)).mul(0.5) * torch.special.erfc(-v.double() / 2 ** 0.5)
    # half steps: the argument's two by its slope, x erfc'(x) / erfc(x) <= 2 x^2 + 1 = v^2 + 1; erfc's own 8 (4 units), two products
    check(run(v, torch.ones(1, 1), act="gelu_erf"), ref, (2 * v.double() ** 2 + 12) * F32 * ref.abs(), "gelu_erf")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("k", [72, 75])
def test_rows_far_apart(k, dtype):
    """Rows of x and of w further from each other than the loads of the fast kernels reach."""
    rows, n, far = 40, 24, (1 << 20) + 8
    x, w = whole(1, rows, k, seed=1, most=4, dtype=dtype), whole(n, k, seed=2, most=4, dtype=dtype)
    xb, wb = (torch.zeros(r * far, dtype=dtype, device="cuda").view(r, far) for r in (rows, n))
    xb[:, :k], wb[:, :k] = x[0].cuda(), w.cuda()
    for a, b in ((xb[:, :k], w.cuda()), (x[0].cuda(), wb[:, :k]), (xb[:, :k], wb[:, :k])):
        out = torch.zeros(rows, n, dtype=dtype, device="cuda")
        with Plan(dtype=dtype) as plan:
            B.difa_linear(plan, a, b, out)
        assert torch.equal(out.cpu(), O.linear(x, w)[0].float().to(dtype))
