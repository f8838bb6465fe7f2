"""Timed cases of the operators around the joint attention of an MMDiT layer: rotary positions over several axes, the
norms of the heads' queries and keys with the rotation in the same pass (forward and backward), and the matrix product
with bias, activation, gate and residual in its epilogue.

`run` computes them in plain form, in elementary torch operations (32 bits, angles in 64), or, where `own` is set, by the
library's calls.  Sizes are the layers of workloads.py (24 heads of 64 or 128; 1K, 2K and video latents) and a hidden size
of 24 heads of 64 with a feed-forward four times as wide.  A case is a dict of plain values:

  kind     "table"     cosines and sines of `tokens` positions for head_dim D on `axes` axes
           "rotate"    queries and keys of a layer rotated by such a table (inverse: by the opposite angles, which is
                       also the gradient)
           "norm"      RMS norms of queries and keys per head, rotation, and the gathering of the text and image streams'
                       packed projections into the attention's joint q, k and v
           "backward"  its gradients: both packed projections' and the four weight vectors'
           "linear"    out = residual + gate * act(x W^T + bias)
  B H D n_text n_img   the layer;  rows, K, N   rows of x per batch entry, input and output features
"""
import math

import torch

own = False

EPS = 1e-6
THETA = 10000.0
DIMS = {(64, 1): (64,), (64, 2): (32, 32), (64, 3): (8, 28, 28), (128, 1): (128,), (128, 2): (64, 64), (128, 3): (16, 56, 56)}


def _table(tokens, D, axes):
    return dict(kind="table", tokens=tokens, D=D, axes=axes)


def _layer(kind, B, H, D, n_text, n_img, **more):
    c = dict(kind=kind, B=B, H=H, D=D, n_text=n_text, n_img=n_img, axes=3, dtype="bf16", layout="bhnd", image_first=False,
             halves=False)
    if kind == "rotate":
        c["inverse"] = False
    c.update(more)
    return c


def _linear(B, rows, K, N, **more):
    c = dict(kind="linear", B=B, rows=rows, K=K, N=N, dtype="bf16", bias=True, act="none", gate=False, residual=False)
    c.update(more)
    return c


def listed():
    def named(name, c):
        return dict(c, name=name)

    return [
        # positions of a 1024 px latent (64 x 64 tokens behind 512 text tokens): once per resolution
        named("table_1k", _table(4608, 128, 3)),
        # ... of a video latent (13 frames of 30 x 52) with 256 text tokens
        named("table_video", _table(20536, 128, 3)),
        # queries and keys of an SD3-like 1K layer, CFG pair, [batch, token, head, feature]
        named("rotate_1k", _layer("rotate", 2, 24, 64, 333, 4096, axes=2, layout="bnhd")),
        # a video layer in fp32, rotated back: the gradient of the rotation
        named("rotate_video_f32", _layer("rotate", 1, 24, 128, 256, 20280, dtype="f32", halves=True, inverse=True)),
        # an 8 x 8 latent, four heads: launch and host latency
        named("norm_tiny", _layer("norm", 1, 4, 64, 16, 64)),
        # FLUX-like 2K layer, from the two packed projections to the attention's q, k and v
        named("norm_2k", _layer("norm", 1, 24, 128, 512, 16384)),
        # gradients of an SD3-like 512 px layer, image tokens first
        named("backward_512", _layer("backward", 2, 24, 64, 154, 1024, image_first=True, layout="bnhd")),
        # ... of a FLUX-like 1K layer
        named("backward_1k", _layer("backward", 1, 24, 128, 512, 4096)),
        # shift, scale and gate vectors of both sub-layers from the time embedding, one row per CFG entry
        named("linear_modulation", _linear(2, 1, 1536, 9216)),
        # feed-forward's second product on the text stream (333 tokens, CFG pair), gated and added to the stream
        named("linear_text_down", _linear(2, 333, 6144, 1536, gate=True, residual=True)),
        # output projection of a 1K layer in fp32
        named("linear_out_f32", _linear(1, 4096, 1536, 1536, dtype="f32", residual=True)),
        # feed-forward's first product on the image stream of a 2K layer, CFG pair
        named("linear_up_2k", _linear(2, 16384, 1536, 6144, act="gelu_tanh")),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        c = _draw(rng)
        w = work(c)
        if w["bytes"] <= 6e8 and w["flops"] <= (6e11 if c.get("dtype") != "f32" else 8e10):
            return c


def _draw(rng):
    kind = rng.choice(["table", "rotate", "norm", "backward", "linear", "linear"])
    if kind == "table":
        return _table(_log_int(rng, 1, 20536), rng.choice([64, 128]), rng.randint(1, 3))
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind != "linear":
        more = dict(axes=rng.randint(1, 3), dtype=dtype, layout=rng.choice(["bhnd", "bnhd"]), halves=rng.random() < 0.3,
                    image_first=rng.random() < 0.3)
        if kind == "rotate":
            more["inverse"] = rng.random() < 0.5
        return _layer(kind, rng.choice([1, 2]), rng.randint(1, 24), rng.choice([64, 128]), rng.choice([0, 77, 154, 256, 333, 512]),
                      _log_int(rng, 1, 20280), **more)
    act = rng.choice(["none", "none", "gelu_tanh", "gelu_erf", "silu"])
    end = act == "none"
    # features in eights, now and then any number of them
    K, N = 8 * _log_int(rng, 1, 768), 8 * _log_int(rng, 1, 1152)
    if rng.random() < 0.2:
        K, N = _log_int(rng, 1, 6144), _log_int(rng, 1, 9216)
    return _linear(rng.choice([1, 2]), _log_int(rng, 1, 16384), K, N, dtype=dtype, bias=rng.random() < 0.8, act=act,
                   gate=end and rng.random() < 0.5, residual=end and rng.random() < 0.5)


def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _pairs(c):
    """Axis and frequency of each of the D / 2 pairs of features."""
    axis, omega = [], []
    for a, d in enumerate(DIMS[(c["D"], c["axes"])]):
        axis += [a] * (d // 2)
        omega += [THETA ** (-2.0 * j / d) for j in range(d // 2)]
    return axis, omega


def _positions(tokens, n_text, axes, shift, dev):
    """Row-major coordinates on the most nearly cubic grid, moved by `shift`; text tokens sit at the origin."""
    n = max(tokens - n_text, 1)
    side = max(int(round(n ** (1.0 / axes))), 1)
    i = torch.arange(n, device=dev)
    cols = []
    for a in range(axes):
        below = side ** (axes - 1 - a)
        cols.append((i // below) % side if a else i // below)
    img = torch.stack(cols, dim=1).float() + float(shift)
    return torch.cat([torch.zeros(n_text, axes, device=dev), img])[:tokens].contiguous()


class _Plan:
    """A plan object that lives as long as the state that holds it."""

    def __init__(self, B, H, D, dtype, layout, tokens, image_first):
        from paper_2503_22796_amd import binding
        self.binding = binding
        self.handle = binding.difa_plan_create(
            B, H, D, dtype=binding.DIFA_DTYPE_F32 if dtype == "f32" else binding.DIFA_DTYPE_BF16,
            layout=binding.DIFA_LAYOUT_BHND if layout == "bhnd" else binding.DIFA_LAYOUT_BNHD,
            max_tokens=tokens, flags=binding.DIFA_FLAG_IMAGE_FIRST if image_first else 0)

    def __del__(self):
        handle = getattr(self, "handle", None)
        if handle is not None:
            self.handle = None
            self.binding.difa_plan_destroy(handle)


def prepare(case, seed):
    c = dict(case)
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(104729 * int(seed) + 11)

    def rand(*shape, scale=1.0, about=0.0, dtype=None):
        return (torch.randn(shape, device=dev, generator=gen) * scale + about).to(dtype or _type(c))

    kind = c["kind"]
    s = {"c": c}
    if kind == "table":
        s["positions"] = _positions(c["tokens"], 0, c["axes"], int(seed) % 97, dev)
        s["out"] = torch.empty(c["tokens"], c["D"] // 2, 2, device=dev)
        if own:
            s["plan"] = _Plan(1, 1, c["D"], "bf16", "bhnd", 1, False)
        return s
    if kind == "linear":
        B, rows, K, N = c["B"], c["rows"], c["K"], c["N"]
        s["x"] = rand(B, rows, K)
        s["w"] = rand(N, K, scale=K ** -0.5)
        s["bias"] = rand(N, scale=0.1) if c["bias"] else None
        s["gate"] = rand(B, N, scale=0.5) if c["gate"] else None
        s["residual"] = rand(B, rows, N) if c["residual"] else None
        s["out"] = torch.empty(B, rows, N, device=dev, dtype=_type(c))
        if own:
            s["plan"] = _Plan(1, 1, 64, c["dtype"], "bhnd", 1, False)
            size = s["plan"].binding.difa_linear_workspace(s["plan"].handle, B, rows, N, K)
            s["workspace"] = torch.zeros(size, device=dev, dtype=torch.uint8) if size else None
        return s
    B, H, D, n_text, n_img = c["B"], c["H"], c["D"], c["n_text"], c["n_img"]
    n = n_text + n_img
    # cosines and sines of the layer's positions, made once per resolution
    axis, omega = _pairs(c)
    pos = _positions(n, n_text, c["axes"], 0, dev)
    if c["image_first"]:
        pos = pos.roll(n_img, 0)
    angle = pos.double()[:, axis] * torch.tensor(omega, device=dev, dtype=torch.float64)
    s["table"] = torch.stack([angle.cos(), angle.sin()], dim=-1).float()
    joint = (B, H, n, D) if c["layout"] == "bhnd" else (B, n, H, D)
    if own:
        s["plan"] = _Plan(B, H, D, c["dtype"], c["layout"], n, c["image_first"])
    if kind == "rotate":
        s["q"], s["k"] = rand(*joint), rand(*joint)
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["q"])
        return s
    # the two streams' packed projections (q, k and v next to each other) and norm weights
    for name, tokens in (("text", n_text), ("image", n_img)):
        s[name] = rand(B, tokens, 3, H, D, scale=2.0)
        s[name + "_wq"], s[name + "_wk"] = rand(D, scale=0.2, about=1.0), rand(D, scale=0.2, about=1.0)
    if kind == "norm":
        s["outs"] = [torch.empty(joint, device=dev, dtype=_type(c)) for _ in range(3)]
        return s
    s["grads"] = [rand(*joint) for _ in range(3)]
    for name in ("text", "image"):
        s["d" + name] = torch.empty_like(s[name])
        s["d" + name + "_w"] = torch.empty(2, D, device=dev)
    if own:
        size = s["plan"].binding.difa_qk_norm_rotate_workspace(s["plan"].handle, n_text, n_img)
        s["workspace"] = torch.empty(size, device=dev, dtype=torch.uint8)
    return s


def _run_own(s):
    c = s["c"]
    b = s["plan"].binding
    handle = s["plan"].handle
    if c["kind"] == "table":
        b.difa_rope_table(handle, s["positions"], DIMS[(c["D"], c["axes"])], THETA, s["out"])
        return s["out"]
    if c["kind"] == "linear":
        act = {"none": b.DIFA_ACT_NONE, "gelu_tanh": b.DIFA_ACT_GELU_TANH, "gelu_erf": b.DIFA_ACT_GELU_ERF, "silu": b.DIFA_ACT_SILU}
        b.difa_linear(handle, s["x"], s["w"], s["out"], bias=s["bias"], activation=act[c["act"]], gate=s["gate"],
                      residual=s["residual"], workspace=s["workspace"])
        return s["out"]
    flags = b.DIFA_ROPE_HALVES if c["halves"] else 0
    if c["kind"] == "rotate":
        if c["inverse"]:
            flags |= b.DIFA_ROPE_INVERSE
        b.difa_rotate(handle, s["q"], s["k"], s["q_out"], s["k_out"], s["table"], c["n_text"] + c["n_img"], flags=flags)
        return s["q_out"], s["k_out"]
    text, image = ((x[:, :, 0], x[:, :, 1], x[:, :, 2], s[name + "_wq"], s[name + "_wk"])
                   for name, x in (("text", s["text"]), ("image", s["image"])))
    if c["kind"] == "norm":
        q, k, v = s["outs"]
        b.difa_qk_norm_rotate(handle, text, image, q, k, v, table=s["table"], eps=EPS, flags=flags)
        return q, k, v
    dtext, dimage = ((x[:, :, 0], x[:, :, 1], x[:, :, 2], w[0], w[1])
                     for x, w in ((s["dtext"], s["dtext_w"]), (s["dimage"], s["dimage_w"])))
    dq, dk, dv = s["grads"]
    b.difa_qk_norm_rotate_backward(handle, text, image, dq, dk, dv, dtext, dimage, s["workspace"], table=s["table"], eps=EPS,
                                   flags=flags)
    return (s["dimage"], s["dimage_w"]) + ((s["dtext"], s["dtext_w"]) if c["n_text"] else ())


def _turn(x, table, halves, sign):
    """x [B, tokens, H, D] in 32 bits, its pairs of features turned by sign * angle."""
    cos, sin = table[:, None, :, 0], sign * table[:, None, :, 1]
    half = x.shape[-1] // 2
    a, b = (x[..., :half], x[..., half:]) if halves else (x[..., 0::2], x[..., 1::2])
    u, v = a * cos - b * sin, a * sin + b * cos
    return torch.cat([u, v], dim=-1) if halves else torch.stack([u, v], dim=-1).flatten(-2)


def _joined(text, image, image_first):
    return torch.cat([image, text] if image_first else [text, image], dim=1)


def _stored(x, c):
    """[B, tokens, H, D] as the layer's layout holds it."""
    return (x.transpose(1, 2) if c["layout"] == "bhnd" else x).to(_type(c)).contiguous()


def _norm(x, w):
    x = x.float()
    return x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * w.float()


def _norm_gradients(x, w, dy):
    """Gradients of _norm for x and w, dy in 32 bits."""
    x, w = x.float(), w.float()
    r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
    n, g = x * r, dy * w
    return r * (g - n * (g * n).mean(dim=-1, keepdim=True)), (dy * n).sum(dim=(0, 1, 2))


def _stream_gradients(s, name, dq, dk, dv):
    x = s[name]
    a, aw = _norm_gradients(x[:, :, 0], s[name + "_wq"], dq)
    b, bw = _norm_gradients(x[:, :, 1], s[name + "_wk"], dk)
    return torch.stack([a, b, dv], dim=2).to(x.dtype), torch.stack([aw, bw])


def run(s):
    if own:
        return _run_own(s)
    c = s["c"]
    if c["kind"] == "table":
        axis, omega = _pairs(c)
        angle = s["positions"].double()[:, axis] * torch.tensor(omega, device=s["positions"].device, dtype=torch.float64)
        return torch.stack([angle.cos(), angle.sin()], dim=-1).float()
    if c["kind"] == "linear":
        B, rows, K = s["x"].shape
        y = (s["x"].float().reshape(B * rows, K) @ s["w"].float().t()).reshape(B, rows, -1)
        if c["bias"]:
            y = y + s["bias"].float()
        if c["act"] == "gelu_tanh":
            y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
        elif c["act"] == "gelu_erf":
            y = 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
        elif c["act"] == "silu":
            y = y / (1 + torch.exp(-y))
        if c["gate"]:
            y = y * s["gate"].float()[:, None]
        if c["residual"]:
            y = y + s["residual"].float()
        return y.to(_type(c))
    t = c["layout"] == "bhnd"
    if c["kind"] == "rotate":
        sign = -1.0 if c["inverse"] else 1.0
        q, k = ((x.transpose(1, 2) if t else x).float() for x in (s["q"], s["k"]))
        return _stored(_turn(q, s["table"], c["halves"], sign), c), _stored(_turn(k, s["table"], c["halves"], sign), c)
    text, image = s["text"], s["image"]
    if c["kind"] == "norm":
        q = _joined(_norm(text[:, :, 0], s["text_wq"]), _norm(image[:, :, 0], s["image_wq"]), c["image_first"])
        k = _joined(_norm(text[:, :, 1], s["text_wk"]), _norm(image[:, :, 1], s["image_wk"]), c["image_first"])
        v = _joined(text[:, :, 2], image[:, :, 2], c["image_first"])
        return _stored(_turn(q, s["table"], c["halves"], 1.0), c), _stored(_turn(k, s["table"], c["halves"], 1.0), c), _stored(v, c)
    dq, dk, dv = ((x.transpose(1, 2) if t else x).float() for x in s["grads"])
    dq, dk = _turn(dq, s["table"], c["halves"], -1.0), _turn(dk, s["table"], c["halves"], -1.0)
    at, n_text, n_img = (0 if c["image_first"] else c["n_text"]), c["n_text"], c["n_img"]
    di, dwi = _stream_gradients(s, "image", *(x.narrow(1, at, n_img) for x in (dq, dk, dv)))
    if not n_text:
        return di, dwi
    at = n_img if c["image_first"] else 0
    dt, dwt = _stream_gradients(s, "text", *(x.narrow(1, at, n_text) for x in (dq, dk, dv)))
    return di, dwi, dt, dwt


def exact(case, seed):
    """The definitions in 64 bits; rotations as products of complex numbers."""
    s = prepare(case, seed)
    c = s["c"]
    if c["kind"] == "table":
        out = torch.zeros(c["tokens"], c["D"] // 2, dtype=torch.complex128, device="cuda:0")
        first = 0
        for a, d in enumerate(DIMS[(c["D"], c["axes"])]):
            j = torch.arange(d // 2, device="cuda:0", dtype=torch.float64)
            angle = s["positions"][:, a:a + 1].double() / torch.pow(torch.tensor(THETA, device="cuda:0", dtype=torch.float64), 2 * j / d)
            out[:, first:first + d // 2] = torch.polar(torch.ones_like(angle), angle)
            first += d // 2
        return torch.view_as_real(out)
    if c["kind"] == "linear":
        y = torch.nn.functional.linear(s["x"].double(), s["w"].double(), s["bias"].double() if c["bias"] else None)
        if c["act"] == "gelu_tanh":
            y = torch.nn.functional.gelu(y, approximate="tanh")
        elif c["act"] == "gelu_erf":
            y = torch.nn.functional.gelu(y)
        elif c["act"] == "silu":
            y = torch.nn.functional.silu(y)
        if c["gate"]:
            y = torch.einsum("btn,bn->btn", y, s["gate"].double())
        return y + s["residual"].double() if c["residual"] else y
    B, H, D, n_text, n_img = c["B"], c["H"], c["D"], c["n_text"], c["n_img"]
    phase = torch.view_as_complex(s["table"].double())

    def turned(x, conj=False):                              # [B, H, tokens, D]
        x = x.unflatten(-1, (2, D // 2)).transpose(-1, -2) if c["halves"] else x.unflatten(-1, (D // 2, 2))
        z = torch.view_as_complex(x.contiguous()) * (phase.conj() if conj else phase)
        z = torch.view_as_real(z.resolve_conj())
        return (z.transpose(-1, -2) if c["halves"] else z).flatten(-2)

    def seen(x):                                            # joint tensor <-> [B, H, tokens, D]
        return x if c["layout"] == "bhnd" else x.transpose(1, 2)

    if c["kind"] == "rotate":
        return tuple(seen(turned(seen(s[n]).double(), conj=c["inverse"])).contiguous() for n in ("q", "k"))
    order = ("image", "text") if c["image_first"] else ("text", "image")
    begin = {order[0]: 0, order[1]: n_img if c["image_first"] else n_text}
    if c["kind"] == "norm":
        got = []
        for i, w in ((0, "_wq"), (1, "_wk"), (2, None)):
            parts = []
            for name in order:
                x = s[name][:, :, i].double().transpose(1, 2)
                if w:
                    x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / D + EPS) * s[name + w].double()
                parts.append(x)
            x = torch.cat(parts, dim=2)
            got.append(seen(turned(x) if w else x).contiguous())
        return tuple(got)
    d = [seen(g).double() for g in s["grads"]]
    d[0], d[1] = turned(d[0], conj=True), turned(d[1], conj=True)
    got = []
    for name, tokens in (("image", n_img), ("text", n_text)):
        if not tokens:
            continue
        dx, dw = torch.empty(s[name].shape, dtype=torch.float64, device="cuda:0"), []
        for i, w in ((0, "_wq"), (1, "_wk")):
            x = s[name][:, :, i].double().transpose(1, 2)
            dy = d[i][:, :, begin[name]:begin[name] + tokens]
            m = torch.sqrt(x.square().sum(-1, keepdim=True) / D + EPS)
            g = dy * s[name + w].double()
            dx[:, :, i] = (g / m - x * (g * x).sum(-1, keepdim=True) / (D * m ** 3)).transpose(1, 2)
            dw.append((dy * x / m).sum(dim=(0, 1, 2)))
        dx[:, :, 2] = d[2][:, :, begin[name]:begin[name] + tokens].transpose(1, 2)
        got += [dx, torch.stack(dw)]
    return tuple(got)


def work(case):
    c = case
    if c["kind"] == "table":
        return {"bytes": c["tokens"] * (4 * c["axes"] + 4 * c["D"]), "flops": c["tokens"] * c["D"] // 2}
    size = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "linear":
        B, rows, K, N = c["B"], c["rows"], c["K"], c["N"]
        values = B * rows * K + N * K + B * rows * N * (2 if c["residual"] else 1) + (N if c["bias"] else 0) + (B * N if c["gate"] else 0)
        return {"bytes": size * values, "flops": 2 * B * rows * K * N}
    n = c["n_text"] + c["n_img"]
    values = c["B"] * n * c["H"] * c["D"]
    table = n * c["D"] * 4
    if c["kind"] == "rotate":
        return {"bytes": 4 * values * size + table, "flops": 6 * values}
    if c["kind"] == "norm":
        return {"bytes": 6 * values * size + table, "flops": 14 * values}
    # backward: q and k and three gradients read, three written
    return {"bytes": 8 * values * size + table, "flops": 30 * values}
