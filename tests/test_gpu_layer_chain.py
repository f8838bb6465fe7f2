"""The operators around the attention together with it, as a layer uses them: eagerly, and captured into a graph."""
import numpy as np
import pytest
import torch

from layer_util import F32, Plan, check, half_step, norm_bound, randn
from oracle import layer_oracle as O
from paper_2503_22796_amd import binding as B
from util import ARROW, FULL, check_against_oracle

pytestmark = pytest.mark.gpu

EPS = 1e-6


class Layer:
    """An attention sub-layer of hidden size 256 (four heads of 64): projections, norms, rotation, attention, output
    projections gated and added to both streams in place."""

    def __init__(self, plan, batch=2, n_text=45, n_img=144, layout="bnhd"):
        H, D, C = 4, 64, 256
        self.plan, self.dims = plan, (batch, H, D, C, n_text, n_img)
        mk = lambda *s, seed, **kw: randn(*s, seed=seed, **kw).cuda()  # noqa: E731
        n = n_text + n_img
        self.x = [mk(batch, t, C, seed=i) for i, t in enumerate((n_text, n_img))]
        self.w_qkv = [mk(3 * C, C, seed=10 + i, scale=C ** -0.5) for i in (0, 1)]
        self.b_qkv = [mk(3 * C, seed=20 + i, scale=0.1) for i in (0, 1)]
        self.norms = [[mk(D, seed=30 + 2 * i + j, scale=0.2, about=1.0) for j in (0, 1)] for i in (0, 1)]
        self.w_out = [mk(C, C, seed=40 + i, scale=C ** -0.5) for i in (0, 1)]
        self.gate = [mk(batch, C, seed=50 + i) for i in (0, 1)]
        pos = torch.zeros(n, 3)
        pos[n_text:, 1], pos[n_text:, 2] = torch.arange(n_img) // 12, torch.arange(n_img) % 12
        self.pos, self.table = pos.cuda(), torch.empty(n, D // 2, 2, device="cuda")
        self.qkv = [torch.empty(batch, t, 3 * C, dtype=torch.bfloat16, device="cuda") for t in (n_text, n_img)]
        self.joint = [torch.empty(batch, n, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
        self.out = [torch.empty_like(x) for x in self.x]
        self.modes, self.windows = np.array([FULL, ARROW, ARROW, FULL], np.int32), np.array([0, 13, 40, 0], np.int32)
        sizes = [B.difa_linear_workspace(plan, batch, t, o, C) for t in (n_text, n_img) for o in (3 * C, C)]
        self.space = torch.zeros(max(sizes + [16]), dtype=torch.uint8, device="cuda")

    def streams(self):
        batch, H, D, C, n_text, n_img = self.dims
        got = []
        for qkv, w in zip(self.qkv, self.norms):
            x = qkv.view(batch, -1, 3, H, D)
            got.append((x[:, :, 0], x[:, :, 1], x[:, :, 2], *w))
        return got

    def run(self):
        batch, H, D, C, n_text, n_img = self.dims
        B.difa_rope_table(self.plan, self.pos, (16, 24, 24), 1e4, self.table)
        for x, w, b, o in zip(self.x, self.w_qkv, self.b_qkv, self.qkv):
            B.difa_linear(self.plan, x, w, o, bias=b, workspace=self.space)
        q, k, v, o = self.joint
        B.difa_qk_norm_rotate(self.plan, *self.streams(), q, k, v, table=self.table, eps=EPS)
        B.difa_joint_attention(self.plan, q, k, v, o, None, self.modes, n_text, n_img, self.windows)
        rows = o.view(batch, n_text + n_img, C)
        for part, x, w, g, y in zip((rows[:, :n_text], rows[:, n_text:]), self.x, self.w_out, self.gate, self.out):
            y.copy_(x)
            B.difa_linear(self.plan, part, w, y, gate=g, residual=y, workspace=self.space)

    def poison(self):
        for t in [self.table, *self.qkv, *self.joint, *self.out]:
            t.fill_(float("nan"))


def plan():
    return Plan(2, 4, 64, torch.bfloat16, "bnhd", 189)


def test_a_layer_step_by_step():
    with plan() as handle:
        layer = Layer(handle)
        layer.poison()
        print("layer chain", flush=True)
        layer.run()
        torch.cuda.synchronize()
    batch, H, D, C, n_text, n_img = layer.dims
    u = half_step(torch.bfloat16)
    table = O.rope_table(layer.pos.cpu(), (16, 24, 24), 1e4, D)
    check(layer.table, table, F32 * table.abs() + 1e-12, "table")
    # each step against the 64-bit form of what the step before it left
    for x, w, b, got in zip(layer.x, layer.w_qkv, layer.b_qkv, layer.qkv):
        ref = O.linear(x.cpu(), w.cpu(), b.cpu())
        check(got, ref, u * ref.abs() * 1.01 + (C + 2) * F32 * O.linear(x.cpu().abs(), w.cpu().abs(), b.cpu().abs()), "projection")
    text, image = ([t.cpu() for t in s] for s in layer.streams())
    t32 = layer.table.cpu()
    refs = O.qk_norm_rotate(text, image, t32, EPS)
    q, k, v, o = (t.cpu().transpose(1, 2) for t in layer.joint)
    for i, got in ((0, q), (1, k)):
        normed = O.joined(*(O.norm(s[i], s[3 + i], EPS) for s in (text, image)), False)
        check(got, refs[i], norm_bound(normed, None, t32.double(), EPS, False, torch.bfloat16, refs[i]), "normed and turned")
    assert torch.equal(v.double(), refs[2])
    check_against_oracle(o.contiguous(), q.contiguous(), k.contiguous(), v.contiguous(), None, layer.modes, layer.windows, n_text, n_img)
    rows = layer.joint[3].cpu().view(batch, -1, C)
    for part, x, w, g, got in zip((rows[:, :n_text], rows[:, n_text:]), layer.x, layer.w_out, layer.gate, layer.out):
        ref = O.linear(part, w.cpu(), gate=g.cpu(), residual=x.cpu())
        size = O.linear(part.abs(), w.cpu().abs(), gate=g.cpu().abs())
        check(got, ref, u * ref.abs() * 1.01 + (C + 4) * F32 * size + 4 * F32 * x.cpu().double().abs(), "output projection")


def test_a_captured_layer_is_replayed():
    with plan() as handle:
        layer = Layer(handle)
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        print("captured layer", flush=True)
        with torch.cuda.stream(stream):
            for _ in range(2):
                layer.run()
            stream.synchronize()
            want = [t.clone() for t in (layer.table, *layer.qkv, *layer.joint[:3])]
            with torch.cuda.graph(graph, stream=stream):
                layer.run()
            for turn in range(4):
                layer.poison()
                graph.replay()
                stream.synchronize()
                first = [t.clone() for t in layer.out]
                for w, t in zip(want, (layer.table, *layer.qkv, *layer.joint[:3])):
                    assert torch.equal(w, t), turn
                # the output projections of this very attention, eagerly
                rows = layer.joint[3].view(2, 189, 256)
                for part, x, w, g, y in zip((rows[:, :45], rows[:, 45:]), layer.x, layer.w_out, layer.gate, first):
                    eager = torch.empty_like(y)
                    B.difa_linear(handle, part, w, eager, gate=g, residual=x, workspace=layer.space)
                    assert torch.equal(eager, y), turn
                stream.synchronize()
        del graph


def test_a_captured_backward_is_replayed():
    heads, D, nt, ni = 4, 64, 33, 100
    with Plan(2, heads, D, max_tokens=nt + ni) as handle:
        xs = [randn(2, t, 3, heads, D, seed=i).cuda() for i, t in enumerate((nt, ni))]
        w = randn(D, seed=5, about=1.0).cuda()
        d = [randn(2, heads, nt + ni, D, seed=6 + i).cuda() for i in range(3)]
        space = torch.empty(B.difa_qk_norm_rotate_workspace(handle, nt, ni), dtype=torch.uint8, device="cuda")
        gx, gw = [torch.empty_like(x) for x in xs], torch.empty(2, 2, D, device="cuda")
        streams = [(x[:, :, 0], x[:, :, 1], x[:, :, 2], w, w) for x in xs]
        grads = [(g[:, :, 0], g[:, :, 1], g[:, :, 2], p[0], p[1]) for g, p in zip(gx, gw)]

        def call():
            B.difa_qk_norm_rotate_backward(handle, *streams, *d, *grads, workspace=space, eps=EPS)

        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            call()
            stream.synchronize()
            want = [t.clone() for t in (*gx, gw)]
            with torch.cuda.graph(graph, stream=stream):
                call()
            for turn in range(4):
                for t in (*gx, gw):
                    t.fill_(float("nan"))
                space.fill_(0xff)
                graph.replay()
                stream.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(want, (*gx, gw))), turn
                call()
                stream.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(want, (*gx, gw))), turn
        del graph
