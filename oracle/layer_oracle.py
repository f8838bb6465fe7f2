"""Plain 64-bit CPU forms of the operators around a layer's joint attention: rotary positions, head norms with the
rotation and their gradients, the matrix product with its epilogue.  Shares no code with the library.

Joint tensors are [B, H, N, D]; streams are [B, T, H, D].
"""
import math

import torch


def rope_table(positions, dims, theta, D):
    """[rows, D / 2, 2]: cosine and sine of every pair."""
    pos = positions.double()
    out = torch.zeros(pos.shape[0], D // 2, 2, dtype=torch.float64)
    out[:, :, 0] = 1.0
    p = 0
    for a, d in enumerate(dims):
        for j in range(d // 2):
            angle = pos[:, a] * float(theta) ** (-2.0 * j / d)
            out[:, p, 0], out[:, p, 1] = torch.cos(angle), torch.sin(angle)
            p += 1
    return out


def pair_features(D, halves):
    """Features (first, second) of every pair."""
    p = torch.arange(D // 2)
    return (p, p + D // 2) if halves else (2 * p, 2 * p + 1)


def rotate(x, table, halves=False, inverse=False):
    """x [B, H, N, D] turned by table [N, D / 2, 2] or [B, N, D / 2, 2]."""
    x, t = x.double(), table.double()
    t = t[None, None] if t.dim() == 3 else t[:, None]
    c, s = t[..., 0], t[..., 1] * (-1 if inverse else 1)
    first, second = pair_features(x.shape[-1], halves)
    out = torch.empty_like(x)
    out[..., first] = x[..., first] * c - x[..., second] * s
    out[..., second] = x[..., first] * s + x[..., second] * c
    return out


def norm(x, w, eps):
    x = x.double()
    n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    return n if w is None else n * w.double()


def joined(text, image, image_first):
    """Streams [B, T, H, D] (either may be None) as the joint [B, H, N, D]."""
    parts = [p for p in ((image, text) if image_first else (text, image)) if p is not None]
    return torch.cat(parts, dim=1).transpose(1, 2)


def qk_norm_rotate(text, image, table, eps, image_first=False, halves=False):
    """text, image: (q, k, v, q_weight, k_weight) or None.  Returns joint q, k, v."""
    outs = []
    for i in (0, 1):
        parts = [None if s is None else norm(s[i], s[3 + i], eps) for s in (text, image)]
        x = joined(*parts, image_first)
        outs.append(x if table is None else rotate(x, table, halves))
    v = joined(*(None if s is None else s[2].double() for s in (text, image)), image_first)
    return outs[0], outs[1], v


def qk_norm_rotate_backward(text, image, table, eps, dq, dk, dv, image_first=False, halves=False):
    """Gradients as the formulas give them: per stream (dq, dk, dv, dq_weight, dk_weight), None for one that is absent."""
    n_text = 0 if text is None else text[0].shape[1]
    n_img = 0 if image is None else image[0].shape[1]
    d = [g.double() if table is None else rotate(g, table, halves, inverse=True) for g in (dq, dk)] + [dv.double()]
    got = []
    for s, begin, count in ((text, n_img if image_first else 0, n_text), (image, 0 if image_first else n_text, n_img)):
        if s is None:
            got.append(None)
            continue
        mine = [g[:, :, begin:begin + count].transpose(1, 2) for g in d]
        dx, dw = [], []
        for i in (0, 1):
            x, w = s[i].double(), s[3 + i]
            r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
            n, g = x * r, mine[i] if w is None else mine[i] * w.double()
            dx.append(r * (g - n * (g * n).mean(-1, keepdim=True)))
            dw.append((mine[i] * n).sum(dim=(0, 1, 2)))
        got.append((dx[0], dx[1], mine[2], dw[0], dw[1]))
    return got


def activation(y, act):
    if act == "gelu_tanh":
        return 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
    if act == "gelu_erf":
        return 0.5 * y * (1 + torch.erf(y / math.sqrt(2)))
    if act == "silu":
        return y / (1 + torch.exp(-y))
    return y


def linear(x, w, bias=None, act="none", gate=None, residual=None):
    """x [B, T, K], w [N, K], bias [N], gate [B, N], residual [B, T, N]."""
    y = x.double() @ w.double().t()
    if bias is not None:
        y = y + bias.double()
    y = activation(y, act)
    if gate is not None:
        y = y * gate.double()[:, None]
    return y if residual is None else y + residual.double()
