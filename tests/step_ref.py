"""Plain 64-bit statements of the norm, the embedding and the clip, for their tests."""
import torch


def norm(h, w, b, layer, eps):
    """y, mean, rstd and the normed rows without weight and bias, of what the norm is taken of."""
    h = h.double()
    mean = h.mean(1) if layer else torch.zeros(h.shape[0], dtype=torch.float64, device=h.device)
    v = h - mean[:, None]
    rstd = 1 / torch.sqrt((v * v).mean(1) + eps)
    xh = v * rstd[:, None]
    y = xh if w is None else xh * w.double()
    return y if b is None else y + b.double(), mean, rstd, xh


def norm_gradients(dy, h, w, mean, rstd, dh):
    """dx, dw, db and the magnitudes behind dx and dw, from the statistics as they were kept (mean None: RMS norm)."""
    dy, v, r = dy.double(), h.double(), rstd.double()[:, None]
    xh = (v if mean is None else v - mean.double()[:, None]) * r
    g = dy if w is None else dy * w.double()
    c2 = (g * xh).mean(1, keepdim=True)
    d = g - xh * c2
    size = g.abs() + xh.abs() * (g * xh).abs().mean(1, keepdim=True)
    if mean is not None:
        d = d - g.mean(1, keepdim=True)
        size = size + g.abs().mean(1, keepdim=True)
    dx = d * r if dh is None else d * r + dh.double()
    return dx, (dy * xh).sum(0), dy.sum(0), size * r, (dy * xh).abs().sum(0), dy.abs().sum(0)


def embed(ids, table, scale):
    live = (ids >= 0) & (ids < table.shape[0])
    y = table.double()[torch.where(live, ids, torch.zeros_like(ids)).long()] * scale
    return torch.where(live[:, None], y, torch.zeros_like(y))


def embed_gradient(ids, dy, V, scale):
    """dtable and the sum of the magnitudes, of the tokens that have an id"""
    live = (ids >= 0) & (ids < V)
    at, d = ids[live].long(), dy[live].double()
    zero = torch.zeros(V, dy.shape[1], dtype=torch.float64, device=dy.device)
    return zero.clone().index_add_(0, at, d) * scale, zero.index_add_(0, at, d.abs()) * abs(scale)


def clip(grads, bound):
    bound = float(torch.tensor(bound, dtype=torch.float32))      # the entry point takes it in fp32: 1e-40 is 71362 2^-149 there, 5e-6 of it less
    norm = sum(float((g.double() ** 2).sum()) for g in grads) ** 0.5
    return norm, min(1.0, bound / (norm + 1e-6))
