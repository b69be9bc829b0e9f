"""Plain 64-bit statements of the operators around the expert layer, for their tests: the dropout mask from the
published generator (NumPy integers), the linear layer and its gradients, the balance loss and its gradient."""
import math

import numpy as np
import torch


def philox4x32(counter, key, rounds=10):
    """Philox4x32 (Salmon et al., SC 2011) on arrays of 32-bit words held in uint64: four counter words, two key words."""
    c = [np.asarray(v, dtype=np.uint64) for v in counter]
    k = [np.uint64(v) for v in key]
    low, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> sh) ^ c[1] ^ k[0], b & low, (a >> sh) ^ c[3] ^ k[1], a & low]
        k = [(k[0] + np.uint64(0x9E3779B9)) & low, (k[1] + np.uint64(0xBB67AE85)) & low]
    return c


def keep_mask(seed, offset, first, n, p):
    """keep of the elements first .. first+n-1 and the factor of the kept ones, as include/rr.h defines them."""
    drop = int(math.floor(65536 * float(np.float32(p)) + 0.5))
    g = np.arange(first // 8, (first + n + 7) // 8, dtype=np.uint64)
    low, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    seed, offset = seed % (1 << 64), offset % (1 << 64)
    w = philox4x32([g & low, g >> sh, np.full_like(g, offset & 0xFFFFFFFF), np.full_like(g, offset >> 32)], [seed & 0xFFFFFFFF, seed >> 32])
    pieces = np.stack([h for v in w for h in (v & np.uint64(0xFFFF), v >> np.uint64(16))], 1).reshape(-1)
    at = first - 8 * (first // 8)
    return pieces[at:at + n] >= drop, (65536 / (65536 - drop) if drop < 65536 else 0.0)


def dropped(v, p, rng):
    """dropout of a float64 tensor (row-major index); rng: the device tensor {seed, offset}"""
    if rng is None or p == 0:
        return v
    keep, factor = keep_mask(int(rng[0]), int(rng[1]), 0, v.numel(), p)
    return torch.where(torch.from_numpy(keep).to(v.device).view(v.shape), v * factor, torch.zeros_like(v))


def act(z, a):
    if a == 1:
        return z.clamp(min=0)
    if a == 2:
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2))
    if a == 3:
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if a == 4:
        return z * torch.sigmoid(z)
    return z


def act_slope(z, a):
    if a == 1:
        return (z > 0).double()
    if a == 2:
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if a == 3:
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    if a == 4:
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def balance(a, topk, k, alpha, beta, S, live):
    """loss [2], count, n, P and the gradient of loss[0] + loss[1], token after token in float64 on the CPU."""
    T, E = a.shape
    a, L = a.double().cpu(), T // S
    live = torch.ones(T, dtype=torch.bool) if live is None else live.cpu() != 0
    topk = topk.cpu()
    count, n, P = torch.zeros(S, E, dtype=torch.int32), torch.zeros(S, dtype=torch.int32), torch.zeros(S, E, dtype=torch.float64)
    for s in range(S):
        m = live[s * L:(s + 1) * L]
        n[s] = int(m.sum())
        if n[s]:
            P[s] = torch.softmax(a[s * L:(s + 1) * L][m], 1).mean(0)
            count[s] = torch.bincount(topk[s * L:(s + 1) * L][m][:, :k].reshape(-1).long(), minlength=E).int()
    segs, tokens = max(1, int((n > 0).sum())), max(1, int(n.sum()))
    f = count.double() / (k * n.clamp(min=1))[:, None]
    z = torch.logsumexp(a[live], 1)
    loss = torch.stack([alpha * E / segs * (f * P).sum(), beta / tokens * (z * z).sum()])
    d = torch.zeros(T, E, dtype=torch.float64)
    at = torch.arange(T)[live] // max(L, 1)
    g = torch.softmax(a[live], 1)
    fi = f[at]
    d[live] = g * (alpha * E / (segs * n[at].double())[:, None] * (fi - (fi * g).sum(1, keepdim=True)) + 2 * beta / tokens * z[:, None])
    return loss, count, n, P, d
