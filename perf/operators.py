"""Workloads of the operators around the rectified MoE layer: the linear layer with its epilogue, dropout with a
counter-based mask, and the balance loss over all choices -- their plain forms in elementary torch operations, the
library's calls, and their values in 64 bits."""
import math

import torch

own = False  # True: run() calls the library; False: the plain form

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
INIT_STD = 0.02  # weights: N(0, 0.02), as everywhere in this repository


# ---- cases --------------------------------------------------------------------------------------------
def _linear(name, op, M, N, K, act, p=0.0, bias=True, residual=False, save=False, pad=0):
    c = {"op": op, "M": M, "N": N, "K": K, "act": act, "p": p, "bias": bias, "pad": pad}
    if op == "linear_fwd":
        c |= {"residual": residual, "save": save}
    return c | ({"name": name} if name else {})


def _dropout(name, op, rows, cols, p, x, y, residual=False):
    c = {"op": op, "rows": rows, "cols": cols, "p": p, "x": x, "y": y}
    if op == "dropout_fwd":
        c |= {"residual": residual}
    return c | ({"name": name} if name else {})


def _balance(name, op, segments, length, E, k, padded, garbage=False):
    c = {"op": op, "segments": segments, "length": length, "E": E, "k": k, "padded": padded, "garbage": garbage}
    return c | ({"name": name} if name else {})


def listed():
    return [
        # one token of a running generation through a d x d projection back into the residual stream (d = 4096)
        _linear("linear one token", "linear_fwd", 1, 4096, 4096, "none", residual=True),
        # an uneven batch of running generations through the up projection of a dense FFN
        _linear("linear 37 tokens", "linear_fwd", 37, 14336, 4096, "silu"),
        # a training micro-batch at d = 1024: FFN up projection with everything its epilogue does, pre-activations kept
        _linear("linear train", "linear_fwd", 2048, 4096, 1024, "gelu", p=0.1, residual=True, save=True),
        # the largest: 8 x 2048 tokens into the FFN width of the 7B layer
        _linear("linear prompt large", "linear_fwd", 16384, 14336, 4096, "gelu_tanh"),
        # gradients of the training micro-batch
        _linear("linear gradients", "linear_bwd", 2048, 4096, 1024, "gelu", p=0.1),
        # gradients with a ragged number of tokens, odd widths, a view of a wider buffer
        _linear("linear gradients ragged", "linear_bwd", 1501, 1416, 2056, "silu", pad=64),
        # gradients of an output projection over 8 x 2048 tokens at d = 4096
        _linear("linear gradients large", "linear_bwd", 16384, 4096, 4096, "none", p=0.1),
        # the residual branch behind the MoE layer for one odd-sized token batch
        _dropout("dropout small", "dropout_fwd", 5, 1023, 0.1, "f32", "bf16", residual=True),
        # the same for a full training batch: fp32 output of the expert layer onto the bf16 residual stream
        _dropout("dropout large", "dropout_fwd", 65536, 1024, 0.1, "f32", "bf16", residual=True),
        # the gradient of that branch, in the type that the expert layer's backward pass reads
        _dropout("dropout gradient", "dropout_bwd", 65536, 1024, 0.1, "bf16", "bf16"),
        # router of 64 experts, top-2, over a batch of 32 padded sequences of 2048
        _balance("balance loss", "balance_fwd", 32, 2048, 64, 2, 0.3, garbage=True),
        # its gradient
        _balance("balance gradient", "balance_bwd", 32, 2048, 64, 2, 0.3, garbage=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["linear_fwd", "linear_fwd", "linear_bwd", "linear_bwd", "dropout_fwd", "dropout_bwd", "balance_fwd", "balance_bwd"])
    if op.startswith("linear"):
        top = 16384 * 14336 * 4096 if op == "linear_fwd" else 16384 * 4096 * 4096
        while True:
            M, N, K = _log(rng, 1, 16384), 8 * _log(rng, 8, 1792), 8 * _log(rng, 8, 1792)
            if M * N * K <= top and max(M * N, M * K, N * K) <= 16384 * 14336:
                break
        return _linear("", op, M, N, K, rng.choice(ACTS), rng.choice([0.0, 0.0, 0.1, 0.25]), rng.random() < 0.7, rng.random() < 0.5, rng.random() < 0.5,
                       rng.choice([0, 0, 8, 64]))
    if op.startswith("dropout"):
        cols = _log(rng, 1, 8192)
        rows = _log(rng, 1, 65536 * 1024 // cols)
        return _dropout("", op, rows, cols, rng.choice([0.05, 0.1, 0.3, 0.5]), rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"]), rng.random() < 0.7)
    E = _log(rng, 2, 256)
    k = rng.randint(1, min(8, E))
    segments = _log(rng, 1, 64)
    length = _log(rng, 1, max(1, 65536 * 64 // (E * segments)))
    return _balance("", op, segments, length, E, k, rng.choice([0.0, 0.1, 0.5]), rng.random() < 0.5)


# ---- inputs -------------------------------------------------------------------------------------------
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    def view(rows, cols, **kw):  # `pad` more columns lie between the rows
        return normal(rows, cols + case["pad"], **kw)[:, :cols]

    op, s = case["op"], {"case": case}
    if op.startswith("linear"):
        M, N, K = case["M"], case["N"], case["K"]
        s |= {"x": view(M, K), "w": normal(N, K, std=INIT_STD), "bias": normal(N, std=0.1) if case["bias"] else None}
        if op == "linear_fwd":
            s["residual"] = view(M, N) if case["residual"] else None
        else:
            s["dy"] = view(M, N)
            s["z"] = view(M, N, std=INIT_STD * math.sqrt(K)) if case["act"] != "none" else None
    elif op.startswith("dropout"):
        s["x"] = normal(case["rows"], case["cols"], dtype=TYPES[case["x"]])
        s["residual"] = normal(case["rows"], case["cols"], dtype=TYPES[case["y"]]) if case.get("residual") else None
    else:
        S, L, E, k = case["segments"], case["length"], case["E"], case["k"]
        a = normal(S * L, E, dtype=torch.float32) + normal(E, std=0.8, dtype=torch.float32)  # some experts are in demand
        top = torch.topk(a, min(k + 1, E), dim=1).indices.int()  # the routing table [T, k+1]: choices by falling score, then the nominee
        if E == k:
            top = torch.cat([top, torch.full_like(top[:, :1], -1)], 1)
        live = torch.ones(S, L, dtype=torch.uint8, device="cuda")
        if case["padded"]:  # every sequence ends early by its own share; the last one may have no token at all
            end = (L * (1 - 2 * case["padded"] * torch.rand(S, generator=g, device="cuda"))).round().clamp(0, L)
            end[-1] = 0 if S > 1 else end[-1].clamp(min=1)
            live = (torch.arange(L, device="cuda")[None] < end[:, None]).to(torch.uint8)
        live = live.reshape(-1)
        if case["garbage"] and case["padded"]:  # nothing has cleared the rows behind the sequences
            a[live == 0] = float("nan")
        s |= {"logits": a, "topk": top.contiguous(), "live": live, "alpha": 1e-2, "beta": 1e-3}
        if op == "balance_bwd":
            m = live.view(S, L) != 0
            hit = (top[:, :k].long().view(S, L, k, 1) == torch.arange(E, device="cuda")) if S * L * k * E <= 1 << 26 else None
            if hit is not None:
                s["count"] = (hit & m[:, :, None, None]).sum((1, 2)).int()
            else:
                flat = torch.arange(S, device="cuda").view(S, 1, 1) * E + top[:, :k].long().view(S, L, k)
                s["count"] = torch.bincount(flat[m].reshape(-1), minlength=S * E).view(S, E).int()
            s["n"] = m.sum(1).int()
    if case.get("p"):
        s["rng"] = torch.randint(0, 1 << 62, (2,), generator=g, device="cuda")
    return s


# ---- the plain forms ------------------------------------------------------------------------------------
M32 = 0xFFFFFFFF


def _mask(rng, n, p):
    """keep[n] and the factor of what is kept: Philox4x32-10 on the counter (i / 8, offset) under the key `seed`; element i takes
    the i % 8-th 16-bit piece of the four words."""
    seed, offset = rng[0], rng[1]
    group = torch.arange((n + 7) // 8, device=rng.device)
    c = [group & M32, (group >> 32) & M32, (offset & M32).expand_as(group), ((offset >> 32) & M32).expand_as(group)]
    k0, k1 = seed & M32, (seed >> 32) & M32
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57  # 64-bit products: the wrapped sign bit does not matter below
        c = [((p1 >> 32) & M32) ^ c[1] ^ k0, p1 & M32, ((p0 >> 32) & M32) ^ c[3] ^ k1, p0 & M32]
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    pieces = torch.stack([c[0] & 0xFFFF, c[0] >> 16, c[1] & 0xFFFF, c[1] >> 16, c[2] & 0xFFFF, c[2] >> 16, c[3] & 0xFFFF, c[3] >> 16], 1)
    drop = int(round(p * 65536))
    return pieces.reshape(-1)[:n] >= drop, 65536 / (65536 - drop)


def _dropped(v, rng, p):
    if not p:
        return v
    keep, factor = _mask(rng, v.numel(), p)
    return torch.where(keep.view(v.shape), v * factor, torch.zeros_like(v))


def _act(z, act):
    if act == "none":
        return z
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z / (1 + torch.exp(-z))


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


def _plain(s):
    c = s["case"]
    op = c["op"]
    if op == "linear_fwd":
        z = s["x"].float() @ s["w"].float().T
        if s["bias"] is not None:
            z = z + s["bias"].float()
        y = _dropped(_act(z, c["act"]), s.get("rng"), c["p"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"y": y.bfloat16()} | ({"z": z.bfloat16()} if c["save"] else {})
    if op == "linear_bwd":
        dz = _dropped(s["dy"].float(), s.get("rng"), c["p"])
        if c["act"] != "none":
            dz = dz * _act_slope(s["z"].float(), c["act"])
        return {"dx": (dz @ s["w"].float()).bfloat16(), "dw": (dz.T @ s["x"].float()).bfloat16()} | ({"dbias": dz.sum(0)} if c["bias"] else {})
    if op.startswith("dropout"):
        y = _dropped(s["x"].float(), s["rng"], c["p"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return y.to(TYPES[c["y"]])
    S, L, E, k = c["segments"], c["length"], c["E"], c["k"]
    m = (s["live"] != 0).view(S, L, 1)
    a = torch.where(m, s["logits"].view(S, L, E), torch.zeros((), device="cuda"))
    top = a.amax(2, keepdim=True)
    e = torch.exp(a - top)
    total = e.sum(2, keepdim=True)
    g = torch.where(m, e / total, torch.zeros_like(e))
    lse = torch.where(m, torch.log(total) + top, torch.zeros_like(total))
    if op == "balance_fwd":
        n = m.sum((1, 2))
        hot = torch.zeros(S, L, E, dtype=torch.int32, device="cuda")
        hot.scatter_add_(2, s["topk"][:, :k].long().view(S, L, k), m.int().expand(S, L, k).contiguous())
        count = hot.sum(1).int()
        P = g.sum(1) / n.clamp(min=1)[:, None]
        f = count / (k * n.clamp(min=1))[:, None]
        segs = (n > 0).sum().clamp(min=1)
        loss = torch.stack([s["alpha"] * E * (f * P).sum() / segs, s["beta"] * (lse * lse).sum() / n.sum().clamp(min=1)])
        return {"loss": loss, "count": count, "n": n.int(), "P": P}
    n = s["n"]
    f = (s["count"] / (k * n.clamp(min=1))[:, None])[:, None]
    segs, tokens = (n > 0).sum().clamp(min=1), n.sum().clamp(min=1)
    from_balance = s["alpha"] * E / (segs * n.clamp(min=1))[:, None, None] * (f - (f * g).sum(2, keepdim=True))
    return (g * (from_balance + 2 * s["beta"] / tokens * lse)).view(S * L, E)


# ---- the library's calls ----------------------------------------------------------------------------------
def _library(s):
    import paper_2402_12399_b200 as rr
    c = s["case"]
    op = c["op"]
    if op.startswith("linear"):
        act = {"none": rr.ACT_NONE, "relu": rr.ACT_RELU, "gelu": rr.ACT_GELU, "gelu_tanh": rr.ACT_GELU_TANH, "silu": rr.ACT_SILU}[c["act"]]
        if "ws" not in s:  # kept by the program, as its output buffers are
            sizes = rr.linear_workspace_bytes(c["M"], c["N"], c["K"])
            s["ws"] = rr.alloc_workspace(sizes[0] if op == "linear_fwd" else sizes[1])
            empty = dict(dtype=torch.bfloat16, device="cuda")
            if op == "linear_fwd":
                s["y"] = torch.empty(c["M"], c["N"], **empty)
                s["z"] = torch.empty(c["M"], c["N"], **empty) if c["save"] else None
            else:
                s["dx"], s["dw"] = torch.empty(c["M"], c["K"], **empty), torch.empty(c["N"], c["K"], **empty)
                s["dbias"] = torch.empty(c["N"], dtype=torch.float32, device="cuda") if c["bias"] else None
        if op == "linear_fwd":
            rr.linear_fwd(s["x"], s["w"], s["bias"], s["residual"], act=act, p=c["p"], rng=s.get("rng"), out=s["y"], z=s["z"], workspace=s["ws"])
            return {"y": s["y"]} | ({"z": s["z"]} if c["save"] else {})
        rr.linear_bwd(s["dy"], s["x"], s["w"], s["z"], act=act, p=c["p"], rng=s.get("rng"), dx=s["dx"], dw=s["dw"], dbias=s["dbias"], workspace=s["ws"])
        return {"dx": s["dx"], "dw": s["dw"]} | ({"dbias": s["dbias"]} if c["bias"] else {})
    if op.startswith("dropout"):
        if "y" not in s:
            s["y"] = torch.empty(c["rows"], c["cols"], dtype=TYPES[c["y"]], device="cuda")
        if op == "dropout_fwd":
            return rr.dropout_fwd(s["x"], c["p"], s["rng"], residual=s["residual"], out=s["y"])
        return rr.dropout_bwd(s["x"], c["p"], s["rng"], out=s["y"])
    S, E, k = c["segments"], c["E"], c["k"]
    if op == "balance_fwd":
        if "ws" not in s:
            s["ws"] = rr.alloc_workspace(rr.balance_workspace_bytes(S * c["length"], E, S))
        loss, count, n, P = rr.balance_fwd(s["logits"], s["topk"], k, s["alpha"], s["beta"], segments=S, live=s["live"], workspace=s["ws"])
        return {"loss": loss, "count": count, "n": n, "P": P}
    return rr.balance_bwd(s["logits"], s["count"], s["n"], k, s["alpha"], s["beta"], live=s["live"])


def run(state):
    return _library(state) if own else _plain(state)


# ---- floors -----------------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op.startswith("linear"):
        M, N, K = case["M"], case["N"], case["K"]
        if op == "linear_fwd":
            values = M * K + N * K + M * N * (1 + case["residual"] + case["save"]) + N * case["bias"]
            return {"bytes": 2 * values, "flops": 2 * M * N * K}
        values = 2 * M * K + 2 * N * K + M * N * (1 + (case["act"] != "none"))
        return {"bytes": 2 * values + 4 * N * case["bias"], "flops": 4 * M * N * K}
    if op.startswith("dropout"):
        size = {"f32": 4, "bf16": 2}
        n = case["rows"] * case["cols"]
        return {"bytes": n * (size[case["x"]] + size[case["y"]] * (1 + bool(case.get("residual")))), "flops": 2 * n}
    S, T, E, k = case["segments"], case["segments"] * case["length"], case["E"], case["k"]
    if op == "balance_fwd":
        return {"bytes": 4 * T * E + 4 * T * k + T + 8 * S * E + 4 * S + 8, "flops": 5 * T * E}
    return {"bytes": 8 * T * E + T + 4 * S * E + 4 * S, "flops": 9 * T * E}


# ---- the same values from the definitions, in 64 bits -----------------------------------------------------
def _pieces64(rng, n):
    """The 16-bit pieces of elements 0..n-1, with 32-bit words held as two 16-bit halves (high, low) so that no product leaves 63 bits."""
    def word(v):
        return (v >> 16) & 0xFFFF, v & 0xFFFF

    def times(w, m):  # (high word, low word) of the 64-bit product of a word and a constant
        h, l = w
        mh, ml = m >> 16, m & 0xFFFF
        ll = l * ml
        mid = h * ml + (ll >> 16)
        cross = l * mh + (mid & 0xFFFF)
        high = h * mh + (mid >> 16) + (cross >> 16)
        return word(high), (cross & 0xFFFF, ll & 0xFFFF)

    seed, offset = (int(v) for v in rng.tolist())
    i = torch.arange((n + 7) // 8, device="cuda", dtype=torch.int64)
    zero = torch.zeros_like(i)
    x0, x1 = word(i % (1 << 32)), word(i // (1 << 32))
    x2, x3 = word(zero + offset % (1 << 32)), word(zero + (offset // (1 << 32)) % (1 << 32))
    for r in range(10):
        ka, kb = word((seed + r * 0x9E3779B9) % (1 << 32)), word(((seed >> 32) + r * 0xBB67AE85) % (1 << 32))
        ha, la = times(x0, 0xD2511F53)
        hb, lb = times(x2, 0xCD9E8D57)
        x0 = (hb[0] ^ x1[0] ^ ka[0], hb[1] ^ x1[1] ^ ka[1])
        x2 = (ha[0] ^ x3[0] ^ kb[0], ha[1] ^ x3[1] ^ kb[1])
        x1, x3 = lb, la
    both = torch.stack([x0[1], x0[0], x1[1], x1[0], x2[1], x2[0], x3[1], x3[0]], -1)
    return both.flatten()[:n]


def _factors64(rng, shape, p):
    """What dropout multiplies each element by: zero with probability p (to 16 bits), else the inverse of the share that is kept."""
    if not p:
        return 1.0
    out = round(65536 * p)
    return (_pieces64(rng, shape[0] * shape[1]) >= out).double().reshape(shape) / (1 - out / 65536)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    phi = lambda z: 0.5 * torch.special.erfc(-z / math.sqrt(2.0))  # noqa: E731  the normal distribution function
    if op.startswith("linear"):
        x, w = s["x"].double(), s["w"].double()
    if op == "linear_fwd":
        z = torch.einsum("mk,nk->mn", x, w)
        if case["bias"]:
            z += s["bias"].double()
        kinds = {"none": lambda: z, "relu": lambda: z.clamp(min=0), "gelu": lambda: z * phi(z), "silu": lambda: z * torch.sigmoid(z),
                 "gelu_tanh": lambda: z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))}
        y = kinds[case["act"]]() * _factors64(s.get("rng"), z.shape, case["p"])
        if case["residual"]:
            y = y + s["residual"].double()
        return {"y": y} | ({"z": z} if case["save"] else {})
    if op == "linear_bwd":
        dz = s["dy"].double() * _factors64(s.get("rng"), s["dy"].shape, case["p"])
        if case["act"] != "none":
            z = s["z"].double()
            if case["act"] == "relu":
                dz *= z > 0
            elif case["act"] == "gelu":
                dz *= phi(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
            else:  # both are z sigmoid(u(z))
                c = 2 * math.sqrt(2 / math.pi)
                u, slope = (z, 1.0) if case["act"] == "silu" else (c * (z + 0.044715 * z ** 3), c * (1 + 0.134145 * z ** 2))
                q = torch.sigmoid(u)
                dz *= q + z * slope * q * torch.sigmoid(-u)
        return {"dx": torch.einsum("mn,nk->mk", dz, w), "dw": torch.einsum("mn,mk->nk", dz, x)} | ({"dbias": dz.sum(0)} if case["bias"] else {})
    if op.startswith("dropout"):
        y = s["x"].double() * _factors64(s["rng"], s["x"].shape, case["p"])
        return y + s["residual"].double() if s["residual"] is not None else y
    S, L, E, k = case["segments"], case["length"], case["E"], case["k"]
    live = s["live"].bool()
    at = torch.arange(S, device="cuda").repeat_interleave(L)[live]  # segment of each live token
    a = s["logits"][live].double()
    lse = torch.logsumexp(a, 1)
    g = torch.softmax(a, 1)
    n = torch.bincount(at, minlength=S).double()
    per = torch.where(n > 0, 1 / n, 0.0)
    counts = torch.bincount((at[:, None] * E + s["topk"][live][:, :k].long()).flatten(), minlength=S * E).view(S, E)
    f = counts.double() / k * per[:, None]
    segs, tokens = max(1, int((n > 0).sum())), max(1, int(n.sum()))
    if op == "balance_fwd":
        P = torch.zeros(S, E, dtype=torch.float64, device="cuda").index_add_(0, at, g) * per[:, None]
        return {"loss": torch.stack([s["alpha"] * E * (f * P).sum() / segs, s["beta"] * lse.square().sum() / tokens]), "count": None, "n": None, "P": P}
    d = torch.zeros(S * L, E, dtype=torch.float64, device="cuda")
    fi = f[at]
    d[live] = g * (s["alpha"] * E / segs * per[at][:, None] * (fi - (fi * g).sum(1, keepdim=True)) + 2 * s["beta"] / tokens * lse[:, None])
    return d
