"""Workloads of the rest of a training step around the rectified MoE layer: the norm with its residual add, the embedding, and the clip
of all gradients by their global norm -- their plain forms in elementary torch operations, the library's calls, and their values
in 64 bits."""
import math

import torch

own = False  # True: run() calls the library; False: the plain form

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


# ---- cases --------------------------------------------------------------------------------------------
def _named(name, c):
    return c | ({"name": name} if name else {})


def _norm(name, rows, cols, kind, x, y, h=None, w="bf16", bias=False, stats=False, pad=0):
    """h: the type of the residual stream that x is added to (None: no residual)."""
    return _named(name, {"op": "norm_fwd", "rows": rows, "cols": cols, "kind": kind, "x": x, "y": y, "h": h or "", "w": w, "bias": bias, "stats": stats,
                         "pad": pad})


def _norm_bwd(name, rows, cols, kind, dy, h, dx, through, w="bf16", bias=False, pad=0):
    """through: whether a gradient comes along the residual stream and is added."""
    return _named(name, {"op": "norm_bwd", "rows": rows, "cols": cols, "kind": kind, "dy": dy, "h": h, "dx": dx, "through": through, "w": w, "bias": bias,
                         "pad": pad})


def _embed(name, op, n, V, d, t, y, scale=1.0, padded=0.0, wide=False):
    """t: type of the table (forward) or of dy (backward); y: type of the result; wide: 64-bit ids."""
    return _named(name, {"op": op, "n": n, "V": V, "d": d, "t": t, "y": y, "scale": scale, "padded": padded, "wide": wide})


def _clip(name, blocks, E, d, d_ff, V, experts="f32", dense="f32", out="f32", flat=False, active=True):
    """Gradients of `blocks` blocks (four d x d projections, two norms, with E experts of width d_ff and their gate) and of an embedding
    of V rows.  flat: they lie back to back in one buffer per type.  active: the norm exceeds the bound; if not, in place."""
    return _named(name, {"op": "clip", "blocks": blocks, "E": E, "d": d, "d_ff": d_ff, "V": V, "experts": experts, "dense": dense, "out": out, "flat": flat,
                         "active": active})


def listed():
    return [
        # one token of a running generation: the branch's fp32 result joins the bf16 residual stream and is normed for the next one
        _norm("norm one token", 1, 4096, "rms", "f32", "bf16", h="bf16"),
        # odd widths and a ragged number of tokens, layer norm with bias
        _norm("norm ragged", 1501, 1023, "layer", "bf16", "f32", w="f32", bias=True, stats=True),
        # a training batch of 4 x 4096 tokens at d = 4096: the expert layer's fp32 output onto the residual stream, statistics kept
        _norm("norm add large", 16384, 4096, "rms", "f32", "bf16", h="bf16", stats=True),
        # gradients of a training micro-batch at d = 1024, rows in a wider buffer
        _norm_bwd("norm gradients", 2048, 1024, "layer", "bf16", "bf16", "bf16", False, bias=True, pad=64),
        # gradients at d = 4096, joined with what comes along the residual stream
        _norm_bwd("norm gradients large", 16384, 4096, "rms", "bf16", "bf16", "bf16", True),
        # the last tokens of an uneven batch of running generations
        _embed("embed 37 tokens", "embed_fwd", 37, 32000, 4096, "bf16", "bf16"),
        # 32 padded sequences of 2048 into d = 1024, scaled by sqrt(d)
        _embed("embed prompt", "embed_fwd", 65536, 32000, 1024, "bf16", "bf16", scale=32.0, padded=0.3, wide=True),
        # gradient of a small model's table, odd sizes
        _embed("embed gradients ragged", "embed_bwd", 1501, 9973, 1000, "f32", "bf16", scale=0.5, padded=0.1),
        # gradient of a 7B-width table over 4 x 4096 tokens of text (a few tokens are most of it)
        _embed("embed gradients large", "embed_bwd", 16384, 32000, 4096, "bf16", "f32", wide=True),
        # the gradients of two small dense blocks
        _clip("clip small", 2, 0, 256, 0, 0),
        # a flattened buffer with odd sizes, experts in fp32, the rest in bf16; the norm stays below the bound
        _clip("clip idle ragged", 3, 5, 333, 777, 4001, dense="bf16", flat=True, active=False),
        # one layer of 64 experts at d = 1024 with its block and the table
        _clip("clip large", 1, 64, 1024, 2816, 32000),
    ]


MOST_CLIP = 64 * 3 * 1024 * 2816


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _round(rng, v, lo=1):
    """widths are multiples of 8 more often than not"""
    return max(lo, v) if rng.random() < 0.3 else max(8, v // 8 * 8)


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_fwd", "norm_bwd", "norm_bwd", "embed_fwd", "embed_bwd", "embed_bwd", "clip", "clip"])
    two = lambda: rng.choice(["f32", "bf16"])  # noqa: E731
    if op.startswith("norm"):
        cols = _round(rng, _log(rng, 1, 16384))
        rows = _log(rng, 1, min(65536, 16384 * 4096 // cols))
        kind, pad = rng.choice(["layer", "rms"]), rng.choice([0, 0, 0, 64])
        bias = kind == "layer" and rng.random() < 0.8
        if op == "norm_fwd":
            return _norm("", rows, cols, kind, two(), two(), rng.choice([None, "f32", "bf16"]), two(), bias, rng.random() < 0.6, pad)
        return _norm_bwd("", rows, cols, kind, two(), two(), two(), rng.random() < 0.5, two(), bias, pad)
    if op.startswith("embed"):
        while True:
            n, V, d = _log(rng, 1, 65536), _log(rng, 2, 262144), _round(rng, _log(rng, 1, 8192))
            if n * d <= 65536 * 1024 and V * d <= 32000 * 4096:
                return _embed("", op, n, V, d, two(), two(), rng.choice([1.0, 1.0, 0.5, 32.0]), rng.choice([0.0, 0.1, 0.3]), rng.random() < 0.5)
    while True:
        E, d, f, V, blocks = rng.choice([0, _log(rng, 1, 64)]), _log(rng, 8, 4096), _log(rng, 8, 8192), rng.choice([0, _log(rng, 8, 64000)]), _log(rng, 1, 16)
        if blocks * (3 * E * d * f + E * d + 4 * d * d) + V * d <= MOST_CLIP:
            active = rng.random() < 0.7
            return _clip("", blocks, E, d, f, V, two(), two(), two(), rng.random() < 0.4, active)


# ---- inputs -------------------------------------------------------------------------------------------
def _ids(g, case):
    """Token ids as text has them: the r-th most frequent of V has probability ~ 1 / (r + 2.7); -1 where a sequence has ended."""
    n, V = case["n"], case["V"]
    weight = torch.cumsum(1 / (torch.arange(V, device="cuda", dtype=torch.float64) + 2.7), 0)
    rank = torch.searchsorted(weight, torch.rand(n, generator=g, device="cuda", dtype=torch.float64) * weight[-1]).clamp(max=V - 1)
    ids = torch.randperm(V, generator=g, device="cuda")[rank]
    if case["padded"]:
        length = max(1, min(2048, n // 2))
        end = length * (1 - 2 * case["padded"] * torch.rand(-(-n // length), generator=g, device="cuda"))
        at = torch.arange(n, device="cuda")
        ids = torch.where(at % length < end[at // length], ids, torch.full_like(ids, -1))
    return ids if case["wide"] else ids.int()


def _shapes(c):
    """(shape, type) of every gradient"""
    out = []
    d, f, E = c["d"], c["d_ff"], c["E"]
    if c["V"]:
        out.append(((c["V"], d), c["dense"]))
    for _ in range(c["blocks"]):
        out += [((d,), c["dense"])] + [((d, d), c["dense"])] * 4 + [((d,), c["dense"])]
        if E:
            out += [((E, d), "f32"), ((E, f, d), c["experts"]), ((E, f, d), c["experts"]), ((E, d, f), c["experts"])]
    return out


def _elements(c):
    return [(math.prod(s), t) for s, t in _shapes(c)]


def _buffers(shapes, flat):
    """uninitialised tensors of these (shape, type), one after the other in one buffer per type or each by itself"""
    if not flat:
        return [torch.empty(s, dtype=TYPES[t], device="cuda") for s, t in shapes]
    whole = {k: torch.empty(sum(math.prod(s) for s, t in shapes if t == k), dtype=TYPES[k], device="cuda") for k in TYPES}
    at, out = dict.fromkeys(TYPES, 0), []
    for s, t in shapes:
        n = math.prod(s)
        out.append(whole[t][at[t]:at[t] + n].view(s))
        at[t] += n
    return out


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)

    def normal(*shape, std=1.0, t="bf16"):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(TYPES[t])

    def view(rows, cols, **kw):  # `pad` more columns lie between the rows
        return normal(rows, cols + case["pad"], **kw)[:, :cols]

    op, s = case["op"], {"case": case}
    if op.startswith("norm"):
        M, N = case["rows"], case["cols"]
        s["w"] = (1 + 0.1 * torch.randn(N, generator=g, device="cuda")).to(TYPES[case["w"]])
        s["b"] = normal(N, std=0.1, t=case["w"]) if case["bias"] else None
        # a residual stream: a few channels are far larger than the rest and off centre
        loud = (torch.rand(N, generator=g, device="cuda") < 0.01).float() * 20

        def stream(t):
            wide = torch.randn(M, N + case["pad"], generator=g, device="cuda")
            wide[:, :N] += loud
            return wide.to(TYPES[t])[:, :N]
        if op == "norm_fwd":
            s["x"] = view(M, N, t=case["x"]) if case["h"] else stream(case["x"])
            s["residual"] = stream(case["h"]) if case["h"] else None
            return s
        s["dy"], s["h"] = view(M, N, t=case["dy"]), stream(case["h"])
        s["dh"] = view(M, N, t=case["dx"]) if case["through"] else None
        h = s["h"].double()
        mean = h.mean(1) if case["kind"] == "layer" else torch.zeros(M, device="cuda", dtype=torch.float64)
        s["mean"] = mean.float() if case["kind"] == "layer" else None
        s["rstd"] = torch.rsqrt((h - mean[:, None]).square().mean(1) + EPS).float()
    elif op == "embed_fwd":
        s["ids"], s["table"] = _ids(g, case), normal(case["V"], case["d"], std=0.02, t=case["t"])
    elif op == "embed_bwd":
        s["ids"], s["dy"] = _ids(g, case), normal(case["n"], case["d"], t=case["t"])
    else:
        shapes = _shapes(case)
        s["grads"] = _buffers(shapes, case["flat"])
        for t in s["grads"]:  # every matrix has its own size of gradient
            t.copy_(torch.randn(t.shape, generator=g, device="cuda") * (0.01 * float(torch.rand(1, generator=g, device="cuda"))))
        total = math.sqrt(sum(float(t.float().square().sum(dtype=torch.float64)) for t in s["grads"]))
        s["bound"] = total / 3 if case["active"] else 2 * total
        s["out"] = _buffers([(sh, case["out"]) for sh, _ in shapes], case["flat"]) if case["active"] else None
    return s


# ---- the plain forms ------------------------------------------------------------------------------------
def _plain(s):
    c = s["case"]
    op = c["op"]
    if op == "norm_fwd":
        h, out = s["x"].float(), {}
        if c["h"]:
            out["h"] = (h + s["residual"].float()).to(TYPES[c["h"]])
            h = out["h"].float()
        mean = h.mean(1, keepdim=True) if c["kind"] == "layer" else torch.zeros(c["rows"], 1, device="cuda")
        v = h - mean
        rstd = 1 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
        y = v * rstd * s["w"].float()
        out["y"] = (y + s["b"].float() if c["bias"] else y).to(TYPES[c["y"]])
        if c["stats"]:
            out["rstd"] = rstd[:, 0]
            if c["kind"] == "layer":
                out["mean"] = mean[:, 0]
        return out
    if op == "norm_bwd":
        dy, v = s["dy"].float(), s["h"].float()
        if c["kind"] == "layer":
            v = v - s["mean"][:, None]
        xh = v * s["rstd"][:, None]
        g = dy * s["w"].float()
        d = g - xh * (g * xh).mean(1, keepdim=True)
        if c["kind"] == "layer":
            d = d - g.mean(1, keepdim=True)
        dx = d * s["rstd"][:, None]
        if c["through"]:
            dx = dx + s["dh"].float()
        return {"dx": dx.to(TYPES[c["dx"]]), "dw": (dy * xh).sum(0)} | ({"db": dy.sum(0)} if c["bias"] else {})
    if op == "embed_fwd":
        ids = s["ids"].long()
        y = s["table"][ids.clamp(min=0)].float() * c["scale"]
        return torch.where((ids >= 0)[:, None], y, torch.zeros((), device="cuda")).to(TYPES[c["y"]])
    if op == "embed_bwd":
        ids = s["ids"].long()
        dy = torch.where((ids >= 0)[:, None], s["dy"].float(), torch.zeros((), device="cuda"))
        return (torch.zeros(c["V"], c["d"], device="cuda").index_add_(0, ids.clamp(min=0), dy) * c["scale"]).to(TYPES[c["y"]])
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    for t in s["grads"]:
        total = total + t.float().square().sum(dtype=torch.float64)
    norm = total.sqrt()
    factor = (s["bound"] / (norm + 1e-6)).clamp(max=1).float()
    if c["active"]:
        out = [t.copy_(g.float() * factor) for t, g in zip(s["out"], s["grads"])]
    else:
        out = [t.copy_(t.float() * factor) for t in s["grads"]]
    return {"norm": torch.stack([norm.float(), factor]), "grads": out}


# ---- the library's calls ----------------------------------------------------------------------------------
def _library(s):
    import paper_2402_12399_b200 as rr
    c = s["case"]
    op = c["op"]

    def empty(*shape, t="f32"):
        return torch.empty(*shape, dtype=TYPES[t], device="cuda")
    first = "out" not in s and "plan" not in s  # buffers, workspace and plan are kept by the program
    kind = {"layer": rr.NORM_LAYER, "rms": rr.NORM_RMS}[c["kind"]] if op.startswith("norm") else None
    if op == "norm_fwd":
        M, N = c["rows"], c["cols"]
        if first:
            layer = c["kind"] == "layer"
            s["out"] = {"y": empty(M, N, t=c["y"])} | ({"h": empty(M, N, t=c["h"])} if c["h"] else {})
            s["out"] |= ({"rstd": empty(M)} | ({"mean": empty(M)} if layer else {})) if c["stats"] else {}
        o = s["out"]
        rr.norm_fwd(s["x"], s["w"], s["b"], residual=s["residual"], kind=kind, eps=EPS, out=o["y"], h=o.get("h"), mean=o.get("mean"), rstd=o.get("rstd"))
        return o
    if op == "norm_bwd":
        M, N = c["rows"], c["cols"]
        if first:
            s["ws"] = rr.alloc_workspace(rr.norm_workspace_bytes(M, N))
            s["out"] = {"dx": empty(M, N, t=c["dx"]), "dw": empty(N)} | ({"db": empty(N)} if c["bias"] else {})
        o = s["out"]
        rr.norm_bwd(s["dy"], s["h"], s["w"], s["mean"], s["rstd"], kind=kind, dh=s["dh"], dx=o["dx"], dw=o["dw"], dbias=o.get("db"), workspace=s["ws"])
        return o
    if op == "embed_fwd":
        if first:
            s["ws"] = rr.alloc_workspace(rr.embed_workspace_bytes(c["n"], c["V"], c["d"])[0])
            s["out"] = empty(c["n"], c["d"], t=c["y"])
        return rr.embed_fwd(s["ids"], s["table"], scale=c["scale"], out=s["out"], workspace=s["ws"])
    if op == "embed_bwd":
        if first:
            s["ws"] = rr.alloc_workspace(rr.embed_workspace_bytes(c["n"], c["V"], c["d"])[1])
            s["out"] = empty(c["V"], c["d"], t=c["y"])
        return rr.embed_bwd(s["ids"], s["dy"], s["out"], scale=c["scale"], workspace=s["ws"])
    if "plan" not in s:
        s["plan"] = rr.grad_plan(s["grads"], out=s["out"])
        s["ws"] = rr.alloc_workspace(rr.clip_workspace_bytes())
        s["norm"] = empty(2)
    rr.clip_grads(s["plan"], s["bound"], norm=s["norm"], workspace=s["ws"])
    return {"norm": s["norm"], "grads": s["out"] if c["active"] else s["grads"]}


def run(state):
    return _library(state) if own else _plain(state)


# ---- floors -----------------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op.startswith("norm"):
        n, rows = case["rows"] * case["cols"], case["rows"]
        params = SIZE[case["w"]] * case["cols"] * (1 + case["bias"])
        if op == "norm_fwd":
            stats = 4 * rows * (1 + (case["kind"] == "layer")) if case["stats"] else 0
            return {"bytes": n * (SIZE[case["x"]] + SIZE[case["y"]] + (2 * SIZE[case["h"]] if case["h"] else 0)) + params + stats, "flops": 8 * n}
        values = n * (SIZE[case["dy"]] + SIZE[case["h"]] + SIZE[case["dx"]] * (1 + case["through"]))
        weight = SIZE[case["w"]] * case["cols"]
        return {"bytes": values + weight + 4 * case["cols"] * (1 + case["bias"]) + 4 * rows * (1 + (case["kind"] == "layer")), "flops": 14 * n}
    if op.startswith("embed"):
        n, V, d, wide = case["n"], case["V"], case["d"], 8 if case["wide"] else 4
        if op == "embed_fwd":  # rows are named more than once: the expected number of different ones
            total = math.log((V + 2.7) / 2.7)
            seen, r = 0.0, 0
            while r < V:  # in strides that grow with the rank
                step = max(1, r // 64)
                m = min(step, V - r)
                seen += m * -math.expm1(-(1 - case["padded"]) * n / ((r + m / 2 + 2.2) * total))
                r += m
            return {"bytes": int(n * wide + n * d * SIZE[case["y"]] + min(seen, n) * d * SIZE[case["t"]]), "flops": n * d}
        return {"bytes": int(n * wide + (1 - case["padded"]) * n * d * SIZE[case["t"]] + V * d * SIZE[case["y"]]), "flops": n * d}
    elements = _elements(case)
    read = sum(n * SIZE[t] for n, t in elements)
    total = sum(n for n, _ in elements)
    return {"bytes": read + (total * SIZE[case["out"]] if case["active"] else 0) + 8, "flops": 3 * total}


# ---- the same values from the definitions, in 64 bits -----------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("norm"):
        w, layer = s["w"].double(), case["kind"] == "layer"
    if op == "norm_fwd":
        out = {}
        a = s["x"].double()
        if case["h"]:
            a = a + s["residual"].double()
            out["h"] = a
            a = a.to(TYPES[case["h"]]).double()  # the norm is that of the stream as it is stored
        N = case["cols"]
        first = a.sum(1) / N if layer else torch.zeros(case["rows"], device="cuda", dtype=torch.float64)
        spread = torch.einsum("mn,mn->m", a - first[:, None], a - first[:, None]) / N
        r = torch.rsqrt(spread + EPS)
        y = torch.einsum("mn,m,n->mn", a - first[:, None], r, w)
        out["y"] = y + s["b"].double() if case["bias"] else y
        if case["stats"]:
            out["rstd"] = r
            if layer:
                out["mean"] = first
        return out
    if op == "norm_bwd":
        dy, r, N = s["dy"].double(), s["rstd"].double(), case["cols"]
        centred = s["h"].double() - (s["mean"].double()[:, None] if layer else 0)
        along = torch.einsum("mn,n,mn->m", dy, w, centred)  # the part of w dy along the row itself
        dx = r[:, None] * (dy * w) - (r ** 3 * along / N)[:, None] * centred
        if layer:
            dx = dx - (r * (dy @ w) / N)[:, None]
        out = {"dx": dx + s["dh"].double() if case["through"] else dx, "dw": torch.einsum("mn,mn,m->n", dy, centred, r)}
        return out | ({"db": dy.sum(0)} if case["bias"] else {})
    if op.startswith("embed"):
        live = s["ids"] >= 0
        ids = s["ids"][live].long()
        if op == "embed_fwd":
            y = torch.zeros(case["n"], case["d"], dtype=torch.float64, device="cuda")
            y[live] = case["scale"] * s["table"].double()[ids]
            return y
        d = torch.zeros(case["V"], case["d"], dtype=torch.float64, device="cuda")
        return d.index_add_(0, ids, s["dy"][live].double(), alpha=case["scale"])
    norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(t, dtype=torch.float64)) ** 2 for t in s["grads"]))
    factor = min(1.0, s["bound"] / (norm + 1e-6))
    return {"norm": torch.tensor([norm, factor], dtype=torch.float64, device="cuda"), "grads": [t.double() * factor for t in s["grads"]]}
