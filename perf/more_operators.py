"""Operators that a model of tokens needs before, between and after its layers, as cases that can be timed:

  embed       rows of an embedding table for given tokens, times a scale
  embed_grad  the gradient of that table: the gradients of all places where a token stands, added; or added to a gradient that is there
  norm        layer norm with the statistics that its gradient needs
  norm_grad   gradients of the input, of the weight and of the bias
  orth        a matrix of update directions made orthogonal by Newton-Schulz steps: every singular value is brought near 1
  muon        an optimiser's step over many matrices: momentum, orthogonal directions, weight decay and update

The plain forms below are elementary torch operations in 32 bits; with `own` the calls of paper_1512_01274_amd.mxc run.
"""
import math

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": 0, "bf16": 1}        # MXC_F32, MXC_BF16
SIZE = {"f32": 4, "bf16": 2}


def _embed(name, kind, N, V, C, dtype, add=False):
    """N tokens of a vocabulary of V, rows of C values; add: the gradient is added to one that is there (of a table that is also the last layer)."""
    return {"name": name, "kind": kind, "N": N, "V": V, "C": C, "dtype": dtype, "add": add}


def _norm(name, kind, N, C, dtype, affine=True):
    return {"name": name, "kind": kind, "N": N, "C": C, "dtype": dtype, "affine": affine}


def _matrices(name, kind, shapes, dtype, steps=5, nesterov=True, copy=False):
    """shapes: rows x columns of each matrix, with *n for n of them; copy: a bf16 copy of the weights too."""
    return {"name": name, "kind": kind, "shapes": shapes, "dtype": dtype, "steps": steps, "nesterov": nesterov, "copy": copy}


def listed():
    return [
        # a step of decoding for 64 sequences: latency
        _embed("embed_token", "embed", 64, 131072, 4096, "bf16"),
        # prompts of 16384 tokens in all: a row read and a row written for each
        _embed("embed_prompt", "embed", 16384, 50257, 4096, "bf16"),
        # a small batch on a table that is also the last layer: a few hundred rows of a gradient that is there
        _embed("embed_grad_tied", "embed_grad", 500, 1000, 512, "f32", True),
        # a training step's text: common tokens stand in it by the thousand, most of the vocabulary does not
        _embed("embed_grad_text", "embed_grad", 32768, 50257, 2048, "bf16"),
        # one token of one sequence: latency
        _norm("norm_token", "norm", 1, 4096, "bf16"),
        # prompts of 16384 tokens
        _norm("norm_prompt", "norm", 16384, 4096, "bf16"),
        # a classifier's batch, microseconds of work
        _norm("norm_grad_classes", "norm_grad", 128, 1000, "f32"),
        # a training step's text, rows of an odd length
        _norm("norm_grad_text", "norm_grad", 16383, 4097, "bf16"),
        # the filter of an image network's first layer, 64 x (3 * 11 * 11): latency
        _matrices("orth_filter", "orth", "64x363", "f32"),
        # a square layer of 8192: the matrix cores' work
        _matrices("orth_large", "orth", "8192x8192", "bf16"),
        # a residual network's 42 filters, each some microseconds of work
        _matrices("muon_deep", "muon", "64x64,256x64*8,64x256*5,64x576*6,512x256,128x512*8,128x1152*7,512x128*6", "bf16"),
        # an image network's filters and the three layers of its head
        _matrices("muon_stack", "muon", "64x363,192x1600,384x1728,256x3456,256x2304,4096x9216,4096x4096,1000x4096", "f32", copy=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "embed_grad", "norm", "norm_grad", "norm_grad", "orth", "muon"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("embed", "embed_grad"):
        C = _log(rng, 1, 8192)
        if rng.random() < 0.5:
            C = -(-C // 8) * 8
        V = _log(rng, 2, min(131072, 50257 * 2048 // C))
        c = _embed("", kind, _log(rng, 1, min(65536, 16384 * 4096 * 2 // (C * SIZE[dtype]))), V, C, dtype, kind == "embed_grad" and rng.random() < 0.5)
    elif kind in ("norm", "norm_grad"):
        C = _log(rng, 4, 16384)         # of two values a norm leaves a sign alone, and of the gradient its rounding errors
        if rng.random() < 0.5:
            C = -(-C // 8) * 8
        c = _norm("", kind, _log(rng, 1, min(65536, 16384 * 4096 * 2 // (C * SIZE[dtype]))), C, dtype, rng.random() < 0.8)
    else:
        shapes, left = [], 8192.0 ** 3 / 4
        for _ in range(rng.choice([1, 1, _log(rng, 1, 12)])):
            r, k = _log(rng, 1, 8192), _log(rng, 1, 8192)
            if rng.random() < 0.5:
                r, k = -(-r // 64) * 64, -(-k // 64) * 64
            cost = float(r) * k * min(r, k)
            if cost > left:
                continue
            n = 1 if rng.random() < 0.6 else _log(rng, 1, min(16, max(1, left / cost)))
            left -= cost * n
            shapes.append(f"{r}x{k}" + (f"*{n}" if n > 1 else ""))
        c = _matrices("", kind, ",".join(shapes) or "100x300", dtype, rng.choice([5, 5, 4, 6]), rng.random() < 0.7, kind == "muon" and rng.random() < 0.5)
    c.pop("name", None)
    return c


# ---- inputs ----------------------------------------------------------------------------------------------------------------

def _shapes(case):
    out = []
    for part in case["shapes"].split(","):
        size, _, n = part.partition("*")
        r, c = size.split("x")
        out += [(int(r), int(c))] * int(n or 1)
    return out


def _buffer(case, dtype):
    """One buffer for all matrices of a case, each on a whole 512 values with zeros behind it, and the matrices in it."""
    at, views = 0, []
    for r, c in _shapes(case):
        views.append((at, r, c))
        at += -(-r * c // 512) * 512
    flat = torch.zeros(at, dtype=dtype, device="cuda")
    return flat, [flat[a:a + r * c].view(r, c) for a, r, c in views]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    new = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    s, kind, dtype = {"case": case}, case["kind"], DTYPE[case["dtype"]]
    if kind in ("embed", "embed_grad"):
        N, V, C = case["N"], case["V"], case["C"]
        # the k-th most common token is as common as 1 / k has it; a few places are padding, which has no token
        tokens = torch.exp(torch.rand(N, generator=gen, device="cuda") * math.log(V + 1.0)).long() - 1
        tokens[torch.rand(N, generator=gen, device="cuda") < 0.03] = -1
        s["tokens"], s["scale"] = tokens.clamp_(-1, V - 1).int(), math.sqrt(C)
        if kind == "embed":
            s["w"], s["y"] = (rand(V, C) * 0.02).to(dtype), new(N, C, dtype=dtype)
        else:
            s["dy"] = (rand(N, C) * 1e-3).to(dtype)
            s["dw"] = rand(V, C) * 1e-3 if case["add"] else new(V, C)
    elif kind in ("norm", "norm_grad"):
        N, C = case["N"], case["C"]
        x = rand(N, C) * torch.exp(rand(N, 1) * 0.5) + rand(N, 1) * 0.5
        s["x"], s["eps"] = x.to(dtype), 1e-5
        s["gamma"], s["beta"] = (1.0 + 0.1 * rand(C), 0.1 * rand(C)) if case["affine"] else (None, None)
        if kind == "norm":
            s["y"], s["stats"] = new(N, C, dtype=dtype), new(N, 2)
        else:
            x = s["x"].double()
            mean = x.mean(1)
            s["stats"] = torch.stack([mean, torch.rsqrt((x - mean[:, None]).square().mean(1) + s["eps"])], 1).float()
            s["dy"], s["dx"] = (rand(N, C) * 1e-3).to(dtype), new(N, C, dtype=dtype)
            s["dgamma"], s["dbeta"] = new(C), new(C)
    else:
        def direction(r, c):        # a gradient: a few strong directions over many weak ones
            k = min(8, r, c)
            return (rand(r, c) + (rand(r, k) * torch.exp2(-torch.arange(k, device="cuda").float())) @ rand(k, c) * 4.0) * 1e-3
        matrices = {"x": dtype, "y": torch.bfloat16} if kind == "orth" else {"g": dtype, "m": torch.float32, "w": torch.float32}
        if case["copy"]:
            matrices["wb"] = torch.bfloat16
        s["flat"] = {}
        for k, t in matrices.items():
            s["flat"][k], s[k] = _buffer(case, t)
        for i, (r, c) in enumerate(_shapes(case)):
            if kind == "orth":
                s["x"][i].copy_(direction(r, c))
            else:
                s["g"][i].copy_(direction(r, c))
                s["m"][i].copy_(direction(r, c) * 10.0)
                s["w"][i].copy_(rand(r, c) * (2.0 / c) ** 0.5)
    return s


# ---- the operators ---------------------------------------------------------------------------------------------------------

HYPER = {"lr": 1e-4, "momentum": 0.95, "wd": 0.1, "rms": 0.2, "grad_scale": 0.5}


def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own(state, kind)
    return {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad, "orth": _plain_orth,
            "muon": _plain_muon}[kind](state)


def _own(s, kind):
    from paper_1512_01274_amd import mxc
    c = s["case"]
    if kind == "embed":
        mxc.mxc_embedding_fwd(c["N"], c["V"], c["C"], CODE[c["dtype"]], s["tokens"], s["w"], s["scale"], s["y"])
        return s["y"]
    if kind == "norm":
        mxc.mxc_layernorm_fwd(c["N"], c["C"], CODE[c["dtype"]], s["x"], s["gamma"], s["beta"], s["eps"], s["y"], s["stats"])
        return {"y": s["y"], "stats": s["stats"]}
    if "workspace" not in s:
        s["workspace"] = mxc.alloc_workspace(
            mxc.mxc_embedding_workspace_bytes(c["N"], c["V"], c["C"], CODE[c["dtype"]]) if kind == "embed_grad" else
            mxc.mxc_layernorm_workspace_bytes(c["N"], c["C"], CODE[c["dtype"]]) if kind == "norm_grad" else
            mxc.mxc_orthogonalize_workspace_bytes(*map(list, zip(*_shapes(c)))))
    if kind == "embed_grad":
        mxc.mxc_embedding_bwd(c["N"], c["V"], c["C"], CODE[c["dtype"]], s["tokens"], s["dy"], s["scale"], c["add"], s["dw"], s["workspace"])
        return s["dw"]
    if kind == "norm_grad":
        mxc.mxc_layernorm_bwd(c["N"], c["C"], CODE[c["dtype"]], s["x"], s["gamma"], s["stats"], s["dy"], s["dx"], s["dgamma"], s["dbeta"], s["workspace"])
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if kind == "orth":
        mxc.mxc_orthogonalize(s["x"], c["steps"], s["y"], s["workspace"])
        return s["flat"]["y"]
    h = HYPER
    mxc.mxc_muon_update(s["w"], s["g"], s["m"], s.get("wb"), h["lr"], h["momentum"], c["nesterov"], h["wd"], h["rms"], h["grad_scale"], c["steps"], s["workspace"])
    return _updated(s)


def _updated(s):
    return {k: s["flat"].get(k) for k in ("w", "m", "wb")}


def _plain_embed(s):
    c, t = s["case"], s["tokens"].long()
    there = (t >= 0) & (t < c["V"])
    return (s["w"][t.clamp(0, c["V"] - 1)].float() * s["scale"] * there[:, None]).to(s["y"].dtype)


def _plain_embed_grad(s):
    c, t = s["case"], s["tokens"].long()
    there = (t >= 0) & (t < c["V"])
    dw = s["dw"] if c["add"] else s["dw"].zero_()
    return dw.index_add_(0, t.clamp(0, c["V"] - 1), s["dy"].float() * (s["scale"] * there)[:, None])


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    x = x - mean
    rstd = 1.0 / torch.sqrt(x.square().mean(1, keepdim=True) + s["eps"])
    y = x * rstd
    if s["gamma"] is not None:
        y = y * s["gamma"] + s["beta"]
    return {"y": y.to(s["y"].dtype), "stats": torch.cat([mean, rstd], 1)}


def _plain_norm_grad(s):
    mean, rstd = s["stats"][:, :1], s["stats"][:, 1:]
    z, dy = (s["x"].float() - mean) * rstd, s["dy"].float()
    g = dy if s["gamma"] is None else dy * s["gamma"]
    dx = (g - g.mean(1, keepdim=True) - z * (g * z).mean(1, keepdim=True)) * rstd
    return {"dx": dx.to(s["dx"].dtype), "dgamma": (dy * z).sum(0), "dbeta": dy.sum(0)}


COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def _orthogonal(x, steps):
    """x over its norm, then steps of x <- a x + (b A + c A A) x, A = x x^T, with the shorter side as rows."""
    a, b, c = COEFFICIENTS
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = x / torch.sqrt(x.square().sum()).clamp_(min=1e-30)
    for _ in range(steps):
        A = x @ x.t()
        x = a * x + (b * A + c * (A @ A)) @ x
    return x.t() if tall else x


def _plain_orth(s):
    for x, y in zip(s["x"], s["y"]):
        y.copy_(_orthogonal(x.float(), s["case"]["steps"]))
    return s["flat"]["y"]


def _plain_muon(s):
    c, h = s["case"], HYPER
    for i, (w, g, m) in enumerate(zip(s["w"], s["g"], s["m"])):
        g = g.float() * h["grad_scale"]
        m.mul_(h["momentum"]).add_(g)
        o = _orthogonal(g + m * h["momentum"] if c["nesterov"] else m, c["steps"])
        w.mul_(1.0 - h["lr"] * h["wd"]).sub_(o * (h["lr"] * h["rms"] * math.sqrt(max(w.shape))))
        if c["copy"]:
            s["wb"][i].copy_(w)
    return _updated(s)


# ---- what a pass cannot do without --------------------------------------------------------------------------------------------

def work(case):
    kind, size = case["kind"], SIZE[case["dtype"]]
    if kind == "embed":
        return {"bytes": case["N"] * (4 + 2 * case["C"] * size), "flops": case["N"] * case["C"]}
    if kind == "embed_grad":
        # added to a gradient that is there: at most a row for each token is read and written
        rows = 2 * min(case["N"], case["V"]) if case["add"] else case["V"]
        return {"bytes": case["N"] * (4 + case["C"] * size) + rows * case["C"] * 4, "flops": 2 * case["N"] * case["C"]}
    if kind in ("norm", "norm_grad"):
        values, weights = case["N"] * case["C"], case["C"] * 4
        if kind == "norm":
            return {"bytes": values * 2 * size + 2 * weights * case["affine"] + 8 * case["N"], "flops": 7 * values}
        return {"bytes": values * 3 * size + weights * (2 + case["affine"]) + 8 * case["N"], "flops": 14 * values}
    nbytes = flops = 0
    for r, c in _shapes(case):
        m, n = min(r, c), max(r, c)
        # A and A A are symmetric: half of each; the third product is whole
        flops += case["steps"] * (m * m * n + m ** 3 + 2 * m * m * n)
        nbytes += r * c * (size + 2 if kind == "orth" else size + 16 + (2 if case["copy"] else 0))
    return {"bytes": nbytes, "flops": flops}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------------

def _exact_orthogonal(x, steps):
    a, b, c = COEFFICIENTS
    norm = torch.linalg.vector_norm(x)
    x = x / norm if norm > 0 else x
    eye = torch.eye(min(x.shape), dtype=torch.float64, device="cuda")
    for _ in range(steps):
        if x.shape[0] <= x.shape[1]:
            A = torch.mm(x, x.t().contiguous())
            x = torch.mm(torch.addmm(eye, A, b * eye + c * A, beta=a), x)
        else:
            A = torch.mm(x.t().contiguous(), x)
            x = torch.mm(x, torch.addmm(eye, A, b * eye + c * A, beta=a))
    return x


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "embed":
        table = torch.cat([s["w"].double() * s["scale"], torch.zeros(1, case["C"], dtype=torch.float64, device="cuda")])
        return table[s["tokens"].long()]        # -1: the row of zeros at its end
    if kind == "embed_grad":
        dw = torch.zeros(case["V"] + 1, case["C"], dtype=torch.float64, device="cuda")
        dw.index_add_(0, s["tokens"].long() % (case["V"] + 1), s["dy"].double(), alpha=s["scale"])
        return dw[:-1] + s["dw"].double() if case["add"] else dw[:-1]
    if kind == "norm":
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + s["eps"]) ** -0.5
        y = (x - mean[:, None]) * rstd[:, None]
        if case["affine"]:
            y = y * s["gamma"].double() + s["beta"].double()
        return {"y": y, "stats": torch.stack([mean, rstd], 1)}
    if kind == "norm_grad":
        stats, dy, C = s["stats"].double(), s["dy"].double(), case["C"]
        z = s["x"].double().sub_(stats[:, :1]).mul_(stats[:, 1:])
        g = dy * s["gamma"].double() if case["affine"] else dy
        along = torch.stack([g.sum(1), (g * z).sum(1)], 1) / C
        return {"dx": stats[:, 1:] * (g - along[:, :1] - z * along[:, 1:]), "dgamma": (z * dy).sum(0), "dbeta": dy.sum(0)}
    if kind == "orth":
        flat, out = _buffer(case, torch.float64)
        for x, y in zip(s["x"], out):
            y.copy_(_exact_orthogonal(x.double(), case["steps"]))
        return flat
    h, (new_w, ws), (new_m, ms) = HYPER, _buffer(case, torch.float64), _buffer(case, torch.float64)
    for w, g, m, w_to, m_to in zip(s["w"], s["g"], s["m"], ws, ms):
        g = g.double() * h["grad_scale"]
        m_to.copy_(h["momentum"] * m.double() + g)
        u = g + h["momentum"] * m_to if case["nesterov"] else m_to
        step = h["lr"] * h["rms"] * max(w.shape) ** 0.5
        w_to.copy_((1 - h["lr"] * h["wd"]) * w.double() - step * _exact_orthogonal(u, case["steps"]))
    return {"w": new_w, "m": new_m, "wb": new_w if case["copy"] else None}
