"""The operators of a dense block and of its update, as cases that can be timed and compared.

  layernorm  layer norm of rows after a residual's addition; its gradients
  linear     rows times a matrix, with bias, activation and residual; its gradients
  muon       momentum, Newton-Schulz products that orthogonalise the update, and the step of the weights
  orthogonalise  those products alone

With `own` false everything is computed in its plain form, from elementary torch operations in 32 bits; with `own` true by the
library's entry points (`paper_2311_13225_amd.binding`).
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-5
BETA, LR, DECAY = 0.95, 0.02, 0.01
A, B, C = 3.4445, -4.7750, 2.0315        # the quintic of a Newton-Schulz step
STEPS = 5
ACTS = ("none", "relu", "gelu", "silu")


def listed():
    return [
        # one token's norm at serving time, with its residual: latency alone
        dict(name="layernorm_one_row", kind="layernorm_fwd", n=1, dim=1024, x="bf16", y="bf16", residual=True),
        # a residual stream's norm in a large batch
        dict(name="layernorm_residual", kind="layernorm_fwd", n=16_384, dim=4096, x="bf16", y="bf16", residual=True),
        # feature rows of a hop, wide and odd, normalised for bf16 products
        dict(name="layernorm_features", kind="layernorm_fwd", n=50_001, dim=602, x="f32", y="bf16", residual=False),
        # the norm's gradients in training, with the residual's gradient joined
        dict(name="layernorm_grad", kind="layernorm_bwd", n=16_384, dim=2048, x="bf16", residual=True),
        # a single token through a wide layer: the matrix is read, little else
        dict(name="linear_one_token", kind="linear_fwd", n=1, d_in=2048, d_out=8192, x="bf16", act="gelu", residual=False, keep=False),
        # a hop's vertices through a hidden layer in 32 bits, the features' width odd
        dict(name="linear_vertices", kind="linear_fwd", n=24_922, d_in=602, d_out=256, x="f32", act="relu", residual=False, keep=True),
        # the second half of a block in a large batch: back to the stream's width, with the residual
        dict(name="linear_residual", kind="linear_fwd", n=16_384, d_in=8192, d_out=2048, x="bf16", act="none", residual=True, keep=False),
        # the first half's gradients
        dict(name="linear_grad", kind="linear_bwd", n=8192, d_in=2048, d_out=8192, x="bf16", act="gelu"),
        # a narrow layer's gradients over a hop's vertices in 32 bits, the classes' number odd
        dict(name="linear_grad_classes", kind="linear_bwd", n=10_001, d_in=256, d_out=47, x="f32", act="relu"),
        # the matrices of a graph layer in one call
        dict(name="muon_graph_layer", kind="muon", matrices=2, rows=602, cols=256, grad="f32", nesterov=True),
        # a large block's matrix
        dict(name="muon_large", kind="muon", matrices=1, rows=4096, cols=4096, grad="bf16", nesterov=True),
        # updates of four layers, orthogonalised for a caller's own step
        dict(name="orthogonalise_wide", kind="orthogonalise", matrices=4, rows=512, cols=2048, grad="f32"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        case = _draw(rng)
        if _cost(case) <= most:
            return case


def _draw(rng):
    kind = rng.choice(("layernorm_fwd", "layernorm_bwd", "linear_fwd", "linear_fwd", "linear_bwd", "muon", "orthogonalise"))
    if kind.startswith("layernorm"):
        case = dict(kind=kind, n=_log(rng, 1, 200_000), dim=_log(rng, 16, 16_384), x=rng.choice(("f32", "bf16")), residual=rng.random() < 0.6)
        if kind == "layernorm_fwd":
            case["y"] = rng.choice(("f32", "bf16"))
        return case
    if kind.startswith("linear"):
        # half of the widths are whole multiples of 64, as models choose them, half are anything
        d_in, d_out = ((64 * _log(rng, 1, 128) if rng.random() < 0.5 else _log(rng, 16, 8192)) for _ in range(2))
        case = dict(kind=kind, n=_log(rng, 1, 50_000), d_in=d_in, d_out=d_out, x=rng.choice(("f32", "bf16", "bf16")), act=rng.choice(ACTS))
        if kind == "linear_fwd":
            case.update(residual=rng.random() < 0.4, keep=rng.random() < 0.5)
        return case
    case = dict(kind=kind, matrices=_log(rng, 1, 8), rows=_log(rng, 16, 4096), cols=_log(rng, 16, 4096), grad=rng.choice(("f32", "bf16")))
    if kind == "muon":
        case["nesterov"] = rng.random() < 0.7
    return case


def work(case):
    kind = case["kind"]
    if kind.startswith("layernorm"):
        n, dim, e = case["n"], case["dim"], SIZE[case["x"]]
        if kind == "layernorm_fwd":
            return {"bytes": n * (dim * (e * (3 if case["residual"] else 1) + SIZE[case["y"]]) + 8) + 8 * dim, "flops": 8 * n * dim}
        return {"bytes": n * (dim * e * (4 if case["residual"] else 3) + 8) + 12 * dim, "flops": 13 * n * dim}
    if kind.startswith("linear"):
        n, d_in, d_out, e = case["n"], case["d_in"], case["d_out"], SIZE[case["x"]]
        if kind == "linear_fwd":
            return {"bytes": e * (n * d_in + d_in * d_out + n * d_out * (1 + case["residual"] + case["keep"])) + 4 * d_out, "flops": 2 * n * d_in * d_out}
        stored = 0 if case["act"] == "none" else 1
        return {"bytes": e * (2 * n * d_in + 2 * d_in * d_out + n * d_out * (1 + stored)) + 4 * d_out, "flops": 4 * n * d_in * d_out}
    k, p, q = case["matrices"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    each = SIZE[case["grad"]] + (16 if kind == "muon" else SIZE[case["grad"]])
    return {"bytes": k * p * q * each, "flops": k * STEPS * (3 * p * p * q + p * p * p)}      # symmetric products by half


# ------------------------------------------------------------------------------------------------------- inputs

def _generator(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * (seed + 1) + tag)
    return g


def _normal(shape, dtype, gen, spread=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * spread).to(dtype)


def prepare(case, seed):
    s = {"case": case}
    gen = _generator(seed, 2)
    kind = case["kind"]
    if kind.startswith("layernorm"):
        n, dim, dt = case["n"], case["dim"], DTYPES[case["x"]]
        level = torch.randn((dim,), generator=gen, device="cuda")         # columns have levels of their own
        s["x"] = (_normal((n, dim), torch.float32, gen, 1.5) + level).to(dt)
        s["weight"] = 1.0 + 0.2 * torch.randn((dim,), generator=gen, device="cuda")
        s["bias"] = 0.1 * torch.randn((dim,), generator=gen, device="cuda")
        s["residual"] = _normal((n, dim), dt, gen) if case["residual"] else None
        if kind == "layernorm_bwd":      # x is the sum that the forward pass stored, residual the gradient that reaches it from above
            s["grad"] = _normal((n, dim), dt, gen)
            x = s["x"].float()
            s["mean"] = x.mean(1)
            s["rstd"] = 1.0 / torch.sqrt(((x - s["mean"][:, None]) ** 2).mean(1) + EPS)
    elif kind.startswith("linear"):
        n, d_in, d_out, dt = case["n"], case["d_in"], case["d_out"], DTYPES[case["x"]]
        s["x"] = _normal((n, d_in), dt, gen)
        s["w"] = _normal((d_in, d_out), dt, gen, 1.0 / math.sqrt(d_in))
        if kind == "linear_fwd":
            s["bias"] = 0.1 * torch.randn((d_out,), generator=gen, device="cuda")
            s["residual"] = _normal((n, d_out), dt, gen) if case["residual"] else None
        else:
            s["grad"] = _normal((n, d_out), dt, gen)
            s["z"] = None if case["act"] == "none" else _normal((n, d_out), dt, gen)        # as the forward pass stored it
    else:
        shape = (case["matrices"], case["rows"], case["cols"])
        # a gradient: a few strong directions above noise
        few = torch.randn((shape[0], shape[1], 4), generator=gen, device="cuda")
        g = 0.3 * torch.randn(shape, generator=gen, device="cuda")
        for j in range(4):
            g += few[:, :, j:j + 1] * torch.randn((shape[0], 1, shape[2]), generator=gen, device="cuda")
        s["grad"] = (0.01 * g).to(DTYPES[case["grad"]])
        if kind == "muon":
            s["w"] = _normal(shape, torch.float32, gen, 1.0 / math.sqrt(shape[1]))
            s["momentum"] = _normal(shape, torch.float32, gen, 0.02)
            s["scale"] = math.sqrt(max(1.0, shape[1] / shape[2]))
    return s


# ------------------------------------------------------------------------------------------------------- one pass

def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "layernorm_fwd":
        return _plain_layernorm(state)
    if kind == "layernorm_bwd":
        return _plain_layernorm_grad(state)
    if kind == "linear_fwd":
        return _plain_linear(state)
    if kind == "linear_bwd":
        return _plain_linear_grad(state)
    return _plain_muon(state) if kind == "muon" else _plain_orthogonalise(state)


def _plain_layernorm(s):
    x, out = s["x"], {}
    if s["residual"] is not None:
        x = out["sum"] = (x.float() + s["residual"].float()).to(x.dtype)
    x = x.float()
    out["mean"] = x.mean(1)
    x = x - out["mean"][:, None]
    out["rstd"] = 1.0 / torch.sqrt((x * x).mean(1) + EPS)
    out["y"] = (x * out["rstd"][:, None] * s["weight"] + s["bias"]).to(DTYPES[s["case"]["y"]])
    return out


def _plain_layernorm_grad(s):
    g, rstd = s["grad"].float(), s["rstd"][:, None]
    u = (s["x"].float() - s["mean"][:, None]) * rstd
    wg = g * s["weight"]
    dx = rstd * (wg - wg.mean(1, keepdim=True) - u * (wg * u).mean(1, keepdim=True))
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    return {"grad_x": dx.to(s["x"].dtype), "grad_weight": (g * u).sum(0), "grad_bias": g.sum(0)}


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z / (1.0 + torch.exp(-z)) if act == "silu" else z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    p = 1.0 / (1.0 + torch.exp(-z))
    return p * (1.0 + z * (1.0 - p))


def _plain_linear(s):
    z = s["x"].float() @ s["w"].float() + s["bias"]
    y = _act(z, s["case"]["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = {"y": y.to(s["x"].dtype)}
    if s["case"]["keep"]:
        out["z"] = z.to(s["x"].dtype)
    return out


def _plain_linear_grad(s):
    g = s["grad"].float()
    if s["z"] is not None:
        g = g * _act_slope(s["z"].float(), s["case"]["act"])
    dt = s["x"].dtype
    return {"grad_x": (g @ s["w"].float().t()).to(dt), "grad_w": (s["x"].float().t() @ g).to(dt), "grad_bias": g.sum(0)}


def _newton_schulz(u):
    x = u / torch.sqrt((u * u).sum((1, 2), keepdim=True))
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2).contiguous() if tall else x
    x = _steps(x)
    return x.transpose(1, 2) if tall else x


def _steps(x):
    for _ in range(STEPS):
        a = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = A * x + torch.matmul(B * a + C * torch.matmul(a, a), x)
    return x


def _plain_orthogonalise(s):
    return {"out": _newton_schulz(s["grad"].float()).to(s["grad"].dtype).contiguous()}


def _plain_muon(s):
    g, m, w = s["grad"].float(), s["momentum"], s["w"]
    m.mul_(BETA).add_(g)
    o = _newton_schulz(g + BETA * m if s["case"]["nesterov"] else m)
    w.mul_(1.0 - LR * DECAY).sub_(o * (LR * s["scale"]))
    return {"w": w, "momentum": m}


def _run_own(s):
    from paper_2311_13225_amd import binding as b
    case, kind = s["case"], s["case"]["kind"]
    if "out" not in s:                   # results and workspaces, which a program makes once
        s["out"] = _room(b, s)
    o = s["out"]
    if kind == "layernorm_fwd":
        b.no_layernorm_fwd(s["x"], s["weight"], s["bias"], EPS, o["y"], residual=s["residual"], sum_out=o.get("sum"), mean=o["mean"], rstd=o["rstd"])
        return {name: o[name] for name in ("sum", "mean", "rstd", "y") if name in o}
    if kind == "layernorm_bwd":
        b.no_layernorm_bwd(s["x"], s["weight"], s["mean"], s["rstd"], s["grad"], o["grad_x"], o["grad_weight"], o["grad_bias"], o["ws"],
                           grad_sum=s["residual"])
        return {name: o[name] for name in ("grad_x", "grad_weight", "grad_bias")}
    if kind == "linear_fwd":
        b.no_linear_fwd(s["x"], s["w"], s["bias"], b.ACT_OF_NAME[case["act"]], o["y"], o["ws"], residual=s["residual"], z=o.get("z"))
        return {name: o[name] for name in ("y", "z") if name in o}
    if kind == "linear_bwd":
        b.no_linear_bwd(s["x"], s["w"], b.ACT_OF_NAME[case["act"]], s["z"], s["grad"], o["grad_x"], o["grad_w"], o["grad_bias"], o["ws"])
        return {name: o[name] for name in ("grad_x", "grad_w", "grad_bias")}
    if kind == "muon":
        b.no_muon_step(s["w"], s["momentum"], s["grad"], LR, BETA, o["ws"], nesterov=case["nesterov"], steps=STEPS, weight_decay=DECAY, scale=s["scale"])
        return {"w": s["w"], "momentum": s["momentum"]}
    b.no_orthogonalise(s["grad"], o["out"], o["ws"], steps=STEPS)
    return {"out": o["out"]}


def _room(b, s):
    case, kind = s["case"], s["case"]["kind"]
    e = lambda *shape, dt=torch.float32: torch.empty(shape, dtype=dt, device="cuda")  # noqa: E731
    room = lambda size: torch.empty(size, dtype=torch.uint8, device="cuda")  # noqa: E731
    if kind.startswith("layernorm"):
        n, dim, dt = case["n"], case["dim"], DTYPES[case["x"]]
        if kind == "layernorm_fwd":
            o = {"y": e(n, dim, dt=DTYPES[case["y"]]), "mean": e(n), "rstd": e(n)}
            if case["residual"]:
                o["sum"] = e(n, dim, dt=dt)
            return o
        return {"grad_x": e(n, dim, dt=dt), "grad_weight": e(dim), "grad_bias": e(dim), "ws": room(b.no_layernorm_ws_bytes(n, dim))}
    if kind.startswith("linear"):
        n, d_in, d_out, dt = case["n"], case["d_in"], case["d_out"], DTYPES[case["x"]]
        o = {"ws": room(b.no_linear_ws_bytes(dt, n, d_in, d_out))}
        if kind == "linear_fwd":
            o["y"] = e(n, d_out, dt=dt)
            if case["keep"]:
                o["z"] = e(n, d_out, dt=dt)
        else:
            o.update(grad_x=e(n, d_in, dt=dt), grad_w=e(d_in, d_out, dt=dt), grad_bias=e(d_out))
        return o
    o = {"ws": room(b.no_orthogonalise_ws_bytes(*s["grad"].shape))}
    if kind == "orthogonalise":
        o["out"] = torch.empty_like(s["grad"])
    return o


# ------------------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind.startswith("layernorm"):
        step = (1 << 24) // case["dim"] + 1
        parts = [_exact_layernorm(case, s, lo, lo + step) for lo in range(0, case["n"], step)]
        return {name: sum(p[name] for p in parts) if name in ("grad_weight", "grad_bias") else torch.cat([p[name] for p in parts]) for name in parts[0]}
    if kind == "linear_fwd":
        z = torch.addmm(s["bias"].double(), s["x"].double(), s["w"].double())
        out = {"z": z.clone()} if case["keep"] else {}
        if case["act"] == "relu":
            z = torch.relu(z)
        elif case["act"] == "gelu":      # z times the normal distribution's probability of less than z
            z = z * 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        elif case["act"] == "silu":
            z = z * torch.sigmoid(z)
        return {"y": z if s["residual"] is None else z + s["residual"].double(), **out}
    if kind == "linear_bwd":
        g = s["grad"].double()
        if case["act"] != "none":
            z = s["z"].double()
            if case["act"] == "relu":
                slope = torch.where(z > 0, 1.0, 0.0).double()
            elif case["act"] == "gelu":
                slope = 0.5 * torch.special.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2) * (2 * math.pi) ** -0.5
            else:
                slope = torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)
            g = g * slope
        return {"grad_x": torch.mm(g, s["w"].double().t()), "grad_w": torch.mm(s["x"].double().t(), g), "grad_bias": torch.sum(g, 0)}
    u = s["grad"].double()
    if kind == "muon":
        m = BETA * s["momentum"].double() + u
        u = u + BETA * m if case["nesterov"] else m
    made = []
    for x in u:                          # the polynomial a x + b (x x') x + c (x x')^2 x, matrix by matrix
        x = x / torch.linalg.norm(x)
        for _ in range(STEPS):
            gram = x @ x.T if x.shape[0] <= x.shape[1] else None
            if gram is None:
                gram = x.T @ x
                x = A * x + x @ (B * gram + C * gram @ gram)
            else:
                x = A * x + (B * gram + C * gram @ gram) @ x
        made.append(x)
    o = torch.stack(made)
    if kind == "orthogonalise":
        return {"out": o}
    return {"w": (1.0 - LR * DECAY) * s["w"].double() - LR * s["scale"] * o, "momentum": m}


def _exact_layernorm(case, s, lo, hi):
    x, w = s["x"][lo:hi].double(), s["weight"].double()
    dim = case["dim"]
    if case["kind"] == "layernorm_bwd":
        g, r = s["grad"][lo:hi].double(), s["rstd"][lo:hi].double().unsqueeze(1)
        u = (x - s["mean"][lo:hi].double().unsqueeze(1)) * r
        dx = r * (w * g - torch.einsum("ij,j->i", g, w).unsqueeze(1) / dim - u * torch.einsum("ij,ij,j->i", g, u, w).unsqueeze(1) / dim)
        if case["residual"]:
            dx = dx + s["residual"][lo:hi].double()
        return {"grad_x": dx, "grad_weight": torch.einsum("ij,ij->j", g, u), "grad_bias": torch.einsum("ij->j", g)}
    out = {}
    if case["residual"]:                 # the stored sum is a value of its own type, by definition
        out["sum"] = (x + s["residual"][lo:hi].double()).to(s["x"].dtype).double()
        x = out["sum"]
    var, mean = torch.var_mean(x, 1, correction=0)
    out["mean"], out["rstd"] = mean, (var + EPS) ** -0.5
    out["y"] = (x - mean.unsqueeze(1)) * out["rstd"].unsqueeze(1) * w + s["bias"].double()
    return out
