"""The operators for learned inputs and large answers, as cases that can be timed and compared.

  embed      rows of a table by id, scaled; its gradient, added up by id (dense, or straight into the table: the SGD update)
  rmsnorm    root-mean-square norm of rows after a residual's addition, into fp32, bf16 or 8 bits with a scale a row; its gradients
  distill    loss against a teacher's top logits, and its gradient, apart and in one call
  logprobs   log probability of a given class, entropy and the largest alternatives; the gradient of the first two

With `own` false everything is computed in its plain form, from elementary torch operations in 32 bits; with `own` true by the
library's entry points (`paper_2311_13225_amd.binding`).
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
SIZE = {"f32": 4, "bf16": 2, "e4m3": 1}
EPS = 1e-5
E4M3_MOST = 448.0            # the largest e4m3 value: a row's largest magnitude is stored as this one
SMALLEST_MOST = 2.0 ** -100  # ... or as less, where the row is smaller than this: an all-zero row has a scale too
LR = 0.01


def listed():
    return [
        # one request's tokens at serving time: latency alone
        dict(name="embed_few_tokens", kind="embed_fwd", n=4, rows=32_000, dim=1024, table="bf16", out="bf16", zipf=True),
        # a bottom hop's vertices out of a table kept in 8 bits, with a scale a row
        dict(name="embed_vertices_8bit", kind="embed_fwd", n=118_000, rows=2_400_000, dim=256, table="e4m3", out="bf16", zipf=False),
        # gradient of a token table: popular tokens with thousands of occurrences, most rows untouched
        dict(name="embed_grad_tokens", kind="embed_bwd", n=65_536, rows=131_072, dim=2048, grad="bf16", accumulate=False, zipf=True),
        # SGD on the learned rows of a small batch's vertices, odd sizes
        dict(name="embed_update_small", kind="embed_bwd", n=777, rows=10_000, dim=100, grad="f32", accumulate=True, zipf=False),
        # a residual stream's norm in a large batch
        dict(name="rmsnorm_residual", kind="rmsnorm_fwd", n=16_384, dim=4096, x="bf16", y="bf16", residual=True),
        # feature rows of a hop, normalised into 8 bits, wide and odd
        dict(name="rmsnorm_features_8bit", kind="rmsnorm_fwd", n=50_001, dim=602, x="f32", y="e4m3", residual=False),
        # the norm's gradients in training, with the residual's gradient joined
        dict(name="rmsnorm_grad", kind="rmsnorm_bwd", n=16_384, dim=2048, x="bf16", residual=True),
        # node classification against a teacher: the classes of the largest graph
        dict(name="distill_classes", kind="distill", n=1024, classes=172, k=8, x="f32", mode="fwd_bwd", temperature=2.0),
        # distillation over a vocabulary: loss and gradient of a large batch
        dict(name="distill_vocabulary", kind="distill", n=4096, classes=131_072, k=64, x="bf16", mode="fwd_bwd", temperature=1.0),
        # one generated token: its log probability, entropy and alternatives
        dict(name="logprobs_one_row", kind="logprobs_fwd", n=1, classes=131_072, k=8, x="bf16", temperature=1.0),
        # scoring a batch of answers, an odd vocabulary in 32 bits
        dict(name="logprobs_scoring", kind="logprobs_fwd", n=4096, classes=50_001, k=20, x="f32", temperature=0.7),
        # gradient of log probability and entropy, as a policy's update takes it
        dict(name="logprobs_grad", kind="logprobs_bwd", n=4096, classes=32_000, x="bf16", temperature=1.0),
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
        if _cost(case) <= most and _values(case) <= 4096 * 131_072:
            return case


def _values(case):
    """Elements of the largest array of a case."""
    return max(case["n"], case.get("rows", 0)) * case.get("dim", 1) * case.get("classes", 1)


def _draw(rng):
    kind = rng.choice(("embed_fwd", "embed_bwd", "rmsnorm_fwd", "rmsnorm_bwd", "distill", "distill", "logprobs_fwd", "logprobs_bwd"))
    if kind == "embed_fwd":
        return dict(kind=kind, n=_log(rng, 1, 300_000), rows=_log(rng, 1000, 2_400_000), dim=_log(rng, 16, 8192),
                    table=rng.choice(("f32", "bf16", "e4m3")), out=rng.choice(("f32", "bf16")), zipf=rng.random() < 0.5)
    if kind == "embed_bwd":
        return dict(kind=kind, n=_log(rng, 1, 300_000), rows=_log(rng, 1000, 500_000), dim=_log(rng, 16, 8192),
                    grad=rng.choice(("f32", "bf16")), accumulate=rng.random() < 0.5, zipf=rng.random() < 0.7)
    if kind == "rmsnorm_fwd":
        return dict(kind=kind, n=_log(rng, 1, 200_000), dim=_log(rng, 16, 16_384), x=rng.choice(("f32", "bf16")),
                    y=rng.choice(("f32", "bf16", "e4m3")), residual=rng.random() < 0.6)
    if kind == "rmsnorm_bwd":
        return dict(kind=kind, n=_log(rng, 1, 200_000), dim=_log(rng, 16, 16_384), x=rng.choice(("f32", "bf16")), residual=rng.random() < 0.6)
    classes = _log(rng, 10, 200_000)
    case = dict(kind=kind, n=_log(rng, 1, 20_000), classes=classes, x=rng.choice(("f32", "bf16")), temperature=rng.choice((1.0, 1.0, 0.7, 2.0)))
    if kind == "distill":
        case.update(k=min(classes, _log(rng, 1, 128)), mode=rng.choice(("fwd", "bwd", "fwd_bwd", "fwd_bwd")))
    elif kind == "logprobs_fwd":
        case.update(k=rng.choice((0, min(classes, _log(rng, 1, 64)))))
    return case


def _distinct(case):
    """How many different rows n ids are expected to name."""
    n, v = case["n"], case["rows"]
    if not case["zipf"]:
        return v * -math.expm1(n * math.log1p(-1.0 / v))
    total, lo, top = 0.0, 1.0, float(v + 1)
    while lo < top:                      # ids follow a log-uniform rank: equal shares of the draws for equal ratios of ranks
        hi = min(top, lo * 1.05 if lo > 20 else lo + 1)
        share = math.log(hi / lo) / math.log(top) / (hi - lo)
        total += (hi - lo) * -math.expm1(n * math.log1p(-min(share, 1 - 1e-12)))
        lo = hi
    return total


def work(case):
    kind, n = case["kind"], case["n"]
    if kind == "embed_fwd":
        rows = _distinct(case)
        return {"bytes": rows * (case["dim"] * SIZE[case["table"]] + (4 if case["table"] == "e4m3" else 0)) + n * (4 + case["dim"] * SIZE[case["out"]]),
                "flops": n * case["dim"]}
    if kind == "embed_bwd":
        table = 8 * _distinct(case) if case["accumulate"] else 4 * case["rows"]
        return {"bytes": n * (4 + case["dim"] * SIZE[case["grad"]]) + table * case["dim"], "flops": n * case["dim"]}
    if kind == "rmsnorm_fwd":
        each = SIZE[case["x"]] * (3 if case["residual"] else 1) + SIZE[case["y"]]
        return {"bytes": n * (case["dim"] * each + 4 + (4 if case["y"] == "e4m3" else 0)) + 4 * case["dim"], "flops": 5 * n * case["dim"]}
    if kind == "rmsnorm_bwd":
        each = SIZE[case["x"]] * (4 if case["residual"] else 3)
        return {"bytes": n * (case["dim"] * each + 4) + 8 * case["dim"], "flops": 9 * n * case["dim"]}
    values = n * case["classes"]
    if kind == "distill":
        passes = 1 if case["mode"] == "fwd" else 2
        return {"bytes": passes * values * SIZE[case["x"]] + n * (8 * case["k"] + 12), "flops": (4 if passes == 1 else 7) * values}
    if kind == "logprobs_fwd":
        return {"bytes": values * SIZE[case["x"]] + n * (8 * case["k"] + 16), "flops": 6 * values}
    return {"bytes": 2 * values * SIZE[case["x"]] + n * 20, "flops": 7 * values}


# ------------------------------------------------------------------------------------------------------- inputs

def _generator(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * (seed + 1) + tag)
    return g


def _normal(shape, dtype, gen, spread=1.0):
    """Normal values, made in parts that fit beside the result."""
    t = torch.empty(shape, dtype=dtype, device="cuda")
    step = max(1, (1 << 28) // max(1, shape[1]))
    for lo in range(0, shape[0], step):
        part = t[lo:lo + step]
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda") * spread)
    return t


def _ids(case, gen):
    n, v = case["n"], case["rows"]
    if case["zipf"]:                     # log-uniform ranks, spread over the table
        u = torch.rand((n,), generator=gen, device="cuda", dtype=torch.float64)
        rank = (torch.exp(u * math.log(v + 1)) - 1).long().clamp_(0, v - 1)
        ids = (rank * 2_654_435_761 + 12_345) % v
    else:
        ids = torch.randint(0, v, (n,), generator=gen, device="cuda")
    if n > 64:
        ids[torch.rand((n,), generator=gen, device="cuda") < 0.01] = -1   # padding
    return ids.to(torch.int32)


def _logits(case, gen):
    z = _normal((case["n"], case["classes"]), DTYPES[case["x"]], gen, 2.0)
    if case["classes"] >= 1000:
        z[:, case["classes"] - case["classes"] // 128:] = -math.inf       # a vocabulary's padding is masked
    return z


def prepare(case, seed):
    s = {"case": case}
    gen = _generator(seed, 1)
    kind, n = case["kind"], case["n"]
    if kind.startswith("embed"):
        s["ids"] = _ids(case, gen)
        s["scale"] = math.sqrt(case["dim"])
    if kind == "embed_fwd":
        s["table"] = _normal((case["rows"], case["dim"]), DTYPES[case["table"]], gen, 1.0 if case["table"] != "e4m3" else 60.0)
        s["row_scale"] = torch.rand((case["rows"],), generator=gen, device="cuda") * 0.01 + 0.002 if case["table"] == "e4m3" else None
    elif kind == "embed_bwd":
        s["grad"] = _normal((n, case["dim"]), DTYPES[case["grad"]], gen)
        s["table"] = _normal((case["rows"], case["dim"]), torch.float32, gen) if case["accumulate"] else None
        if case["accumulate"]:
            s["scale"] = -LR             # the step of plain SGD, added into the table itself
    elif kind.startswith("rmsnorm"):
        dt = DTYPES[case["x"]]
        s["x"] = _normal((n, case["dim"]), dt, gen, 1.5)
        s["weight"] = 1.0 + 0.2 * torch.randn((case["dim"],), generator=gen, device="cuda")
        s["residual"] = _normal((n, case["dim"]), dt, gen) if case["residual"] else None
        if kind == "rmsnorm_bwd":        # x is the sum that the forward pass stored, residual the gradient that reaches it from above
            s["grad"] = _normal((n, case["dim"]), dt, gen)
            s["rstd"] = (1.0 / torch.sqrt((s["x"].float() ** 2).mean(1) + EPS))
    else:
        s["z"] = _logits(case, gen)
        rows = torch.arange(n, device="cuda")
        real = case["classes"] - (case["classes"] // 128 if case["classes"] >= 1000 else 0)
        if kind == "distill":
            k = case["k"]
            first = torch.randint(0, real, (n, 1), generator=gen, device="cuda")
            step = max(1, real // max(1, k))
            ids = (first + torch.arange(k, device="cuda") * step) % real  # k different classes
            s["teacher_logits"] = torch.sort(2.5 * torch.randn((n, k), generator=gen, device="cuda"), dim=1, descending=True).values
            if k > 2:                                                     # fewer entries than k in some rows
                ids[torch.rand((n,), generator=gen, device="cuda") < 0.1, k - 1] = -1
            s["teacher_ids"] = ids.to(torch.int32)
            top = ids[:, 0].clamp(min=0)
            s["z"][rows, top] = 6.0                                       # the student has learned something
            w = torch.full((n,), 1.0 / n, device="cuda")
            if n > 16:
                w[torch.rand((n,), generator=gen, device="cuda") < 0.05] = 0.0   # rows outside the training set
            s["row_weight"] = w
        else:
            tok = torch.randint(0, real, (n,), generator=gen, device="cuda")
            s["z"][rows, tok] = 5.0
            if n > 16:
                tok[torch.rand((n,), generator=gen, device="cuda") < 0.05] = -1  # positions without an answer
            s["tokens"] = tok.to(torch.int32)
        if kind == "logprobs_bwd":
            s["grad_logprob"] = torch.randn((n,), generator=gen, device="cuda")
            s["grad_entropy"] = 0.1 * torch.randn((n,), generator=gen, device="cuda")
        if kind == "logprobs_bwd" or case.get("mode") == "bwd":           # what the forward pass left
            lse, ent = _row_sums(s["z"], case["temperature"])
            s["lse"], s["entropy"] = lse, ent
    return s


def _row_sums(z, temperature):
    """(log of the sum of exponentials, entropy) of every row, fp32, made in parts."""
    lse, ent = [], []
    step = max(1, (1 << 27) // z.shape[1])
    for lo in range(0, z.shape[0], step):
        x = z[lo:lo + step].float() / temperature
        m = x.amax(1, keepdim=True)
        e = torch.exp(x - m)
        t = e.sum(1)
        lse.append(m[:, 0] + torch.log(t))
        ent.append(torch.log(t) - torch.where(e > 0, e * (x - m), 0.0).sum(1) / t)
    return torch.cat(lse), torch.cat(ent)


# ------------------------------------------------------------------------------------------------------- one pass

def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "embed_fwd":
        return _plain_embed(state)
    if kind == "embed_bwd":
        return _plain_embed_grad(state)
    if kind == "rmsnorm_fwd":
        return _plain_rmsnorm(state)
    if kind == "rmsnorm_bwd":
        return _plain_rmsnorm_grad(state)
    if kind == "distill":
        return _plain_distill(state)
    if kind == "logprobs_fwd":
        return _plain_logprobs(state)
    return _plain_logprobs_grad(state)


def _plain_embed(s):
    ids, table = s["ids"], s["table"]
    inside = (ids >= 0) & (ids < table.shape[0])
    at = torch.where(inside, ids, 0).long()
    if s["row_scale"] is not None:       # (indexing bytes: the 8-bit type itself has no such operation)
        rows = table.view(torch.uint8)[at].view(table.dtype).float()
        by = s["row_scale"][at] * s["scale"]
        rows = rows * torch.where(inside, by, 0.0)[:, None]
    else:
        rows = table[at].float() * torch.where(inside, s["scale"], 0.0)[:, None]
    return {"out": rows.to(DTYPES[s["case"]["out"]])}


def _plain_embed_grad(s):
    ids, case = s["ids"], s["case"]
    inside = (ids >= 0) & (ids < case["rows"])
    at = torch.where(inside, ids, 0).long()
    g = s["grad"].float() * torch.where(inside, s["scale"], 0.0)[:, None]
    if case["accumulate"]:
        return {"table": s["table"].index_add_(0, at, g)}
    return {"grad_table": torch.zeros((case["rows"], case["dim"]), device="cuda").index_add_(0, at, g)}


def _plain_rmsnorm(s):
    case, x = s["case"], s["x"]
    out = {}
    if s["residual"] is not None:
        x = out["sum"] = (x.float() + s["residual"].float()).to(x.dtype)
    x = x.float()
    rstd = 1.0 / torch.sqrt((x * x).mean(1) + EPS)
    y = x * rstd[:, None] * s["weight"]
    out["rstd"] = rstd
    if case["y"] == "e4m3":
        out["scale"] = torch.clamp(y.abs().amax(1), min=SMALLEST_MOST) / E4M3_MOST
        y = torch.clamp(y / out["scale"][:, None], -E4M3_MOST, E4M3_MOST)
    out["y"] = y.to(DTYPES[case["y"]])
    return out


def _plain_rmsnorm_grad(s):
    x, g, rstd = s["x"].float(), s["grad"].float(), s["rstd"][:, None]
    u = x * rstd
    wg = g * s["weight"]
    dx = rstd * (wg - u * (wg * u).mean(1, keepdim=True))
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    return {"grad_x": dx.to(s["x"].dtype), "grad_weight": (g * u).sum(0)}


def _plain_teacher(s):
    """(ids made safe, probabilities, their logarithms) of the teacher's entries."""
    ids, inside = s["teacher_ids"].long(), (s["teacher_ids"] >= 0) & (s["teacher_ids"] < s["case"]["classes"])
    t = torch.where(inside, s["teacher_logits"].float() / s["case"]["temperature"], -math.inf)
    t = t - t.amax(1, keepdim=True)
    e = torch.exp(t)
    total = e.sum(1, keepdim=True)
    return torch.where(inside, ids, 0), e / total, t - torch.log(total)


def _plain_distill(s):
    case, z, w = s["case"], s["z"], s["row_weight"]
    temperature, mode = case["temperature"], case["mode"]
    at, p, log_p = _plain_teacher(s)
    x = z.float() / temperature
    if mode == "bwd":
        q = torch.exp(x - s["lse"][:, None])
    else:
        x = x - (most := x.amax(1, keepdim=True))
        q = torch.exp(x)
        total = q.sum(1, keepdim=True)
        q = q / total if mode == "fwd_bwd" else q
    out = {}
    if mode != "bwd":
        log_q = x.gather(1, at) - torch.log(total)
        loss = torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1)
        out["loss"] = torch.where(w != 0, w * temperature ** 2 * loss, 0.0)
        out["lse"] = (most + torch.log(total))[:, 0]
    if mode != "fwd":
        dz = q.scatter_add_(1, at, -p)
        out["grad"] = torch.where((w != 0)[:, None], (w * temperature)[:, None] * dz, 0.0).to(z.dtype)
    return out


def _plain_logprobs(s):
    case, z, tok = s["case"], s["z"], s["tokens"].long()
    x = z.float() / case["temperature"]
    most = x.amax(1, keepdim=True)
    x = x - most
    e = torch.exp(x)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    there = (tok >= 0) & (tok < case["classes"])
    lp = x.gather(1, torch.where(there, tok, 0)[:, None]) - log_total
    out = {"logprob": torch.where(there, lp[:, 0], 0.0), "lse": (most + log_total)[:, 0],
           "entropy": (log_total - torch.where(e > 0, e * x, 0.0).sum(1, keepdim=True) / total)[:, 0]}
    if case["k"]:                        # by value, then by the lower index: both in one whole number
        bits = z.float().view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        key = order * (1 << 32) + (0x7FFFFFFF - torch.arange(case["classes"], device="cuda"))
        top = 0x7FFFFFFF - (torch.topk(key, case["k"], dim=1).values & 0xFFFFFFFF)
        out["top_ids"] = top.to(torch.int32)
        out["top_logprobs"] = x.gather(1, top) - log_total
    return out


def _plain_logprobs_grad(s):
    case, z, tok = s["case"], s["z"], s["tokens"].long()
    there = (tok >= 0) & (tok < case["classes"])
    g = torch.where(there, s["grad_logprob"], 0.0)[:, None]
    log_p = z.float() / case["temperature"] - s["lse"][:, None]
    p = torch.exp(log_p)
    gh = s["grad_entropy"][:, None]
    dz = torch.where(p > 0, -p * (g + gh * (log_p + s["entropy"][:, None])), 0.0)
    dz.scatter_add_(1, torch.where(there, tok, 0)[:, None], g)
    return {"grad": (dz / case["temperature"]).to(z.dtype)}


def _buffers(s, b):
    """Outputs and workspace of a state, made by its first pass and kept as a program's loop keeps them."""
    case, dev = s["case"], "cuda"
    n, kind = case["n"], case["kind"]
    o = s["buffers"] = {}
    if kind == "embed_fwd":
        o["out"] = torch.empty((n, case["dim"]), dtype=DTYPES[case["out"]], device=dev)
    elif kind == "embed_bwd":
        o["grad_table"] = s["table"] if case["accumulate"] else torch.empty((case["rows"], case["dim"]), device=dev)
        o["ws"] = torch.empty((b.no_embed_ws_bytes(n, case["dim"]),), dtype=torch.uint8, device=dev)
    elif kind == "rmsnorm_fwd":
        o["y"] = torch.empty((n, case["dim"]), dtype=DTYPES[case["y"]], device=dev)
        o["sum"] = torch.empty_like(s["x"]) if case["residual"] else None
        o["rstd"] = torch.empty((n,), device=dev)
        o["scale"] = torch.empty((n,), device=dev) if case["y"] == "e4m3" else None
    elif kind == "rmsnorm_bwd":
        o["grad_x"] = torch.empty_like(s["x"])
        o["grad_weight"] = torch.empty((case["dim"],), device=dev)
        o["ws"] = torch.empty((b.no_rmsnorm_ws_bytes(n, case["dim"]),), dtype=torch.uint8, device=dev)
    elif kind == "distill":
        o["loss"], o["lse"] = torch.empty((n,), device=dev), torch.empty((n,), device=dev)
        o["grad"] = torch.empty_like(s["z"]) if case["mode"] != "fwd" else None
        o["ws"] = torch.empty((b.no_distill_ws_bytes(n, case["classes"]),), dtype=torch.uint8, device=dev)
    elif kind == "logprobs_fwd":
        for name in ("logprob", "entropy", "lse"):
            o[name] = torch.empty((n,), device=dev)
        if case["k"]:
            o["top_ids"] = torch.empty((n, case["k"]), dtype=torch.int32, device=dev)
            o["top_logprobs"] = torch.empty((n, case["k"]), device=dev)
        o["ws"] = torch.empty((b.no_logprobs_ws_bytes(n, case["classes"], case["k"]),), dtype=torch.uint8, device=dev)
    else:
        o["grad"] = torch.empty_like(s["z"])
    return o


def _run_own(s):
    from paper_2311_13225_amd import binding as b
    case = s["case"]
    kind, o = case["kind"], s.get("buffers") or _buffers(s, b)
    if kind == "embed_fwd":
        b.no_embed_fwd(s["table"], s["ids"], o["out"], scale=s["scale"], row_scale=s["row_scale"])
        return {"out": o["out"]}
    if kind == "embed_bwd":
        b.no_embed_bwd(s["grad"], s["ids"], o["grad_table"], o["ws"], scale=s["scale"], accumulate=case["accumulate"])
        return {"table" if case["accumulate"] else "grad_table": o["grad_table"]}
    if kind == "rmsnorm_fwd":
        b.no_rmsnorm_fwd(s["x"], s["weight"], EPS, o["y"], residual=s["residual"], sum_out=o["sum"], row_scale=o["scale"], rstd=o["rstd"])
        return {name: o[name] for name in ("y", "sum", "rstd", "scale") if o[name] is not None}
    if kind == "rmsnorm_bwd":
        b.no_rmsnorm_bwd(s["x"], s["weight"], s["rstd"], s["grad"], o["grad_x"], o["grad_weight"], o["ws"], grad_sum=s["residual"])
        return {"grad_x": o["grad_x"], "grad_weight": o["grad_weight"]}
    if kind == "distill":
        teacher = (s["teacher_ids"], s["teacher_logits"], case["temperature"], s["row_weight"])
        if case["mode"] == "fwd":
            b.no_distill_fwd(s["z"], *teacher, o["loss"], o["lse"], o["ws"])
            return {"loss": o["loss"], "lse": o["lse"]}
        if case["mode"] == "bwd":
            b.no_distill_bwd(s["z"], *teacher, s["lse"], o["grad"])
            return {"grad": o["grad"]}
        b.no_distill_fwd_bwd(s["z"], *teacher, o["loss"], o["lse"], o["grad"], o["ws"])
        return {"loss": o["loss"], "lse": o["lse"], "grad": o["grad"]}
    if kind == "logprobs_fwd":
        b.no_logprobs_fwd(s["z"], s["tokens"], case["temperature"], o["logprob"], o["entropy"], o["lse"], o["ws"],
                          top_ids=o.get("top_ids"), top_logprobs=o.get("top_logprobs"))
        return {name: o[name] for name in ("logprob", "entropy", "lse", "top_ids", "top_logprobs") if name in o}
    b.no_logprobs_bwd(s["z"], s["tokens"], case["temperature"], s["lse"], s["entropy"], s["grad_logprob"], s["grad_entropy"], o["grad"])
    return {"grad": o["grad"]}


# ------------------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    kind, f64 = case["kind"], torch.float64
    if kind == "embed_fwd":
        out = torch.zeros((case["n"], case["dim"]), dtype=f64, device="cuda")
        rows = torch.nonzero((s["ids"] >= 0) & (s["ids"] < case["rows"]))[:, 0]
        picked = s["ids"][rows].long()
        if s["row_scale"] is None:
            out[rows] = s["table"][picked].to(f64) * s["scale"]
        else:
            out[rows] = s["table"].view(torch.uint8)[picked].view(torch.float8_e4m3fn).to(f64) * (s["row_scale"][picked].to(f64) * s["scale"])[:, None]
        return {"out": out}
    if kind == "embed_bwd":
        rows = torch.nonzero((s["ids"] >= 0) & (s["ids"] < case["rows"]))[:, 0]
        total = torch.zeros((case["rows"], case["dim"]), dtype=f64, device="cuda")
        total.index_add_(0, s["ids"][rows].long(), s["grad"][rows].to(f64))
        if case["accumulate"]:
            return {"table": s["table"].to(f64) + s["scale"] * total}
        return {"grad_table": total * s["scale"]}
    if kind.startswith("rmsnorm"):
        parts = [_exact_rmsnorm(case, s, lo, lo + (1 << 24) // case["dim"] + 1) for lo in range(0, case["n"], (1 << 24) // case["dim"] + 1)]
        return {name: sum(p[name] for p in parts) if name == "grad_weight" else torch.cat([p[name] for p in parts]) for name in parts[0]}
    step = (1 << 26) // case["classes"] + 1
    parts = [(_exact_distill if kind == "distill" else _exact_logprobs)(case, s, slice(lo, min(case["n"], lo + step)))
             for lo in range(0, case["n"], step)]
    return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}


def _exact_rmsnorm(case, s, lo, hi):
    x = s["x"][lo:hi].double()
    w = s["weight"].double()
    if case["kind"] == "rmsnorm_bwd":
        g, r = s["grad"][lo:hi].double(), s["rstd"][lo:hi].double().unsqueeze(1)
        dx = r * w * g - r ** 3 * x * torch.einsum("ij,ij->i", w * g, x).unsqueeze(1) / case["dim"]
        if case["residual"]:
            dx += s["residual"][lo:hi].double()
        return {"grad_x": dx, "grad_weight": torch.einsum("ij,ij->j", g, x * r)}
    out = {}
    if case["residual"]:                 # the stored sum is a value of its own type, by definition
        out["sum"] = (x + s["residual"][lo:hi].double()).to(s["x"].dtype).double()
        x = out["sum"]
    out["rstd"] = (x.square().sum(1) / case["dim"] + EPS) ** -0.5
    out["y"] = torch.einsum("ij,i,j->ij", x, out["rstd"], w)
    if case["y"] == "e4m3":
        out["scale"] = out["y"].abs().max(1).values.clamp(min=SMALLEST_MOST) / E4M3_MOST
        out["y"] = out["y"] / out["scale"].unsqueeze(1)
    return out


def _exact_distill(case, s, part):
    t = case["temperature"]
    z, w = s["z"][part].double() / t, s["row_weight"][part].double()
    ids, given = s["teacher_ids"][part].long(), s["teacher_logits"][part].double() / t
    p = torch.zeros_like(z)              # the teacher over all classes: zero outside its entries
    given[(ids < 0) | (ids >= case["classes"])] = -math.inf
    p.scatter_add_(1, ids.clamp(0, case["classes"] - 1), torch.softmax(given, 1))
    lse = s["lse"][part].double() if case["mode"] == "bwd" else torch.logsumexp(z, 1)
    log_q = z - lse.unsqueeze(1)
    out = {}
    if case["mode"] != "bwd":
        out["loss"] = w * t * t * (torch.xlogy(p, p) - torch.where(p > 0, p * log_q, 0.0)).sum(1)
        out["lse"] = lse
    if case["mode"] != "fwd":
        out["grad"] = (w * t).unsqueeze(1) * (log_q.exp() - p)
    return out


def _exact_logprobs(case, s, part):
    t = case["temperature"]
    z, tok = s["z"][part].double() / t, s["tokens"][part].long()
    there = (tok >= 0) & (tok < case["classes"])
    given = case["kind"] == "logprobs_bwd"
    lse = s["lse"][part].double() if given else torch.logsumexp(z, 1)
    log_p = z - lse.unsqueeze(1)
    plogp = torch.where(log_p > -math.inf, log_p.exp() * log_p, 0.0)
    hit = torch.zeros_like(z)
    hit[torch.nonzero(there)[:, 0], tok[there]] = 1.0
    if given:
        gl, gh, ent = (s[name][part].double().unsqueeze(1) for name in ("grad_logprob", "grad_entropy", "entropy"))
        p = log_p.exp()
        return {"grad": (torch.where(there.unsqueeze(1), gl, 0.0) * (hit - p) - gh * (plogp + p * ent)) / t}
    out = {"logprob": torch.where(hit > 0, log_p, 0.0).sum(1), "entropy": -plogp.sum(1), "lse": lse}
    if case["k"]:
        value, at = torch.sort(log_p, dim=1, descending=True, stable=True)
        out["top_ids"], out["top_logprobs"] = at[:, :case["k"]].to(torch.int32), value[:, :case["k"]].contiguous()
    return out
