"""The operators of a dense block and of its update (layer norm, dense layer, orthogonalised updates) against their formulas in 64 bits, element by element, and as
differences.

u = 2^-24 is the unit roundoff of fp32, half(t) half a step of an output type, relative. Element bounds count roundings: a sum whose longest chain of additions has k terms is
off by at most k roundings of the sum of magnitudes (2 u each in a matrix instruction, which may cut instead of rounding). Where a chain is long such a bound says little, so long
sums are held to a norm as well: k roundings of random sign, each of a partial sum that grows like its root, leave a relative error of about u sqrt(k) / 2 in the 2-norm; 2 u sqrt(k) is
four times that."""
import math

import pytest
import torch

from .test_operators import BF16, F32, INF, MARK, NAN, TINY, U, Rows, chain, close, count, half, nb, randn, rng, ws_of

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])


# ------------------------------------------------------------------------------------------------------- layer norm

NORM_SIZES = [(1, 1, 0, 0), (1, 64, 0, 0), (3, 5, 2, 1), (7, 63, 0, 0), (64, 100, 4, 4), (100, 602, 0, 0), (65, 256, 0, 0), (1000, 128, 0, 0), (33, 1025, 3, 1),
              (19, 2048, 0, 0), (5, 4096, 8, 8), (3, 4099, 0, 0), (2, 8192, 0, 0), (2, 16_385, 1, 0), (1, 40_000, 0, 0), (2, 65_536, 0, 0), (9000, 32, 0, 0),
              (300, 777, 0, 1), (4, 12_000, 0, 0), (3, 33_000, 1, 1)]


def norm_ref(x, residual, weight, bias, eps):
    s = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    v = s.double()
    mean = v.mean(1)
    d = v - mean[:, None]
    rstd = 1.0 / torch.sqrt(d.square().mean(1) + eps)
    y = d * rstd[:, None] * (1.0 if weight is None else weight.double())
    return s, mean, rstd, y + (0.0 if bias is None else bias.double())


@pytest.mark.parametrize("n,dim,pad,off", NORM_SIZES)
@BOTH
@pytest.mark.parametrize("dt_y", [F32, BF16], ids=["to_f32", "to_bf16"])
@pytest.mark.parametrize("residual", [False, True])
def test_layernorm_fwd(n, dim, pad, off, dt, dt_y, residual):
    b, g, eps = nb(), rng(n + dim), 1e-5
    level = 3.0 if n % 2 else 0.0           # rows with a level of their own
    x = Rows(n, dim, dt, pad, off, (randn((n, dim), g, F32, 2.0) + level).to(dt))
    r = Rows(n, dim, dt, 0, off, randn((n, dim), g, dt)) if residual else None
    weight = 1 + 0.3 * randn((dim,), g) if n != 65 else None
    bias = randn((dim,), g) if n != 100 else None
    if n > 4:
        x.t[2] = 1.5                        # a row of equal values: nothing but the bias is left
        if residual:
            r.t[2] = 0
    s, y = (Rows(n, dim, dt, pad, off) if residual or n % 2 else None), Rows(n, dim, dt_y, pad, off)
    mean, rstd = torch.full((n,), MARK, device="cuda"), torch.full((n,), MARK, device="cuda")
    b.no_layernorm_fwd(x.t, weight, bias, eps, y.t, residual=r.t if r else None, sum_out=s.t if s else None, mean=mean, rstd=rstd)
    ref_s, ref_mean, ref_rstd, ref_y = norm_ref(x.t, r.t if r else None, weight, bias, eps)
    if s:
        assert torch.equal(s.t, ref_s) and s.untouched()
    v = ref_s.double()
    mean_tol = (chain(dim) + 4) * U * v.abs().mean(1)
    close(mean, ref_mean, mean_tol, "mean")
    # a mean that is off by e moves the sum of squared differences by n e^2 (the differences themselves add up to nothing); each difference is rounded
    var = (v - ref_mean[:, None]).square().mean(1)
    var_tol = (chain(dim) + 8) * U * var + (mean_tol + U * ref_mean.abs()).square() + 2 * mean_tol * var.sqrt() * dim * U
    # half of the relative error of var + eps, while that is small
    rel = 0.5 * var_tol / (var + eps) * (1 + var_tol / (var + eps)) + 6 * U
    close(rstd, ref_rstd, rel * ref_rstd, "rstd")
    w = torch.ones((dim,), device="cuda").double() if weight is None else weight.double().abs()
    d = (v - ref_mean[:, None]).abs()
    tol = w * ref_rstd[:, None] * ((mean_tol[:, None] + U * d) * (1 + rel[:, None]) + d * (rel[:, None] + 3 * U)) + U * ref_y.abs()
    close(y.t, ref_y, tol + half(dt_y) * (ref_y.abs() + tol) + TINY, "y")
    assert y.untouched()


def test_layernorm_fwd_in_place_counts_and_extremes():
    b, g = nb(), rng(4)
    for dt, n, dim in ((BF16, 9, 1000), (F32, 9, 1000), (BF16, 3, 20_000), (F32, 5, 7)):
        x, r, w, c = randn((n, dim), g, dt), randn((n, dim), g, dt), randn((dim,), g), randn((dim,), g)
        s, y = torch.empty_like(x), torch.empty_like(x)
        b.no_layernorm_fwd(x, w, c, 1e-6, y, residual=r, sum_out=s)
        x1, r1 = x.clone(), r.clone()
        b.no_layernorm_fwd(x1, w, c, 1e-6, x1, residual=r1, sum_out=r1)          # the sum over the residual, the result over x
        assert torch.equal(x1, y) and torch.equal(r1, s)
        out = Rows(n, dim, dt)
        b.no_layernorm_fwd(x, w, c, 1e-6, out.t, residual=r, n_rows=count(2))
        assert torch.equal(out.t[:2], y[:2]) and out.untouched(rows=2)
        for none in (0, -3):
            b.no_layernorm_fwd(x, w, c, 1e-6, out.t, n_rows=count(none))
            assert out.untouched(rows=2)
        b.no_layernorm_fwd(x, w, c, 1e-6, out.t, residual=r, n_rows=count(n + 5))
        assert torch.equal(out.t, y) and out.untouched()
    b.no_layernorm_fwd(torch.empty((0, 8), device="cuda"), None, None, 1e-6, torch.empty((0, 8), device="cuda"))
    x = torch.arange(256, device="cuda").float().view(4, 64)
    x[0, 5], x[1, 6], x[2] = NAN, INF, 4.0
    y, mean, rstd = torch.empty((4, 64), device="cuda"), torch.empty((4,), device="cuda"), torch.empty((4,), device="cuda")
    b.no_layernorm_fwd(x, None, None, 0.0, y, mean=mean, rstd=rstd)
    assert y[:2].isnan().all() and mean[0].isnan() and mean[1] == INF and rstd[:2].isnan().all()
    assert mean[2] == 4 and rstd[2] == INF and y[2].isnan().all() and y[3].isfinite().all()
    # one value: it is its own mean
    y1 = torch.full((3, 1), MARK, device="cuda")
    b.no_layernorm_fwd(torch.tensor([[1e30], [-2.0], [0.0]], device="cuda"), torch.full((1,), 5.0, device="cuda"), torch.full((1,), 0.25, device="cuda"), 1e-5, y1)
    assert (y1 == 0.25).all()
    # a level of 2^12 above a spread of 1: the differences are what counts
    x = randn((8, 1024), g)
    near, far = torch.empty_like(x), torch.empty_like(x)
    x = (x * 256).round() / 256                # (so that adding 4096 rounds nothing)
    b.no_layernorm_fwd(x, None, None, 1e-5, near)
    b.no_layernorm_fwd(x + 4096, None, None, 1e-5, far)
    close(far, near, (chain(1024) + 4) * U * 4096 * 1.2 + 1e-5, "level")      # the mean's error, over a deviation of about 1


@pytest.mark.parametrize("n,dim,pad,off", NORM_SIZES + [(3000, 7, 0, 0), (70_000, 16, 0, 0), (600, 2049, 1, 1)])
@BOTH
@pytest.mark.parametrize("joined", [False, True])
def test_layernorm_bwd(n, dim, pad, off, dt, joined):
    b, g = nb(), rng(n + dim)
    s = Rows(n, dim, dt, pad, off, (randn((n, dim), g, F32, 2.0) + 1.0).to(dt))
    gy = Rows(n, dim, dt, 0, off, randn((n, dim), g, dt))
    gs = Rows(n, dim, dt, pad, 0, randn((n, dim), g, dt)) if joined else None
    weight = 1 + 0.3 * randn((dim,), g) if n != 65 else None
    v = s.t.double()
    mean = v.mean(1).float()
    rstd = (1.0 / torch.sqrt((v - v.mean(1, keepdim=True)).square().mean(1) + 1e-5)).float()
    gx, gw, gb = Rows(n, dim, dt, pad, off), torch.full((dim,), MARK, device="cuda"), torch.full((dim,), MARK, device="cuda")
    ws = ws_of(b.no_layernorm_ws_bytes(n, dim))
    b.no_layernorm_bwd(s.t, weight, mean, rstd, gy.t, gx.t, gw, gb, ws, grad_sum=gs.t if gs else None)
    r = rstd.double()[:, None]
    u_, wg = (v - mean.double()[:, None]) * r, gy.t.double() * (1.0 if weight is None else weight.double())
    dot, size = (wg * u_).mean(1, keepdim=True), (wg * u_).abs().mean(1, keepdim=True)
    flat, flat_size = wg.mean(1, keepdim=True), wg.abs().mean(1, keepdim=True)
    ref = r * (wg - flat - u_ * dot)
    # the means: their products, chains, divisions; then the products and differences of the formula
    tol = r * (5 * U * (wg.abs() + flat.abs()) + (chain(dim) + 4) * U * flat_size + u_.abs() * ((chain(dim) + 9) * U * size + 5 * U * dot.abs()))
    if joined:
        ref = ref + gs.t.double()
        tol = tol + U * ref.abs()
    close(gx.t, ref, tol + half(dt) * (ref.abs() + tol) + TINY, "grad_x")
    close(gw, (gy.t.double() * u_).sum(0), (n + 5) * U * (gy.t.double() * u_).abs().sum(0), "grad_weight")
    close(gb, gy.t.double().sum(0), (n + 2) * U * gy.t.double().abs().sum(0), "grad_bias")
    assert gx.untouched()
    again, gw2, gb2 = torch.empty((n, dim), device="cuda", dtype=dt), torch.empty_like(gw), torch.empty_like(gw)
    ws.fill_(0x3C)
    b.no_layernorm_bwd(s.t, weight, mean, rstd, gy.t, again, gw2, None, ws, grad_sum=gs.t if gs else None)
    b.no_layernorm_bwd(s.t, weight, mean, rstd, gy.t, again, None, gb2, ws, grad_sum=gs.t if gs else None)
    assert torch.equal(again, gx.t) and torch.equal(gw, gw2) and torch.equal(gb, gb2)
    b.no_layernorm_bwd(s.t, weight, mean, rstd, gy.t, again, None, None, ws, grad_sum=gs.t if gs else None)
    assert torch.equal(again, gx.t)
    for over in ("gy", "s", "gs") if joined else ("gy", "s"):
        inputs = {"gy": gy.t.clone(), "s": s.t.clone(), "gs": gs.t.clone() if gs else None}
        b.no_layernorm_bwd(inputs["s"], weight, mean, rstd, inputs["gy"], inputs[over], gw2, gb2, ws, grad_sum=inputs["gs"])
        assert torch.equal(inputs[over], again) and torch.equal(gw, gw2) and torch.equal(gb, gb2), over


def test_layernorm_bwd_counts():
    b, g = nb(), rng(6)
    n, dim = 500, 96
    s, gy, mean, rstd = randn((n, dim), g), randn((n, dim), g), randn((n,), g), torch.rand((n,), generator=g, device="cuda")
    ws = ws_of(b.no_layernorm_ws_bytes(n, dim))
    for here in (499, 130, 1, 0):
        s[here:], rstd[here:], mean[here:], gy[here:] = NAN, NAN, NAN, NAN
        gx, gw, gb = Rows(n, dim, F32), torch.full((dim,), MARK, device="cuda"), torch.full((dim,), MARK, device="cuda")
        b.no_layernorm_bwd(s, None, mean, rstd, gy, gx.t, gw, gb, ws, n_rows=count(here))
        terms = gy[:here].double() * ((s[:here].double() - mean[:here, None].double()) * rstd[:here, None].double())
        close(gw, terms.sum(0), (here + 5) * U * terms.abs().sum(0))
        close(gb, gy[:here].double().sum(0), (here + 2) * U * gy[:here].double().abs().sum(0))
        assert gx.untouched(rows=here) and not gx.t[:here].isnan().any()
    b.no_layernorm_bwd(s[:0], None, mean[:0], rstd[:0], gy[:0], gx.t[:0], gw, gb, ws)
    assert (gw == 0).all() and (gb == 0).all()


def test_layernorm_gradient_against_differences():
    b, g = nb(), rng(8)
    n, dim, h = 3, 40, 1e-3
    x, w, c, gy = randn((n, dim), g), 1 + 0.2 * randn((dim,), g), randn((dim,), g), randn((n, dim), g)
    mean, rstd, y = torch.empty((n,), device="cuda"), torch.empty((n,), device="cuda"), torch.empty((n, dim), device="cuda")
    b.no_layernorm_fwd(x, w, c, 1e-5, y, mean=mean, rstd=rstd)
    gx, gw, gb = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
    b.no_layernorm_bwd(x, w, mean, rstd, gy, gx, gw, gb, ws_of(b.no_layernorm_ws_bytes(n, dim)))
    f = lambda xx, ww, cc: (norm_ref(xx, None, ww, cc, 1e-5)[3] * gy.double()).sum().item()  # noqa: E731
    for i, at in ((0, 0), (1, 17), (2, 39)):
        d = torch.zeros((n, dim), device="cuda", dtype=torch.float64)
        d[i, at] = h
        # central differences of a smooth function: off by about h^2 of its third derivative
        assert abs((f(x.double() + d, w, c) - f(x.double() - d, w, c)) / (2 * h) - gx[i, at].item()) < 1e-4
        assert abs((f(x, w.double() + d[i], c) - f(x, w.double() - d[i], c)) / (2 * h) - gw[at].item()) < 1e-4
        assert abs((f(x, w, c.double() + d[i]) - f(x, w, c.double() - d[i])) / (2 * h) - gb[at].item()) < 1e-4


# ------------------------------------------------------------------------------------------------------- dense layer

# rows, sides, elements between rows and in front: few rows; tiles of each width; sides that are no multiple of 8; rows off 16 bytes
LINEAR_SIZES = [(1, 1, 1, 0, 0), (1, 7, 5, 0, 0), (1, 300, 129, 1, 1), (2, 64, 64, 0, 0), (3, 100, 47, 0, 0), (5, 33, 130, 3, 0), (8, 1100, 70, 0, 0), (9, 17, 9, 0, 0),
                (16, 64, 128, 0, 0), (33, 130, 70, 0, 1), (64, 256, 256, 0, 0), (65, 257, 300, 1, 1), (128, 8, 8, 0, 0), (129, 64, 1, 0, 0), (130, 1, 65, 0, 0),
                (200, 602, 256, 0, 0), (300, 96, 513, 8, 8), (1000, 128, 172, 0, 0), (31, 72, 136, 4, 0), (70, 2000, 40, 0, 0), (12, 3000, 500, 8, 8), (2000, 56, 24, 0, 0)]
ACTS = ("none", "relu", "gelu", "silu")


def act_ref(z, act):
    if act == "relu":
        return torch.relu(z)
    if act == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    return z * torch.sigmoid(z) if act == "silu" else z


def slope_ref(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        return torch.sigmoid(z) * (1 + z * torch.sigmoid(-z))
    return torch.ones_like(z)


def product(a, bb):
    """(product, bound of an fp32 one): exact sums of magnitudes by the chain's length."""
    a, bb = a.double(), bb.double()
    # pieces of fp32 values: three more sums of at most 2^-8 of the magnitude, and what is left out, below 2^-22 of it
    return a @ bb, (2 * (a.shape[1] + 40) + 8) * U * (a.abs() @ bb.abs())


def near(got, ref, k, dt, what):
    """Long sums: the 2-norm (four roundings of the output type's for good measure: its own, and an operand's)."""
    norm = ref.norm().item()
    if norm:
        rel = (got.double() - ref).norm().item() / norm
        assert rel <= 2 * U * math.sqrt(k + 64) + half(dt) * (1.0 if dt == BF16 else 0.0), (what, rel)


@pytest.mark.parametrize("n,d_in,d_out,pad,off", LINEAR_SIZES)
@BOTH
@pytest.mark.parametrize("act", ACTS)
def test_linear(n, d_in, d_out, pad, off, dt, act):
    b, g = nb(), rng(n + d_in + d_out)
    code = b.ACT_OF_NAME[act]
    x = Rows(n, d_in, dt, pad, off, randn((n, d_in), g, dt))
    w = Rows(d_in, d_out, dt, pad, off, randn((d_in, d_out), g, dt, d_in ** -0.5))
    bias = randn((d_out,), g) if d_out != 64 else None
    r = Rows(n, d_out, dt, 0, off, randn((n, d_out), g, dt)) if act in ("none", "silu") else None
    z, y = (Rows(n, d_out, dt, pad, off) if act != "relu" or n % 2 else None), Rows(n, d_out, dt, pad, off)
    ws = ws_of(b.no_linear_ws_bytes(dt, n, d_in, d_out))
    b.no_linear_fwd(x.t, w.t, bias, code, y.t, ws, residual=r.t if r else None, z=z.t if z else None)
    ref_z, tol_z = product(x.t, w.t)
    if bias is not None:
        ref_z = ref_z + bias.double()
        tol_z = tol_z + U * ref_z.abs()
    if z:
        close(z.t, ref_z, tol_z + half(dt) * (ref_z.abs() + tol_z) + TINY, "z")
        assert z.untouched()
    ref, tol = act_ref(ref_z, act), 1.2 * tol_z + 8 * U * ref_z.abs()       # (no slope is above 1.13)
    if r:
        ref = ref + r.t.double()
        tol = tol + U * ref.abs()
    close(y.t, ref, tol + half(dt) * (ref.abs() + tol) + TINY, "y")
    assert y.untouched()
    ws.fill_(0x3C)
    again = torch.empty((n, d_out), device="cuda", dtype=dt)
    b.no_linear_fwd(x.t, w.t, bias, code, again, ws, residual=r.t if r else None)
    assert torch.equal(again, y.t)
    if r:
        b.no_linear_fwd(x.t, w.t, bias, code, r.t, ws, residual=r.t)          # over the residual
        assert torch.equal(r.t, again) and r.untouched()

    gy = Rows(n, d_out, dt, pad, off, randn((n, d_out), g, dt))
    kept = Rows(n, d_out, dt, pad, off, ref_z.to(dt)) if act != "none" else None
    gx, gw, gb = Rows(n, d_in, dt, pad, off), Rows(d_in, d_out, dt, pad, off), torch.full((d_out,), MARK, device="cuda")
    b.no_linear_bwd(x.t, w.t, code, kept.t if kept else None, gy.t, gx.t, gw.t, gb, ws)
    slope = slope_ref(kept.t.double(), act) if kept else torch.ones((n, d_out), device="cuda", dtype=torch.float64)
    gz = gy.t.double() * slope
    smooth = act in ("gelu", "silu")
    gz_tol = (10 * U * gy.t.double().abs() * (1 + (kept.t.double().abs() if kept else 0))) if smooth else torch.zeros_like(gz)
    close(gb, gz.sum(0), gz_tol.sum(0) + (n + 2) * U * gz.abs().sum(0), "grad_bias")
    rounded = gz_tol + (half(dt) * (gz.abs() + gz_tol) if smooth else 0)
    for name, got, (ref, tol), more in (("grad_x", gx, product(gz, w.t.double().t()), rounded @ w.t.double().abs().t()),
                                        ("grad_w", gw, product(x.t.double().t(), gz), x.t.double().abs().t() @ rounded)):
        tol = tol + more
        close(got.t, ref, tol + half(dt) * (ref.abs() + tol) + TINY, name)
        assert got.untouched()
    gx2, gw2, gb2 = torch.empty((n, d_in), device="cuda", dtype=dt), torch.empty((d_in, d_out), device="cuda", dtype=dt), torch.empty_like(gb)
    ws.fill_(0x3C)
    b.no_linear_bwd(x.t, w.t, code, kept.t if kept else None, gy.t, gx2, None, None, ws)
    b.no_linear_bwd(x.t, w.t, code, kept.t if kept else None, gy.t, None, gw2, None, ws)
    b.no_linear_bwd(x.t, w.t, code, kept.t if kept else None, gy.t, None, None, gb2, ws)
    assert torch.equal(gx2, gx.t) and torch.equal(gw2, gw.t) and torch.equal(gb2, gb)


@pytest.mark.parametrize("n,d_in,d_out", [(4100, 1000, 4104), (2049, 1027, 1500), (700, 5000, 900), (16, 4096, 2048), (9000, 512, 768), (20_000, 300, 100), (40, 8192, 8192), (1, 8192, 8200)])
@BOTH
def test_linear_of_long_sums(n, d_in, d_out, dt):
    """Every tile width, whole and ragged, with and without splits of the reduction."""
    b, g = nb(), rng(n)
    x, w, gy = randn((n, d_in), g, dt), randn((d_in, d_out), g, dt, d_in ** -0.5), randn((n, d_out), g, dt)
    bias, y = randn((d_out,), g), torch.empty((n, d_out), device="cuda", dtype=dt)
    ws = ws_of(b.no_linear_ws_bytes(dt, n, d_in, d_out))
    b.no_linear_fwd(x, w, bias, b.NO_ACT_NONE, y, ws)
    near(y, torch.addmm(bias.double(), x.double(), w.double()), d_in, dt, "y")
    gx, gw, gb = torch.empty_like(x), torch.empty_like(w), torch.empty_like(bias)
    b.no_linear_bwd(x, w, b.NO_ACT_NONE, None, gy, gx, gw, gb, ws)
    near(gx, gy.double() @ w.double().t().contiguous(), d_out, dt, "grad_x")
    near(gw, x.double().t().contiguous() @ gy.double(), n, dt, "grad_w")
    near(gb, gy.double().sum(0), n, F32, "grad_bias")


@pytest.mark.parametrize("n,d_in,d_out", [(8, 40, 48), (100, 40, 48), (100, 41, 47), (700, 256, 300), (3000, 1024, 2048)])
@BOTH
def test_linear_counts(n, d_in, d_out, dt):
    """Rows from the device's count on are neither read nor written."""
    b, g = nb(), rng(n)
    x, w, bias, gy = randn((n, d_in), g, dt), randn((d_in, d_out), g, dt), randn((d_out,), g), randn((n, d_out), g, dt)
    z = randn((n, d_out), g, dt)
    ws = ws_of(b.no_linear_ws_bytes(dt, n, d_in, d_out))
    y, gx, gw, gb = (torch.empty_like(t) for t in (gy, x, w, bias))
    for here in (n, n // 2 + 1, 1, 0, -4):
        real = max(0, here)
        for t in (x, gy, z):
            t[real:] = NAN
        for act in (b.NO_ACT_GELU, b.NO_ACT_NONE):
            out, got = Rows(n, d_out, dt), Rows(n, d_in, dt)
            b.no_linear_fwd(x, w, bias, act, out.t, ws, n_rows=count(here))
            b.no_linear_bwd(x, w, act, z, gy, got.t, gw, gb, ws, n_rows=count(here))
            assert out.untouched(rows=real) and got.untouched(rows=real)
            ref = act_ref(torch.addmm(bias.double(), x[:real].double(), w.double()), "gelu" if act else "none")
            close(out.t[:real], ref, 1e-3 * d_in ** 0.5 + half(dt) * 2 * ref.abs(), "y")
            gz = gy[:real].double() * (slope_ref(z[:real].double(), "gelu") if act else 1.0)
            ref = gz @ w.double().t().contiguous()
            close(got.t[:real], ref, (1e-3 + 4 * half(dt)) * d_out ** 0.5 * 4 + half(dt) * 2 * ref.abs(), "grad_x")
            ref = x[:real].double().t().contiguous() @ gz
            close(gw, ref, (1e-3 + 4 * half(dt)) * n ** 0.5 * 4 + half(dt) * 2 * ref.abs(), "grad_w")
            if real == 0:
                assert (gw == 0).all() and (gb == 0).all()
    e = lambda *s: torch.empty(s, device="cuda", dtype=dt)  # noqa: E731
    b.no_linear_fwd(e(0, d_in), w, bias, b.NO_ACT_RELU, e(0, d_out), ws)
    b.no_linear_bwd(e(0, d_in), w, b.NO_ACT_RELU, e(0, d_out), e(0, d_out), e(0, d_in), gw, gb, ws)
    assert (gw == 0).all() and (gb == 0).all()


@pytest.mark.parametrize("n,d_in,d_out,pad,off", [(40_000, 602, 256, 0, 0), (40_001, 64, 250, 0, 0), (38_000, 67, 258, 1, 1), (70_000, 127, 130, 3, 0), (12_345, 1030, 1000, 2, 3), (20_000, 96, 512, 4, 4), (2000, 4100, 300, 0, 1),
                                                      (8192, 33, 1024, 0, 0), (9000, 32, 1024, 1, 0)])
def test_linear_rows_cut_inside_the_product(n, d_in, d_out, pad, off):
    """fp32 rows of a large product are read where they are, in whole steps of 32 and a rest: rows that are aligned to 4 bytes alone, a count, NaN behind it and in two rows."""
    b, g = nb(), rng(n)
    x = Rows(n, d_in, F32, pad, off, randn((n, d_in), g))
    w, bias, r = randn((d_in, d_out), g, F32, d_in ** -0.5), randn((d_out,), g), randn((n, d_out), g)
    ws = ws_of(b.no_linear_ws_bytes(F32, n, d_in, d_out))
    y = Rows(n, d_out, F32, pad, off)
    b.no_linear_fwd(x.t, w, bias, b.NO_ACT_NONE, y.t, ws, residual=r)
    ref, tol = product(x.t, w)
    ref = ref + bias.double() + r.double()
    close(y.t, ref, tol + 3 * U * (ref.abs() + bias.double().abs() + r.double().abs()) + TINY, "y")
    near(y.t, ref, d_in, F32, "y")
    assert y.untouched()
    whole, real = y.t.clone(), n - 777
    x.t[real:], x.t[3, 0], x.t[700, d_in - 1], x.t[900, d_in // 2] = NAN, NAN, NAN, INF
    ws.fill_(0xFF)                          # (NaN wherever a word of it is read unwritten)
    out = Rows(n, d_out, F32, pad, off)
    b.no_linear_fwd(x.t, w, bias, b.NO_ACT_NONE, out.t, ws, residual=r, n_rows=count(real))
    assert out.untouched(rows=real)
    assert out.t[3].isnan().all() and out.t[700].isnan().all() and not out.t[900].isfinite().any()
    fine = torch.ones(real, dtype=torch.bool, device="cuda")
    fine[[3, 700, 900]] = False
    assert torch.equal(out.t[:real][fine], whole[:real][fine])


@pytest.mark.parametrize("n,d_in,d_out", [(3000, 1000, 2900), (2900, 3000, 392), (1100, 700, 1100), (130, 300, 9000)])
@BOTH
def test_linear_of_middling_sizes(n, d_in, d_out, dt):
    b, g = nb(), rng(n)
    x, w, gy = randn((n, d_in), g, dt), randn((d_in, d_out), g, dt, d_in ** -0.5), randn((n, d_out), g, dt)
    r, y = randn((n, d_out), g, dt), torch.empty((n, d_out), device="cuda", dtype=dt)
    ws = ws_of(b.no_linear_ws_bytes(dt, n, d_in, d_out))
    b.no_linear_fwd(x, w, None, b.NO_ACT_NONE, y, ws, residual=r)
    near(y, x.double() @ w.double() + r.double(), d_in, dt, "y")
    gx, gw = torch.empty_like(x), torch.empty_like(w)
    b.no_linear_bwd(x, w, b.NO_ACT_NONE, None, gy, gx, gw, None, ws)
    near(gx, gy.double() @ w.double().t().contiguous(), d_out, dt, "grad_x")
    near(gw, x.double().t().contiguous() @ gy.double(), n, dt, "grad_w")


@pytest.mark.parametrize("n", [9, 500, 60_000])
def test_linear_by_the_identity_gives_the_rows(n):
    """The pieces' sum is the value, to the last bit, whichever kernel cuts them."""
    b, g = nb(), rng(n)
    x = randn((n, 250), g) * torch.pow(2.0, torch.randint(-60, 60, (n, 250), generator=g, device="cuda").float())
    y = torch.empty_like(x)
    b.no_linear_fwd(x, torch.eye(250, device="cuda"), None, b.NO_ACT_NONE, y, ws_of(b.no_linear_ws_bytes(F32, n, 250, 250)))
    assert torch.equal(y, x)


def test_linear_rows_whose_small_tiles_no_launch_holds():
    """1.2 billion rows of one value: 18.75 million tiles of 64 rows, whose threads would pass 2^32."""
    b, g, n, here = nb(), rng(1), 1_200_000_000, 1000
    x, y = torch.empty((n, 1), device="cuda", dtype=BF16), torch.empty((n, 1), device="cuda", dtype=BF16)
    x[:here], w = randn((here, 1), g, BF16), randn((1, 1), g, BF16)
    y[:here + 1] = MARK
    ws = torch.empty((b.no_linear_ws_bytes(BF16, n, 1, 1),), device="cuda", dtype=torch.uint8)
    b.no_linear_fwd(x, w, None, b.NO_ACT_NONE, y, ws, n_rows=count(here))
    ref = x[:here].double() * w.double()
    close(y[:here], ref, half(BF16) * ref.abs() + TINY)
    assert (y[here:here + 1] == MARK).all()


def test_linear_pieces_keep_what_fp32_holds():
    """Values of very different size in one sum, which meet only their like: each column of x is 2^-k w's row. And small values, and rows of zeros."""
    b, g = nb(), rng(3)
    n, d_in, d_out = 128, 192, 128
    scale = torch.pow(2.0, torch.linspace(-40, 40, d_in, device="cuda").round())
    x, w = randn((n, d_in), g) * scale, randn((d_in, d_out), g) / scale[:, None]
    y, ws = torch.empty((n, d_out), device="cuda"), ws_of(b.no_linear_ws_bytes(F32, n, d_in, d_out))
    b.no_linear_fwd(x, w, None, 0, y, ws)
    close(y, *product(x, w), "spread")
    b.no_linear_fwd(x * 0 + 1e-30, w * 0 + 1.0, None, 0, y, ws)
    close(y, torch.full_like(y, 1e-30).double() * d_in, 1e-30 * 1e-4)
    x[5], x[7, 3], x[9, 4] = 0.0, NAN, INF
    b.no_linear_fwd(x, w, None, 0, y, ws)
    assert (y[5] == 0).all() and y[7].isnan().all() and not y[9].isfinite().any() and y[10:].isfinite().all()


def test_linear_values_that_are_no_numbers_stay_in_their_rows():
    b, g = nb(), rng(5)
    for dt, n, d_in, d_out in ((BF16, 300, 96, 200), (F32, 300, 96, 200), (BF16, 4, 96, 200), (F32, 4, 96, 200), (BF16, 300, 97, 201)):
        x, w, gy, z = randn((n, d_in), g, dt), randn((d_in, d_out), g, dt), randn((n, d_out), g, dt), randn((n, d_out), g, dt)
        ws = ws_of(b.no_linear_ws_bytes(dt, n, d_in, d_out))
        y, gx, gw, gb = torch.empty_like(gy), torch.empty_like(x), torch.empty_like(w), torch.empty((d_out,), device="cuda")
        x[1, 3], gy[2, 7] = NAN, INF
        for act in (b.NO_ACT_NONE, b.NO_ACT_RELU, b.NO_ACT_GELU, b.NO_ACT_SILU):
            b.no_linear_fwd(x, w, None, act, y, ws)
            b.no_linear_bwd(x, w, act, z.abs(), gy, gx, gw, gb, ws)
            assert y[1].isnan().all() and y[0].isfinite().all() and y[2:].isfinite().all(), act
            assert not gx[2].isfinite().any() and gx[:2].isfinite().all() and gx[3:].isfinite().all()
            assert gw[3].isnan().all() and not gw[:, 7].isfinite().any() and gw[:3, :7].isfinite().all() and gw[4:, 8:].isfinite().all()
            assert gb[7] == INF and gb[:7].isfinite().all()


def test_linear_gradient_against_differences():
    b, g = nb(), rng(8)
    n, d_in, d_out, h = 10, 12, 14, 1e-4
    x, w, bias, gy = randn((n, d_in), g), randn((d_in, d_out), g), randn((d_out,), g), randn((n, d_out), g)
    ws = ws_of(b.no_linear_ws_bytes(F32, n, d_in, d_out))
    for act in ("gelu", "silu", "none"):
        z, y, gx, gw, gb = torch.empty_like(gy), torch.empty_like(gy), torch.empty_like(x), torch.empty_like(w), torch.empty_like(bias)
        b.no_linear_fwd(x, w, bias, b.ACT_OF_NAME[act], y, ws, z=z)
        b.no_linear_bwd(x, w, b.ACT_OF_NAME[act], z, gy, gx, gw, gb, ws)
        f = lambda xx, ww, cc: (act_ref(xx @ ww + cc, act) * gy.double()).sum().item()  # noqa: E731
        args = [t.double() for t in (x, w, bias)]
        for at, got in enumerate((gx, gw, gb)):
            for place in (0, got.numel() // 2, got.numel() - 1):
                d = torch.zeros_like(args[at]).view(-1)
                d[place] = h
                up, down = list(args), list(args)
                up[at], down[at] = args[at] + d.view_as(args[at]), args[at] - d.view_as(args[at])
                assert abs((f(*up) - f(*down)) / (2 * h) - got.view(-1)[place].item()) < 1e-4, (act, at)


# ------------------------------------------------------------------------------------------------------- orthogonalised updates

A, B, C = 3.4445, -4.7750, 2.0315


def steps_ref(x, steps):
    """The polynomial's steps in x's own type, matrix by matrix."""
    made = []
    for m in x:
        tall = m.shape[0] > m.shape[1]
        m = m.t().contiguous() if tall else m
        norm = torch.linalg.norm(m.double())
        m = (m.double() / norm).to(x.dtype) if norm > 0 else m
        for _ in range(steps):
            g = m @ m.t().contiguous()
            m = A * m + (B * g + C * (g @ g)) @ m
        made.append(m.t() if tall else m)
    return torch.stack(made)


def apart(got, ref):
    return ((got.double() - ref).norm() / ref.norm()).item()


# A step's rounding, in parts of |X|: a x, b G x and c G G x of singular values up to 1.21 add up to 34 |X| in magnitude, their factors are off by 2^-22 and the sums over k by 2 u sqrt(k), random in
# sign. Over five steps a perturbation grows up to 3.9-fold in each, which is no bound worth having; there the same formula in fp32 is the measure: its operands are held to 2^-24 and its
# sums rounded alike, so twice its error, and 8 x 2^-22 where that is smaller.
def one_step_tol(k):
    return 34 * (2.0 ** -22 + 2 * U * math.sqrt(k + 64))


@pytest.mark.parametrize("n,rows,cols", [(1, 1, 1), (2, 1, 9), (3, 9, 1), (1, 7, 5), (2, 64, 64), (3, 65, 130), (2, 130, 65), (1, 256, 602), (2, 602, 256), (1, 100, 1001), (4, 300, 41),
                                         (1, 1030, 1500), (1, 1500, 1030), (2, 520, 2048), (1, 2050, 2050)])
@BOTH
def test_orthogonalise(n, rows, cols, dt):
    b, g = nb(), rng(rows + cols)
    x = randn((n, rows, cols), g, dt, 0.01)
    x[0, 0] *= 30                           # a strong direction
    ws = ws_of(b.no_orthogonalise_ws_bytes(n, rows, cols))
    small = min(rows, cols)
    for steps in (1, 5):
        out = torch.empty_like(x)
        wide = torch.empty((n, rows, cols), device="cuda")
        b.no_orthogonalise(x, out, ws, steps=steps)
        ws.fill_(0x3C)
        b.no_orthogonalise(x, wide, ws, steps=steps)
        ref = steps_ref(x.double(), steps)
        tol = one_step_tol(max(rows, cols)) if steps == 1 else max(2 * apart(steps_ref(x.float(), steps), ref), 8 * 2.0 ** -22)
        assert apart(wide, ref) <= tol, (steps, apart(wide, ref), tol)
        assert torch.equal(out, wide.to(dt))
    # what it is for: every singular value of x / |x| went through the polynomial five times (a matrix of small difference has singular values that differ by no more than its norm)
    sv = torch.linalg.svdvals(x.double())
    sv = sv / sv.norm(dim=1, keepdim=True)
    for _ in range(5):
        sv = A * sv + B * sv ** 3 + C * sv ** 5
    diff = torch.linalg.svdvals(wide.double()).sort().values - sv.sort().values
    assert diff.abs().max() <= tol * ref.norm() + 1e-9 and sv.max() < 1.21
    again = x.clone()
    b.no_orthogonalise(again, again, ws)
    assert torch.equal(again, out)
    one = torch.empty((rows, cols), device="cuda")
    b.no_orthogonalise(x[n - 1], one, ws_of(b.no_orthogonalise_ws_bytes(1, rows, cols)))
    assert apart(one, wide[n - 1].double()) <= 2 * tol


@pytest.mark.parametrize("n,rows,cols", [(1, 117, 3860), (1, 3860, 117), (4, 96, 2500), (2, 3001, 260)])
@BOTH
def test_orthogonalise_long_and_narrow(n, rows, cols, dt):
    """Gram matrices whose long reduction is split."""
    b, g = nb(), rng(rows + cols)
    x = randn((n, rows, cols), g, dt, 0.01)
    ws, out, again = ws_of(b.no_orthogonalise_ws_bytes(n, rows, cols)), torch.empty((n, rows, cols), device="cuda"), torch.empty((n, rows, cols), device="cuda")
    for steps in (1, 5):
        b.no_orthogonalise(x, out, ws, steps=steps)
        ref = steps_ref(x.double(), steps)
        tol = one_step_tol(max(rows, cols)) if steps == 1 else max(2 * apart(steps_ref(x.float(), steps), ref), 8 * 2.0 ** -22)
        assert apart(out, ref) <= tol, (steps, apart(out, ref), tol)
        ws.fill_(0xFF)
        b.no_orthogonalise(x, again, ws, steps=steps)
        assert torch.equal(out, again)


@BOTH
def test_orthogonalise_strides_and_extremes(dt):
    b, g = nb(), rng(2)
    rows, cols = 40, 67
    base = randn((3, rows + 2, cols + 5), g, dt)
    x = base[:, 1:rows + 1, 3:cols + 3]
    marked = torch.full((3, rows + 2, cols + 5), MARK, device="cuda", dtype=dt)
    out = marked[:, 1:rows + 1, 3:cols + 3]
    ws = ws_of(b.no_orthogonalise_ws_bytes(3, rows, cols))
    b.no_orthogonalise(x, out, ws)
    dense = torch.empty((3, rows, cols), device="cuda", dtype=dt)
    b.no_orthogonalise(x.contiguous(), dense, ws)
    assert torch.equal(out, dense)
    marked[:, 1:rows + 1, 3:cols + 3] = MARK
    assert (marked == MARK).all()
    b.no_orthogonalise(x.contiguous() * 2.0 ** -60, out, ws)                # the size of a matrix does not count
    assert torch.equal(out, dense)
    if dt == F32:
        b.no_orthogonalise(x.contiguous() * 2.0 ** 100, out, ws)            # (squares beyond fp32)
        assert torch.equal(out, dense)
    y = x.contiguous()
    y[0], y[1, 3, 4] = 0.0, NAN
    b.no_orthogonalise(y, out, ws)
    assert (out[0] == 0).all() and out[1].isnan().all() and torch.equal(out[2], dense[2])
    y[1, 3, 4] = INF
    b.no_orthogonalise(y, out, ws)
    assert out[1].isnan().all() and torch.equal(out[2], dense[2])
    b.no_orthogonalise(y[:0], out[:0], ws_of(b.no_orthogonalise_ws_bytes(0, rows, cols)))


@pytest.mark.parametrize("n,rows,cols", [(1, 1, 3), (2, 602, 256), (3, 41, 300), (1, 777, 777)])
@BOTH
@pytest.mark.parametrize("nesterov", [False, True])
def test_muon_step(n, rows, cols, dt, nesterov):
    b, g = nb(), rng(rows + 1)
    w, m = randn((n, rows, cols), g), randn((n, rows, cols), g, F32, 0.1)
    ws = ws_of(b.no_orthogonalise_ws_bytes(n, rows, cols))
    lr, beta, decay, scale = 0.05, 0.9, 0.1, 1.5
    for _ in range(3):
        grad = randn((n, rows, cols), g, dt)
        w0, m0, g0 = w.double(), m.double(), grad.double()
        b.no_muon_step(w, m, grad, lr, beta, ws, nesterov=nesterov, weight_decay=decay, scale=scale)
        beta32, keep, step = (torch.tensor(v, dtype=F32).item() for v in (beta, 1 - lr * decay, lr * scale))
        ref_m = beta32 * m0 + g0
        close(m, ref_m, 2 * U * ((beta32 * m0).abs() + ref_m.abs()), "momentum")
        u = (g0 + beta32 * m.double()) if nesterov else m.double()
        ref_o = steps_ref(u, 5)
        tol = max(2 * apart(steps_ref(u.float(), 5), ref_o), 8 * 2.0 ** -22)
        got = (w0 * keep - w.double()) / step
        # the update by difference: the weights' own rounding besides (three operations, and their constants)
        assert (got - ref_o).norm() <= tol * ref_o.norm() + 4 * U * w0.norm() / step
    one_w, one_m = w[0].clone(), m[0].clone()
    b.no_muon_step(one_w, one_m, grad[0], 0.0, 0.0, ws, nesterov=nesterov)
    assert torch.equal(one_w, w[0]) and torch.equal(one_m, grad[0].float())
