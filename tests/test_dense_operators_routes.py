"""The products of the dense layer and of updates by every kind of tile, and every way of splitting a reduction, that sizes lead to, on whole tiles and ragged ones, element by element (test_products_plan.py holds
the lists below to what the library plans); and workspaces made for larger sizes.

Element bounds: a sum of k products takes no more than k roundings, each of a partial sum and so of 2 u of the sum of magnitudes at most (u = 2^-24, twice that in a matrix instruction, which may cut). Their signs are
random: eight standard deviations are 16 u sqrt(k) of the magnitudes, which the 10^8 elements of a test do not reach. A value in its wrong place is off by a term or more."""
import math

import pytest
import torch

from .test_dense_operators import ACTS, act_ref, apart, slope_ref, steps_ref
from .test_operators import BF16, F32, INF, NAN, TINY, U, Rows, close, half, nb, randn, rng, ws_of

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])

# rows, sides
LINEAR_F32 = [(132, 192, 145), (192, 192, 160), (164, 1664, 130), (136, 192, 1728), (1536, 192, 192), (6144, 136, 153), (192, 5632, 162),
              (192, 192, 7104), (16832, 141, 144), (192, 1457, 2304), (133, 5832, 928), (8399, 384, 384), (1120, 1088, 1139), (1536, 256, 4224),
              (512, 6400, 768), (6144, 3968, 130), (32, 1344, 1152), (1024, 1280, 1152), (5632, 151, 2176), (7424, 4864, 128), (6144, 640, 6272),
              (1024, 10, 8), (1088, 32, 32)]
LINEAR_BF16 = [(285, 280, 303), (384, 448, 384), (266, 7053, 264), (2040, 261, 1838), (384, 8128, 384), (17412, 316, 271), (384, 597, 8813),
               (607, 6528, 624), (11008, 793, 320), (10752, 384, 896), (512, 1024, 7808), (718, 7432, 1296), (1280, 1000, 6912), (5632, 333, 6144),
               (9984, 1536, 768), (544, 32, 768), (4480, 547, 9), (17152, 8, 3008), (2432, 128, 2304), (17629, 3704, 11), (64, 4240, 4608),
               (4864, 64, 4224), (128, 2616, 5952), (768, 8064, 576), (16744, 5840, 72), (1351, 8832, 768), (56704, 1280, 128), (4618, 7296, 512),
               (8420, 256, 8352), (9216, 256, 8576), (38976, 192, 4224), (23040, 192, 8048), (34944, 32, 32), (2067, 6971, 8), (8, 2070, 7184),
               (1216, 32, 6688), (64, 8384, 512), (264, 4864, 2304), (256, 4224, 5344), (4224, 6080, 256), (5760, 192, 7968), (192, 7744, 6464),
               (768, 6024, 2880), (256, 8296, 8832), (16616, 228, 6912), (16640, 256, 7592), (1812, 8225, 2397), (53896, 256, 3328)]
# matrices, rows, columns
UPDATES = [(1, 130, 136), (1, 192, 192), (1, 196, 196), (1, 240, 224), (1, 1152, 1064), (1, 1408, 1152), (8, 816, 669), (7, 768, 917), (6, 1109, 1096),
           (6, 1152, 1184), (7, 1552, 1584), (8, 1536, 1664), (1, 224, 256), (5, 2267, 129), (8, 1792, 256), (8, 256, 2240), (8, 232, 3328),
           (6, 2560, 320), (8, 256, 3200), (8, 3328, 264), (7, 384, 2304), (7, 328, 3840), (5, 2496, 592), (5, 1536, 768), (8, 3840, 512),
           (4, 2048, 1024), (4, 768, 3840), (1, 2020, 16), (1, 3295, 16), (1, 16, 3356), (1, 3136, 32), (1, 32, 3264), (1, 320, 256), (5, 297, 1064),
           (7, 710, 835), (5, 3080, 584), (5, 588, 3136), (7, 1028, 1144), (6, 1192, 1152), (8, 1447, 968), (8, 656, 3408), (3, 3198, 1120),
           (3, 3328, 1152), (7, 768, 3692), (7, 1649, 1548), (6, 1920, 1792)]
# sizes of real use: a block's two layers, forward and back, a hop's vertices, a narrow layer, updates of large matrices
LARGE_F32 = [(24_922, 602, 256), (10_001, 256, 47)]
LARGE_BF16 = [(16_384, 8192, 2048), (8192, 2048, 8192), (8200, 2056, 8200), (8192, 8192, 2048), (16_384, 1000, 2048)]
LARGE_UPDATES = [(2, 602, 256), (1, 4096, 4096), (4, 512, 2048), (6, 1664, 3722), (6, 2089, 907), (2, 3784, 2859)]


def t(m):
    return m.t().contiguous()


def product(a, b):
    """(sum, bound of its error) in fp32, of pieces or not: what pieces leave out lies below 2^-22 of a product, twice."""
    return a @ b, (16 * U * math.sqrt(a.shape[1] + 64) + 2.0 ** -21) * (a.abs() @ b.abs())


def close_rounded(got, ref, tol, dt, what):
    close(got, ref, tol + half(dt) * (ref.abs() + tol) + TINY, what)


def linear(n, d_in, d_out, dt, act):
    """Forward with everything that its epilogue can do, and the three gradients; every element, every byte beside them, and the same bits again."""
    b, g = nb(), rng(n + d_in + d_out)
    x, w, gy = randn((n, d_in), g, dt), randn((d_in, d_out), g, dt, d_in ** -0.5), randn((n, d_out), g, dt)
    bias, r = randn((d_out,), g), randn((n, d_out), g, dt)
    ws = ws_of(b.no_linear_ws_bytes(dt, n, d_in, d_out))
    y, z, gx, gw, gb = Rows(n, d_out, dt, 8, 0), Rows(n, d_out, dt, 8, 0), Rows(n, d_in, dt, 8, 0), Rows(d_in, d_out, dt, 8, 0), torch.empty((d_out,), device="cuda")
    code = b.ACT_OF_NAME[act]
    b.no_linear_fwd(x, w, bias, code, y.t, ws, residual=r, z=z.t)
    b.no_linear_bwd(x, w, code, z.t if act != "none" else None, gy, gx.t, gw.t, gb, ws)
    assert y.untouched() and z.untouched() and gx.untouched() and gw.untouched()
    again = [torch.empty_like(v) for v in (gy, gy, x, w, bias)]
    ws.fill_(0xFF)
    b.no_linear_fwd(x, w, bias, code, again[0], ws, residual=r, z=again[1])
    b.no_linear_bwd(x, w, code, again[1] if act != "none" else None, gy, again[2], again[3], again[4], ws)
    assert all(torch.equal(a, o) for a, o in zip(again, (y.t, z.t, gx.t, gw.t, gb)))
    del again
    xd, wd = x.double(), w.double()
    ref, tol = product(xd, wd)
    ref = ref + bias.double()
    tol = tol + U * ref.abs()
    close_rounded(z.t, ref, tol, dt, "z")
    ref, tol = act_ref(ref, act) + r.double(), 1.2 * tol + 8 * U * ref.abs()          # (no slope is above 1.13)
    close_rounded(y.t, ref, tol + U * ref.abs(), dt, "y")
    del ref, tol
    slope, smooth = slope_ref(z.t.double(), act), act in ("gelu", "silu")
    gz = gy.double() * slope
    # a smooth slope's own error, and where gz is rounded: errors of half a step at most and random sign, eight standard deviations of their sum
    slope_tol = 10 * U * gy.double().abs() * (1 + z.t.double().abs()) if smooth else None
    step = 8 * half(dt) if smooth else 0.0
    for what, got, a, c in (("grad_x", gx, gz, t(wd)), ("grad_w", gw, t(xd), gz)):
        ref, tol = product(a, c)
        if smooth:
            tol = tol + step * ((a * a) @ (c * c)).sqrt() + (slope_tol @ c.abs() if what == "grad_x" else a.abs() @ slope_tol)
        close_rounded(got.t, ref, tol, dt, what)
        if dt == BF16:      # two roundings of a value by half a step at most, spread evenly: sqrt(2 / 3) of it in the 2-norm
            assert apart(got.t, ref) <= half(dt) * math.sqrt(2 / 3), what
        del ref, tol
    close(gb, gz.sum(0), (8 * U * math.sqrt(n + 64)) * gz.abs().sum(0) + (slope_tol.sum(0) if smooth else 0), "grad_bias")


@pytest.mark.parametrize("n,d_in,d_out", LINEAR_F32)
def test_linear_f32_by_every_route(n, d_in, d_out):
    linear(n, d_in, d_out, F32, "none")


@pytest.mark.parametrize("n,d_in,d_out", LINEAR_BF16)
def test_linear_bf16_by_every_route(n, d_in, d_out):
    linear(n, d_in, d_out, BF16, "none")


@pytest.mark.parametrize("n,d_in,d_out", LARGE_F32)
@pytest.mark.parametrize("act", ACTS)
def test_linear_f32_of_real_use(n, d_in, d_out, act):
    linear(n, d_in, d_out, F32, act)


@pytest.mark.parametrize("n,d_in,d_out", LARGE_BF16)
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_linear_bf16_of_real_use(n, d_in, d_out, act):
    linear(n, d_in, d_out, BF16, act)


@pytest.mark.parametrize("n,rows,cols", UPDATES + LARGE_UPDATES)
def test_updates_by_every_route(n, rows, cols):
    """One step element by element: what a product adds to its factors' errors is 16 u sqrt(k) of the magnitudes, and each factor is held to 2^-22; three products follow one another, so four times that of the magnitudes
    a |X| + |b| |G| |X| + c |G| |G| |X| bounds all. Then five steps, against the same formula in fp32 (see test_dense_operators.py)."""
    b, g = nb(), rng(rows + cols)
    x = randn((n, rows, cols), g, F32, 0.01)
    x[0, 0] *= 30
    ws, out, again = ws_of(b.no_orthogonalise_ws_bytes(n, rows, cols)), torch.full((n, rows, cols + 8), 77.0, device="cuda"), torch.empty((n, rows, cols), device="cuda")
    b.no_orthogonalise(x, out[:, :, :cols], ws, steps=1)
    assert (out[:, :, cols:] == 77.0).all()
    ref = steps_ref(x.double(), 1)
    for got, made, one in zip(out[:, :, :cols], ref, x.double()):
        m = (one / one.norm()).abs()
        m = m if rows <= cols else t(m)
        gram = m @ t(m)
        size = 3.4445 * m + (4.7750 * gram + 2.0315 * (gram @ gram)) @ m
        size = size if rows <= cols else t(size)
        close(got, made, 4 * (2.0 ** -22 + 16 * U * math.sqrt(max(rows, cols) + 64)) * size + U * made.abs(), "one step")
    b.no_orthogonalise(x, out[:, :, :cols], ws, steps=5)
    ws.fill_(0xFF)
    b.no_orthogonalise(x, again, ws, steps=5)
    assert torch.equal(again, out[:, :, :cols]) and (out[:, :, cols:] == 77.0).all()
    ref = steps_ref(x.double(), 5)
    assert apart(again, ref) <= max(2 * apart(steps_ref(x, 5), ref), 8 * 2.0 ** -22)


@pytest.mark.parametrize("n,rows,cols", [(2, 602, 256), (1, 4096, 4096), (2, 3784, 2859)])
@BOTH
def test_muon_step_is_that_of_the_orthogonalised_momentum(n, rows, cols, dt):
    b, g = nb(), rng(rows)
    w, m, grad = randn((n, rows, cols), g), randn((n, rows, cols), g, F32, 0.1), randn((n, rows, cols), g, dt)
    w0, m0, made, ws = w.double(), m.double(), torch.empty_like(w), ws_of(b.no_orthogonalise_ws_bytes(n, rows, cols))
    lr, beta, decay, scale = 0.05, 0.9, 0.1, 1.5
    b.no_muon_step(w, m, grad, lr, beta, ws, nesterov=False, weight_decay=decay, scale=scale)
    beta32, lr32, decay32 = (torch.tensor(v, dtype=F32).double().item() for v in (beta, lr, decay))
    ref = beta32 * m0 + grad.double()
    close(m, ref, 2 * U * ((beta32 * m0).abs() + ref.abs()), "momentum")
    b.no_orthogonalise(m, made, ws)
    # (1 - lr decay and lr scale are rounded once or twice, each product and the difference once)
    kept, step = (1 - lr32 * decay32) * w0, lr32 * scale * made.double()
    close(w, kept - step, 4 * U * (kept.abs() + step.abs()), "weights")


@pytest.mark.parametrize("most,fewer", [((9, 256, 256), (8, 256, 256)), ((9, 256, 256), (1, 255, 256)), ((2504, 2048, 8192), (2276, 2048, 8192)), ((130, 3000, 500), (97, 2990, 493))])
@BOTH
def test_linear_in_a_workspace_of_larger_sizes(most, fewer, dt):
    b, g = nb(), rng(fewer[0])
    n, d_in, d_out = fewer
    x, w, gy, z = randn((n, d_in), g, dt), randn((d_in, d_out), g, dt, d_in ** -0.5), randn((n, d_out), g, dt), randn((n, d_out), g, dt)
    made = []
    for sizes in (most, fewer):
        size = b.no_linear_ws_bytes(dt, *sizes)
        ws = ws_of(size + 4096)             # (and what lies behind it stays)
        ws[size:] = 0x5A
        y, gx, gw, gb = Rows(n, d_out, dt), Rows(n, d_in, dt), Rows(d_in, d_out, dt), torch.empty((d_out,), device="cuda")
        b.no_linear_fwd(x, w, gb.fill_(0.5), b.NO_ACT_GELU, y.t, ws[:size])
        b.no_linear_bwd(x, w, b.NO_ACT_GELU, z, gy, gx.t, gw.t, gb, ws[:size])
        assert y.untouched() and gx.untouched() and gw.untouched() and (ws[size:] == 0x5A).all()
        made.append((y.t, gx.t, gw.t, gb))
    for a, c in zip(*made):
        assert torch.equal(a, c)


@pytest.mark.parametrize("most,fewer", [((1, 256, 3900), (1, 256, 3300)), ((4, 100, 2600), (3, 96, 2500)), ((7, 3608, 63), (7, 3496, 63))])
@BOTH
def test_updates_in_a_workspace_of_larger_sizes(most, fewer, dt):
    b, g = nb(), rng(fewer[1])
    x, made = randn(fewer, g, dt, 0.01), []
    for sizes in (most, fewer):
        size = b.no_orthogonalise_ws_bytes(*sizes)
        ws = ws_of(size + 4096)
        ws[size:] = 0x5A
        made.append(b.no_orthogonalise(x, torch.empty(fewer, device="cuda"), ws[:size]))
        assert (ws[size:] == 0x5A).all()
    assert torch.equal(*made)


# ------------------------------------------------------------------------------------------------------- far rows, long sides

FAR = (1 << 22) + 64            # bytes between rows above what a tile's 31-bit offsets take


@pytest.mark.parametrize("n,d_in,d_out", [(1, 100, 264), (5, 256, 64), (300, 256, 320), (300, 130, 70)])
@BOTH
def test_linear_with_rows_far_apart(n, d_in, d_out, dt):
    """Rows (and rows of the matrix) more than 4 MB apart are laid out first."""
    b, g = nb(), rng(n)
    pitch = FAR // (2 if dt == BF16 else 4)

    def far(rows, cols, like=None):
        m = torch.empty((rows * pitch,), device="cuda", dtype=dt).view(rows, pitch)[:, :cols + 1]
        m[:, cols] = 77.0                   # behind each row
        if like is not None:
            m[:, :cols] = like
        return m[:, :cols], m[:, cols]
    x, w, gy = randn((n, d_in), g, dt), randn((d_in, d_out), g, dt), randn((n, d_out), g, dt)
    ws, bias = ws_of(b.no_linear_ws_bytes(dt, n, d_in, d_out)), torch.zeros((d_out,), device="cuda")
    made = []
    for place in (lambda r, c, like=None: (torch.empty((r, c), device="cuda", dtype=dt) if like is None else like, None), far):
        (xx, _), (ww, _), (gg, _) = place(n, d_in, x), place(d_in, d_out, w), place(n, d_out, gy)
        outs = place(n, d_out), place(n, d_out), place(n, d_in), place(d_in, d_out)
        y, z, gx, gw = (o[0] for o in outs)
        gb = torch.empty_like(bias)
        b.no_linear_fwd(xx, ww, bias, b.NO_ACT_SILU, y, ws, residual=gg, z=z)
        b.no_linear_bwd(xx, ww, b.NO_ACT_SILU, z, gg, gx, gw, gb, ws)
        assert all(o[1] is None or (o[1] == 77.0).all() for o in outs)
        made.append([o.clone() for o in (y, z, gx, gw, gb)])
        ref, tol = product(x.double(), w.double())
        close_rounded(z, ref, tol, dt, "z")
        ref = act_ref(ref, "silu") + gy.double()
        close_rounded(y, ref, 1.2 * tol + 8 * U * ref.abs() + 2 * U * gy.double().abs(), dt, "y")
    for a, c in zip(*made):                 # (the same products on copies of the same values; few rows may be read as they are, in another order)
        if n > 8:
            assert torch.equal(a, c)


def test_linear_rows_far_apart_in_large_tiles():
    """fp32 rows whose tile's offsets would leave 31 bits are not cut inside the product."""
    b, g, n, d_in, d_out = nb(), rng(3), 4096, 256, 4096
    pitch = FAR // 4
    assert n * pitch * 4 < 20 << 30
    x = torch.empty((n * pitch,), device="cuda").view(n, pitch)[:, :d_in]
    x.copy_(randn((n, d_in), g))
    w, y, near = randn((d_in, d_out), g), torch.empty((n, d_out), device="cuda"), torch.empty((n, d_out), device="cuda")
    ws = ws_of(b.no_linear_ws_bytes(F32, n, d_in, d_out))
    b.no_linear_fwd(x, w, None, b.NO_ACT_NONE, y, ws)
    b.no_linear_fwd(x.contiguous(), w, None, b.NO_ACT_NONE, near, ws)
    ref, tol = product(x.double(), w.double())
    close_rounded(y, ref, tol, F32, "far")
    close_rounded(near, ref, tol, F32, "near")


LONGEST = 1 << 20


@pytest.mark.parametrize("n,d_in,d_out", [(1, LONGEST, 3), (3, LONGEST - 1, 40), (3, 40, LONGEST), (20, 9, LONGEST - 5), (300, LONGEST, 16), (300, 64, LONGEST)])
@BOTH
def test_linear_of_the_longest_sides(n, d_in, d_out, dt):
    linear(n, d_in, d_out, dt, "none")


@pytest.mark.parametrize("rows,cols", [(32_768, 9), (9, 32_768), (32_768, 130), (130, 32_767), (32_768, 1)])
def test_updates_of_the_longest_sides(rows, cols):
    test_updates_by_every_route(1, rows, cols)


# ------------------------------------------------------------------------------------------------------- values at the ends of the range

def alike(got, ref, tol, what):
    """NaN and infinities where the formula has them, the others close."""
    got = got.double()
    assert torch.equal(got.isnan(), ref.isnan()), what
    wide = ref.isinf()
    assert torch.equal(got[wide], ref[wide]), what
    fine = ref.isfinite()
    close(got[fine], ref[fine], tol[fine] + TINY, what)


def scale_of(a, c):
    """Magnitudes of a product of which some factors are no numbers: the others'."""
    fine = lambda m: torch.where(m.isfinite(), m, 0.0).abs()  # noqa: E731
    return (16 * U * math.sqrt(a.shape[1] + 64) + 2.0 ** -21) * (fine(a) @ fine(c))


@pytest.mark.parametrize("n,d_in,d_out", [(8, 64, 72), (9, 64, 72), (300, 301, 263), (300, 8000, 40), (40, 24, 8000), (10_001, 256, 47), (24_922, 602, 256), (40_001, 64, 250), (2000, 4100, 300), (4096, 24, 4096),
                                          (2048, 2048, 1100)])
def test_linear_f32_at_the_ends_of_the_range(n, d_in, d_out):
    """Infinite operands, and finite ones that round to none of bf16, give what products in fp32 give, whatever the number of rows."""
    b, g = nb(), rng(n + d_out)
    x, w, gy = randn((n, d_in), g), randn((d_in, d_out), g), randn((n, d_out), g)
    x[1, 2], x[2, 5], x[n - 1, d_in - 1], x[4, 1], x[4, d_in // 2] = INF, -INF, INF, INF, INF
    x[5, 3], x[6, 4] = 3.3999e38, -3.4e38           # above the largest bf16, 3.3895e38
    w[3], w[4] = w[3] * 1e-3, w[4] * 1e-3
    w[2, 0], w[5, d_out - 1] = 0.0, 2.0             # (a product of infinity and 0; a value of one piece)
    gy[1, 2], gy[3, d_out - 1] = -INF, INF
    gy[5, 6], gy[7, 7] = 3.3999e38, NAN
    ws = ws_of(b.no_linear_ws_bytes(F32, n, d_in, d_out))
    y, gx, gw, gb = torch.empty((n, d_out), device="cuda"), torch.empty_like(x), torch.empty_like(w), torch.empty((d_out,), device="cuda")
    b.no_linear_fwd(x, w, None, b.NO_ACT_NONE, y, ws)
    ref = x.double() @ w.double()
    assert ref[5].isfinite().all() and ref[5].abs().max() > 1e34 and ref[2, :d_out - 1].isinf().all() and ref[1, 0].isnan()
    alike(y, ref, scale_of(x.double(), w.double()), "y")
    w[:, 6] *= 1e-3
    x[5] = x[5] * 1e-3                              # (so that what meets the gradient's large value stays in range)
    b.no_linear_bwd(x, w, b.NO_ACT_NONE, None, gy, gx, gw, gb, ws)
    ref = gy.double() @ t(w.double())
    assert ref[5].isfinite().all() and ref[5].abs().max() > 1e34
    alike(gx, ref, scale_of(gy.double(), t(w.double())), "grad_x")
    ref = t(x.double()) @ gy.double()
    ref = torch.where(ref.abs() > 3.4028235e38, ref.sign() * INF, ref)
    alike(gw, ref, scale_of(t(x.double()), gy.double()), "grad_w")
