"""The operators of a dense block and of its update on a stream of the caller's whose inputs arrive late, captured and replayed among eager work, in two graphs that share a workspace, at rows whose
offsets pass 2^32 bytes, on a given stream that is not the current one, and together as a training step uses them."""
import pytest
import torch

from .test_dense_operators import act_ref, apart, norm_ref, slope_ref, steps_ref
from .test_operators import BF16, F32, Rows, U, close, count, nb, randn, rng, ws_of

pytestmark = pytest.mark.gpu


def layernorm(n, d, dt):
    b, g = nb(), rng(n + d)
    x, gy, w, c = randn((n, d), g, dt), randn((n, d), g, dt), 1 + 0.2 * randn((d,), g), randn((d,), g)
    e = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
    y, mean, rstd, gx, gw, gb, ws = torch.empty_like(x), e(n), e(n), torch.empty_like(x), e(d), e(d), ws_of(b.no_layernorm_ws_bytes(n, d))

    def call():
        b.no_layernorm_fwd(x, w, c, 1e-5, y, mean=mean, rstd=rstd)
        b.no_layernorm_bwd(x, w, mean, rstd, gy, gx, gw, gb, ws)
    return [x, gy, w], [y, mean, rstd, gx, gw, gb], call


def linear(n, d_in, d_out, dt, act="gelu"):
    b, g = nb(), rng(n + d_in)
    x, w, bias, gy = randn((n, d_in), g, dt), randn((d_in, d_out), g, dt, d_in ** -0.5), randn((d_out,), g), randn((n, d_out), g, dt)
    y, z, gx, gw, gb, ws = (torch.empty_like(t) for t in (gy, gy, x, w, bias)), None, None, None, None, ws_of(b.no_linear_ws_bytes(dt, n, d_in, d_out))
    y, z, gx, gw, gb = y

    def call():
        b.no_linear_fwd(x, w, bias, b.ACT_OF_NAME[act], y, ws, z=z)
        b.no_linear_bwd(x, w, b.ACT_OF_NAME[act], z, gy, gx, gw, gb, ws)
    return [x, w, gy], [y, z, gx, gw, gb], call


def orthogonalise(n, r, c, dt):
    b, g = nb(), rng(r + c)
    x = randn((n, r, c), g, dt)
    out, ws = torch.empty_like(x), ws_of(b.no_orthogonalise_ws_bytes(n, r, c))
    return [x], [out], lambda: b.no_orthogonalise(x, out, ws)


def muon(n, r, c, dt):
    b, g = nb(), rng(r + c)
    w, m, grad = randn((n, r, c), g), randn((n, r, c), g), randn((n, r, c), g, dt)
    out, ws = [torch.empty_like(w), torch.empty_like(m)], ws_of(b.no_orthogonalise_ws_bytes(n, r, c))

    def call():                                    # (in place: on copies, so that every replay starts alike)
        out[0].copy_(w)
        out[1].copy_(m)
        b.no_muon_step(out[0], out[1], grad, 0.1, 0.9, ws, weight_decay=0.1)
    return [w, m, grad], out, call


ROUTES = [(layernorm, 700, 2049, BF16), (layernorm, 300, 100, F32), (layernorm, 70, 20_000, F32),
          (linear, 1, 512, 2048, BF16), (linear, 5, 300, 1001, F32), (linear, 33, 2048, 72, BF16), (linear, 1000, 256, 300, F32), (linear, 300, 1027, 129, BF16),
          (linear, 4100, 512, 2048, BF16), (linear, 9000, 100, 47, F32), (linear, 3000, 1000, 2000, F32),
          (orthogonalise, 2, 300, 100, F32), (orthogonalise, 1, 1500, 1600, BF16), (muon, 2, 256, 602, BF16), (muon, 1, 2100, 2050, F32),
          (layernorm, 200, 16_384, BF16), (linear, 25_000, 602, 256, F32), (linear, 2000, 4100, 300, F32), (orthogonalise, 1, 117, 3860, F32)]


@pytest.mark.parametrize("route", ROUTES, ids=lambda r: "-".join(getattr(x, "__name__", str(x)) for x in r))
def test_routes_on_another_stream_and_in_a_graph(route):
    inputs, outputs, call = route[0](*route[1:])
    call()
    torch.cuda.synchronize()
    eager = [t.clone() for t in outputs]
    kept = [t.clone() for t in inputs]
    side, late = torch.cuda.Stream(), torch.empty(1 << 28, device="cuda")

    def spoil():
        for t in inputs:
            t.zero_()
        for t in outputs:
            t.fill_(7)
        torch.cuda.synchronize()
    spoil()
    with torch.cuda.stream(side):                  # some milliseconds before the inputs are there
        for _ in range(8):
            late.add_(1.0)
        for t, k in zip(inputs, kept):
            t.copy_(k)
        call()
    side.synchronize()
    for at, (t, want) in enumerate(zip(outputs, eager)):
        assert torch.equal(t, want), at
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for turn in range(4):
        spoil()
        for t, k in zip(inputs, kept):
            t.copy_(k)
            if turn == 2:                          # new inputs under the same graph
                t.mul_(0.5).add_(0.125)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in outputs]
        for t in outputs:
            t.fill_(7)
        call()
        torch.cuda.synchronize()
        for at, (t, want) in enumerate(zip(outputs, replayed)):
            assert torch.equal(t, want), (turn, at)
        if turn != 2:
            for at, (t, want) in enumerate(zip(replayed, eager)):
                assert torch.equal(t, want), (turn, at)


def test_two_graphs_share_a_workspace_in_turn():
    """Nothing in a workspace has to survive a call."""
    b, g = nb(), rng(1)
    x, w, v = randn((300, 200), g), randn((200, 100), g), randn((150, 260), g)
    y, o = torch.empty((300, 100), device="cuda"), torch.empty((150, 260), device="cuda")
    ws = ws_of(max(b.no_linear_ws_bytes(F32, 300, 200, 100), b.no_orthogonalise_ws_bytes(1, 150, 260)))
    calls = [lambda: b.no_linear_fwd(x, w, None, b.NO_ACT_SILU, y, ws), lambda: b.no_orthogonalise(v, o, ws)]
    graphs = []
    for c in calls:
        c()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            c()
    want = [y.clone(), o.clone()]
    for order in ((0, 1), (1, 0), (0, 0), (1, 1, 0)):
        y.fill_(7)
        o.fill_(7)
        for k in order:
            graphs[k].replay()
        torch.cuda.synchronize()
        assert (0 not in order or torch.equal(y, want[0])) and (1 not in order or torch.equal(o, want[1]))


def test_rows_whose_offsets_pass_32_bits():
    b, g = nb(), rng(2)
    n, d_in, d_out = 2_200_000, 1024, 16           # x: 4.5 GB
    x = torch.zeros((n, d_in), dtype=BF16, device="cuda")
    rows = torch.tensor([0, 1, 1_048_575, 2_097_151, 2_097_152, n - 1], device="cuda")
    x[rows] = randn((6, d_in), g, BF16)
    w, bias, y = randn((d_in, d_out), g, BF16), randn((d_out,), g), torch.empty((n, d_out), dtype=BF16, device="cuda")
    ws = ws_of(b.no_linear_ws_bytes(BF16, n, d_in, d_out))
    b.no_linear_fwd(x, w, bias, b.NO_ACT_NONE, y, ws)
    ref = torch.addmm(bias.double(), x[rows].double(), w.double())
    close(y[rows], ref, 2.0 ** -8 * ref.abs() + 1e-3)
    other = torch.ones((n,), dtype=torch.bool, device="cuda")
    other[rows] = False
    assert (y[other] == bias.to(BF16)).all()
    gy = torch.zeros((n, d_out), dtype=BF16, device="cuda")
    gy[rows] = randn((6, d_out), g, BF16)
    gw, gx = torch.empty_like(w), torch.empty_like(x)
    b.no_linear_bwd(x, w, b.NO_ACT_NONE, None, gy, gx, gw, None, ws)
    ref = x[rows].double().t().contiguous() @ gy[rows].double()
    close(gw, ref, 2.0 ** -8 * ref.abs() + 1e-3)
    ref = gy[rows].double() @ w.double().t().contiguous()
    close(gx[rows], ref, 2.0 ** -8 * ref.abs() + 1e-3)
    del ws, gy
    mean, rstd, s = torch.empty((n,), device="cuda"), torch.empty((n,), device="cuda"), gx
    b.no_layernorm_fwd(x, None, None, 1e-5, s, mean=mean, rstd=rstd)
    _, ref_mean, ref_rstd, ref_y = norm_ref(x[rows], None, None, None, 1e-5)
    close(s[rows], ref_y, 2.0 ** -8 * ref_y.abs() + 1e-4)
    close(mean[rows], ref_mean, 1e-5)
    grad = torch.empty_like(x)
    gw = torch.empty((d_in,), device="cuda")
    gy = torch.zeros_like(x)
    gy[rows] = randn((6, d_in), g, BF16)
    b.no_layernorm_bwd(x, None, mean, rstd, gy, grad, gw, None, ws_of(b.no_layernorm_ws_bytes(n, d_in)))
    u_ = (x[rows].double() - mean[rows, None].double()) * rstd[rows, None].double()
    close(gw, (gy[rows].double() * u_).sum(0), 1e-4)
    want = rstd[rows, None].double() * (gy[rows].double() - gy[rows].double().mean(1, keepdim=True) - u_ * (gy[rows].double() * u_).mean(1, keepdim=True))
    close(grad[rows], want, 2.0 ** -8 * want.abs() + 1e-4)


def test_a_block_and_its_update_together():
    """norm -> layer -> layer with residual, back, and a step of both matrices, against the same in 64 bits; rows past the device's count are not touched by any of it."""
    b, g = nb(), rng(9)
    n, here, d, h = 300, 271, 96, 200
    e = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
    x, gamma, beta = randn((n, d), g), 1 + 0.1 * randn((d,), g), 0.1 * randn((d,), g)
    w1, b1, w2, b2 = randn((d, h), g, F32, d ** -0.5), randn((h,), g), randn((h, d), g, F32, h ** -0.5), randn((d,), g)
    target, k = randn((n, d), g), count(here)
    ws = ws_of(max(b.no_linear_ws_bytes(F32, n, d, h), b.no_linear_ws_bytes(F32, n, h, d), b.no_layernorm_ws_bytes(n, d), b.no_orthogonalise_ws_bytes(1, d, h), b.no_orthogonalise_ws_bytes(1, h, d)))
    u_, mean, rstd, z1, a1, y = Rows(n, d, F32), e(n), e(n), Rows(n, h, F32), Rows(n, h, F32), Rows(n, d, F32)
    b.no_layernorm_fwd(x, gamma, beta, 1e-5, u_.t, mean=mean, rstd=rstd, n_rows=k)
    b.no_linear_fwd(u_.t, w1, b1, b.NO_ACT_GELU, a1.t, ws, z=z1.t, n_rows=k)
    b.no_linear_fwd(a1.t, w2, b2, b.NO_ACT_NONE, y.t, ws, residual=x, n_rows=k)
    grad_y = y.t - target                           # of half the squared distance
    ga, gu, gx, gw1, gb1, gw2, gb2, gg, gbeta = Rows(n, h, F32), Rows(n, d, F32), Rows(n, d, F32), e(d, h), e(h), e(h, d), e(d), e(d), e(d)
    b.no_linear_bwd(a1.t, w2, b.NO_ACT_NONE, None, grad_y, ga.t, gw2, gb2, ws, n_rows=k)
    b.no_linear_bwd(u_.t, w1, b.NO_ACT_GELU, z1.t, ga.t, gu.t, gw1, gb1, ws, n_rows=k)
    b.no_layernorm_bwd(x, gamma, mean, rstd, gu.t, gx.t, gg, gbeta, ws, grad_sum=grad_y, n_rows=k)
    m1, m2, w1_0, w2_0 = torch.zeros_like(w1), torch.zeros_like(w2), w1.clone(), w2.clone()
    b.no_muon_step(w1, m1, gw1, 0.02, 0.95, ws)
    b.no_muon_step(w2, m2, gw2, 0.02, 0.95, ws)
    for t in (u_, z1, a1, y, ga, gu, gx):
        assert t.untouched(rows=here)
    d64 = lambda t: t.double()  # noqa: E731
    xs = d64(x[:here])
    _, _, r_, un = norm_ref(x[:here], None, gamma, beta, 1e-5)
    z = un @ d64(w1_0) + d64(b1)
    a = act_ref(z, "gelu")
    out = a @ d64(w2_0) + d64(b2) + xs
    gy = out - d64(target[:here])
    gz = (gy @ d64(w2_0).t().contiguous()) * slope_ref(z, "gelu")
    gun = gz @ d64(w1_0).t().contiguous()
    v = (un - d64(beta)) / d64(gamma)
    wg = gun * d64(gamma)
    want = {"y": (y.t[:here], out), "gw2": (gw2, a.t().contiguous() @ gy), "gb2": (gb2, gy.sum(0)), "gw1": (gw1, un.t().contiguous() @ gz), "gb1": (gb1, gz.sum(0)),
            "gg": (gg, (gun * v).sum(0)), "gbeta": (gbeta, gun.sum(0)), "gx": (gx.t[:here], gy + r_[:, None] * (wg - wg.mean(1, keepdim=True) - v * (wg * v).mean(1, keepdim=True)))}
    for name, (got, ref) in want.items():           # a chain of five sums of up to 271 terms: u sqrt(271) each, and some room for what they pass on
        assert apart(got, ref) < 5 * 8 * U * 271 ** 0.5, name
    for w0, w, m, gw in ((w1_0, w1, m1, gw1), (w2_0, w2, m2, gw2)):
        assert torch.equal(m, gw)
        o = steps_ref(d64(gw)[None] * 1.95, 5)[0]
        assert apart(d64(w0) - d64(w), 0.02 * o) < 1e-4


def test_a_given_stream_is_used_and_not_the_current_one():
    """The stream argument alone says where a call runs: given explicitly while another stream is current."""
    b, g = nb(), rng(3)
    x, w = randn((64, 96), g), randn((96, 32), g)
    y, ws = torch.zeros((64, 32), device="cuda"), ws_of(b.no_linear_ws_bytes(F32, 64, 96, 32))
    torch.cuda.synchronize()
    given, current = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(current):
        b.no_linear_fwd(x, w, None, 0, y, ws, stream=given)
    given.synchronize()
    close(y, x.double() @ w.double(), 1e-3)
