"""The routes of the operators that take several launches, with a workspace between them: on a stream of the caller's whose inputs arrive late, and captured and replayed
among eager work; and the outputs that may stand in an input's place."""
import pytest
import torch

from .test_operators import BF16, F32, MARK, Rows, nb, randn, rng, teacher, ws_of

pytestmark = pytest.mark.gpu


def embed(n, v, d, dt):
    b, g = nb(), rng(n)
    ids = torch.randint(-1, v + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
    ids[torch.rand((n,), generator=g, device="cuda") < 0.4] = v // 2         # (sums over many borders)
    grad, ws, out = randn((n, d), g, dt), ws_of(b.no_embed_ws_bytes(n, d)), torch.empty((v, d), device="cuda")
    return [grad, ids], [out], lambda: b.no_embed_bwd(grad, ids, out, ws, scale=0.5)


def norm(n, d, dt):
    b, g = nb(), rng(n + d)
    s, gy, w, rstd = randn((n, d), g, dt), randn((n, d), g, dt), 1 + 0.2 * randn((d,), g), torch.rand((n,), generator=g, device="cuda") + 0.5
    gx, gw, ws = torch.empty_like(s), torch.empty_like(w), ws_of(b.no_rmsnorm_ws_bytes(n, d))
    return [s, gy, w, rstd], [gx, gw], lambda: b.no_rmsnorm_bwd(s, w, rstd, gy, gx, gw, ws)


def distill(n, c, dt):
    b, g = nb(), rng(n + c)
    z, (ids, tl) = randn((n, c), g, dt), teacher(n, c, 5, g)
    ws = ws_of(b.no_distill_ws_bytes(n, c))
    out = [torch.empty((n,), device="cuda") for _ in range(4)] + [torch.empty_like(z) for _ in range(2)]

    def call():
        b.no_distill_fwd_bwd(z, ids, tl, 1.5, None, out[0], out[1], out[4], ws)
        b.no_distill_fwd(z, ids, tl, 1.5, None, out[2], out[3], ws)
        b.no_distill_bwd(z, ids, tl, 1.5, None, out[3], out[5])
    return [z, tl], out, call


def logprobs(n, c, dt):
    b, g = nb(), rng(n + c)
    z, tok, k = randn((n, c), g, dt), torch.randint(0, c, (n,), generator=g, device="cuda", dtype=torch.int32), 9
    ws, one = ws_of(b.no_logprobs_ws_bytes(n, c, k)), torch.ones((n,), device="cuda")
    out = [torch.empty((n,), device="cuda") for _ in range(3)] + [torch.empty((n, k), dtype=torch.int32, device="cuda"), torch.empty((n, k), device="cuda"), torch.empty_like(z)]

    def call():
        b.no_logprobs_fwd(z, tok, 1.5, *out[:3], ws, top_ids=out[3], top_logprobs=out[4])
        b.no_logprobs_bwd(z, tok, 1.5, out[2], out[1], one, one, out[5])
    return [z], out, call


ROUTES = [(embed, 1500, 500, 96, F32), (embed, 6000, 500, 96, BF16), (embed, 6000, 5_000_000, 4, F32), (embed, 140_000, 900, 20, BF16),     # by counting, tiles of either width, radix passes
          (norm, 600, 2049, BF16), (norm, 70, 20_000, F32), (norm, 5, 40_000, BF16),                                                        # parts joined; rows past registers
          (distill, 6, 90_001, F32), (distill, 300, 33_001, F32), (distill, 3, 200_001, BF16), (distill, 40, 76_001, BF16),                 # pieces
          (logprobs, 300, 33_001, F32), (logprobs, 6, 90_001, F32), (logprobs, 3, 200_001, BF16)]                                           # joined by a wavefront, by a block


@pytest.mark.parametrize("route", ROUTES, ids=lambda r: "-".join(getattr(x, "__name__", str(x)) for x in r))
def test_routes_of_several_launches_on_another_stream_and_in_a_graph(route):
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
            if turn == 2 and t.is_floating_point() and t.dim() == 2:         # new inputs under the same graph
                t.mul_(0.5)
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


@pytest.mark.parametrize("n,dim,pad,off", [(7, 63, 0, 0), (64, 100, 4, 4), (1000, 128, 0, 0), (33, 1025, 3, 1), (600, 2049, 1, 1), (5, 4096, 8, 8), (3, 8191, 0, 1), (70, 16_385, 1, 0), (3, 40_000, 0, 0)])
@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("over", ["s", "grad_sum"])
def test_rmsnorm_input_gradient_over_its_other_inputs(n, dim, pad, off, dt, over):
    b, g = nb(), rng(n + dim)
    s, gy, gs = (Rows(n, dim, dt, pad, off, randn((n, dim), g, dt, 2.0)) for _ in range(3))
    w, rstd = 1 + 0.3 * randn((dim,), g), torch.rand((n,), generator=g, device="cuda") + 0.5
    ws, want, want_w, got_w = ws_of(b.no_rmsnorm_ws_bytes(n, dim)), Rows(n, dim, dt, pad, off), torch.full((dim,), MARK, device="cuda"), torch.full((dim,), MARK, device="cuda")
    b.no_rmsnorm_bwd(s.t, w, rstd, gy.t, want.t, want_w, ws, grad_sum=gs.t)
    to = s if over == "s" else gs
    b.no_rmsnorm_bwd(s.t, w, rstd, gy.t, to.t, got_w, ws, grad_sum=gs.t)
    assert torch.equal(to.t, want.t) and torch.equal(got_w, want_w) and to.untouched()
