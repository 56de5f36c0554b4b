"""Rows of norms and logits whose byte offsets pass 2^32: the first, the last and those beside the border; norms against a call on these rows alone (a row's result depends
on that row, so the bits are the same), logits against their formulas in 64 bits. All other rows are zeros."""
import pytest
import torch

from .test_operators import BF16, F32, U, close, half, nb, randn, rng, teacher, ws_of

pytestmark = pytest.mark.gpu


def far(n, c, dt):
    """(a matrix of more than 2^32 bytes, zeros but for some rows; those rows' numbers)."""
    x = torch.zeros((n, c), dtype=dt, device="cuda")
    border = (1 << 32) // (c * x.element_size())
    at = torch.tensor([0, 1, border - 1, border, border + 1, n - 1], device="cuda")
    x[at] = randn((6, c), rng(c), dt)
    return x, at


def test_rmsnorm_far_rows():
    b, n, d = nb(), 1_050_000, 2055
    x, at = far(n, d, BF16)
    w, near = 1 + 0.1 * randn((d,), rng(1)), x[at]
    y, rstd, y6, rstd6 = torch.empty_like(x), torch.empty((n,), device="cuda"), torch.empty_like(near), torch.empty((6,), device="cuda")
    b.no_rmsnorm_fwd(x, w, 1e-5, y, rstd=rstd)
    b.no_rmsnorm_fwd(near, w, 1e-5, y6, rstd=rstd6)
    assert torch.equal(y[at], y6) and torch.equal(rstd[at], rstd6)
    y[at] = 0
    assert not y.any()
    gx, gw, gx6, gw6 = y, torch.empty((d,), device="cuda"), torch.empty_like(near), torch.empty((d,), device="cuda")
    b.no_rmsnorm_bwd(x, w, rstd, x, gx, gw, ws_of(b.no_rmsnorm_ws_bytes(n, d)))
    b.no_rmsnorm_bwd(near, w, rstd6, near, gx6, gw6, ws_of(b.no_rmsnorm_ws_bytes(6, d)))
    assert torch.equal(gx[at], gx6)
    terms = near.double().square() * rstd6.double()[:, None]
    close(gw, terms.sum(0), 10 * U * terms.sum(0), "grad_weight")       # six terms that are not 0, three roundings each
    gx[at] = 0
    assert not gx.any()


@pytest.mark.parametrize("n,c,dt", [(540_000, 4003, BF16), (27_000, 40_003, F32), (17_000, 131_072, BF16)])
def test_logits_far_rows(n, c, dt):
    b = nb()
    z, at = far(n, c, dt)
    assert n * c * z.element_size() > 1 << 32
    ids, tl = teacher(n, c, 5, rng(2))
    tok = torch.full((n,), 7, dtype=torch.int32, device="cuda")
    loss, lse, grad = torch.empty((n,), device="cuda"), torch.empty((n,), device="cuda"), torch.empty_like(z)
    b.no_distill_fwd_bwd(z, ids, tl, 1.0, None, loss, lse, grad, ws_of(b.no_distill_ws_bytes(n, c)))
    x = z[at].double()
    log_q = torch.log_softmax(x, 1)
    log_p = torch.log_softmax(tl[at].double(), 1)
    p, k_at = log_p.exp(), ids[at].long()
    bound = (c / 256 + 64) * U
    ql = log_q.gather(1, k_at)
    close(loss[at], (p * (log_p - ql)).sum(1), 42 * U * (p * (log_p.abs() + ql.abs())).sum(1) + bound + 8 * U, "loss")
    close(lse[at], torch.logsumexp(x, 1), bound + 8 * U * torch.logsumexp(x, 1).abs() + 4 * U * x.amax(1).abs(), "lse")
    want = log_q.exp().scatter_add(1, k_at, -p)
    tol = log_q.exp() * (bound + 8 * U * (1 + log_q.abs())) + U * torch.zeros_like(want).scatter_add(1, k_at, p * (26 + 8 * log_p.abs())) + 2 * U * want.abs()
    close(grad[at], want, tol + half(dt) * (want.abs() + tol), "grad")
    lp, ent, lse2, top, top_ids = (torch.empty(s, device="cuda") for s in ((n,), (n,), (n,), (n, 3), (n, 3)))
    top_ids = top_ids.to(torch.int32)
    b.no_logprobs_fwd(z, tok, 1.0, lp, ent, lse2, ws_of(b.no_logprobs_ws_bytes(n, c, 3)), top_ids=top_ids, top_logprobs=top)
    close(lp[at], log_q[:, 7], bound + 8 * U * (1 + log_q[:, 7].abs()), "logprob")
    h = -(log_q.exp() * log_q).sum(1)
    close(ent[at], h, 5 * bound * (1 + h) + 16 * U * h, "entropy")
    assert torch.equal(top_ids[at], torch.sort(z[at].float(), dim=1, descending=True, stable=True).indices[:, :3].to(torch.int32))
    other = torch.ones((n,), dtype=torch.bool, device="cuda")
    other[at] = False
    assert (top_ids[other] == torch.arange(3, device="cuda")).all()         # equal logits: the lowest classes
    close(lse2[other], torch.full((n - 6,), c, dtype=torch.float64, device="cuda").log(), bound + 8 * U * 12, "lse of zeros")
    one = torch.ones((n,), device="cuda")
    b.no_logprobs_bwd(z, tok, 1.0, lse2, ent, one, None, grad)
    log_p = x - lse2[at].double()[:, None]
    want = -log_p.exp()
    want[:, 7] += 1
    tol = log_p.exp() * (4 * U * (x.abs() + lse2[at].double().abs()[:, None]) + 8 * U * (1 + log_p.abs())) + 8 * U * want.abs()
    close(grad[at], want, tol + half(dt) * (want.abs() + tol), "grad of log probabilities")
