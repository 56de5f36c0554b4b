"""Log probabilities and distillation of rows whose classes are masked with finite values: the lowest of the type, -1e38, -1e35, -1e9.

References take the row's largest logit off first, in 64 bits, so that a row that is masked throughout keeps its shares there. Bounds: a sum of C
exponentials is off by its chain and tree, C / 256 + 64 roundings with those of its exponents (at most 3 log2 C + 2 on the average under the shares themselves); its
logarithm and the differences around it by 8 more of 1 + |log p|; the entropy is made of two such sums."""
import pytest
import torch

from .test_operators import BF16, F32, INF, NAN, TINY, U, close, half, nb, randn, rng, teacher, ws_of

pytestmark = pytest.mark.gpu

LOW = {F32: torch.finfo(F32).min, BF16: torch.finfo(BF16).min}
# rows of a wavefront, of a block, in pieces joined by a block and by a wavefront a row, in the shortest pieces; ends inside a run
ROUTES = [(10, 172), (10, 1003), (10, 5003), (10, 40_003), (300, 33_001), (10, 131_072)]


def masked_rows(n, c, dt, low, g):
    """Rows 0 .. 8 masked in nine ways, the others like row 0: (logits, classes that are left in all but rows 5 and 6)."""
    z = randn((n, c), g, dt)
    z[:, c - 8:] = low                              # one aligned run and what is around it
    z[1, : c // 4] = low                            # the front, so that a lane begins with nothing else
    left = torch.randperm(c - 8, generator=g, device="cuda")[:10]
    keep = z[2, left].clone()
    z[2] = low
    z[2, left] = keep                               # all but ten
    z[3, c // 8: 7 * c // 8] = low                  # whole pieces
    z[4, ::2] = low                                 # every other class
    z[5] = low                                      # nothing is left
    z[6], z[6, : c // 2] = low, -INF                # ... and half of it is -inf
    z[7, : c // 2] = -INF                           # both kinds
    z[8, : c - 9] = low                             # one class is left
    return z


def exact_rows(z, t):
    """(log p, entropy, lse) in 64 bits."""
    x = z.double()
    m = x.amax(1, keepdim=True)
    d = (x - m) / t
    log_s = d.exp().sum(1, keepdim=True).log()
    log_p = d - log_s
    p = log_p.exp()
    return log_p, -torch.where(p > 0, p * log_p, 0.0).sum(1), (m / t + log_s)[:, 0]


def sum_bound(c):
    return (c / 256 + 64) * U


def answers_of(z, tok, t, k=0):
    b, (n, c) = nb(), z.shape
    lp, ent, lse, top = (torch.full(s, 77.0, device="cuda") for s in ((n,), (n,), (n,), (n, k)))
    ids = torch.full((n, k), 77, dtype=torch.int32, device="cuda")
    b.no_logprobs_fwd(z, tok, t, lp, ent, lse, ws_of(b.no_logprobs_ws_bytes(n, c, k)), top_ids=ids if k else None, top_logprobs=top if k else None)
    return lp, ent, lse, ids, top


@pytest.mark.parametrize("n,c", ROUTES)
@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("low", [None, -1e38, -1e35, -1e9], ids=["lowest", "-1e38", "-1e35", "-1e9"])
@pytest.mark.parametrize("t", [1.0, 2.0, 0.7])
def test_entropy_of_rows_with_finite_masks(n, c, dt, low, t):
    g = rng(c)
    z = masked_rows(n, c, dt, LOW[dt] if low is None else low, g)
    tok = z.float().argmax(1).to(torch.int32)       # (a class that is left, where one is)
    log_p, want, want_lse = exact_rows(z, t)
    for k in (0, 8):
        lp, ent, lse, _, _ = answers_of(z, tok, t, k)
        want_lp = log_p.gather(1, tok.long()[:, None])[:, 0]
        close(ent, want, 5 * sum_bound(c) * (1 + want) + 16 * U * want, "entropy")
        close(lp, want_lp, sum_bound(c) + 8 * U * (1 + want_lp.abs()), "logprob")
        m = z.double().amax(1).abs() / t
        close(lse, want_lse.float(), sum_bound(c) + 4 * U * (m + want_lse.abs()), "lse")


@pytest.mark.parametrize("n,c", ROUTES)
@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("low", [None, -2.5e38, -1e9], ids=["lowest", "-2.5e38", "-1e9"])
@pytest.mark.parametrize("t", [1.0, 2.0, 0.7])
def test_log_probabilities_of_masked_classes(n, c, dt, low, t):
    """A finite logit has a finite log probability wherever fp32 holds it: of an answer, and of an alternative."""
    g = rng(c + 1)
    z = masked_rows(n, c, dt, LOW[dt] if low is None else low, g)
    z[9 % n] = LOW[dt]
    z[9 % n, 3] = -LOW[dt]                          # differences that leave fp32 before their division by T
    tok = torch.full((n,), c - 5, dtype=torch.int32, device="cuda")     # masked, but in a row with nothing left
    log_p, _, _ = exact_rows(z, t)
    k = 20
    lp, _, _, ids, top = answers_of(z, tok, t, k)
    bound = lambda want: sum_bound(c) + 8 * U * (1 + torch.where(want.isfinite(), want.abs(), 0.0))  # noqa: E731
    want = log_p[:, c - 5].float()
    close(lp, want, bound(want.double()), "logprob")
    value, at = torch.sort(z.float(), dim=1, descending=True, stable=True)
    want_ids = torch.where(value[:, :k] > -INF, at[:, :k], -1).to(torch.int32)
    assert torch.equal(ids, want_ids)
    want = log_p.gather(1, at[:, :k]).float()
    close(top, want, bound(want.double()), "top")


@pytest.mark.parametrize("n,c", ROUTES)
@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("low", [None, -2.5e38, -1e9], ids=["lowest", "-2.5e38", "-1e9"])
@pytest.mark.parametrize("t", [1.0, 2.0, 0.7])
def test_losses_against_a_teacher_that_names_masked_classes(n, c, dt, low, t):
    b, g = nb(), rng(c + 2)
    z = masked_rows(n, c, dt, LOW[dt] if low is None else low, g)
    k = 6
    ids, tl = teacher(n, c, k, g)
    ids[:, 0] = c - 5                               # masked, but in a row with nothing left
    ids[:, 1:] = torch.randperm(c - 9, generator=g, device="cuda")[:k - 1].to(torch.int32)      # some of them masked too
    log_q, _, want_lse = exact_rows(z, t)
    log_p = torch.log_softmax(tl.double() / t, 1)
    p, at = log_p.exp(), ids.long()
    w = torch.rand((n,), generator=g, device="cuda") * 0.4 + 0.1
    ql = log_q.gather(1, at)
    by = w.double() * t * t
    want = by * (p * (log_p - ql)).sum(1)
    # a share's exponent, sum, quotient; its logarithm; the difference; the sum of k; log q's own sum
    size = (p * (log_p.abs() + ql.abs())).sum(1)
    tol = by * ((2 * k + 32) * U * size.nan_to_num(0.0, 0.0, 0.0) + sum_bound(c) + 8 * U)
    loss, lse, grad = torch.empty((n,), device="cuda"), torch.empty((n,), device="cuda"), torch.empty_like(z)
    ws = ws_of(b.no_distill_ws_bytes(n, c))
    # the gradient, from the row's own sums: three roundings of an exponent, the sum's, quotient and products; the teacher's shares likewise
    q = log_q.exp()
    dense = torch.zeros_like(q).scatter_add_(1, at, p)
    dense_size = torch.zeros_like(q).scatter_add_(1, at, p * (2 * k + 16 + 8 * log_p.abs()))
    want_grad = (w.double() * t)[:, None] * (q - dense)
    exponent = torch.where(q > 0, log_q, 0.0).abs()
    grad_tol = (w.double() * t)[:, None] * (q * (sum_bound(c) + 8 * U * (1 + exponent)) + U * dense_size) + 2 * U * want_grad.abs() + TINY
    for both in (True, False):
        loss.fill_(77.0)
        lse.fill_(77.0)
        if both:
            b.no_distill_fwd_bwd(z, ids, tl, t, w, loss, lse, grad, ws)
            close(grad, want_grad, grad_tol + half(dt) * (want_grad.abs() + grad_tol), "grad")
        else:
            b.no_distill_fwd(z, ids, tl, t, w, loss, lse, ws)
        close(loss, torch.where(want.isnan(), INF, want).float(), tol, "loss")
        m = z.double().amax(1).abs() / t
        close(lse, want_lse.float(), sum_bound(c) + 4 * U * (m + want_lse.abs()), "lse")


@pytest.mark.parametrize("n,c", ROUTES)
@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
def test_gradient_of_log_probabilities_does_not_read_an_entropy_without_a_gradient(n, c, dt):
    b, g = nb(), rng(c + 3)
    z = randn((n, c), g, dt)
    tok = torch.randint(0, c, (n,), generator=g, device="cuda", dtype=torch.int32)
    _, ent, lse, _, _ = answers_of(z, tok, 1.0)
    gl, want, got = randn((n,), g), torch.empty_like(z), torch.empty_like(z)
    b.no_logprobs_bwd(z, tok, 1.0, lse, ent, gl, torch.zeros_like(gl), want)
    for other in (NAN, INF):
        b.no_logprobs_bwd(z, tok, 1.0, lse, torch.full_like(ent, other), gl, None, got)
        assert torch.equal(got, want)


def given_shares(z, lse, t):
    """(log p, bound of p's relative error) by a stored lse, which stands rounded: exponents are off by its rounding and theirs."""
    log_p = (z.double() / t - lse.double()[:, None]).clamp(max=0.0)
    there = log_p > -200
    size = torch.where(there, (z.double() / t).nan_to_num(0.0, 0.0, 0.0).abs() + lse.double().nan_to_num(0.0, 0.0, 0.0).abs()[:, None] + log_p.abs(), 0.0)
    return log_p, 4 * U * size + 8 * U


@pytest.mark.parametrize("n,c", ROUTES)
@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("low", [None, -1e38, -1e9], ids=["lowest", "-1e38", "-1e9"])
@pytest.mark.parametrize("t", [1.0, 2.0, 0.7])
def test_gradient_of_log_probabilities_of_masked_rows(n, c, dt, low, t):
    """Rows with classes left have their gradient; rows without, whose lse is rounded by more than their shares' logarithm or leaves fp32, stay within what shares of at most
    1 can give."""
    b, g = nb(), rng(c + 4)
    z = masked_rows(n, c, dt, LOW[dt] if low is None else low, g)
    tok = z.float().argmax(1).to(torch.int32)
    _, ent, lse, _, _ = answers_of(z, tok, t)
    gl, gh, grad = randn((n,), g), randn((n,), g), torch.empty_like(z)
    for entropy in (True, False):
        grad.fill_(77.0)
        b.no_logprobs_bwd(z, tok, t, lse, ent, gl, gh if entropy else None, grad)
        e, h = (gh.double()[:, None], ent.double()[:, None]) if entropy else (torch.zeros((n, 1), device="cuda", dtype=torch.float64),) * 2
        l = gl.double()[:, None]
        assert grad.isfinite().all()
        most = (l.abs() + (l.abs() + e.abs() * (1 + h))).expand(n, c) / t
        assert (grad.double().abs()[5:7] <= most[5:7] * (1 + half(dt) + 16 * U) + TINY).all()
        rows = [i for i in range(n) if i not in (5, 6)]
        log_p, rel = given_shares(z[rows], lse[rows], t)
        p = log_p.exp()
        hit = torch.zeros_like(p).scatter_(1, tok[rows].long()[:, None], 1.0)
        lp = torch.where(p > 0, log_p, 0.0)
        ref = (l[rows] * (hit - p) - e[rows] * p * (lp + h[rows])) / t
        size = (l[rows].abs() * (hit + p) + e[rows].abs() * p * (lp.abs() + h[rows])) / t
        tol = (rel + 8 * U) * size + rel * p * e[rows].abs() / t + TINY
        close(grad[rows], ref, tol + half(dt) * (ref.abs() + tol), "grad")


@pytest.mark.parametrize("n,c", ROUTES)
@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("low", [None, -1e38, -1e9], ids=["lowest", "-1e38", "-1e9"])
@pytest.mark.parametrize("t", [1.0, 2.0, 0.7])
def test_gradient_of_the_loss_of_masked_rows_from_an_lse(n, c, dt, low, t):
    b, g = nb(), rng(c + 5)
    z = masked_rows(n, c, dt, LOW[dt] if low is None else low, g)
    k = 6
    ids, tl = teacher(n, c, k, g)
    w = torch.rand((n,), generator=g, device="cuda") * 0.4 + 0.1
    loss, lse, grad = torch.empty((n,), device="cuda"), torch.empty((n,), device="cuda"), torch.full_like(z, 77.0)
    b.no_distill_fwd(z, ids, tl, t, w, loss, lse, ws_of(b.no_distill_ws_bytes(n, c)))
    b.no_distill_bwd(z, ids, tl, t, w, lse, grad)
    assert grad.isfinite().all()
    log_p = torch.log_softmax(tl.double() / t, 1)
    dense = torch.zeros_like(z, dtype=torch.float64).scatter_add_(1, ids.long(), log_p.exp())
    dense_size = torch.zeros_like(dense).scatter_add_(1, ids.long(), log_p.exp() * (2 * k + 16 + 8 * log_p.abs()))
    by = (w.double() * t)[:, None]
    assert (grad.double().abs()[5:7] <= (by * (1 + dense))[5:7] * (1 + half(dt) + 128 * U)).all()      # nothing left: shares of at most 1
    rows = [i for i in range(n) if i not in (5, 6)]
    log_q, rel = given_shares(z[rows], lse[rows], t)
    q = log_q.exp()
    ref = by[rows] * (q - dense[rows])
    tol = by[rows] * (rel * q + U * dense_size[rows]) + 2 * U * ref.abs() + TINY
    close(grad[rows], ref, tol + half(dt) * (ref.abs() + tol), "grad")


@pytest.mark.parametrize("n,c", [(10, 172), (10, 40_003), (2, 131_072), (3, 200_001)])
@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
def test_an_id_that_stands_twice_counts_entry_by_entry_in_the_loss_and_once_in_the_gradient(n, c, dt):
    """Halved shares of the same classes: the gradient of the whole shares, and a loss that is less by log 2, whatever the logits."""
    b, g, t = nb(), rng(c + 6), 2.0
    z, k = randn((n, c), g, dt), 4
    ids, tl = teacher(n, c, k, g)
    w = torch.rand((n,), generator=g, device="cuda") + 0.5
    ws = ws_of(b.no_distill_ws_bytes(n, c))
    loss, grad = [torch.empty((n,), device="cuda") for _ in range(2)], [torch.empty_like(z) for _ in range(2)]
    b.no_distill_fwd_bwd(z, ids, tl, t, w, loss[0], None, grad[0], ws)
    b.no_distill_fwd_bwd(z, ids.repeat(1, 2).contiguous(), tl.repeat(1, 2).contiguous(), t, w, loss[1], None, grad[1], ws)
    log_q, _, _ = exact_rows(z, t)
    log_p = torch.log_softmax(tl.double() / t, 1)
    p, ql = log_p.exp(), log_q.gather(1, ids.long())
    by = w.double() * t * t
    want = by * (p * (log_p - ql)).sum(1)
    tol = by * ((4 * k + 32) * U * (p * (log_p.abs() + 1 + ql.abs())).sum(1) + sum_bound(c) + 8 * U)
    close(loss[0], want, tol, "loss")
    close(loss[1], want - by * torch.log(torch.tensor(2.0, dtype=torch.float64)), tol, "loss of halved shares")
    # each of the two gradients: its own bound around the same value
    size = (w.double() * t)[:, None] * (log_q.exp() * (sum_bound(c) + 8 * U * (1 + log_q.abs())) + U * torch.zeros_like(log_q).scatter_add_(1, ids.long(), p * (4 * k + 16 + 8 * (log_p.abs() + 1))))
    ref = (w.double() * t)[:, None] * (log_q.exp() - torch.zeros_like(log_q).scatter_add_(1, ids.long(), p))
    for at in (0, 1):
        close(grad[at], ref, size + 2 * U * ref.abs() + half(dt) * (ref.abs() + size) + TINY, "grad")
