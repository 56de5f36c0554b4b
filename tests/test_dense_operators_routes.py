"""The products of the dense layer and of updates by every kind of tile that sizes lead to, whole and ragged, and workspaces made for larger sizes."""
import pytest
import torch

from .test_operators import BF16, F32, Rows, nb, randn, rng, ws_of

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])


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
