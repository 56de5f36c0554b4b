"""Workspaces of the operators on learned inputs and large answers, and of norms: one made for larger sizes holds for smaller ones, on the host."""
import math
import os
import random

import pytest

MOST_ROWS, MOST_CLASSES = 60_000, 300_000
SIZES = {"no_embed_ws_bytes": ((300_000, 5000), (20_000, 200)), "no_rmsnorm_ws_bytes": ((60_000, 60_000),), "no_layernorm_ws_bytes": ((60_000, 60_000),),
         "no_distill_ws_bytes": ((MOST_ROWS, MOST_CLASSES), (2000, 20_000)), "no_logprobs_ws_bytes": ((MOST_ROWS, MOST_CLASSES, 64), (2000, 20_000, 20))}


@pytest.fixture(scope="module")
def lib():
    from paper_2311_13225_amd import binding as b
    if not os.path.exists(b.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return b.lib()


def up(v, to):
    return -(-v // to) * to


def needs(name, sizes):
    """What the call takes of it, at the least."""
    if name == "no_embed_ws_bytes":         # two sums a chunk
        n, dim = sizes
        if n <= 1024:
            return 16
        units, chunk = -(-dim // 8), 64
        lanes = 1 << (min(units, 64) - 1).bit_length()
        while chunk > 8 and n * -(-units // 64) * lanes // 64 // chunk < 1024:
            chunk >>= 1
        return up(n, 1024) * 4 * (2 if n <= 4096 else 4) + -(-n // chunk) * 2 * dim * 4 + 16
    if name in ("no_distill_ws_bytes", "no_logprobs_ws_bytes"):        # three fp32 sums and k keys of 8 bytes a piece
        n, classes = sizes[:2]
        u = 8
        while u > 1 and n * -(-classes // (1024 * u)) < 1024:
            u >>= 1
        return n * -(-classes // (1024 * u)) * (12 + 8 * (sizes[2] if len(sizes) > 2 else 0)) if classes > 8192 else 0
    return 0


@pytest.mark.parametrize("name", sorted(SIZES))
def test_workspaces_grow_with_every_size(lib, name):
    rng, size = random.Random(3), getattr(lib, name)
    for _ in range(20_000):
        sizes = [round(math.exp(rng.uniform(0, math.log(hi)))) for hi in rng.choice(SIZES[name])]
        which = rng.randrange(len(sizes) + 1)
        less = [max(1, int(v * rng.uniform(0.3, 1.0))) if which in (i, len(sizes)) else v for i, v in enumerate(sizes)]
        assert needs(name, less) <= size(*less) <= size(*sizes) and size(*less) > 0, (less, sizes)
    rest = [100] * (len(SIZES[name][0]) - 1)
    for n in (1, 65, 256, 257, 1024, 1025, 4096, 4097, 131_072, 131_073):        # (where the ways change)
        assert size(n - 1, *rest) <= size(n, *rest), n


@pytest.mark.gpu
def test_calls_in_a_workspace_of_larger_sizes():
    """What a call needs besides lies within: the bytes behind the workspace stay."""
    import torch

    from .test_operators import nb, randn, rng, ws_of
    b, g = nb(), rng(1)

    def both(size_of, most, fewer, call):
        made = []
        for sizes in (most, fewer):
            size = size_of(*sizes)
            ws = ws_of(size + 4096)
            ws[size:] = 0x5A
            made.append(call(ws[:size]))
            assert (ws[size:] == 0x5A).all()
        for x, y in zip(*made):
            assert torch.equal(x, y)

    n, classes, k = 719, 4671, 5
    z, tokens = randn((1281, 9000), g), torch.arange(1281, dtype=torch.int32, device="cuda")
    for rows, wide in ((n, classes), (719, 8500), (3, 9000)):
        zz, ids = z[:rows, :wide], tokens[:rows, None] + torch.arange(k, dtype=torch.int32, device="cuda")

        def distill(ws):
            loss, lse = torch.empty((rows,), device="cuda"), torch.empty((rows,), device="cuda")
            b.no_distill_fwd(zz, ids.contiguous(), ids.float() * 0.01, 2.0, None, loss, lse, ws)
            return loss, lse

        def logprobs(ws):
            e = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
            out = e(rows), e(rows), e(rows), torch.empty((rows, k), dtype=torch.int32, device="cuda"), e(rows, k)
            b.no_logprobs_fwd(zz, tokens[:rows], 1.0, out[0], out[1], out[2], ws, top_ids=out[3], top_logprobs=out[4])
            return out
        both(b.no_distill_ws_bytes, (1281, 9000), (rows, wide), distill)
        both(b.no_logprobs_ws_bytes, (1281, 9000, 6), (rows, wide, k), logprobs)
    for most, n, dim in (((140_000, 40), 131_072, 33), ((5000, 40), 4096, 40), ((30_000, 600), 15_000, 512)):
        grad, ids = randn((n, dim), g), torch.randint(0, 3000, (n,), generator=g, device="cuda", dtype=torch.int32)

        def embed(ws):
            table = torch.empty((3000, dim), device="cuda")
            b.no_embed_bwd(grad, ids, table, ws)
            return (table,)
        both(b.no_embed_ws_bytes, most, (n, dim), embed)
