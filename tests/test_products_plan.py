"""Which tiles and how many parts the library plans for its products, and the workspaces that those need, on the host.

The products of the dense layer: forward [n, d_out] over d_in, input gradient [n, d_in] over d_out, weight gradient [d_in, d_out] over n; of an update: the smaller side's symmetric product over the longer side,
its square, and the product with the matrix."""
import ctypes as C
import math
import os
import random
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
HIPCC = os.environ.get("HIPCC") or shutil.which("hipcc", path="/opt/rocm/bin") or shutil.which("hipcc")
F32, BF16 = 0, 1
LINEAR_PARTS, UPDATE_PARTS, FEW = 128 << 20, 64 << 20, 8


@pytest.fixture(scope="session")
def plan(tmp_path_factory):
    """plan(M, N, K, pieces, matrices, half, parts_most, elsewhere) -> (kind, parts)"""
    if not HIPCC:
        pytest.skip("no hipcc here")
    from paper_2311_13225_amd import build
    path = str(tmp_path_factory.mktemp("plan") / "plan.so")
    subprocess.run([HIPCC] + build.FLAGS + ["-w", "-shared", os.path.join(HERE, "products_plan.hip"), "-o", path], check=True)
    f = C.CDLL(path).products_plan
    f.argtypes = [C.c_int64, C.c_int64, C.c_int64, C.c_int32, C.c_int64, C.c_int32, C.c_uint64, C.c_double, C.POINTER(C.c_int32)]
    out = (C.c_int32 * 2)()

    def ask(m, n, k, pieces, matrices=1, half=False, parts_most=0, elsewhere=0.0):
        f(m, n, k, pieces, matrices, half, parts_most, elsewhere, out)
        return out[0], out[1]
    return ask


@pytest.fixture(scope="module")
def lib():
    from paper_2311_13225_amd import binding as b
    if not os.path.exists(b.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return b.lib()


def up(v, to):
    return -(-v // to) * to


def linear_plans(plan, dt, n, d_in, d_out):
    """Per product of a dense layer: (name, kind, parts, bytes of parts)"""
    pieces = 3 if dt == F32 else 1
    layout = max(0.0, n * d_in * 10 / 8e6 - 5) if dt == F32 and d_in >= 32 else 0.0        # (other tiles than the large ones take fp32 rows behind a launch that lays them out)
    for name, m, c, k, elsewhere in (("fwd", n, d_out, d_in, layout), ("grad_x", n, d_in, d_out, 0.0), ("grad_w", d_in, d_out, n, 0.0)):
        kind, parts = plan(m, c, k, pieces, parts_most=LINEAR_PARTS, elsewhere=elsewhere)
        yield name, kind, parts, parts * m * up(c, 8) * 4 if parts > 1 else 0


def few_parts(dt, n, d_in, d_out):
    size, splits = 4 if dt == F32 else 2, 1
    while splits < 32 and splits * 2 <= max(1, d_in // 128) and d_in * min(d_out, 128 // size) * size > splits * (128 << 10):
        splits *= 2
    return (1 if splits == 2 and n < 4 else splits) * n * up(d_out, 8) * 4


def linear_bytes(plan, dt, n, d_in, d_out):
    """What the calls take of their workspace, at most."""
    operand = lambda rows, dim: up(rows * up(dim, 8) * 2 * (3 if dt == F32 else 1), 256)  # noqa: E731
    parts = max(p[3] for p in linear_plans(plan, dt, n, d_in, d_out))
    if n <= FEW:
        parts = max(parts, few_parts(dt, n, d_in, d_out))
    return operand(n, d_in) + operand(d_in, d_out) + operand(n, d_out) + up(max(1, min(512, -(-n // 64))) * d_out * 4, 256) + parts


def log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(hi))))))


def smaller(rng, sizes):
    """The sizes with one or all of them made smaller."""
    which = rng.randrange(len(sizes) + 1)
    return tuple(max(1, int(v * rng.uniform(0.3, 1.0))) if which in (i, len(sizes)) else v for i, v in enumerate(sizes))


@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
def test_linear_workspaces_grow_with_every_size(lib, plan, dt):
    rng, size = random.Random(1), lambda s: lib.no_linear_ws_bytes(dt, *s)  # noqa: E731
    for _ in range(6000):
        sizes = tuple(log_int(rng, 1, hi) for hi in rng.choice(((64, 9000, 9000), (60_000, 9000, 9000), (60_000, 600, 600))))
        less = smaller(rng, sizes)
        assert size(less) <= size(sizes), (less, sizes)
        assert size(less) >= linear_bytes(plan, dt, *less), less
    assert size((8, 256, 256)) <= size((9, 256, 256)) and size((2276, 2048, 8192)) <= size((2504, 2048, 8192)) and size((0, 64, 64)) <= size((1, 64, 64))


def update_plans(plan, n, rows, cols):
    """Per product of an update: (name, kind, parts, bytes of parts)"""
    side, longer = min(rows, cols), max(rows, cols)
    kind, parts = plan(side, side, longer, 2, n, True, UPDATE_PARTS)
    yield "gram", kind, parts, parts * n * side * up(side, 8) * 4 if parts > 1 else 0
    yield ("square",) + plan(side, side, side, 2, n, True) + (0,)
    yield ("with_x",) + plan(rows, cols, side, 2, n) + (0,)


def update_bytes(plan, n, rows, cols):
    pieces = lambda r, c: up(n * r * up(c, 8) * 4, 256)  # noqa: E731
    side = min(rows, cols)
    return n * 1024 * 8 + 2 * pieces(rows, cols) + 2 * pieces(side, side) + max(p[3] for p in update_plans(plan, n, rows, cols))


def test_update_workspaces_grow_with_every_size(lib, plan):
    rng, size = random.Random(2), lambda s: lib.no_orthogonalise_ws_bytes(*s)  # noqa: E731
    for _ in range(6000):
        sizes = tuple(log_int(rng, 1, hi) for hi in rng.choice(((8, 5000, 5000), (300, 300, 300), (2, 300, 5000))))
        less = smaller(rng, sizes)
        assert size(less) <= size(sizes), (less, sizes)
        assert size(less) >= update_bytes(plan, *less), less
    assert size((7, 3496, 63)) <= size((7, 3608, 63)) and size((0, 9, 9)) <= size((1, 9, 9))


# ------------------------------------------------------------------------------------------------------- what the tests on the GPU take

KINDS = ((256, 256), (192, 192), (128, 128), (128, 128), (64, 64), (64, 64), (64, 64), (32, 32))        # tiles; the first is 256 x 128 of three pieces
STEPS = 5           # of a reduction: enough for every copy in LDS to be filled again


def tiles(kind, pieces):
    return (256, 128) if kind == 0 and pieces == 3 else KINDS[kind]


def linear_routes(plan, dt, n, d_in, d_out):
    """(product, kind, split) -> whether its tiles are whole"""
    pieces, step = (3, 32) if dt == F32 else (1, 64)
    shapes = {"fwd": (n, d_out, d_in), "grad_x": (n, d_in, d_out), "grad_w": (d_in, d_out, n)}
    for name, kind, parts, _ in linear_plans(plan, dt, n, d_in, d_out):
        m, c, k = shapes[name]
        if k > step * (STEPS - 1) and not (name == "fwd" and n <= FEW):
            bm, bn = tiles(kind, pieces)
            yield (dt, name, kind, parts > 1), m % bm == 0 and c % bn == 0


def update_routes(plan, n, rows, cols):
    side, longer, tall = min(rows, cols), max(rows, cols), rows > cols
    shapes = {"gram": (side, side, longer), "square": (side, side, side), "with_x": (rows, cols, side)}
    for name, kind, parts, _ in update_plans(plan, n, rows, cols):
        m, c, k = shapes[name]
        if k > 32 * (STEPS - 1):
            bm, bn = tiles(kind, 2)
            yield (name, tall and name != "square", kind, parts > 1), m % bm == 0 and c % bn == 0


def on_the_gpu(plan):
    from . import test_dense_operators_routes as r
    seen = {}
    for dt, sizes in ((F32, r.LINEAR_F32 + r.LARGE_F32), (BF16, r.LINEAR_BF16 + r.LARGE_BF16)):
        for s in sizes:
            for route, whole in linear_routes(plan, dt, *s):
                seen.setdefault(route, set()).add(whole)
    for s in r.UPDATES + r.LARGE_UPDATES:
        for route, whole in update_routes(plan, *s):
            seen.setdefault(route, set()).add(whole)
    return seen


def test_every_route_is_tested_on_the_gpu(plan):
    """Sizes drawn over what the operators are measured at lead to no kind of tile, in no product, that the tests leave out, neither whole nor ragged."""
    seen, rng, asked = on_the_gpu(plan), random.Random(4), set()

    def side(lo, hi):
        v, to = log_int(rng, lo, hi), rng.choice((1, 8, 64, 128, 192, 256))
        return max(lo, v // to * to)
    for _ in range(8000):
        for dt in (F32, BF16):
            n, d_in, d_out = side(1, 60_000), side(16, 9000), side(16, 9000)
            if n * d_in * d_out <= 3e11:
                asked.update(linear_routes(plan, dt, n, d_in, d_out))
        n, rows, cols = log_int(rng, 1, 8), side(16, 4100), side(16, 4100)
        if n * rows * cols * min(rows, cols) <= 1.4e11:
            asked.update(update_routes(plan, n, rows, cols))
    missing = sorted(str((route, "whole" if whole else "ragged")) for route, whole in asked if whole not in seen.get(route, ()))
    assert len(asked) > 200 and not missing, (len(missing), missing)


def test_the_cases_that_are_measured_take_tested_routes(plan):
    from perf import more_operators
    seen = on_the_gpu(plan)
    for case in more_operators.listed():
        kind = case["kind"]
        if kind.startswith("linear"):
            routes = linear_routes(plan, F32 if case["x"] == "f32" else BF16, case["n"], case["d_in"], case["d_out"])
            routes = [r for r in routes if (r[0][1] == "fwd") == (kind == "linear_fwd")]
        elif kind in ("muon", "orthogonalise"):
            routes = update_routes(plan, case["matrices"], case["rows"], case["cols"])
        else:
            continue
        for route, whole in routes:
            assert whole in seen.get(route, ()), (case["name"], route, whole)
