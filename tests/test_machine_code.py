"""Waits that the chip asks of a program between two instructions, in the library's own device code. The compiler keeps them between instructions of its own; what is written by hand it does not look into, so
they are read off the code that was built."""
import os
import re
import shutil
import struct
import subprocess

import pytest

OBJDUMP = shutil.which("llvm-objdump", path="/opt/rocm/llvm/bin") or shutil.which("llvm-objdump")
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"
M0_WAIT = 1         # instructions, or states of an s_nop, between a scalar write of m0 and a load into LDS, whose place m0 gives
SCALAR_WAIT = 5     # between a vector instruction that writes a scalar register and a memory request that reads it
MFMA_WAIT = 2       # between a vector instruction's result and a matrix instruction that reads it
SUM_WAIT = 11       # between a matrix instruction of 16 x 16 x 32 and another that reads its sums, but for the next one that adds to them


def code_objects(path):
    """The gfx950 images of a library's bundles."""
    data, at = open(path, "rb").read(), 0
    while (at := data.find(MAGIC, at)) >= 0:
        (entries,), place = struct.unpack_from("<Q", data, at + len(MAGIC)), at + len(MAGIC) + 8
        for _ in range(entries):
            offset, size, length = struct.unpack_from("<QQQ", data, place)
            name = data[place + 24:place + 24 + length]
            place += 24 + length
            if b"gfx950" in name and size:
                yield data[at + offset:at + offset + size]
        at += len(MAGIC)


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    """Per code object the instructions in order: (kernel, operation, operands), with (kernel, '', []) where a jump may arrive or a kernel begins."""
    if not OBJDUMP:
        pytest.skip("no llvm-objdump here")
    from paper_2311_13225_amd import binding as b
    if not os.path.exists(b.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    made = []
    for i, image in enumerate(code_objects(b.LIB_PATH)):
        path = tmp_path_factory.mktemp("code") / ("%d.elf" % i)
        path.write_bytes(image)
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--symbolize-operands", str(path)], capture_output=True, text=True, check=True).stdout
        kernel, out = "", []
        for line in text.splitlines():
            line = line.split("//")[0].rstrip()
            if line.endswith(">:"):
                name = re.search(r"<([^>]+)>:", line).group(1)
                if not re.match(r"L\d+$", name):
                    kernel = name
                out.append((kernel, "", []))
            elif line.startswith("\t"):
                op, _, rest = line.strip().partition(" ")
                out.append((kernel, op, [t.strip() for t in rest.split(",")] if rest else []))
        made.append(out)
    assert made, "the library holds no gfx950 code"
    return made


def registers(operand, kind):
    """Numbers of the vector ('v') or scalar ('s') registers that an operand names."""
    m = re.match(r"%s\[(\d+):(\d+)\]" % kind, operand) or re.match(r"%s(\d+)\b" % kind, operand)
    return set(range(int(m.group(1)), int(m.group(m.lastindex)) + 1)) if m else set()


def named(operands):
    """Vector registers of either kind, by name."""
    return {kind + str(r) for a in operands for kind in "va" for r in registers(a, kind)}


def too_near(out, i, states, writes):
    """The instruction before out[i], fewer than `states` wait states away on the straight way there, for which `writes` holds."""
    passed = 0
    for kernel, op, args in reversed(out[max(0, i - states - 1):i]):
        if passed >= states or op == "":
            return None
        if writes(op, args):
            return op, args
        passed += int(args[0], 0) + 1 if op == "s_nop" else 1
    return None


def test_a_load_into_lds_waits_for_its_place(listings):
    """And nothing else in those kernels has m0 hold a value."""
    seen, bad, written, loads = 0, [], {}, {}
    for out in listings:
        for i, (kernel, op, args) in enumerate(out):
            if not re.match(r"(buffer|global|scratch)_load", op) or not any(re.search(r"\blds\b", a) for a in args) and "_lds_" not in op:
                continue
            seen += 1
            loads[kernel] = loads.get(kernel, 0) + 1
            if too_near(out, i, M0_WAIT, lambda o, a: o.startswith("s_") and a and a[0] == "m0"):
                bad.append(kernel)
        for kernel, op, args in out:
            if args and args[0] == "m0":
                written[kernel] = written.get(kernel, 0) + 1
    assert seen > 1000, "the products' loads are not found"
    assert {k: written.get(k, 0) for k in loads} == loads
    assert not bad, "%d of %d loads stand right behind the write of m0, in %d kernels, the first %s" % (len(bad), seen, len(set(bad)), bad[0])


def test_a_request_waits_for_scalars_that_vector_instructions_wrote(listings):
    bad = []
    for out in listings:
        for i, (kernel, op, args) in enumerate(out):
            if not op.startswith("buffer_"):
                continue
            used = set().union(*(registers(a.split(" ")[0], "s") for a in args))
            hit = too_near(out, i, SCALAR_WAIT, lambda o, a: o.startswith("v_") and a and registers(a[0], "s") & used)
            if hit:
                bad.append((kernel, hit))
    assert not bad, (len(bad), bad[0])


def test_a_matrix_instruction_waits_for_its_operands(listings):
    seen, bad = 0, []
    for out in listings:
        for i, (kernel, op, args) in enumerate(out):
            if not op.startswith("v_mfma"):
                continue
            seen += 1
            used = named(args[1:])
            hit = too_near(out, i, MFMA_WAIT, lambda o, a: o.startswith("v_") and not o.startswith("v_mfma") and a and named(a[:1]) & used)
            if hit:
                bad.append((kernel, hit, args))
    assert seen > 1000 and not bad, (len(bad), bad[:1])


def test_sums_are_read_when_they_are_there(listings):
    seen, bad = 0, []
    for out in listings:
        for i, (kernel, op, args) in enumerate(out):
            if not re.match(r"v_mfma\w*_16x16x32", op):
                continue
            seen += 1
            made, passed = named(args[:1]), 0
            for _, later, its in out[i + 1:i + 1 + SUM_WAIT]:
                if passed >= SUM_WAIT or later == "":
                    break
                if not later.startswith(("v_mfma", "s_")) and named(its) & made:
                    bad.append((kernel, args, later, its))
                passed += int(its[0], 0) + 1 if later == "s_nop" else 1
    assert seen > 1000 and not bad, (len(bad), bad[:1])
