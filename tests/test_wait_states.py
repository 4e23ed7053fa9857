"""Wait states around the loads into LDS, read off the built kernels (no GPU).

These loads are written as inline assembly, so that the compiler does not wait for them by itself; it then fills in no wait states either.
gfx9 asks for them between a scalar write of M0 and a load into LDS, which takes its LDS address from there (1), and between a vector
instruction that writes a scalar register, as one that brings back a spilled register does, and a memory instruction that reads it (5)."""
import os
import re
import struct
import subprocess

import pytest

OBJDUMP = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def code_objects(library):
    """The gfx950 code objects of a library: bundles of a count and entries of offset, size and name."""
    data = open(library, "rb").read()
    at = data.find(MAGIC)
    while at >= 0:
        count, = struct.unpack_from("<Q", data, at + 24)
        p = at + 32
        for _ in range(count if count < 16 else 0):
            offset, size, length = struct.unpack_from("<QQQ", data, p)
            if b"gfx950" in data[p + 24:p + 24 + length] and size:
                yield data[at + offset:at + offset + size]
            p += 24 + length
        at = data.find(MAGIC, at + 24)


def kernels(text):
    """(name, [(instruction, operands)]) of a disassembly."""
    name, body = None, []
    for line in text.splitlines():
        head = re.match(r"[0-9a-f]+ <(.+)>:", line)
        if head:
            if name:
                yield name, body
            name, body = head[1], []
            continue
        line = line.split("//")[0].strip()
        if name and line:
            op, _, args = line.partition(" ")
            body.append((op, [a.strip() for a in args.split(",")]))
    if name:
        yield name, body


def wait_states(op, args):
    return int(args[0], 0) + 1 if op == "s_nop" else 1


def loads_to_lds(body):
    return [i for i, (op, args) in enumerate(body) if op.startswith(("global_load_lds", "buffer_load")) and ("_lds_" in op or "lds" in args[-1].split())]


def m0_too_late(body):
    """Loads into LDS with less than one wait state between them and a scalar write of M0."""
    return [i for i in loads_to_lds(body) if i > 0 and body[i - 1][0].startswith("s_") and body[i - 1][1][0] == "m0"]


def scalars(operand):
    """The scalar registers that an operand names."""
    word = operand.split()[0] if operand.split() else ""
    one, many = re.fullmatch(r"s(\d+)", word), re.fullmatch(r"s\[(\d+):(\d+)\]", word)
    if one:
        return {int(one[1])}
    if many:
        return set(range(int(many[1]), int(many[2]) + 1))
    return {"vcc"} if word.startswith("vcc") else set()


def written_by_vector(op, args):
    """What a vector instruction writes of the scalar registers: lanes that are read, comparisons, carries."""
    if op.startswith(("v_readlane", "v_readfirstlane", "v_cmp")):
        return scalars(args[0])
    return scalars(args[1]) if op.startswith("v_") and len(args) > 3 and ("_co_" in op or "div_scale" in op or "_u64_u32" in op or "_i64_i32" in op) else set()


def scalars_too_late(body):
    """Memory instructions that read a scalar register less than five wait states behind the vector instruction that wrote it."""
    late = []
    for i, (op, args) in enumerate(body):
        if not op.startswith(("global_", "buffer_", "flat_", "scratch_")):
            continue
        read = set().union(*map(scalars, args))
        states, j = 0, i - 1
        while read and j >= 0 and states < 5:
            if written_by_vector(*body[j]) & read:
                late.append(i)
                break
            states += wait_states(*body[j])
            j -= 1
    return late


@pytest.fixture(scope="module")
def built(tmp_path_factory):
    from paper_2401_14021_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    found = []
    for n, code in enumerate(code_objects(binding.LIB_PATH)):
        file = tmp_path_factory.mktemp("code") / f"{n}.o"
        file.write_bytes(code)
        found += kernels(subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(file)], capture_output=True, text=True, check=True).stdout)
    return found


def test_the_checks_themselves():
    listing = """
0000000000001000 <one>:
\ts_mov_b32 m0, s4            // 000000001000
\tglobal_load_lds_dwordx4 v1, s[2:3] nt
\ts_mov_b32 m0, s4
\ts_nop 0
\tglobal_load_lds_dwordx4 v1, s[2:3]
\ts_mov_b32 m0, s4
\tglobal_load_dwordx4 v[4:7], v1, s[2:3]
"""
    (name, body), = kernels(listing)
    assert name == "one" and loads_to_lds(body) == [1, 4] and m0_too_late(body) == [1]
    listing = """
0000000000001000 <two>:
\tv_readlane_b32 s3, v168, 11
\ts_mov_b32 m0, s4
\ts_nop 2
\tglobal_load_lds_dwordx4 v1, s[2:3] nt
\tglobal_load_lds_dwordx4 v1, s[2:3]
\tv_add_co_u32 v1, vcc, v1, v2
\tv_add_co_u32 v1, s[6:7], v1, v2
\ts_nop 3
\tglobal_load_lds_dwordx4 v1, s[6:7]
\ts_nop 0
\tglobal_load_lds_dwordx4 v1, s[6:7]
"""
    (name, body), = kernels(listing)
    assert m0_too_late(body) == [] and scalars_too_late(body) == [3, 8]


def test_m0_is_written_in_time(built):
    assert sum(len(loads_to_lds(body)) for _, body in built) > 1000
    late = {name: len(m0_too_late(body)) for name, body in built if m0_too_late(body)}
    assert not late, f"{sum(late.values())} loads, first in {next(iter(late))}"


def test_scalars_are_written_in_time(built):
    late = {name: len(scalars_too_late(body)) for name, body in built if scalars_too_late(body)}
    assert not late, f"{sum(late.values())} reads, first in {next(iter(late))}"
