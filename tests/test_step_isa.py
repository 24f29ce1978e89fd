"""The assembly of the ring kernels (csrc/step_tile.h), whose matrix instructions
are written out: the compiler puts no wait states between one of them and an
instruction beside it.  Here the built library is looked at, along every path: no
vector instruction writes a register that one of the next two matrix instructions
reads, and nothing but a matrix instruction touches an accumulator before 20 wait
states have gone by since the last of them."""

from __future__ import annotations

import os
import re
import struct
import subprocess

import pytest

from paper_2411_00284_amd import _native

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def code_objects(path):
    """The gfx950 code objects that a library carries."""
    data = open(path, "rb").read()
    at = data.find(MAGIC)
    while at >= 0:
        count, = struct.unpack_from("<Q", data, at + 24)
        pos = at + 32
        for _ in range(count):
            offset, size, length = struct.unpack_from("<QQQ", data, pos)
            name = data[pos + 24:pos + 24 + length]
            pos += 24 + length
            if b"gfx950" in name:
                yield data[at + offset:at + offset + size]
        at = data.find(MAGIC, at + 24)


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """name -> [(address, instruction)] of every ring kernel."""
    if not os.path.exists(OBJDUMP):
        pytest.skip("no disassembler")
    found = {}
    for i, blob in enumerate(code_objects(_native.STEP_LIB_PATH)):
        path = str(tmp_path_factory.mktemp("isa") / f"{i}.co")
        open(path, "wb").write(blob)
        out = subprocess.run([OBJDUMP, "-d", path], capture_output=True, text=True, check=True).stdout
        name = None
        for line in out.splitlines():
            head = re.match(r"[0-9a-f]+ <(\S+)>:", line)
            if head:
                name = head.group(1) if "ring_kernel" in head.group(1) else None
                if name:
                    found[name] = []
            elif name and line.startswith("\t") and "//" in line:
                text, _, comment = line.partition("//")
                found[name].append((int(comment.split(":")[0], 16), text.strip()))
    return found


def registers(text):
    """The vector registers ("v" or "a", number) of an operand."""
    got = set()
    for kind, single, low, high in re.findall(r"\b([va])(?:(\d+)\b|\[(\d+):(\d+)\])", text):
        got |= {(kind, n) for n in (range(int(single), int(single) + 1) if single else range(int(low), int(high) + 1))}
    return got


def operands(line):
    return [p.strip() for p in line.split(None, 1)[1].split(", ")] if " " in line else []


def successors(code, place, i):
    """Indices that may follow instruction i."""
    op = code[i][1].split()[0]
    if op == "s_endpgm":
        return []
    following = [i + 1] if op != "s_branch" and i + 1 < len(code) else []
    if op == "s_branch" or op.startswith("s_cbranch"):
        offset = int(operands(code[i][1])[0])
        following.append(place[code[i][0] + 4 + 4 * (offset - 0x10000 if offset >= 0x8000 else offset)])
    return following


def waits_of(text):
    return int(operands(text)[0], 0) + 1 if text.startswith("s_nop") else 1


ENOUGH = 20


def analyse(code):
    """For every instruction, over all paths: the fewest wait states since a matrix instruction, and the registers that
    the last two wait states' vector instructions wrote."""
    place = {address: n for n, (address, _) in enumerate(code)}
    assert len(place) == len(code)
    after = [successors(code, place, i) for i in range(len(code))]
    far, near = [ENOUGH] * len(code), [(frozenset(), frozenset())] * len(code)
    todo = list(range(len(code)))
    while todo:
        i = todo.pop()
        text = code[i][1]
        op = text.split()[0]
        n = waits_of(text)
        out_far = 0 if op.startswith("v_mfma") else min(ENOUGH, far[i] + n)
        wrote = frozenset(registers(operands(text)[0])) if op.startswith("v_") and not op.startswith(("v_mfma", "v_cmp")) else frozenset()
        out_near = (wrote, near[i][0] if n == 1 else frozenset())
        for k in after[i]:
            new_far, new_near = min(far[k], out_far), tuple(a | b for a, b in zip(near[k], out_near))
            if (new_far, new_near) != (far[k], near[k]):
                far[k], near[k] = new_far, new_near
                todo.append(k)
    return far, near


def test_there_are_ring_kernels(kernels):
    assert len(kernels) == 18                                   # two types, three products, three forms
    assert all(sum(i.startswith("v_mfma") for _, i in v) in (5 * 128, 5 * 32) for v in kernels.values())


def test_nothing_comes_near_a_matrix_instruction(kernels):
    for name, code in kernels.items():
        far, near = analyse(code)
        for i, (_, text) in enumerate(code):
            parts = operands(text)
            if text.startswith("v_mfma"):
                assert parts[0] == parts[3] and parts[0].startswith("a"), (name, text)
                assert not (registers(parts[1]) | registers(parts[2])) & (near[i][0] | near[i][1]), (name, text)
            elif any(k == "a" for part in parts for k, _ in registers(part)):
                assert far[i] >= ENOUGH, (name, text, far[i])
