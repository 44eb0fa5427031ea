"""The compiled kernels of the calls on new tokens (assembly of this repository's own sources, made here), read for the
waits that the compiler does not place by itself: around inline assembly, and before a barrier that orders memory."""

import os
import re
import subprocess

import pytest

from paper_2510_13223_amd import build


@pytest.fixture(scope="module", params=["rows_attn.hip", "tokens.hip", "blocks.hip"])
def kernels(request, tmp_path_factory):
    """{kernel: its lines, labels among them} of one source, with the product build's flags."""
    out = str(tmp_path_factory.mktemp("asm") / "kernels.s")
    subprocess.run([build.HIPCC, *build.CFLAGS, "-x", "hip", "--cuda-device-only", "-S",
                    os.path.join(build.CSRC, request.param), "-o", out], check=True, capture_output=True, timeout=300)
    found, name = {}, None
    for line in open(out):
        line = line.split(";")[0].strip()
        if re.match(r"_Z\w+:$", line):
            name = line[:-1]
            found[name] = []
        elif line.startswith(".Lfunc_end"):
            name = None
        elif name and (re.match(r"\.LBB\w+:$", line) or re.match(r"[a-z]\w+(\s|$)", line)):
            found[name].append(line)
    assert found and all("s_endpgm" in x for x in found.values())
    return found


def predecessors(lines):
    """Lines that may run just before each line."""
    before = [[i - 1] if i and not re.match(r"s_(branch|endpgm|setpc)", lines[i - 1]) else [] for i in range(len(lines))]
    at = {line[:-1]: i for i, line in enumerate(lines) if line.endswith(":")}
    for i, line in enumerate(lines):
        jump = re.match(r"s_c?branch\w*\s+(\.LBB\w+)$", line)
        if jump:
            before[at[jump.group(1)]].append(i)
    return before


def scalars(operand):
    """Numbers of the scalar registers that an operand names."""
    one = re.match(r"s(\d+)$", operand)
    pair = re.match(r"s\[(\d+):(\d+)\]$", operand)
    return {int(one.group(1))} if one else set(range(int(pair.group(1)), int(pair.group(2)) + 1)) if pair else set()


def operands(line):
    return [x.split()[0] for x in line.partition(" ")[2].replace("\t", " ").split(",") if x.split()]


def scalars_written(line):
    """Of a vector instruction: a lane read out, a comparison, a carry."""
    if not line.startswith("v_"):
        return set()
    x = operands(line.replace("\t", " ", 1))
    carry = x[1:2] if re.match(r"v_(\w+_co_|div_scale|mad_[ui]64)", line) else []
    return set().union(*(scalars(o) for o in x[:1] + carry))


def wait_states(line):
    nop = re.match(r"s_nop\s+(\d+)", line)
    return 0 if line.endswith(":") else int(nop.group(1)) + 1 if nop else 1


def test_memory_instructions_wait_for_scalars_that_vector_instructions_wrote(kernels):
    """Five wait states between a vector instruction that writes a scalar register and a memory instruction that reads it,
    on every path."""
    seen = 0
    for name, lines in kernels.items():
        before = predecessors(lines)
        for i, line in enumerate(lines):
            if not re.match(r"(global|buffer|flat|scratch)_", line):
                continue
            reads = set().union(*(scalars(o) for o in operands(line.replace("\t", " ", 1))))
            if not reads:
                continue
            seen += 1
            todo, done = [(p, 0) for p in before[i]], set()
            while todo:
                p, waited = todo.pop()
                if waited >= 5 or (p, waited) in done:
                    continue
                done.add((p, waited))
                assert not scalars_written(lines[p]) & reads, f"{name}: {lines[p]!r} {waited} before {line!r}"
                todo += [(q, waited + wait_states(lines[p])) for q in before[p]]
    assert seen > 0


def test_in_place_moves_have_read_before_the_barrier(kernels):
    """Compaction in place: at the barrier between a step's reads and its writes, every wavefront's own loads have
    arrived, on every path back from the barrier to them."""
    found = [n for n in kernels if "compact" in n]
    for name in found:
        lines = kernels[name]
        before = predecessors(lines)
        barriers = [i for i, line in enumerate(lines) if line.startswith("s_barrier")]
        assert barriers
        for i in barriers:
            todo, done = list(before[i]), set()
            while todo:
                p = todo.pop()
                if p in done or re.match(r"s_waitcnt.*vmcnt\(0\)", lines[p]):
                    continue
                done.add(p)
                assert not lines[p].startswith("global_load"), f"{name}: {lines[p]!r} may be under way at the barrier"
                todo += before[p]
    assert found or not any("append" in n for n in kernels)
