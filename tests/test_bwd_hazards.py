"""The wait states around the matrix products that csrc/bwd.hip writes as assembly (CPU).

The compiler keeps the wait states that gfx950 asks for between a matrix instruction and
its neighbours, but not for instructions inside inline assembly.  This test compiles the
backward kernels to assembly and follows every path of the control flow for the last
few instructions: a plain register that a matrix instruction wrote must not be used by
anything but a matrix accumulation for 12 wait states (what the compiler holds itself for
this instruction), and a matrix instruction must not read a register that a vector
instruction wrote less than 2 wait states before.
"""
from __future__ import annotations

import os
import re
import subprocess

import pytest

from paper_2609_29219_amd import build

RESULT, OPERAND = 12, 2


def registers(text):
    m = re.match(r"^([va])\[(\d+):(\d+)\]$", text)
    if m:
        return {(m[1], i) for i in range(int(m[2]), int(m[3]) + 1)}
    m = re.match(r"^([va])(\d+)$", text)
    return {(m[1], int(m[2]))} if m else set()


class Instr:
    def __init__(self, line):
        self.line = line
        self.op, _, rest = line.partition(" ")
        ops = [registers(x.split()[0]) if x.split() else set() for x in rest.split(",")]
        self.mfma = self.op.startswith("v_mfma")
        self.valu = self.op.startswith("v_") and not self.mfma
        self.states = int(rest, 0) + 1 if self.op == "s_nop" else 1
        stores = self.op.startswith(("ds_write", "global_store", "buffer_store", "scratch_store",
                                     "v_cmp"))
        self.writes = set() if stores or not ops else ops[0]
        self.reads = set().union(*(ops if stores else ops[1:]))
        self.ab = ops[1] | ops[2] if self.mfma else set()


def blocks(body):
    """(label, instructions, labels it may go to) of each basic block, in order."""
    found, label, code = [], "", []
    for line in body.splitlines():
        line = line.split(";")[0].strip()
        m = re.match(r"^(\.LBB\w+):", line)
        if m:
            found.append([label, code, [], True])
            label, code = m[1], []
        elif line and not line.startswith(".") and not line.endswith(":"):
            code.append(Instr(line))
            if code[-1].op.startswith(("s_cbranch", "s_branch")) or code[-1].op == "s_endpgm":
                to = line.split()[-1] if code[-1].op != "s_endpgm" else None
                found.append([label, code, [to] if to else [], code[-1].op.startswith("s_cbranch")])
                label, code = label + "'", []
    found.append([label, code, [], False])
    for i, b in enumerate(found):
        if b[3] and i + 1 < len(found):
            b[2].append(found[i + 1][0])
    return found


def violations(asm, kernel):
    bad, products = [], 0
    for m in re.finditer(r"^(_ZN\w*%s\w*):" % kernel, asm, re.M):
        body = asm[m.end():]
        found = blocks(body[:body.index(".Lfunc_end")])
        before = {b[0]: [] for b in found}
        for b in found:
            for to in b[2]:
                before[to].append(b)

        def tails(b, states, seen=()):
            """Instruction sequences of at least `states` wait states that end with b."""
            have = sum(i.states for i in b[1])
            if have >= states or not before[b[0]] or b[0] in seen:
                return [b[1]]
            return [t + b[1] for p in before[b[0]]
                    for t in tails(p, states - have, seen + (b[0],))]

        for b in found:
            histories = [t for p in before[b[0]] for t in tails(p, RESULT)] or [[]]
            for h in histories:
                seq = h + b[1]
                for at in range(len(h), len(seq)):
                    i, waited = seq[at], 0
                    products += i.mfma
                    for j in reversed(seq[:at]):
                        if waited >= RESULT:
                            break
                        hit = {r for r in j.writes if r[0] == "v"}
                        if j.mfma and not i.mfma and hit & (i.reads | i.writes):
                            bad.append((waited, i.line, j.line))
                        if j.mfma and i.mfma and hit & i.ab:
                            bad.append((waited, i.line, j.line))
                        if j.valu and i.mfma and waited < OPERAND and j.writes & i.reads:
                            bad.append((waited, i.line, j.line))
                        waited += j.states
    return bad, products


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("asm") / "bwd.s")
    cmd = [build.HIPCC, *build.CFLAGS, "--offload-device-only", "-S",
           os.path.join(build.CSRC, "bwd.hip"), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    return open(out).read()


def test_wait_states_around_the_products(assembly):
    bad, products = violations(assembly, "bwd_kernel")
    assert products > 300
    assert not bad, f"{len(bad)}: {bad[:5]}"


def test_a_missing_wait_is_seen(assembly):
    # the same code with settle's wait states taken out
    bad, _ = violations(assembly.replace("s_nop 11", "s_nop 0"), "bwd_kernel")
    assert bad
