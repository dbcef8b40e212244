"""More of the wait states around the written-out matrix products of csrc/bwd.hip (CPU).

tests/test_bwd_hazards.py follows results and the operands A and B.  Here: the addend C, which
a product reads as late as it writes its result where that lies elsewhere, and results that
overlap another product's addend or result in part.  A product of 32x32x16 takes eight passes,
each as long as a wait state, and has read its operands by the end of the last: a vector
instruction that writes a plain register of its addend within RELEASE = 8 of them might be too
early.  Addends and results of two products may follow each other at once only where they are
the same registers (an accumulation), else after RESULT wait states as any other use.
"""
from __future__ import annotations

import re

from tests.test_bwd_hazards import RESULT, assembly, blocks, registers  # noqa: F401  (a fixture)

RELEASE = 8
KERNELS = {(d, mask) for d in (64, 128) for mask in (0, 1, 2)}


def bodies(asm):
    """(d, mask): code of each backward kernel."""
    found = {}
    for m in re.finditer(r"^(_ZN\w*10bwd_kernelILi(\d+)ELi(\d+)E\w*):", asm, re.M):
        body = asm[m.end():]
        key = int(m[2]), int(m[3])
        assert key not in found
        found[key] = body[:body.index(".Lfunc_end")]
    return found


def addend(i):
    """Plain registers of a product's C (none where it is a constant)."""
    ops = i.line.partition(" ")[2].split(",")
    return {r for r in registers(ops[3].split()[0]) if r[0] == "v"}


def plain(registers_):
    return {r for r in registers_ if r[0] == "v"}


def violations(body):
    """(of addends, of overlaps) and the number of products with an addend elsewhere."""
    found = blocks(body)
    before = {b[0]: [] for b in found}
    for b in found:
        for to in b[2]:
            before[to].append(b)

    def tails(b, states, seen=()):
        have = sum(i.states for i in b[1])
        if have >= states or not before[b[0]] or b[0] in seen:
            return [b[1]]
        return [t + b[1] for p in before[b[0]] for t in tails(p, states - have, seen + (b[0],))]

    released, overlaps, elsewhere = [], [], 0
    for b in found:
        for h in [t for p in before[b[0]] for t in tails(p, RESULT)] or [[]]:
            seq = h + b[1]
            for at in range(len(h), len(seq)):
                i, waited = seq[at], 0
                vector = not i.mfma and i.op.startswith(("v_", "ds_read", "buffer_load",
                                                         "global_load", "scratch_load"))
                c = addend(i) if i.mfma else set()
                elsewhere += bool(c) and c != plain(i.writes)
                for j in reversed(seq[:at]):
                    if waited >= RESULT:
                        break
                    if j.mfma and vector and waited < RELEASE and addend(j) & i.writes:
                        released.append((waited, i.line, j.line))
                    if j.mfma and i.mfma:
                        result = plain(j.writes)
                        same = c == result == plain(i.writes)
                        if result & (c | plain(i.writes)) and not same and c != result:
                            overlaps.append((waited, i.line, j.line))
                        if addend(j) & plain(i.writes) and addend(j) != plain(j.writes) and \
                                waited < RELEASE:
                            overlaps.append((waited, i.line, j.line))
                    waited += j.states
    return released, overlaps, elsewhere


def test_all_kernels_are_there(assembly):  # noqa: F811
    found = bodies(assembly)
    assert set(found) == KERNELS
    for key, body in found.items():
        # seven products of each block of 32 x 32 in the loops of both kinds of workgroups:
        # D / 16 of each, of one or two blocks, in one or two forms of the loop
        assert body.count("v_mfma_f32_32x32x16_bf16") >= 7 * key[0] // 16, key


def test_addends_and_overlaps(assembly):  # noqa: F811
    for key, body in bodies(assembly).items():
        released, overlaps, elsewhere = violations(body)
        assert elsewhere, f"{key}: no product adds to another register"
        assert not released, f"{key}: {len(released)}: {released[:3]}"
        assert not overlaps, f"{key}: {len(overlaps)}: {overlaps[:3]}"


def planted(body, plant):
    """The body with plant(line, its registers of D and C) behind each product whose addend
    lies elsewhere."""
    out = []
    for line in body.splitlines():
        out.append(line)
        m = re.match(r"\s*v_mfma_f32_32x32x16_bf16 v\[(\d+):\d+\], [^,]+, [^,]+, v\[(\d+):\d+\]\s*$",
                     line)
        if m and m[1] != m[2]:
            out.append("\t" + plant(int(m[1]), int(m[2])))
    return "\n".join(out)


def test_planted_mistakes_are_seen(assembly):  # noqa: F811
    for key, body in bodies(assembly).items():
        # the addend written too early, by the VALU or a load
        for code in ("v_mov_b32_e32 v%d, 0", "ds_read_b32 v%d, v0"):
            bad = violations(planted(body, lambda d, c: code % c))[0]
            assert bad, (key, code)
        # behind seven wait states it is still seen, behind eight no longer
        assert violations(planted(body, lambda d, c: "s_nop 6\n\tv_mov_b32_e32 v%d, 0" % c))[0]
        assert not violations(planted(body, lambda d, c: "s_nop 7\n\tv_mov_b32_e32 v%d, 0" % c))[0]
        # a product that adds to, or writes, a part of the result
        for code in ("v_mfma_f32_32x32x16_bf16 a[0:15], v[0:3], v[0:3], v[%d:%d]",
                     "v_mfma_f32_32x32x16_bf16 v[%d:%d], v[0:3], v[0:3], 0"):
            bad = violations(planted(body, lambda d, c: code % (d + 4, d + 19)))[1]
            assert bad, (key, code)
        # and one that writes the addend
        bad = violations(planted(
            body, lambda d, c: f"v_mfma_f32_32x32x16_bf16 v[{c}:{c + 15}], v[0:3], v[0:3], 0"))[1]
        assert bad, key
