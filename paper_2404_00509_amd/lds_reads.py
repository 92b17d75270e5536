"""Reads of LDS by inline assembly, checked on the assembly that goes into the library.

The matrix kernels of csrc/matmul.hpp read LDS by inline assembly and wait for it themselves, so that the compiler does
not make every read wait for all direct loads in flight.  The compiler takes such a read's registers as written at once:
where it spills or moves one of them before the wait, the value that arrives later is lost or overwrites another.  No
source can rule that out, so every build looks at what its compiler made, over every path through every kernel."""
from __future__ import annotations

import re

READ = ("ds_read_b128", "ds_read_b64_tr_b16")


def registers(text):
    """("v" or "a", number) of each vector register that an instruction's operands name."""
    out = set()
    for m in re.finditer(r"\b([va])\[(\d+):(\d+)\]|\b([va])(\d+)\b", text):
        if m.group(1):
            out |= {(m.group(1), i) for i in range(int(m.group(2)), int(m.group(3)) + 1)}
        else:
            out.add((m.group(4), int(m.group(5))))
    return out


def blocks_of(body):
    """[(label or None, [(instruction, from inline assembly), ...]), ...], ended by labels and branches."""
    blocks, own = [(None, [])], False
    for line in body.split("\n"):
        if "#ASMSTART" in line or "#ASMEND" in line:
            own = "#ASMSTART" in line
            continue
        text = line.split(";")[0].strip()
        label = re.match(r"^(\.LBB\S+):", text)
        if label:
            blocks.append((label.group(1), []))
        elif text and not text.startswith("."):
            blocks[-1][1].append((text, own))
            if text.startswith(("s_branch", "s_cbranch", "s_endpgm")):
                blocks.append((None, []))
    return blocks


def _walk(block, in_flight, found=None):
    flying = set(in_flight)
    for text, own in block:
        op, _, rest = text.partition(" ")
        if op == "s_waitcnt" and "lgkmcnt(0)" in text:
            flying = set()
            continue
        if found is not None and registers(rest) & flying:
            found.append(text)
        if own and op in READ:
            flying |= registers(rest.split(",")[0])
    return frozenset(flying)


def touched_in_flight(body):
    """Of one kernel: the instructions that touch a register whose read has not been waited for, and the number of reads."""
    blocks = blocks_of(body)
    at = {label: i for i, (label, _) in enumerate(blocks) if label}
    states = [None] * len(blocks)
    states[0] = frozenset()
    todo = [0]
    while todo:
        i = todo.pop()
        out = _walk(blocks[i][1], states[i])
        last = blocks[i][1][-1][0] if blocks[i][1] else ""
        after = [] if last.startswith(("s_branch", "s_endpgm")) else [i + 1]
        if last.startswith(("s_branch", "s_cbranch")):
            after.append(at[last.split()[1]])
        for j in after:
            if j < len(blocks) and (states[j] is None or not out <= states[j]):
                states[j] = out | (states[j] or frozenset())
                todo.append(j)
    found = []
    for (_, block), state in zip(blocks, states):
        if state is not None:
            _walk(block, state, found)
    return found, sum(own and t.startswith(READ) for _, b in blocks for t, own in b)


def check(assembly: str, where: str) -> int:
    """Raises if a kernel of this assembly touches a register whose read is in flight; the number of reads."""
    reads = 0
    for m in re.finditer(r"^(\w+):[^\n]*\n(.*?)^\s*\.size", assembly, re.S | re.M):
        found, n = touched_in_flight(m.group(2))
        if found:
            raise RuntimeError(f"{where}: {m.group(1)} touches registers whose LDS read is in flight: {found[:3]}; the "
                               f"compiler ran out of registers there or moved them, results could be wrong")
        reads += n
    if reads == 0:
        raise RuntimeError(f"{where}: no LDS read by inline assembly found in what the compiler made")
    return reads
