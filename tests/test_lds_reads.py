"""The matrix kernels read LDS by inline assembly and wait for it themselves (so that the compiler does not make every
read wait for all direct loads in flight).  The compiler takes such a read's registers as written at once: nothing it
schedules may touch them before the wait.  Checked on the assembly that this compiler makes of the sources, over every
path through every kernel."""
import os
import re
import subprocess

import pytest

from paper_2404_00509_amd import build

READ = ("ds_read_b128", "ds_read_b64_tr_b16")


def registers(text):
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


def walk(block, in_flight, found=None):
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
    """Instructions that touch a register whose read by inline assembly has not been waited for; number of reads."""
    blocks = blocks_of(body)
    at = {label: i for i, (label, _) in enumerate(blocks) if label}
    states = [None] * len(blocks)
    states[0] = frozenset()
    todo = [0]
    while todo:
        i = todo.pop()
        out = walk(blocks[i][1], states[i])
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
            walk(block, state, found)
    return found, sum(own and t.startswith(READ) for _, b in blocks for t, own in b)


def test_the_check_sees_a_register_that_is_touched_too_early():
    read = "\t;;#ASMSTART\n\tds_read_b128 v[4:7], v9\n\t;;#ASMEND\n"
    wait = "\ts_waitcnt lgkmcnt(0)\n"
    use = "\tv_mfma_f32_32x32x16_bf16 a[0:15], v[4:7], v[10:13], a[0:15]\n"
    end = "\ts_endpgm\n"
    assert touched_in_flight(read + wait + use + end) == ([], 1)
    assert len(touched_in_flight(read + use + wait + end)[0]) == 1
    assert len(touched_in_flight(read + "\tv_mov_b32_e32 v20, v6\n" + wait + use + end)[0]) == 1
    assert len(touched_in_flight(read + "\tscratch_store_dwordx4 off, v[4:7], off\n" + wait + end)[0]) == 1
    # ... on one of two paths
    fork = read + "\ts_cbranch_scc1 .LBB0_2\n" + wait + ".LBB0_2:\n" + use + end
    assert len(touched_in_flight(fork)[0]) == 1
    loop = ".LBB0_1:\n" + use + read + "\ts_cbranch_scc1 .LBB0_1\n" + wait + end
    assert len(touched_in_flight(loop)[0]) == 2  # (the read of the next turn overwrites it, too)


@pytest.mark.parametrize("source", ["class_loss.hip", "embed_grad.hip"])
def test_no_register_is_touched_while_its_read_is_in_flight(source, tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    out = str(tmp_path / "kernels.s")
    flags = [f for f in build.HIPCC_FLAGS if f != "-shared"]
    subprocess.run([hipcc] + flags + ["--cuda-device-only", "-S", "-o", out, os.path.join(build.CSRC, source)], check=True,
                   stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    text = open(out).read()
    reads = 0
    for m in re.finditer(r"^(_ZN3mae\w+):[^\n]*\n(.*?)^\s*\.size", text, re.S | re.M):
        found, n = touched_in_flight(m.group(2))
        assert not found, (m.group(1), found[:5])
        reads += n
    assert reads > 100
