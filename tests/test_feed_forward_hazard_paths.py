"""A memory instruction may read a scalar register five wait states after a
vector instruction wrote it, not sooner: the compiled loads of the feed-forward
products, along every path through the code, loops' back edges among them (no
GPU needed)."""

import os
import re
import subprocess

import pytest

from paper_2412_02962_amd import build

WAIT_STATES = 5
MEMORY = ("buffer_", "global_", "flat_", "scratch_")
# scalar instructions whose first operand is read, or is no register
NO_RESULT = ("s_cmp", "s_bitcmp", "s_setreg", "s_nop", "s_wait", "s_branch", "s_cbranch", "s_barrier", "s_endpgm",
             "s_setprio", "s_sleep", "s_sendmsg", "s_trap", "s_icache", "s_set_gpr", "s_code_end")


def _scalars(operand):
    m = re.fullmatch(r"(s|ttmp)\[(\d+):(\d+)\]|(s|ttmp)(\d+)", operand)
    if m:
        kind, first, last = (m[1], m[2], m[3]) if m[1] else (m[4], m[5], m[5])
        return {f"{kind}{i}" for i in range(int(first), int(last) + 1)}
    if operand in ("vcc", "exec", "flat_scratch"):
        return {operand + "_lo", operand + "_hi"}
    return {operand} if operand in ("m0", "vcc_lo", "vcc_hi", "exec_lo", "exec_hi") else set()


def _instructions(assembly):
    """[(operation, operands, line)], and every label's position: that of the
    instruction after it."""
    code, labels = [], {}
    for line in assembly.splitlines():
        text = line.split(";")[0].split("//")[0].strip()
        label = re.fullmatch(r"([.\w$]+):", text)
        if label:
            labels[label[1]] = len(code)
        elif text and not text.startswith("."):
            t = text.replace(",", " ").split()
            code.append((t[0], t[1:], text))
    return code, labels


def _after(op, operands, since):
    """Wait states since the vector writes of `since`, after an instruction."""
    states = int(operands[0], 0) + 1 if op == "s_nop" else 1
    since = {r: n + states for r, n in since.items() if n + states < WAIT_STATES}
    if op.startswith("v_"):
        # the result, and a carry or a comparison's mask beside a vector result
        results = set().union(*map(_scalars, operands[:1]))
        if re.match(r"v_(add|sub|subrev|addc|subb|subbrev)_co_|v_mad_[ui]64_|v_div_scale_", op):
            results |= set().union(*map(_scalars, operands[1:2]))
        since.update(dict.fromkeys(results, 0))
    elif op.startswith("s_") and not op.startswith(NO_RESULT) and operands:
        for r in _scalars(operands[0]):
            since.pop(r, None)
    return since


def early_reads(assembly):
    """The memory instructions that some path reaches with a scalar register
    of theirs written by a vector instruction too short a time before."""
    code, labels = _instructions(assembly)
    assert not [op for op, _, _ in code if op.startswith(("s_setpc", "s_swappc", "s_call"))], "paths unknown"
    state, found = {0: {}}, {}
    state.update({at: {} for at in labels.values()})  # functions begin at labels
    work = list(state)
    while work:
        at = work.pop()
        if at >= len(code):
            continue
        op, operands, line = code[at]
        since = state[at]
        if op.startswith(MEMORY):
            read = set().union(*map(_scalars, operands)) | ({"m0"} if "lds" in operands else set())
            if read & set(since):
                found[at] = line
        since = _after(op, operands, since)
        follow = [] if op in ("s_branch", "s_endpgm") else [at + 1]
        if op.startswith(("s_branch", "s_cbranch")):
            follow.append(labels[operands[0]])
        for n in follow:  # the shortest time over the paths that meet
            old = state.get(n)
            new = dict(since)
            for r, s in (old or {}).items():
                new[r] = min(s, new.get(r, s))
            if old is None or new != old:
                state[n] = new
                work.append(n)
    return [found[at] for at in sorted(found)]


LOAD = "buffer_load_dwordx4 v2, s[4:7], 0 offen lds"


@pytest.mark.parametrize("early,code", [
    (1, ["v_readfirstlane_b32 s6, v1", "s_nop 3", LOAD]),
    (0, ["v_readfirstlane_b32 s6, v1", "s_nop 4", LOAD]),
    (0, ["v_readfirstlane_b32 s6, v1", "s_mov_b32 s6, s9", LOAD]),
    # a comparison reads its scalar registers, a bit test too
    (1, ["v_readfirstlane_b32 s6, v1", "s_cmp_lg_u32 s6, 0", LOAD]),
    (1, ["v_readfirstlane_b32 s6, v1", "s_bitcmp1_b32 s6, 0", LOAD]),
    # a loop: the write at its end, the load at its head
    (1, ["v_mov_b32_e32 v2, 0", ".LBB0_1:", LOAD, "s_add_i32 s8, s8, 1", "s_cmp_lt_i32 s8, s9",
         "v_readfirstlane_b32 s6, v1", "s_cbranch_scc1 .LBB0_1", "s_endpgm"]),
    (0, ["v_mov_b32_e32 v2, 0", ".LBB0_1:", "s_nop 3", LOAD, "v_readfirstlane_b32 s6, v1", "s_cbranch_scc1 .LBB0_1",
         "s_endpgm"]),
    # a branch over the wait, and one that the load does not follow
    (1, ["v_readfirstlane_b32 s6, v1", "s_cbranch_scc0 .LBB0_2", "s_nop 7", ".LBB0_2:", LOAD, "s_endpgm"]),
    (0, ["v_readfirstlane_b32 s6, v1", "s_branch .LBB0_2", LOAD, ".LBB0_2:", "s_endpgm"]),
    # masks and carries of vector instructions
    (1, ["v_cmp_gt_u32_e64 s[4:5], v0, v1", LOAD]),
    (1, ["v_add_co_u32_e64 v0, s[6:7], v1, v2", LOAD]),
    (1, ["v_readfirstlane_b32 m0, v1", LOAD]),
    (0, ["v_readfirstlane_b32 s8, v1", LOAD]),
])
def test_the_reader_of_paths(early, code):
    assert len(early_reads("\n".join(code))) == early


def test_no_path_reads_a_buffer_too_early():
    src = os.path.join(build.CSRC, "ff_product.hip")
    r = subprocess.run([build.hipcc()] + build.flags_of(src) + ["--cuda-device-only", "-S", "-o", "-", src],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert len([line for line in r.stdout.splitlines() if "offen lds" in line]) > 100
    assert early_reads(r.stdout) == []
