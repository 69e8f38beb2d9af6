"""Listings of the kernels whose matrix instructions' results cross branches (built here from source, CPU): on every path between a matrix instruction and
the first other use of its result lie as many wait states as the compiler itself puts there within a block - an instruction counts one, s_nop n
counts n + 1: 8 for a 16 x 16 instruction (4 passes), 12 for a 32 x 32 one (8 passes; the block-scaled ones on 4-bit codes take as many)."""
import os
import re
import subprocess

import pytest

from paper_2505_20932_amd import build

_REG = re.compile(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)")
_FLOW = re.compile(r"^(s_branch|s_cbranch\w*)$")


def _regs(operand):
    out = set()
    for kind, lo, hi, one in _REG.findall(operand):
        out |= {(kind, i) for i in range(int(lo or one), int(hi or one) + 1)}
    return out


def kernels(text):
    """{name: (instructions [(opcode, operands, their registers)], {label: index})}"""
    out, cur = {}, None
    for line in text.splitlines():
        line = line.split(";")[0].rstrip()
        label = re.match(r"^([\w.$]+):", line)
        if label:
            if label.group(1).startswith("_Z"):
                cur = out.setdefault(label.group(1), ([], {}))
            elif cur:
                cur[1][label.group(1)] = len(cur[0])
            continue
        word = line.split(None, 1)
        if cur and word and re.match(r"^(v|s|ds|global|buffer|flat|scratch)_", word[0]):
            operands = [x.strip() for x in re.split(r",(?![^\[]*\])", word[1])] if len(word) > 1 else []
            cur[0].append((word[0], operands, [_regs(x) for x in operands]))
    return out


def too_near(code, labels):
    """[(matrix instruction, user, wait states between them)] of uses that come too early on some path."""
    found = []
    for i, (op, _, regs) in enumerate(code):
        if not op.startswith("v_mfma"):
            continue
        need, seen, todo = (12 if "32x32" in op else 8), {}, [(i + 1, 0)]
        while todo:
            j, waits = todo.pop()
            if j >= len(code) or waits >= need or seen.get(j, 99) <= waits:
                continue
            seen[j] = waits
            user, operands, used = code[j]
            if user == "s_endpgm":
                continue
            if user.startswith("v_mfma"):
                if used[0] == regs[0]:                                 # the next sum in the same registers: it has a scan of its own
                    if not (used[1] | used[2]) & regs[0]:
                        continue
                hit = (used[1] | used[2]) & regs[0]
            else:
                hit = any(u & regs[0] for u in used)
            if hit:
                found.append((f"{i}: {op}", f"{j}: {user}", waits))
                continue
            if _FLOW.match(user):
                todo.append((labels[operands[-1]], waits + 1))
                if user == "s_branch":
                    continue
            todo.append((j + 1, waits + (int(operands[0], 0) + 1 if user == "s_nop" else 1)))
    return found


@pytest.mark.parametrize("source", ["mx4_linear.hip", "llm_attention.hip"])
def test_results_are_read_late_enough(source, tmp_path):
    if not os.path.exists(build._hipcc()):
        pytest.skip("needs hipcc")
    out = tmp_path / "k.s"
    subprocess.run([build._hipcc(), *build.HIPCC_FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o", str(out)], check=True,
                   stderr=subprocess.DEVNULL)
    all_kernels = kernels(out.read_text())
    assert sum(op.startswith("v_mfma") for code, _ in all_kernels.values() for op, _, _ in code) > 300
    for name, (code, labels) in all_kernels.items():
        assert not too_near(code, labels), name


def test_the_scan_finds_what_it_looks_for():
    """A result that is read on the back edge of a loop, one short and just far enough; behind a straight line; as an operand of the next one."""
    mfma = "v_mfma_f32_16x16x32_f16 a[0:3], v[0:3], v[4:7], a[0:3]"

    def scan(*lines):
        return len(too_near(*kernels("\n".join(("_Zk:",) + lines))["_Zk"]))
    for nops, want in ((5, 1), (6, 0)):
        assert scan(".L1:", f"s_nop {nops}", "v_accvgpr_read_b32 v9, a2", mfma, "s_cbranch_scc0 .L1", "s_branch .L2", ".L2:", "s_endpgm") == want
    assert scan(mfma, "s_nop 6", "v_add_f32 v1, v2, a3") == 1 and scan(mfma, "s_nop 7", "v_add_f32 v1, v2, a3") == 0
    assert scan(mfma, mfma, "s_nop 7", "global_store_dwordx4 v[8:9], a[0:3], off") == 0
    assert scan(mfma, "v_mfma_f32_16x16x32_f16 a[4:7], a[0:3], v[4:7], a[4:7]") == 1
