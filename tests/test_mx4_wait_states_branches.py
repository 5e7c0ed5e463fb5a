"""The wait states around the matrix instructions that the large MXFP4 tiles
write as text, over every path: backwards from an instruction through what
falls into it and every branch to its label, until the states are covered.  A
vector instruction's result may be read by a matrix instruction two wait states
later; a sum may be read, written or set otherwise 18 behind the matrix
instruction that makes it, and is used by another one no sooner than 16 steps
later."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2603_04359_amd import build as b

HIPCC = shutil.which("hipcc") or os.path.join(b.ROCM, "bin", "hipcc")


def _registers(text, kind):
    regs = set()
    for lo, hi in re.findall(r"\b%s\[(\d+):(\d+)\]" % kind, text):
        regs |= set(range(int(lo), int(hi) + 1))
    return regs | {int(r) for r in re.findall(r"\b%s(\d+)\b" % kind, text)}


def _states(ins):
    return int(ins.split()[1], 0) + 1 if ins.startswith("s_nop") else 1


def _flow(body):
    """The instructions and, of each, those that may run right before it."""
    code, at = [], {}
    for line in body.split("\n"):
        line = line.split(";")[0].strip()
        if line.endswith(":"):
            at[line[:-1]] = len(code)
        elif line and not line.startswith("."):
            code.append(line)
    before = [[] for _ in code]
    for i, ins in enumerate(code):
        op = ins.split()[0]
        assert not op.startswith(("s_setpc", "s_swappc", "s_call", "s_cbranch_g_fork")), ins
        if op.startswith(("s_branch", "s_cbranch")):
            to = at[ins.split()[1]]
            if to < len(code):
                before[to].append(i)
        if op not in ("s_branch", "s_endpgm") and i + 1 < len(code):
            before[i + 1].append(i)
    return code, before


def _within(code, before, i, states):
    """Instructions that may end fewer than `states` wait states before
    instruction i, over all paths."""
    least = {}
    todo = [(p, 0) for p in before[i]]
    while todo:
        k, waited = todo.pop()
        if waited >= states or least.get(k, states) <= waited:
            continue
        least[k] = waited
        todo += [(p, waited + _states(code[k])) for p in before[k]]
    return least


def _violations(body):
    code, before = _flow(body)
    bad = []
    for i, ins in enumerate(code):
        ops = ins.split(None, 1)[1] if " " in ins or "\t" in ins else ""
        if ins.startswith("v_mfma"):
            reads, sums = _registers(ops, "v"), _registers(ops, "a")
            for k in _within(code, before, i, 2):
                prev = code[k]
                if prev.startswith("v_") and not prev.startswith(("v_mfma", "v_cmp")):
                    dst = prev.split(None, 1)[1].split(",")[0]
                    if _registers(dst, "v") & reads or _registers(dst, "a") & sums:
                        bad.append((prev, ins))
            for k in _within(code, before, i, 15):
                if code[k].startswith("v_mfma") and _registers(code[k].split(",")[0], "a") & sums:
                    bad.append((code[k], ins))
        elif _registers(ops, "a"):
            for k in _within(code, before, i, 18):
                if code[k].startswith("v_mfma") and _registers(code[k].split(",")[0], "a") & _registers(ops, "a"):
                    bad.append((code[k], ins))
    return bad


MFMA = "v_mfma_scale_f32_16x16x128_f8f6f4 a[0:3], v[0:3], v[4:7], a[0:3], v8, v9"


@pytest.mark.parametrize("body,count", [
    # a result at the end of a loop, read by its first matrix instruction
    ("v_mov_b32 v0, 0\ns_nop 1\n.L1:\n" + MFMA + "\ns_nop 15\nv_add_u32 v8, v8, v1\ns_cbranch_scc1 .L1\ns_endpgm", 1),
    ("v_mov_b32 v0, 0\ns_nop 1\n.L1:\n" + MFMA + "\ns_nop 15\nv_add_u32 v8, v8, v1\ns_nop 0\n"
     "s_cbranch_scc1 .L1\ns_endpgm", 0),
    # what stands above a label behind an unconditional branch does not run before it
    ("s_cbranch_scc0 .L2\ns_nop 1\nv_mov_b32 v0, 0\ns_branch .L3\n.L2:\n" + MFMA + "\n.L3:\ns_endpgm", 0),
    # a sum read too early on one of two paths, and again by a matrix instruction
    (MFMA + "\ns_cbranch_scc1 .L4\ns_nop 15\ns_nop 15\n.L4:\nv_accvgpr_read_b32 v1, a2\ns_endpgm", 1),
    (".L5:\n" + MFMA + "\ns_nop 7\ns_cbranch_scc1 .L5\ns_endpgm", 1)])
def test_the_reader_follows_branches(body, count):
    assert len(_violations(body)) == count


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")
def test_wait_states_over_every_path(tmp_path):
    out = tmp_path / "k.s"
    flags = [f for f in b.HIP_FLAGS if f != "-fPIC"]
    subprocess.run([HIPCC, *flags, "--cuda-device-only", "-S", os.path.join(b.CSRC, "k_mx4_gemm.hip"),
                    "-o", str(out)], check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    kernels = re.findall(r"^(_ZN4catk15mx4_tile_kernel\w+):(.*?)\.Lfunc_end", out.read_text(), re.S | re.M)
    assert len(kernels) == 12
    for name, body in kernels:
        assert "s_cbranch" in body, name
        assert not _violations(body), (name, _violations(body)[:3])
