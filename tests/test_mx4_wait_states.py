"""The matrix instructions that the large MXFP4 tiles write as text are not
seen by the compiler, which therefore does not insert the two wait states
between a vector instruction's result and a matrix instruction that reads it.
The generated code is checked for them: no vector instruction writes an
operand or a sum within the two instructions before a matrix instruction
that reads it, nor does anything but a matrix instruction or a store
preparation touch the sums while one may still be in flight (the reads come
behind at least 32 wait states)."""
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


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")
def test_no_vector_result_reaches_a_matrix_instruction_too_early(tmp_path):
    out = tmp_path / "k.s"
    flags = [f for f in b.HIP_FLAGS if f != "-fPIC"]
    subprocess.run([HIPCC, *flags, "--cuda-device-only", "-S", os.path.join(b.CSRC, "k_mx4_gemm.hip"),
                    "-o", str(out)], check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    kernels = re.findall(r"^(_ZN4catk15mx4_tile_kernel\w+):(.*?)\.Lfunc_end", out.read_text(), re.S | re.M)
    assert len(kernels) == 12
    seen = 0
    for name, body in kernels:
        lines = [line.strip() for line in body.split("\n")]
        code = [x for x in lines if x and not x.startswith((";", "."))]
        code = [x for x in code if not x.endswith(":")]
        assert not any(x.startswith("scratch_") for x in code), name
        since = 99                          # wait states since the last matrix instruction
        for i, ins in enumerate(code):
            if ins.startswith("v_mfma"):
                seen += 1
                since = 0
                ops = ins.split(None, 1)[1]
                reads, sums = _registers(ops, "v"), _registers(ops, "a")
                k, waited = i - 1, 0
                while k >= 0 and waited < 2:
                    prev = code[k]
                    if prev.startswith("v_") and not prev.startswith(("v_mfma", "v_cmp")):
                        dst = prev.split(None, 1)[1].split(",")[0]
                        assert not _registers(dst, "v") & reads, (name, prev, ins)
                        assert not _registers(dst, "a") & sums, (name, prev, ins)
                    waited += _states(prev)
                    k -= 1
            else:
                if ins.startswith("v_accvgpr_read"):
                    assert since >= 18, (name, ins, since)
                since += _states(ins)
    assert seen == 4 * (64 + 128 + 256)     # of the four stages of a kernel, by its tile
