"""The products of the losses keep their accumulators in a0..a255 behind the compiler's back (see test_gemm16_registers.py): generated code between their assembly templates names no accumulation
register, no kernel spills, and kernels start on multiples of 4 KiB.  No GPU needed (hipcc cross-compiles)."""
import os
import re
import subprocess
import tempfile

import pytest

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_03220_amd", "csrc", "symb_loss.hip")


@pytest.fixture(scope="module")
def loss_asm():
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as d:
        out = os.path.join(d, "loss.s")
        subprocess.check_call([hipcc, "-O3", "--offload-arch=gfx950", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "--cuda-device-only",
                               "-S", "-o", out, SRC], stderr=subprocess.DEVNULL)
        return open(out).read()


def test_compiler_code_never_touches_accumulation_registers(loss_asm):
    kernels = re.findall(r"^(_ZN4symb\d+symb_loss_(?:scores|grad)_kernel\w+):(.*?)^\.Lfunc_end", loss_asm, re.S | re.M)
    assert len(kernels) == 26                              # {256x256, 256x128, 128x128} x {gradient or not} x {capped or not} x {labels, teacher}; the second product's two
    for name, text in kernels:
        inside, products = False, 0
        for raw in text.splitlines():
            s = raw.strip()
            if "ASMSTART" in s or "ASMEND" in s:
                inside = "ASMSTART" in s
                continue
            code = s.split(";")[0]
            products += inside and "v_mfma_f32_16x16x32_bf16" in code
            assert inside or not (re.search(r"\ba\d+\b|\ba\[\d+", code) or "accvgpr" in code or "v_mfma" in code), (name, code)
        blocks = 64 if "ILi8ELi8E" in name else 32 if "ILi8ELi4E" in name else 16
        assert products >= 7 * blocks, name                # six halves of a stage at least, and one of what is left of the inner dimension


def test_registers_memory_and_alignment(loss_asm):
    found = re.findall(r"\.amdhsa_kernel (\S+)(.*?)\.end_amdhsa_kernel", loss_asm, re.S)
    assert len(found) >= 15
    for name, body in found:
        assert re.search(r"\.amdhsa_private_segment_fixed_size 0\b", body), name
        if "scores_kernel" in name or "grad_kernel" in name:               # one workgroup a CU with tiles of 256 rows, two with 128; the templates' registers and none below them in the compiler's way
            free, accum = (int(re.search(r"\.amdhsa_%s (\d+)" % w, body).group(1)) for w in ("next_free_vgpr", "accum_offset"))
            if "ILi8ELi4E" in name:
                assert 224 <= accum <= 256 and accum + 128 == free, name
            else:
                assert (free, accum) == ((512, 256) if "ILi8E" in name else (256, 192)), name
    kernels = re.findall(r"\.amdhsa_kernel (_ZN4symb\w+)", loss_asm)
    aligned = re.findall(r"\.p2align\s+12[^\n]*\n(?:[^\n]*@function\n)?(_ZN4symb\w+):", loss_asm)
    assert sorted(kernels) == sorted(aligned)
