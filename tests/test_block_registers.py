"""Generated code of the norm and cache kernels, compiled to assembly: no scratch memory where a loop would meet it, kernels on multiples of 4 KiB, and, along every path,
the wait states that the results of a matrix instruction need before any other instruction touches them (the hardware does not wait by itself).  No GPU needed."""
import os
import re
import subprocess
import tempfile

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = os.path.join(ROOT, "paper_2507_03220_amd", "csrc", "symb_block.hip")
# passes of four clocks + 3
WAIT = {"v_mfma_scale_f32_16x16x128_f8f6f4": 11, "v_mfma_scale_f32_32x32x64_f8f6f4": 19, "v_mfma_f32_16x16x32_bf16": 7, "v_mfma_f32_32x32x16_bf16": 11}


@pytest.fixture(scope="module")
def block_asm():
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as d:
        out = os.path.join(d, "block.s")
        subprocess.check_call([hipcc, "-O3", "--offload-arch=gfx950", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "--cuda-device-only",
                               "-S", "-o", out, SRC], stderr=subprocess.DEVNULL)
        return open(out).read()


def _regs(text):
    """Registers named in an operand list: {("v", 3), ("a", 7), ...}"""
    out = set()
    for kind, lo, hi, one in re.findall(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+))", text):
        out |= {(kind, i) for i in (range(int(lo), int(hi) + 1) if lo else [int(one)])}
    return out


def _kernels(text, pattern):
    for m in re.finditer(r"^(_ZN4symb\d+" + pattern + r"\w*):(.*?)^\.Lfunc_end", text, re.S | re.M):
        code, labels = [], {}
        for raw in m.group(2).splitlines():
            s = raw.split(";")[0].strip()
            if re.match(r"^\.LBB\w+:", s):
                labels[s[:-1]] = len(code)
            elif s and not s.startswith((".", "//")) and not s.endswith(":"):
                code.append(s)
        yield m.group(1), code, labels


def _next(code, labels, i):
    op, _, rest = code[i].partition(" ")
    if op in ("s_endpgm",):
        return []
    if op == "s_branch":
        return [labels[rest.strip()]]
    if op.startswith("s_cbranch"):
        return [labels[rest.strip()], i + 1]
    return [i + 1] if i + 1 < len(code) else []


def test_results_of_matrix_instructions_are_waited_for(block_asm):
    checked = 0
    for name, code, labels in _kernels(block_asm, r"symb_kv_(?:rows|attention)_kernel"):
        touched = [_regs(c.partition(" ")[2]) if not c.startswith(("s_", "ds_nop")) else set() for c in code]
        for i, c in enumerate(code):
            op, _, rest = c.partition(" ")
            if not op.startswith("v_mfma"):
                continue
            checked += 1
            need, dst = WAIT[op], _regs(rest.split(",")[0])
            seen, todo = {}, [(j, 0) for j in _next(code, labels, i)]
            while todo:
                j, waited = todo.pop()
                if waited >= need or seen.get(j, need) <= waited:
                    continue
                seen[j] = waited
                o, _, r = code[j].partition(" ")
                if not o.startswith("v_mfma"):                  # (one matrix instruction behind another: interlocked, or an operand of it, which the compiler spaces)
                    assert not (touched[j] & dst), (name, c, waited, code[j])
                todo += [(k, waited + (int(r, 0) + 1 if o == "s_nop" else 1)) for k in _next(code, labels, j)]
    assert checked > 500


def test_no_scratch_memory(block_asm):
    found = re.findall(r"\.amdhsa_kernel (\S+)(.*?)\.end_amdhsa_kernel", block_asm, re.S)
    assert len(found) >= 20
    for name, body in found:
        m = re.search(r"\.amdhsa_private_segment_fixed_size (\d+)", body)
        assert m and int(m.group(1)) == 0, (name, m and m.group(1))


def test_kernels_start_on_multiples_of_4_kib(block_asm):
    kernels = re.findall(r"\.amdhsa_kernel (_ZN4symb\w+)", block_asm)
    aligned = re.findall(r"\.p2align\s+12[^\n]*\n(?:[^\n]*@function\n)?(_ZN4symb\w+):", block_asm)
    assert kernels and sorted(kernels) == sorted(aligned)
