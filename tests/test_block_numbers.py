"""What the attention kernels' comments and include/symb_block.h say of their number formats, worked out in numpy: queries as two E4M3 terms, capped scores in fp32.  No GPU needed."""
import re
from pathlib import Path

import numpy as np

from oracle import block as ob
from paper_2507_03220_amd import binding as sb

KERNELS = (Path(sb.__file__).parent / "csrc" / "kv_attention_kernels.hpp").read_text()
f32 = np.float32


def test_a_query_is_two_terms_exact_to_a_8192th_of_its_largest():
    """Every bf16 value from 2^-25 of a row's largest on, largest ones of both ends of [128, 256): hi + lo / 16 is it from 2^-13 of the largest on, and off by 2^-21 of the largest at most below."""
    mantissas = 1 + np.arange(128) / 128
    x = np.concatenate([mantissas * 2.0 ** e for e in range(-18, 8)])
    hi = ob.e4m3(x)
    lo = ob.e4m3(np.abs(x - hi) * 16) * np.sign(x - hi)
    off = np.abs(hi + lo / 16 - x)
    for largest in (128.0, 255.0):
        row = x <= largest
        assert not off[row & (x >= largest * 2.0 ** -13)].any()
        assert (off[row] <= largest * 2.0 ** -21).all()
    assert off[x == 2.0 ** -7 + 2.0 ** -14] > 0                             # at 2^-14 of 128 the last bit goes


def test_capped_scores_are_good_to_a_part_in_half_a_million():
    """The formula and the series on their sides of a quarter of the cap, every operation rounded to fp32, exp2 and the reciprocal an ulp off either way: 2^-19 of the score."""
    root, a, b = (f32(re.search(p, KERNELS)[1]) for p in (r"kKvRoot = ([\d.]+)f", r"z, -([\d.]+)f\), x\)", r"fmaf\(z, ([\d.]+)f - z"))
    assert abs(root ** 6 - 17 / 315) < 1e-7 and abs(a * root ** 2 - 1 / 3) < 1e-6 and abs(b * root ** 4 - 2 / 15) < 1e-6
    x = np.linspace(1e-4, 30, 1500001).astype(f32)
    x = np.concatenate([-x[::-1], x])
    for to_cap in (f32(root), f32(root) / f32(3.7), f32(root) / f32(77)):
        u = x * to_cap
        want = np.tanh(x.astype(float) * (to_cap / root)) / (to_cap / root)
        near = np.abs(u) <= f32(0.25) * root
        z = u[near] * u[near]
        fma = lambda p, q, r: (p.astype(float) * q + r).astype(f32)  # noqa: E731
        got = fma(x[near] * z, fma(z, b - z, -a), x[near])
        assert (np.abs(got - want[near]) <= 2.0 ** -19 * np.abs(want[near])).all()
        for de in (-1, 0, 1):
            e = np.exp2((u[~near] * f32(2.885390082 / root)).astype(float)).astype(f32)
            e = e + de * np.spacing(e)
            for dr in (-1, 0, 1):
                r = (1 / (e + f32(1)).astype(float)).astype(f32)
                r = r + dr * np.spacing(r)
                got = (f32(1) / (to_cap / root)) * (f32(1) - f32(2) * r)
                assert got.dtype == f32 and (np.abs(got - want[~near]) <= 2.0 ** -19 * np.abs(want[~near])).all()
