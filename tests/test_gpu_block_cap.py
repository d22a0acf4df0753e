"""Capped scores, cap tanh(x / cap), over the whole range of caps: from one that flattens every score to one that changes none (include/symb_block.h)."""
import numpy as np
import pytest
import torch

from block_harness import host
from block_paths import PATHS, Path, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,P", [(64, 32), (128, 64)])
@pytest.mark.parametrize("path", PATHS)
def test_caps_of_every_size(path, D, P):
    """Scores of size 1, some of size 10: a cap below, about and far above them, to the end of fp32."""
    p = Path(path, D, P, 40 + D)
    q = p.queries()
    q[::3] *= 8
    for cap in (0.3, 4.0, 50.0, 1e4, 1e6, 1e9, 3e38):
        check(p.run(q, cap), p.formula(q, cap), (path, cap))


@pytest.mark.parametrize("path", PATHS)
def test_a_large_cap_is_none(path):
    """Behind a cap of 1e9 scores of size 10 move by 1e-17 of themselves.  What may differ is their last fp32 bits, 2^-22 of 10 or 2^-18 of a weight, and with it the rounding of an output to bf16
    (a step of 2^-8) once in 2^10 of them: 2^-13 of the tensor in the 2-norm, held to 2^-10."""
    p = Path(path, 128, 64, 41)
    q = p.queries(3.0)
    plain, capped = host(p.run(q)), host(p.run(q, 1e9))
    assert np.linalg.norm(capped - plain) < 2.0 ** -10 * np.linalg.norm(plain)


@pytest.mark.parametrize("cap", [1e-30, 1e-42])
def test_a_vanishing_cap_weighs_all_tokens_alike(cap):
    """Scores of 1e-30 at most: every weight is 1, also those of a query of zeros."""
    p = Path("rows", 64, 32, 42)
    q = p.queries()
    q[0] = 0.0
    want = p.formula(torch.zeros_like(q))
    check(p.run(q, cap), want, cap)
