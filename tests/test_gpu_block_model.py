"""paper_2507_03220_amd/block.py as a model uses it: on streams of its own, with the score scale and the biases that the model has."""
import numpy as np
import pytest
import torch

import gpu_harness as gh
from block_harness import bf16, stream
from paper_2507_03220_amd import binding as sb
from paper_2507_03220_amd import block as blk

pytestmark = pytest.mark.gpu


def _lora(rng, d_in, d_out, r, grads=False):
    a = sb.Adapter(sb.SYMB_ADAPTER_LORA, r, 1.5, bf16(rng, r, d_in, std=d_in ** -0.5), bf16(rng, d_out, r, std=r ** -0.5))
    if grads:
        a.dA, a.dB = torch.empty(r, d_in, device="cuda"), torch.empty(d_out, r, device="cuda")
    return a


def test_a_normed_projection_on_streams_of_its_own():
    """The same bits on torch's current stream, on another, and forward on one with backward on a third; torch's own work between the passes takes what memory it is given."""
    rng = np.random.default_rng(1)
    width, d_out, lens = 256, 384, [70, 3, 0, 129]
    W, X, dY = bf16(rng, d_out, width, std=width ** -0.5), bf16(rng, 202, width, mean=0.3), bf16(rng, 202, d_out)
    weights, ads = [bf16(rng, width, std=0.1, mean=1.0) for _ in lens], [_lora(rng, width, d_out, r, True) for r in (8, 16, 4, 5)]
    grads = [torch.empty(width, device="cuda") for _ in lens]

    def step(first, second):
        run = blk.NormedProjection(gh.handle(), W, lens, [sb.Norm(w, None, g) for w, g in zip(weights, grads)], ads, sb.SYMB_NORM_RMS, 1e-6)
        for g in grads + [t for a in ads for t in (a.dA, a.dB)]:
            g.fill_(float("nan"))
        torch.cuda.synchronize()
        out = []
        for _ in range(3):
            y = run.forward(X, None, first)
            torch.full((202, d_out), float("nan"), device="cuda", dtype=torch.bfloat16)
            if first != second:
                torch.cuda.synchronize()
            d = run.backward(X, dY, stream=second)
            torch.full((202, width), float("nan"), device="cuda", dtype=torch.bfloat16)
            torch.cuda.synchronize()
            out += [y.clone(), d.clone()]
        return out + [t.clone() for a in ads for t in (a.dA, a.dB)] + [g.clone() for g in grads]
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    want = step(stream(), stream())
    assert all(torch.isfinite(t).all() for t in want)
    for first, second in ((a.cuda_stream, a.cuda_stream), (a.cuda_stream, b.cuda_stream), (stream(), a.cuda_stream)):
        for x, y in zip(want, step(first, second)):
            assert torch.equal(x, y)
