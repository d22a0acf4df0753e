"""What a segment's bits hang on: norm outputs, input gradients and the cache's bytes on its own rows and pages alone, whoever else is in the batch."""
import numpy as np
import pytest
import torch

import gpu_harness as gh
from block_harness import Pages, bf16, offsets, stream
from paper_2507_03220_amd import binding as sb
from paper_2507_03220_amd import block as blk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("width", [136, 768, 4096, 6152, 16384])
def test_norm_rows_alone_and_in_company(width, rms):
    """Alone without gradients, and in a batch of thousands of rows in which others want both."""
    rng = np.random.default_rng(width)
    lens = [3, 2000, 1, 7]
    off, T = offsets(lens), sum(lens)
    X, dY, w, b = bf16(rng, T, width, std=1.5, mean=0.3), bf16(rng, T, width), [bf16(rng, width, std=0.2, mean=1.0) for _ in lens], [bf16(rng, width) for _ in lens]
    dw, db = torch.empty(4, width, device="cuda"), torch.empty(4, width, device="cuda")

    def run(at, norms, X, dY):
        batch = sb.NormBatch(width, at, norms, int(rms), 1e-5)
        Y, dX, ws = torch.empty_like(X), torch.empty_like(X), torch.empty(max(sb.symb_norm_workspace_bytes(batch), 16), device="cuda", dtype=torch.uint8)
        sb.symb_norm_fwd(gh.handle(), batch, X, Y, stream())
        sb.symb_norm_bwd(gh.handle(), batch, X, dY, dX, 0, ws, stream())
        return Y, dX
    Y, dX = run(off, [sb.Norm(w[i], b[i], dw[i], db[i]) for i in range(4)], X, dY)
    for i in (0, 2, 3):
        rows = slice(off[i], off[i + 1])
        y, dx = run([0, lens[i]], [sb.Norm(w[i], b[i])], X[rows].clone(), dY[rows].clone())
        assert torch.equal(y, Y[rows]) and torch.equal(dx, dX[rows])


@pytest.mark.parametrize("pairs", [sb.SYMB_ROTATE_HALVES, sb.SYMB_ROTATE_ADJACENT])
@pytest.mark.parametrize("D,P", [(64, 32), (128, 64)])
def test_appended_rows_alone_and_in_company(D, P, pairs):
    """A few rows by themselves (a wavefront a head) and beside a prompt (workgroups of four, eight query heads in one): the same bytes of keys and values, the same scales, the same queries."""
    rng = np.random.default_rng(D)
    H, Hq, lens, past = 2, 9, [5, 300, 1], [30, 7, 200]
    off, T = offsets(lens), sum(lens)
    q, k, v = bf16(rng, T, Hq, D), bf16(rng, T, H, D), bf16(rng, T, H, D)
    rot = sb.Rotation(blk.rotation_table(400, D), pairs)
    pg = Pages(rng, lens, past, H, D, P)
    pg.fill(rng, tokens=past)
    cache = pg.cache
    before = [t.view(torch.uint8).clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]

    def run(which):
        for t, b in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), before):
            t.view(torch.uint8).copy_(b)
        rows = torch.cat([torch.arange(off[i], off[i + 1], device="cuda") for i in which])
        out = torch.empty(len(rows), Hq, D, device="cuda", dtype=torch.bfloat16)
        sb.symb_kv_append(gh.handle(), sb.KvBatch(offsets([lens[i] for i in which]), [past[i] for i in which], pg.table[which].contiguous()), cache, rot, q[rows], out, k[rows], v[rows], stream())
        torch.cuda.synchronize()
        return out, [t.view(torch.uint8).clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    together, pages = run([0, 1, 2])
    for i in (0, 2):
        alone, own = run([i])
        assert torch.equal(alone, together[off[i]:off[i + 1]])
        mine = torch.tensor([int(x) for x in pg.ids[i, :-(-(lens[i] + past[i]) // P)]], device="cuda")
        for a, b in zip(own, pages):
            assert torch.equal(a[mine], b[mine])
