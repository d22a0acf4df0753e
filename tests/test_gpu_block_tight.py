"""Attention held to bounds that a lost or doubled chunk, part or row cannot pass: whole tensors in the 2-norm, and sums in which every chunk of tokens has a channel to itself, so that each output says
exactly whose tokens it counted.  And the norms' backward pass over batches of every way that its rows are cut."""
import numpy as np
import pytest
import torch

import gpu_harness as gh
from block_harness import Pages, attend, bf16, close, host, offsets, stream
from block_paths import PATHS, Path, check
from oracle import block as ob
from paper_2507_03220_amd import binding as sb
from test_gpu_block_wide import _copies

pytestmark = pytest.mark.gpu
CHUNK = 64                                                 # tokens that the kernels take at a time


# ---- whole tensors ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("D,P", [(64, 32), (64, 128), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("window", [0, 1, 65, 300])
@pytest.mark.parametrize("path", PATHS)
def test_every_kernel_in_the_norm(path, window, D, P):
    p = Path(path, D, P, 90 + D + window, window)
    q = p.queries(1.5)
    check(p.run(q), p.formula(q), (path, window))


@pytest.mark.parametrize("path", PATHS)
def test_scores_that_differ_by_hundreds(path):
    """Nearly all of a row's weight on one token, wherever it lies.  A score's products are good to 2^-14 of the largest of them, 2^-7 / 64 of 60 here, and where two large scores meet, weights move by as much:
    the 2-norm keeps its bound of 5e-3, as rows with one token alone have none of it."""
    p = Path(path, 128, 64, 91, std=448.0)
    q = p.queries(20.0)
    want = p.formula(q)
    got = host(p.run(q))
    for copy in got:
        assert np.linalg.norm(copy - want[0]) / np.linalg.norm(want[0]) < 5e-3


# ---- who was counted -------------------------------------------------------------------------------------------------------------------
def _marked(rng, lens, past, H, D, P, first):
    """Pages of zeros but for the chunks first .. first + D - 1 of every segment: a token of chunk first + c holds 448 in channel c.  Returns the pages and, per segment, the marked tokens."""
    pg = Pages(rng, lens, past, H, D, P)
    marks = []
    for i, (n, p) in enumerate(zip(lens, past)):
        m = n + p
        k, v = np.zeros((m, H, D)), np.zeros((m, H, D))
        at = np.array([t for t in ((first + c) * CHUNK + int(rng.integers(0, CHUNK)) for c in range(D)) if t < m], int)
        v[at, :, np.arange(len(at))] = 448.0
        pages = -(-m // P)
        pg.put(i, k, v, np.zeros((pages, H), int), np.zeros((pages, H), int))
        marks.append(at)
    return pg, marks


def _counted(got, lens, past, marks, window, what):
    """Zero queries: every weight is 1.  A row's output is 448 / (tokens it sees) in the channels of the marked tokens among them, half a bf16 step of it off at most with 2^-20 for the division, and exactly 0 in the
    others: nothing else is added to them."""
    off = offsets(lens)
    for i, (n, p) in enumerate(zip(lens, past)):
        pos = p + np.arange(n)
        lo = np.maximum(pos + 1 - window, 0) if window else np.zeros(n, int)
        seen = (marks[i][None] <= pos[:, None]) & (marks[i][None] >= lo[:, None])
        want = np.zeros((n, got.shape[-1]))
        want[:, :len(marks[i])] = seen * (448.0 / (pos + 1 - lo))[:, None]
        rows = got[..., off[i]:off[i + 1], :, :]
        close(rows, np.broadcast_to(want[:, None], rows.shape), np.broadcast_to((2.0 ** -8 * want * 1.01)[:, None], rows.shape), (what, i))


@pytest.mark.parametrize("D,P", [(64, 64), (128, 32)])
@pytest.mark.parametrize("H,group,lens,past,window", [
    (1, 4, [1, 2, 1], [9000, 5000, 130], 0),               # decode steps, split and joined row by row
    (1, 4, [1, 2], [9000, 5000], 3000),
    (1, 16, [2, 3], [30000, 9000], 0),                     # runs of 32 and 48 rows of long contexts, split
    (1, 48, [1] * 4, [30000, 20000, 1000, 63], 0),
    (2, 8, [600, 1, 9], [205, 700, 64], 0),                # prompts in tiles that are split, joined 16 rows at a time
    (2, 8, [600, 1, 9], [205, 700, 64], 400),
    (1, 8, [300], [5000], 0),                              # a prompt behind a long context
])
def test_every_chunk_of_a_split_context_counts_once(H, group, lens, past, window, D, P):
    rng = np.random.default_rng(D + H * group)
    copies = _copies(lens, past, H, group, window)         # (so many that runs of 17 to 48 rows have kernels of their own, and prompts are tiles)
    chunks = -(-max(n + p for n, p in zip(lens, past)) // CHUNK)
    for first in range(0, chunks, D):
        pg, marks = _marked(rng, lens, past, H, D, P, first)
        pg.batch = sb.KvBatch(offsets(lens * copies), past * copies, pg.table.repeat(copies, 1))
        assert sb.symb_kv_workspace_bytes(pg.batch, pg.cache, H * group, window) > 0
        q = torch.zeros(sum(lens) * copies, H * group, D, device="cuda", dtype=torch.bfloat16)
        got = host(attend(pg, q, D ** -0.5, window)).reshape(copies, sum(lens), -1, D)
        _counted(got, lens, past, marks, window, first)


@pytest.mark.parametrize("D,P", [(64, 32), (128, 64)])
@pytest.mark.parametrize("window", [0, 200])
@pytest.mark.parametrize("path", PATHS)
def test_every_chunk_counts_once(path, window, D, P):
    c = PATHS[path]
    rng = np.random.default_rng(92)
    copies = _copies(c["lens"], c["past"], c["H"], c["group"], window) if c["many"] else 1
    pg, marks = _marked(rng, c["lens"], c["past"], c["H"], D, P, 0)
    pg.batch = sb.KvBatch(offsets(c["lens"] * copies), c["past"] * copies, pg.table.repeat(copies, 1))
    T = sum(c["lens"])
    q = torch.zeros(T * copies, c["H"] * c["group"], D, device="cuda", dtype=torch.bfloat16)
    got = host(attend(pg, q, D ** -0.5, window)).reshape(copies, T, -1, D)
    _counted(got, c["lens"], c["past"], marks, window, path)


# ---- the norms' backward pass over many rows ---------------------------------------------------------------------------------------------
def _ragged(rng, S, T):
    cuts = np.sort(rng.integers(0, T + 1, S - 1))
    return np.diff(np.concatenate([[0], cuts, [T]])).tolist()


@pytest.mark.parametrize("rms,bias", [(False, True), (True, False), (True, True)])
@pytest.mark.parametrize("width,lens,shared", [
    (64, [8000], 0),                                       # 768 chunks, one segment: hundreds of partial sums
    (64, [2000] * 4, 2),                                   # in pairs that share their gradients
    (72, "600 of 8000", 0),                                # ragged segments: rows a chunk grow until 768 chunks hold them
    (72, "900 of 8000", 3),                                # more segments than chunks
    (136, [3000], 0),                                      # 512 chunks
    (136, "40 of 3000", 5),
    (520, [1200], 0),                                      # 256
    (520, "7 of 1200", 2),
    (4104, [1000, 0, 1500], 0),                            # wide: chunks of more rows
])
def test_norm_backward_over_many_rows(width, lens, shared, rms, bias):
    """dX: half a bf16 step, and fp32 terms of size |dy w| r to 2^-20 (r is 1 / 1.5 here, |dy w| up to 10).  Weight gradients: fp32 sums of n terms good to 2^-24 n of the sum of their magnitudes at worst, the
    terms themselves to 2e-6; and in the 2-norm, where roundings add up as their square root, to 1e-5."""
    rng = np.random.default_rng(width + (0 if isinstance(lens, str) else len(lens)))
    if isinstance(lens, str):
        lens = _ragged(rng, *map(int, lens.split(" of ")))
    S, T, off = len(lens), sum(lens), offsets(lens)
    X, dY, w = bf16(rng, T, width, std=1.5, mean=0.5), bf16(rng, T, width), [bf16(rng, width, std=0.2, mean=1.0) for _ in range(3)]
    owner = [i // shared if shared else i for i in range(S)]
    dw = torch.full((owner[-1] + 1, width), 3.0, device="cuda")
    db = torch.full((owner[-1] + 1, width), -2.0, device="cuda")
    batch = sb.NormBatch(width, off, [sb.Norm(w[i % 3], None, dw[o].data_ptr(), db[o].data_ptr() if bias else None) for i, o in enumerate(owner)],
                         sb.SYMB_NORM_RMS if rms else sb.SYMB_NORM_LAYER, 1e-5, 0.0)
    ws = torch.full((sb.symb_norm_workspace_bytes(batch),), 255, device="cuda", dtype=torch.uint8)
    dX = torch.full_like(X, float("nan"))
    hw, x, dy = [host(t) for t in w], host(X), host(dY)
    want, ww, wb = ob.norm_bwd(off, x, dy, [hw[i % 3] for i in range(S)], not rms, 1e-5, 0.0)
    z = ob.norm_fwd(off, x, [None] * S, [None] * S, not rms, 1e-5, 0.0)
    sums = [np.zeros((owner[-1] + 1, width)) for _ in range(4)]
    rows = np.zeros(owner[-1] + 1)
    for i, o in enumerate(owner):
        part = slice(off[i], off[i + 1])
        for total, add in zip(sums, (ww[i], wb[i], np.abs(dy[part] * z[part]).sum(0), np.abs(dy[part]).sum(0))):
            total[o] += add
        rows[o] += lens[i]
    gw, gb, mw, mb = sums
    for times, flags in ((1, sb.SYMB_GRAD_OVERWRITE), (2, sb.SYMB_GRAD_ACCUMULATE)):
        sb.symb_norm_bwd(gh.handle(), batch, X, dY, dX, flags, ws, stream())
        slack = ((2e-6 + 2.0 ** -24 * rows) * times)[:, None]
        close(dX, want, 1.01 * 2.0 ** -8 * np.abs(want) + 1e-4 * np.abs(want).max(), "dX")
        close(dw, times * gw, slack * mw + 1e-6, "dweight")
        assert np.linalg.norm(host(dw) - times * gw) < 1e-5 * times * np.linalg.norm(gw)
        if bias:
            close(db, times * gb, slack * mb + 1e-6, "dbias")
            assert np.linalg.norm(host(db) - times * gb) < 1e-5 * times * np.linalg.norm(gb)
        else:
            assert (db == -2).all()
