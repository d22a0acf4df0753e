"""Cross entropy and distillation through the vocabulary matrix, with their gradients, through the C ABI, against the 64-bit forms of oracle/loss.py: sizes and masks where they can go wrong.
Bounds are worked out from the formats (loss_harness.py); none is fitted."""
import numpy as np
import pytest
import torch

import gpu_harness as gh
from block_harness import host
from loss_harness import NAN, Case, close, stream
from paper_2507_03220_amd import binding as sb

pytestmark = pytest.mark.gpu

SIZES = [([1], 8, 1), ([1], 8, 2), ([3], 64, 63), ([1, 0, 2], 72, 64), ([5], 56, 65), ([17], 128, 255), ([40, 3], 264, 257), ([128], 192, 1000), ([129, 0, 0, 31], 768, 1025), ([1], 4096, 3001),
         ([255, 2, 300], 136, 2047), ([700], 512, 513), ([33] * 20, 320, 5003), ([2], 1032, 40001), ([600], 64, 30011), ([16], 2048, 17000), ([9, 8], 2056, 17001), ([0, 32], 4160, 129),
         ([30], 2104, 16385), ([33], 2048, 300)]


@pytest.mark.parametrize("lens,width,vocab", SIZES)
def test_cross_entropy(lens, width, vocab):
    Case(width + vocab, lens, width, vocab).check("all rows")
    Case(width + vocab + 1, lens, width, vocab, prompt=0.6, mean=False, cap=3.0).check("capped sums, prompts left out")


@pytest.mark.parametrize("entries", [1, 5, 64, 65, 200])
@pytest.mark.parametrize("lens,width,vocab", [s for s in SIZES if s[2] >= 63])
def test_distillation(lens, width, vocab, entries):
    Case(width + vocab + entries, lens, width, vocab, entries).check("all rows")
    Case(width + vocab + entries + 1, lens, width, vocab, entries, prompt=0.4, mean=False, cap=4.0, ragged=True).check("capped sums, prompts and entries left out")


@pytest.mark.parametrize("std", [0.01, 20.0, 60.0])
def test_scores_of_any_size(std):
    """Flat distributions; labels that lie hundreds below the largest score; and those that are all there is."""
    Case(5, [70, 200], 256, 3000, std=std, sure=0.0).check(f"scores of {std}")
    Case(6, [70, 200], 256, 3000, std=std, sure=1.0).check(f"scores of {std}, sure rows")
    Case(7, [70, 200], 256, 3000, 9, std=std, sure=0.5).check(f"entries, scores of {std}")
    for entries in (0, 5):
        Case(8, [20], 256, 3000, entries, std=std, sure=0.5).check(f"few rows, scores of {std}")


def test_weights_in_different_units():
    """Rows whose label lies far below the scores of some columns and not of others: one column alone, one in every part, in the first and the last."""
    width, vocab = 64, 1500
    for columns, rows in [(c, n) for c in ([1499], [0], [700, 701], list(range(5, 1500, 64)), [3, 300, 1400]) for n in (300, 30, 12)]:
        c = Case(11, [rows], width, vocab, std=1.0, sure=0.0)
        w = host(c.W)
        w[:, 0] = 0
        for k, v in enumerate(columns):
            w[v, 0] = 20.0 + k                                 # times x[0]: 0 to 400 above the rest
        x = host(c.X)
        x[:, 0] = np.arange(rows) * 20 / rows
        c.W, c.X = (torch.from_numpy(t.astype(np.float32)).to(torch.bfloat16).cuda() for t in (w, x))
        c.check(f"columns {columns[:4]}, {rows} rows")


def test_sure_rows_keep_their_precision():
    """Losses from 1 down to 1e-12, relative to themselves."""
    c = Case(12, [64], 128, 900, std=1.0, sure=0.0)
    x = host(c.X) * 0.1 + np.linspace(1, 30, 64)[:, None] * host(c.W)[c.labels]
    c.X = torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).cuda()
    _, row, _ = c.check("sure rows")
    assert float(row.min()) < 1e-9


@pytest.mark.parametrize("rows", [20, 60, 200])
@pytest.mark.parametrize("entries", [0, 7])
def test_caps_and_temperatures_of_any_size(entries, rows):
    """From caps that flatten every score to caps that change none, and the ends of what a temperature may be."""
    for cap in (1e-30, 1e-3, 0.5, 4.0, 30.0, 1e6, 1e30, 3e38):
        Case(21, [rows], 128, 900, entries, cap=cap, std=3.0).check(f"cap {cap}")
    if entries:
        for T in (2.0 ** -20, 0.01, 100.0, 2.0 ** 20):
            for cap in (0.0, 8.0, 3e38):
                c = Case(22, [rows], 128, 900, entries, cap=cap, std=3.0, temperatures=[T])
                if T < 1e-3:                               # (the scores themselves to 2^-20 of 1e7: which one is the largest is all that is left to check)
                    loss, row, dX = c.run()
                    assert torch.isfinite(row).all() and torch.isfinite(loss).all() and torch.isfinite(dX).all()
                else:
                    c.check(f"temperature {T}, cap {cap}")


def test_a_token_twice():
    c = Case(13, [9, 30], 64, 300, 12)
    c.ids[:, 5] = c.ids[:, 2]
    c.ids[::2, 9] = c.ids[::2, 2]
    c.check("two and three entries of one token")
    c.ids[:] = 17
    c.check("all entries of one token")


def test_teacher_logits_of_any_size():
    c = Case(14, [8], 64, 300, 4)
    c.logits[0] = [-3.4e38, -3.4e38, -3.4e38, -3.4e38]
    c.logits[1] = [3.4e38, -3.4e38, 3.4e38, 0]
    c.logits[2, 1:] = -np.inf
    c.logits[3] = 1e-38
    c.check("lowest, highest and infinite logits")


def _poisoned(c, change, rows, others=True):
    """Outputs with some rows' inputs changed: these are NaN, the others as they were."""
    clean = c.run()
    undo = change(c)
    loss, row, dX = c.run()
    undo()
    rows = np.asarray(rows)
    keep = np.setdiff1d(np.arange(c.T), rows)
    assert torch.isnan(row[rows]).all() and torch.isnan(dX[rows]).all()
    assert torch.equal(row[keep], clean[1][keep]) and torch.equal(dX[keep], clean[2][keep])
    for i in range(c.S):
        hit = ((rows >= c.off[i]) & (rows < c.off[i + 1])).any()
        assert torch.isnan(loss[i]) if hit else torch.equal(loss[i], clean[0][i])


@pytest.mark.parametrize("entries", [0, 6])
def test_rows_without_an_answer_are_nan_and_no_others(entries):
    c = Case(15, [20, 140, 30], 128, 700, entries, mean=False)

    def outside(c):
        if entries:
            old = c.ids.copy()
            c.ids[[3, 50], 2] = [700, 2 ** 31 - 1]
            return lambda: c.ids.__setitem__(slice(None), old)
        old = c.labels.copy()
        c.labels[[3, 50]] = [700, 2 ** 31 - 1]
        return lambda: c.labels.__setitem__(slice(None), old)
    _poisoned(c, outside, [3, 50])
    for value in (NAN, float("inf"), -float("inf")):
        def poison(c, value=value):
            old = c.X.clone()
            c.X[30, 5] = c.X[189, 127] = value
            return lambda: c.X.copy_(old)
        _poisoned(c, poison, [30, 189])


@pytest.mark.parametrize("entries", [0, 6])
def test_rows_that_take_no_part(entries):
    """All of a batch, all of a segment; what they hold is not looked at (Case puts NaN there) and their gradient is zeros."""
    c = Case(16, [4, 7, 1], 64, 200, entries, prompt=1.0)
    loss, row, dX = c.run()
    assert not loss.any() and not row.any() and not dX.any()
    c = Case(17, [4, 7, 1], 64, 200, entries)
    if entries:
        c.ids[4:11] = -1
    else:
        c.labels[4:11] = -1
    c.X[4:11] = NAN
    c.out[4:11] = True
    loss, _, dX = c.check("a segment without any")
    assert loss[1] == 0 and not dX[4:11].any()


@pytest.mark.parametrize("entries", [0, 4])
def test_holes_and_many_clients(entries):
    """Rows left out here and there, over several lists of 256; thousands of clients, many of them without a row or without one that takes part."""
    rng = np.random.default_rng(23)
    for lens in ([1000, 3, 0, 530], [int(n) for n in rng.integers(0, 4, 2500)]):
        c = Case(24, lens, 64, 300, entries)
        hole = rng.random(c.T) < 0.6
        if entries:
            c.ids[hole] = -3
        else:
            c.labels[hole] = -1
        c.X[torch.from_numpy(hole).cuda()] = NAN
        c.out |= hole
        _, row, dX = c.check("holes")
        assert not row[torch.from_numpy(c.out).cuda()].any() and not dX[torch.from_numpy(c.out).cuda()].any()


def test_in_place():
    for entries in (0, 8):
        c = Case(18, [100, 300], 192, 700, entries, prompt=0.3)
        loss, row, dX = c.run()
        X = c.X.clone()
        got = c.run(X=X, dX=X)
        assert torch.equal(got[2].view(torch.int16), dX.view(torch.int16)) and torch.equal(got[0], loss) and torch.equal(got[1], row)


def test_outputs_one_by_one():
    c = Case(19, [30, 5], 64, 500)
    loss, row, dX = c.run()
    batch = c.batch()
    ws = torch.empty(sb.symb_loss_workspace_bytes(batch), device="cuda", dtype=torch.uint8)
    for k in range(3):
        out = [torch.full_like(t, NAN) if i == k else None for i, t in enumerate((loss, row, dX))]
        sb.symb_cross_entropy(gh.handle(), batch, c.X, c.W, *c.taught(), *out, ws, stream())
        if k == 2:
            assert torch.equal(out[k], dX)
        else:                                              # (losses alone: sums in the same order)
            close(out[k], host((loss, row)[k]), 2.0 ** -20 * host((loss, row)[k]), "one output")


def test_batches_without_rows():
    ws = torch.empty(256, device="cuda", dtype=torch.uint8)
    empty = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16)
    W, loss = torch.zeros(9, 64, device="cuda", dtype=torch.bfloat16), torch.full((2,), NAN, device="cuda")
    none = torch.empty(0, device="cuda", dtype=torch.int32)
    sb.symb_cross_entropy(gh.handle(), sb.LossBatch(64, 9, [0, 0, 0], [sb.Loss(), sb.Loss()]), empty, W, none, loss, None, empty, ws, stream())
    assert not loss.any()
    sb.symb_cross_entropy(gh.handle(), sb.LossBatch(64, 9, [0], []), empty, W, none, None, None, empty, ws, stream())
