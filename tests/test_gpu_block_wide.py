"""Attention of segments with 17 to 48 rows for a key head, many enough that these rows go through kernels of their own, and of prompts large enough for tiles, also for tiles that are
split and joined (include/symb_block.h)."""
import re
from pathlib import Path

import numpy as np
import pytest
import torch

from block_harness import Pages, attend, attention_bound, bf16, close, host, offsets
from oracle import block as ob
from paper_2507_03220_amd import binding as sb

pytestmark = pytest.mark.gpu
SOURCE = Path(sb.__file__).parent / "csrc" / "symb_block.hip"
ENOUGH, RUNS = map(int, re.search(r"kKvWideWork = (\d+), kKvFewRuns = (\d+);", SOURCE.read_text()).groups())


def _copies(lens, past, H, group, window):
    """How often the segments have to be in the batch for that: chunks of 64 tokens times 16 rows of all key heads, or for tiles their runs of 16 rows."""
    work = runs = 0
    for n, p in zip(lens, past):
        of16 = H * -(-n * group // 16)
        if 16 < n * group <= 48:
            begin = max(p + 1 - window, 0) // 64 * 64 if window else 0
            work += -(-(p + n - begin) // 64) * of16
        elif n * group > 48:
            runs += of16
    return max(-(-ENOUGH // work) if work else 1, RUNS // runs + 1 if runs else 1)


def _many(rng, H, D, P, lens, past, copies, std=60.0):
    """Segments `copies` times over, all reading the first ones' pages; K and V of the first ones."""
    pg = Pages(rng, lens, past, H, D, P)
    K, V = pg.fill(rng, std=std)
    return pg, K, V, lambda table: sb.KvBatch(offsets(lens * copies), past * copies, table.repeat(copies, 1))


def _check(pg, K, V, q, copies, want_of, window=0, cap=0.0):
    """The same queries in every copy: every copy's rows against the formula's for one of them."""
    D, T = pg.D, q.shape[0]
    want, mass, big = want_of(K, V, host(q), D ** -0.5, window, cap)
    fin = lambda x: np.where(np.isnan(x), 0.0, x)  # noqa: E731
    many = q.repeat(copies, 1, 1)
    got = attend(pg, many, D ** -0.5, window, cap)
    tile = lambda x: np.broadcast_to(x, (copies, *x.shape))  # noqa: E731
    close(host(got).reshape(copies, *want.shape), tile(want), tile(attention_bound(fin(want), fin(mass), fin(big))), (T, copies, window, cap))
    assert torch.equal(got.view(torch.int16), attend(pg, many, D ** -0.5, window, cap).view(torch.int16))


def _attention(seed, H, group, D, P, lens, past, window=0, cap=0.0, q_std=1.0):
    rng = np.random.default_rng(seed)
    copies = _copies(lens, past, H, group, window)
    pg, K, V, batch = _many(rng, H, D, P, lens, past, copies)
    pg.batch = batch(pg.table)
    _check(pg, K, V, bf16(rng, sum(lens), H * group, D, std=q_std), copies, lambda *a: ob.attention(offsets(lens), past, *a), window, cap)
    return pg


@pytest.mark.parametrize("D,P", [(64, 32), (64, 128), (128, 32), (128, 64)])
@pytest.mark.parametrize("H,group,lens,past", [
    (16, 1, [17, 48, 1, 33], [700, 0, 90, 63]),            # 17 to 48 tokens of heads of their own, and one below
    (8, 4, [8, 5, 12, 30], [640, 31, 1000, 2]),            # rows of four query heads; one segment of tiles
    (5, 7, [3, 4, 0, 6], [1500, 0, 10, 257]),              # odd head counts, an empty segment
    (3, 32, [1, 1], [900, 2001]),                          # one token of 32 query heads
])
def test_wide_runs(D, P, H, group, lens, past):
    _attention(D + P + H, H, group, D, P, lens, past)


@pytest.mark.parametrize("D,P", [(64, 32), (128, 64)])
@pytest.mark.parametrize("window", [1, 40, 65, 300])
@pytest.mark.parametrize("cap", [0.0, 5.0])
def test_wide_runs_with_window_and_cap(D, P, window, cap):
    _attention(window + D, 32, 1, D, P, [20, 45, 1, 40], [700, 0, 3, 260], window, cap, q_std=2.0)


@pytest.mark.parametrize("D", [64, 128])
def test_wide_runs_in_parts(D):
    """One key head and long contexts: fewer runs than the chip has places, each split and joined."""
    pg = _attention(D, 1, 16, D, 64, [2, 3], [30000, 9000])
    assert sb.symb_kv_workspace_bytes(pg.batch, pg.cache, 16) > 0


@pytest.mark.parametrize("D,window", [(64, 0), (128, 0), (128, 100)])
def test_wide_runs_with_nan_in_hidden_and_in_seen_tokens(D, window):
    rng = np.random.default_rng(3)
    H, P, lens, past = 16, 32, [20, 40, 33], [500, 130, 0]
    copies = _copies(lens, past, H, 1, window)
    pg, K, V, batch = _many(rng, H, D, P, lens, past, copies)
    pg.batch = batch(pg.table)
    for i, (n, p) in enumerate(zip(lens, past)):           # one channel of some tokens' values, early, in the middle of the new ones, last; a key
        for t in {3, p + n // 2, p + n - 1}:
            at = int(pg.ids[i, t // P])
            pg.cache.v.view(torch.uint8)[at, 1, 5, t % P] = 0xff
            V[i][t, 1, 5] = np.nan
        at = int(pg.ids[i, p // P])
        pg.cache.k.view(torch.uint8)[at, 0, p % P, 7] = 0x7f
        K[i][p, 0, 7] = np.nan
    _check(pg, K, V, bf16(rng, sum(lens), H, D), copies, lambda *a: ob.attention(offsets(lens), past, *a), window)


def test_wide_runs_with_a_page_outside_the_pool():
    rng = np.random.default_rng(4)
    H, D, P, lens, past = 16, 128, 64, [20, 40, 20], [500, 130, 400]
    copies = _copies(lens, past, H, 1, 60)
    pg, K, V, batch = _many(rng, H, D, P, lens, past, copies)
    q = bf16(rng, sum(lens), H, D)
    table = pg.table.clone()
    table[0, 2], table[1, 0] = pg.N, -1

    def unknown(*a):
        want, mass, big = ob.attention(offsets(lens), past, *a)
        want[:60] = np.nan
        return want, mass, big

    pg.batch = batch(table)
    _check(pg, K, V, q, copies, unknown)
    table = pg.table.clone()
    table[0, :6], table[2, :5] = -1, 1 << 30               # behind the window nothing is looked up
    pg.batch = batch(table)
    _check(pg, K, V, q, copies, lambda *a: ob.attention(offsets(lens), past, *a), 60)


@pytest.mark.parametrize("D,P,window,cap", [(128, 32, 400, 0.0), (128, 128, 0, 0.0), (64, 64, 500, 5.0), (64, 32, 0, 0.0)])
def test_prompts_in_parts(D, P, window, cap):
    """Long prompts of few key heads: too few tiles for the chip, so each is split, and thousands of rows are joined.  In a window some rows see nothing of a part."""
    rng = np.random.default_rng(D + P)
    H, group, lens, past = 2, 8, [600, 1, 9], [205, 700, 64]
    pg = Pages(rng, lens, past, H, D, P)
    K, V = pg.fill(rng)
    assert sb.symb_kv_workspace_bytes(pg.batch, pg.cache, H * group, window) >= 8192 * H * (D + 2) * 4
    V[0][410, 1, 5] = np.nan                               # a NaN that later rows see
    pg.cache.v.view(torch.uint8)[int(pg.ids[0, 410 // P]), 1, 5, 410 % P] = 0xff
    _check(pg, K, V, bf16(rng, sum(lens), H * group, D), 1, lambda *a: ob.attention(offsets(lens), past, *a), window, cap)
    table = pg.table.clone()
    table[0, 420 // P] = pg.N                              # a page outside the pool: NaN in the rows of the tiles that come to it
    pg.batch = sb.KvBatch(offsets(lens), past, table)
    out = host(attend(pg, bf16(rng, sum(lens), H * group, D), D ** -0.5, window, cap))
    first = 420 // P * P - past[0]
    assert np.isnan(out[max(first, 0):min(first + (window or 600), 600)]).all() and not np.isnan(out[:150]).any() and not np.isnan(out[600:]).any()


# ---- tiles ---------------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("D,P", [(64, 32), (64, 64), (64, 128), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("H,group,lens,past", [
    (2, 3, [17, 1, 40, 43], [0, 200, 90, 64]),             # tiles of 51 to 129 rows, one token beside them
    (1, 8, [100, 3], [33, 1500]),
    (3, 1, [150, 129, 64, 128], [0, 1, 63, 700]),          # tiles that end with, before and behind their last row
    (4, 5, [77, 0, 11], [500, 3, 5]),
])
def test_tiles(D, P, H, group, lens, past):
    _attention(D + P + H, H, group, D, P, lens, past)


@pytest.mark.parametrize("D,P", [(64, 32), (128, 64)])
@pytest.mark.parametrize("window", [1, 5, 100, 129, 4096])
@pytest.mark.parametrize("cap", [0.0, 5.0])
def test_tiles_with_window_and_cap(D, P, window, cap):
    _attention(window + D, 2, 2, D, P, [70, 1, 130], [700, 3, 260], window, cap, q_std=2.0)


@pytest.mark.parametrize("D,window", [(64, 0), (128, 0), (128, 40), (64, 100)])
def test_tiles_with_nan_in_hidden_and_in_seen_tokens(D, window):
    rng = np.random.default_rng(5)
    H, P, group, lens, past = 2, 32, 2, [150, 3, 60], [10, 300, 130]
    copies = _copies(lens, past, H, group, window)
    pg, K, V, batch = _many(rng, H, D, P, lens, past, copies)
    pg.batch = batch(pg.table)
    for i, (n, p) in enumerate(zip(lens, past)):           # one channel of some tokens' values, early, in the middle of the new ones, last; a key
        for t in {3, p + n // 2, p + n - 1}:
            at = int(pg.ids[i, t // P])
            pg.cache.v.view(torch.uint8)[at, 1, 5, t % P] = 0xff
            V[i][t, 1, 5] = np.nan
        at = int(pg.ids[i, p // P])
        pg.cache.k.view(torch.uint8)[at, 0, p % P, 7] = 0x7f
        K[i][p, 0, 7] = np.nan
    _check(pg, K, V, bf16(rng, sum(lens), H * group, D), copies, lambda *a: ob.attention(offsets(lens), past, *a), window)


def test_tiles_of_one_large_score_and_of_queries_that_are_zero_infinite_nan_or_tiny():
    rng = np.random.default_rng(6)
    H, D, P, lens, past = 1, 128, 64, [160, 60], [400, 0]
    copies = _copies(lens, past, H, 2, 0)
    pg, K, V, batch = _many(rng, H, D, P, lens, past, copies)
    pg.batch = batch(pg.table)
    q = bf16(rng, sum(lens), 2, D)
    q[0] = 0.0
    q[1, 0, 3], q[2, 1, 9] = float("nan"), float("inf")
    q[3] = q[3] * 1e-30
    q[4, 0, 1:] = q[4, 0, 1:] * 2.0 ** -18
    q[5:20] = q[5:20] * 8                                  # scores that differ by dozens: the maximum moves, weights vanish

    def formula(K, V, h, *a):
        h[2, 1] = np.nan                                   # inf x finite, both signs
        return ob.attention(offsets(lens), past, K, V, h, *a)

    _check(pg, K, V, q, copies, formula)
