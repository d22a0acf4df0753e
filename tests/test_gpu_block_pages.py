"""Pages that some rows of a prompt see and others do not, with contents that spoil what they meet: scales at the end of E8M0, page numbers outside the pool.  The rows that do not see them, in the
same tile, item or wavefront, have the formula's outputs (include/symb_block.h)."""
import numpy as np
import pytest
import torch

from block_harness import Pages, attend, bf16, host, offsets
from block_paths import EDGES, Path, check
from oracle import block as ob
from paper_2507_03220_amd import binding as sb

pytestmark = pytest.mark.gpu
SIZES = pytest.mark.parametrize("D,P", [(64, 32), (128, 64), (128, 32), (64, 64)])


@SIZES
@pytest.mark.parametrize("windowed", [False, True])
@pytest.mark.parametrize("path", EDGES)
def test_value_scales_up_to_the_largest_byte(path, windowed, D, P):
    """Every code at scales from 2^119 up: from code (262 - byte) << 3 on a value is 2^128 or more, infinite or NaN to a row that sees it; a scale of 0xff is NaN for every code."""
    p = Path.with_edge(path, D, P, 50 + D, windowed)
    q = p.queries()
    want = p.formula(q)
    codes = p.rng.integers(0, 256, (p.H, D, P)).astype(np.uint8)
    codes[:, 0] = 0                                        # (zeros too: 0 x infinity)
    p.pg.cache.v.view(torch.uint8)[p.page] = torch.from_numpy(codes).cuda()
    at = 0 if not windowed else P - 1                      # the slot that every row that sees the page sees
    for byte in range(246, 256):
        p.pg.cache.v_scale.view(torch.uint8)[p.page] = byte
        got = p.run(q)
        check(got, want, (path, byte), ~p.sees)
        limit = 0 if byte == 255 else (262 - byte) << 3 if byte > 246 else 127
        spoilt = np.repeat((codes[:, :, at] & 127) >= limit, p.group, 0)            # [heads][D]
        assert not np.isfinite(host(got)[:, p.sees][:, :, spoilt]).any(), (path, byte)
        if byte == 255:
            assert np.isnan(host(got)[:, p.sees]).all()


@SIZES
@pytest.mark.parametrize("windowed", [False, True])
@pytest.mark.parametrize("path", EDGES)
def test_key_scales_at_the_end(path, windowed, D, P):
    p = Path.with_edge(path, D, P, 60 + D, windowed)
    q = p.queries()
    want = p.formula(q)
    p.pg.cache.k.view(torch.uint8)[p.page] = torch.from_numpy(p.rng.integers(0, 256, (p.H, P, D)).astype(np.uint8)).cuda()
    for byte in (250, 254, 255):
        p.pg.cache.k_scale.view(torch.uint8)[p.page] = byte
        got = p.run(q)
        check(got, want, (path, byte), ~p.sees)
    assert np.isnan(host(got)[:, p.sees]).all()


@SIZES
@pytest.mark.parametrize("windowed", [False, True])
@pytest.mark.parametrize("path", EDGES)
def test_a_page_outside_the_pool_is_nan_to_the_rows_that_see_it_and_to_no_other(path, windowed, D, P):
    """Whatever page 0 holds, which is read in its place."""
    p = Path.with_edge(path, D, P, 70 + D, windowed)
    q = p.queries()
    want = p.formula(q)
    if not (p.pg.ids == 0).any():
        p.pg.cache.v.view(torch.uint8)[0] = 0x7f
        p.pg.cache.k_scale.view(torch.uint8)[0], p.pg.cache.v_scale.view(torch.uint8)[0] = 255, 254
    for number in (-1, p.pg.N, (1 << 31) - 1):
        p.table[p.seg, p.first // P] = number
        got = p.run(q)
        check(got, want, (path, number), ~p.sees)
        assert np.isnan(host(got)[:, p.sees]).all(), (path, number)


@pytest.mark.parametrize("D", [64, 128])
def test_a_page_outside_the_pool_in_one_of_many_parts(D):
    """Long contexts split over the tokens, and prompts whose tiles are: the parts are joined, by either kernel, with NaN in the rows that see the page."""
    rng = np.random.default_rng(80 + D)
    for H, group, lens, past, at in ((1, 4, [3, 1], [8958, 5000], 8960), (2, 8, [600, 1], [205, 700], 600)):
        pg = Pages(rng, lens, past, H, D, 64)
        K, V = pg.fill(rng)
        q = bf16(rng, sum(lens), H * group, D)
        assert sb.symb_kv_workspace_bytes(pg.batch, pg.cache, H * group) > 0
        table, at = pg.table.clone(), at // 64
        table[0, at] = pg.N
        pg.batch = sb.KvBatch(offsets(lens), past, table)
        sees = np.arange(sum(lens)) + past[0] >= at * 64
        sees[lens[0]:] = False
        assert 0 < sees.sum() < lens[0]
        got = attend(pg, q, D ** -0.5)
        check(got[None], ob.attention(offsets(lens), past, K, V, host(q), D ** -0.5, 0, 0.0), (H, group), ~sees)
        assert np.isnan(host(got)[sees]).all()
