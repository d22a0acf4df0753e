"""Pages that some rows of a prompt see and others do not, with contents that spoil what they meet: scales at the end of E8M0, page numbers outside the pool.  The rows that do not see them, in the
same tile, item or wavefront, have the formula's outputs (include/symb_block.h)."""
import numpy as np
import pytest
import torch

from block_harness import host
from block_paths import EDGES, Path, check

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
