"""Batches that reach each of the attention kernels of include/symb_block.h, and the check of a whole tensor against the formula."""
import numpy as np
import torch

from block_harness import Pages, attend, attention_bound, bf16, close, host, offsets
from oracle import block as ob
from paper_2507_03220_amd import binding as sb
from test_gpu_block_wide import _copies

# rows of one key head: up to 16; 17 to 32 and 33 to 48 of enough segments; prompts that go 16 rows at a time; prompts in tiles of 128
PATHS = {
    "rows": dict(H=2, group=2, lens=[1, 5, 1], past=[700, 126, 0], many=False),
    "runs": dict(H=2, group=2, lens=[60, 1, 40], past=[300, 130, 0], many=False),
    "rows32": dict(H=16, group=1, lens=[17, 30, 1], past=[500, 33, 90], many=True),
    "rows48": dict(H=16, group=1, lens=[40, 48], past=[300, 0], many=True),
    "tiles": dict(H=2, group=3, lens=[100, 43], past=[260, 64], many=True),
}

# of one segment of each: (segment, first token of a page that only its later rows see; window, end of a page that only its earlier rows see)
EDGES = {"rows": (1, 128, 64, 64), "runs": (0, 320, 60, 256), "rows32": (0, 512, 60, 448), "rows48": (0, 320, 60, 256), "tiles": (0, 320, 60, 256)}


class Path:
    """One of them, filled: the segments so often that their rows go to that kernel, every copy on the same pages.  `run` gives the outputs of all copies, [copies][T][heads][D]."""

    def __init__(self, name, D, P, seed, window=0, std=60.0):
        c = PATHS[name]
        self.rng = np.random.default_rng(seed)
        self.H, self.group, self.lens, self.past, self.D, self.P, self.window = c["H"], c["group"], c["lens"], c["past"], D, P, window
        self.copies = _copies(self.lens, self.past, self.H, self.group, window) if c["many"] else 1
        self.pg = Pages(self.rng, self.lens, self.past, self.H, D, P)
        self.K, self.V = self.pg.fill(self.rng, std=std)
        self.table = self.pg.table.clone()
        self.T, self.heads, self.off = sum(self.lens), self.H * self.group, offsets(self.lens)

    @classmethod
    def with_edge(cls, name, D, P, seed, windowed):
        """... with `page`, a page (of 32 or 64 tokens) of one segment that some of its rows see and others do not, its first token `first`, and `sees`, which of the batch's rows do."""
        seg, first, window, end = EDGES[name]
        self = cls(name, D, P, seed, window if windowed else 0)
        self.seg, self.first = seg, end - P if windowed else first
        self.page = int(self.pg.ids[seg, self.first // P])
        pos = self.past[seg] + np.arange(self.lens[seg])
        self.sees = np.zeros(self.T, bool)
        self.sees[self.off[seg]:self.off[seg + 1]] = (pos >= self.first) & (not windowed or pos - window < self.first + P - 1)
        assert 0 < self.sees.sum() < self.lens[seg]
        return self

    def queries(self, std=1.0):
        return bf16(self.rng, self.T, self.heads, self.D, std=std)

    def run(self, q, cap=0.0, scale=None):
        self.pg.batch = sb.KvBatch(offsets(self.lens * self.copies), self.past * self.copies, self.table.repeat(self.copies, 1))
        out = attend(self.pg, q.repeat(self.copies, 1, 1), self.D ** -0.5 if scale is None else scale, self.window, cap)
        return out.view(self.copies, self.T, self.heads, self.D)

    def formula(self, q, cap=0.0, scale=None):
        return ob.attention(self.off, self.past, self.K, self.V, host(q), self.D ** -0.5 if scale is None else scale, self.window, cap)


def check(got, formula, what, rows=None):
    """Every copy against the formula, elementwise (block_harness.attention_bound) and as a whole: the output's rounding to bf16 is 1.7e-3 of a tensor, that of the weights as much again at most,
    so 5e-3 of it in the 2-norm.  rows: those that are compared (all)."""
    want, mass, big = formula
    rows = slice(None) if rows is None else rows
    want, mass, big, got = want[rows], mass[rows], big[rows], host(got)[:, rows]
    tile = lambda x: np.broadcast_to(x, (got.shape[0], *x.shape))  # noqa: E731
    fin = lambda x: np.where(np.isnan(x), 0.0, x)  # noqa: E731
    close(got, tile(want), tile(attention_bound(fin(want), fin(mass), fin(big))), what)
    for copy in got:
        rel = np.linalg.norm(fin(copy - want)) / np.linalg.norm(fin(want))
        assert rel < 5e-3, (what, rel)
