"""Inputs, calls and bounds for the tests of include/symb_loss.h."""
import numpy as np
import torch

import gpu_harness as gh
from block_harness import bf16, close, host, offsets, stream
from oracle import loss as ol
from paper_2507_03220_amd import binding as sb

NAN = float("nan")


class Case:
    """A batch of losses.  std: of the scores; sure: how much of its token's vector a row has in it, up to that; prompt: share of a segment's first rows that take no part (they hold NaN);
    entries 0: labels."""

    def __init__(self, seed, lens, width, vocab, entries=0, std=2.0, sure=1.5, prompt=0.0, mean=True, cap=0.0, temperatures=None, ragged=False):
        rng = np.random.default_rng(seed)
        self.lens, self.off, self.T, self.width, self.vocab, self.K = lens, offsets(lens), sum(lens), width, vocab, entries
        self.mean, self.cap, self.S = mean, cap, len(lens)
        self.W = bf16(rng, vocab, width, std=std * width ** -0.5)
        token = rng.integers(0, vocab, self.T)
        x = rng.standard_normal((self.T, width)) + sure * rng.random((self.T, 1)) * host(self.W)[token] * (2.0 / std)
        self.out = np.zeros(self.T, bool)
        for i, n in enumerate(lens):
            self.out[self.off[i]:self.off[i] + int(n * prompt)] = True
        x[self.out] = NAN
        self.X = torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).cuda()
        self.scales = [0.5 + 0.25 * i for i in range(self.S)]
        self.temperatures = temperatures or [1.0 + 0.5 * (i % 3) for i in range(self.S)]
        if entries:
            self.ids = np.stack([rng.permutation(vocab)[:entries] if vocab >= entries else rng.integers(0, vocab, entries) for _ in range(self.T)]).astype(np.int32).reshape(self.T, entries)
            self.ids[:, 0] = token
            if ragged:
                self.ids[rng.random(self.ids.shape) < 0.3] = -7
            self.ids[self.out] = -1
            self.out |= (self.ids < 0).all(1)
            self.logits = (rng.standard_normal((self.T, entries)) * 3).astype(np.float32)
            self.logits[self.ids < 0] = NAN                # (absent: not looked at)
        else:
            self.labels = np.where(self.out, -100, token).astype(np.int32)

    def batch(self):
        return sb.LossBatch(self.width, self.vocab, self.off, [sb.Loss(a, t) for a, t in zip(self.scales, self.temperatures)], sb.SYMB_LOSS_MEAN if self.mean else sb.SYMB_LOSS_SUM, self.cap)

    def want(self):
        x = np.nan_to_num(host(self.X), nan=0.0)
        if self.K:
            return ol.distillation(self.off, x, host(self.W), self.ids, self.logits, self.scales, self.temperatures, self.mean, self.cap)
        return ol.cross_entropy(self.off, x, host(self.W), self.labels, self.scales, self.mean, self.cap)

    def taught(self):
        """What the call is given beside X and W."""
        return (torch.from_numpy(self.ids).cuda(), torch.from_numpy(self.logits).cuda()) if self.K else (torch.from_numpy(self.labels).cuda(),)

    def run(self, gradient=True, X=None, dX=None, batch=None):
        """(loss, row_loss, dX): outputs and workspace start as NaN."""
        batch = batch or self.batch()
        loss, row = torch.full((self.S,), NAN, device="cuda"), torch.full((self.T,), NAN, device="cuda")
        X = self.X if X is None else X
        dX = (torch.full_like(X, NAN) if dX is None else dX) if gradient else None
        ws = torch.full((max(sb.symb_loss_workspace_bytes(batch, self.K, gradient), 16),), 255, device="cuda", dtype=torch.uint8)
        call = sb.symb_distillation if self.K else sb.symb_cross_entropy
        call(gh.handle(), batch, X, self.W, *self.taught(), loss, row, dX, ws, stream())
        torch.cuda.synchronize()
        return loss, row, dX

    def score_error(self):
        """How far the weights of a row may be off, relative: fp32 sums of `width` exact products (2^-24 of their magnitudes each, in any order), of a and of b; capping to 2^-21 and the exponent's own
        rounding, 2^-24 of what it is made of; an exponential's 2^-22."""
        x, w = np.abs(np.nan_to_num(host(self.X), nan=0.0)), np.abs(host(self.W))
        most = (x @ w.T).max(1)
        T = np.repeat(np.asarray(self.temperatures), self.lens) if self.K else np.ones(self.T)
        z = np.minimum(most, self.cap) if self.cap else most
        return (2 * self.width * 2.0 ** -24 * most + (2.0 ** -20 if self.cap else 2.0 ** -22) * z) / T + 2.0 ** -20

    def slope_error(self):
        """How far 1 - tanh^2(s / cap) may be off, relative: 2 / cap times what the score may be, 2^-21 of |s / cap| (that quotient's and the exponential's roundings), 2^-18 for a polynomial of 2^-22 in it."""
        if not self.cap:
            return np.zeros(self.T)
        x, w = np.abs(np.nan_to_num(host(self.X), nan=0.0)), np.abs(host(self.W))
        most = (x @ w.T).max(1)
        return np.expm1(np.minimum(2 * self.width * 2.0 ** -24 * most / self.cap, 50)) + 2.0 ** -18 + 2.0 ** -21 * np.minimum(most / self.cap, 100)

    def check(self, what):
        loss, row, dX = self.run()
        want_loss, want_row, want, mass, both = self.want()
        e = self.score_error()
        if self.K:
            T = np.repeat(np.asarray(self.temperatures), self.lens)
            # sum q (log q - log p): every log p off by e, sums of terms that are rounded to 2^-21 of the largest
            bound = T * T * (1.1 * e + 2.0 ** -20 * (1 + np.abs(self.want_log())))
        else:
            # log(1 + S), S off by e of it; weights below 2^-126 are no numbers of the format and may be zeros, each of the vocabulary's
            bound = 1.1 * e * np.minimum(want_row, 1.0) + 2.0 ** -20 * want_row + self.vocab * 2.0 ** -126
        bound = np.where(self.out, 0.0, bound)
        close(row, want_row, bound, what + ": rows")
        n = np.array([max((~self.out[a:b]).sum(), 1) if self.mean else 1 for a, b in zip(self.off[:-1], self.off[1:])])
        total = np.array([bound[a:b].sum() + 2.0 ** -20 * np.abs(want_row[a:b]).sum() for a, b in zip(self.off[:-1], self.off[1:])])
        close(loss, want_loss, total / n + 1e-30, what + ": segments")
        # half a step of the output, half a step of each weight (of its second term, up to 64 rows), the weights' own errors (p's and, in l, once more; the slope's), sums over the vocabulary in fp32
        held = 2.0 ** -16 if self.T <= 64 else 2.0 ** -8
        tol = 1.02 * 2.0 ** -8 * np.abs(want) + (1.02 * held + self.vocab * 2.0 ** -24) * mass + (2.2 * e + self.slope_error())[:, None] * both + 1e-30
        close(dX, want, tol, what + ": gradient")
        again = self.run()
        assert all(torch.equal(a, b) for a, b in zip((loss, row, dX), again)), what
        alone = self.run(gradient=False)
        close(alone[1], want_row, bound, what + ": rows, losses alone")
        close(alone[0], want_loss, total / n + 1e-30, what + ": segments, losses alone")
        return loss, row, dX

    def want_log(self):
        """The largest log p of a row's entries, in magnitude."""
        x = np.nan_to_num(host(self.X), nan=0.0)
        s = x @ host(self.W).T
        z = (self.cap * np.tanh(s / self.cap) if self.cap else s) / np.repeat(np.asarray(self.temperatures), self.lens)[:, None]
        return np.abs(z).max(1) * 2 + np.log(self.vocab)
