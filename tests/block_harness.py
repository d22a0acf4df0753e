"""Inputs, pages and bounds for the tests of include/symb_block.h."""
import numpy as np
import torch

import gpu_harness as gh
from oracle import block as ob
from paper_2507_03220_amd import binding as sb

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
stream = gh.stream_ptr


def host(t):
    return t.detach().to(torch.float32).cpu().numpy().astype(np.float64)


def bf16(rng, *shape, std=1.0, mean=0.0):
    return torch.from_numpy((rng.standard_normal(shape) * std + mean).astype(np.float32)).to(torch.bfloat16).cuda()


def offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(int)


def close(got, want, tol, what):
    """|got - want| <= tol elementwise, NaN where and only where `want` has it."""
    got = host(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, what
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want), err_msg=what)
    d = np.where(np.isnan(want), 0.0, np.abs(got - want))
    bad = d > np.broadcast_to(tol, d.shape)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.nanmax(d / np.maximum(tol, 1e-300)):.2f} times the bound at {np.argwhere(bad)[0]}"


class Pages:
    """A cache whose every byte is something (NaN among it, where nothing was stored), the page table of a batch, and what its tokens stand for."""

    def __init__(self, rng, lens, past, H, D, P, spare=3, last_pages=0, fill="nan"):
        self.lens, self.past, self.H, self.D, self.P = list(lens), list(past), H, D, P
        pages = [-(-(n + p) // P) if n else 0 for n, p in zip(lens, past)]
        self.N = max(sum(pages) + spare, last_pages)
        ids = self.N - 1 - rng.permutation(sum(pages) + spare)
        self.stride = max(pages + [1]) + 1
        table = np.full((len(lens), self.stride), -1, np.int32)
        at = 0
        for i, n in enumerate(pages):
            table[i, :n] = ids[at:at + n]
            at += n
        self.table = torch.from_numpy(table).cuda()
        self.ids = table
        self.cache = sb.KvCache.empty(self.N, H, D, P)
        if fill == "nan":                                  # what nobody stored: every byte value, NaN too
            for t in (self.cache.k, self.cache.v):
                u = t.view(torch.uint8)
                u[-4096:].copy_(torch.from_numpy(rng.integers(0, 256, u[-4096:].shape).astype(np.uint8)))
            for t in (self.cache.k_scale, self.cache.v_scale):
                t.view(torch.uint8).fill_(255)
        self.batch = sb.KvBatch(offsets(lens), past, self.table)

    def put(self, i, k, v, ks, vs):
        """Tokens 0.. of segment i as codes [tokens][H][D] (values of e4m3) with scales 2^ks, 2^vs [pages][H] (exponents)."""
        n, P = k.shape[0], self.P
        for page in range(-(-n // P)):
            at, m = int(self.ids[i, page]), min(P, n - page * P)
            part = slice(page * P, page * P + m)
            self.cache.k[at, :, :m] = torch.from_numpy(np.ascontiguousarray(k[part].transpose(1, 0, 2))).float().cuda().to(E4M3)
            self.cache.v[at, :, :, :m] = torch.from_numpy(np.ascontiguousarray(v[part].transpose(1, 2, 0))).float().cuda().to(E4M3)
            self.cache.k_scale.view(torch.uint8)[at] = torch.from_numpy((ks[page] + 127).astype(np.uint8)).cuda()
            self.cache.v_scale.view(torch.uint8)[at] = torch.from_numpy((vs[page] + 127).astype(np.uint8)).cuda()

    def fill(self, rng, spread=2, std=60.0, tokens=None):
        """Random tokens for every segment; returns their real values, [tokens][H][D] per segment."""
        K, V = [], []
        for i, (n, p) in enumerate(zip(self.lens, self.past)):
            m = (n + p if tokens is None else tokens[i]) if n else 0
            k, v = (ob.e4m3(np.clip(rng.standard_normal((m, self.H, self.D)) * std, -448, 448)) for _ in range(2))
            np_ = max(-(-m // self.P), 1)
            ks, vs = (rng.integers(-6 - spread, -5 + spread, (np_, self.H)) for _ in range(2))
            self.put(i, k, v, ks, vs)
            page = np.arange(m) // self.P
            K.append(k * 2.0 ** ks[page][:, :, None] if m else k)
            V.append(v * 2.0 ** vs[page][:, :, None] if m else v)
        return K, V

    def read(self, i, tokens):
        """What the cache says that segment i's first tokens are: (K, V), and their pages' scales."""
        ids = self.ids[i, :-(-tokens // self.P)].astype(np.int64)
        at = torch.from_numpy(ids).cuda()
        codes = lambda t: host(t.view(torch.uint8)[at].view(E4M3))  # noqa: E731
        scale = lambda t: 2.0 ** (t.view(torch.uint8)[at].cpu().numpy().astype(float) - 127)  # noqa: E731
        k, v, ks, vs = codes(self.cache.k), codes(self.cache.v), scale(self.cache.k_scale), scale(self.cache.v_scale)
        out = [np.empty((tokens, self.H, self.D)) for _ in range(2)] + [np.empty((tokens, self.H)) for _ in range(2)]
        for t in range(tokens):
            page, slot = t // self.P, t % self.P
            out[0][t], out[1][t] = k[page, :, slot] * ks[page][:, None], v[page, :, :, slot] * vs[page][:, None]
            out[2][t], out[3][t] = ks[page], vs[page]
        return out


def attend(pg, q, scale, window=0, cap=0.0, out=None, ws_fill=None):
    heads = q.shape[1]
    out = torch.full((q.shape[0], heads, pg.D), float("nan"), device="cuda", dtype=torch.bfloat16) if out is None else out
    n = sb.symb_kv_workspace_bytes(pg.batch, pg.cache, heads, window)
    ws = torch.full((n,), 255, device="cuda", dtype=torch.uint8) if n else None             # (all NaN as floats)
    sb.symb_kv_attention(gh.handle(), pg.batch, pg.cache, q, out, scale, window, cap, ws, stream())
    torch.cuda.synchronize()
    return out


def attention_bound(want, mass, big):
    """What the kernel's roundings allow.  Output: half a bf16 step, 2^-8 |out| with room.  Weights: bf16, 2^-9 of each, their sum as much with room; a
    score's products lose up to 2^-14 of the largest of them each (128 terms in two instructions), 2^-7 of the largest in all, e^d - 1 < 1.1 d of a weight."""
    score = 1.1 * 2.0 ** -7 * big + 1e-5
    return 1.02 * 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2 * score) * mass + 1e-30
