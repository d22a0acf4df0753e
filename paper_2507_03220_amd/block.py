"""What a client runs around the shared projections, for many clients at once: a norm with a shared projection behind it (forward and backward, as a fine-tuning step needs them), and the
attention half of a transformer block over paged 8-bit caches (prompts and decode steps in one flattened batch).  Marshalling only: buffers are torch tensors, all arithmetic happens inside
libsymb.so.

    python -m paper_2507_03220_amd.block        # four clients: prompts, decode steps, one fine-tuning step; prints the time of each
"""
from __future__ import annotations

import contextlib
from dataclasses import dataclass, field
from typing import Dict, List, Optional, Sequence

import torch

from . import binding as sb

BF16 = torch.bfloat16


def _offsets(lens: Sequence[int]) -> List[int]:
    off = [0]
    for n in lens:
        off.append(off[-1] + int(n))
    return off


def _workspace(n: int) -> torch.Tensor:
    return torch.empty(max(n, 256), device="cuda", dtype=torch.uint8)


def _stream(stream: int):
    return torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()


def _on(stream: int):
    """Torch's own work (what it allocates, what it copies) in the order of `stream`."""
    return contextlib.nullcontext() if stream == torch.cuda.current_stream().cuda_stream else torch.cuda.stream(_stream(stream))


def _also_on(t: torch.Tensor, stream: int) -> None:
    """The memory of a tensor that was allocated in another stream's order is given on only when what `stream` has been given so far is done as well."""
    t.record_stream(_stream(stream))


def rotation_table(positions: int, dim: int, base: float = 10000.0) -> torch.Tensor:
    """Cosines and sines of position / base^(2j / dim), formed in 64 bits: [positions][dim] fp32 on the GPU."""
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * base ** (-torch.arange(dim // 2, dtype=torch.float64) * 2 / dim)
    return torch.cat([angle.cos(), angle.sin()], 1).float().cuda()


class NormedProjection:
    """x -> adapter_i(W norm_i(x)) for the rows of every client i, and its backward pass.  `norms` and `adapters` hold each client's own parameters and where its gradients go.
    Its buffers are allocated in the order of the stream that uses them, and again when another one does: results are there in that stream's order, and stay until the next call of the same pass."""

    def __init__(self, handle, W: torch.Tensor, lens: Sequence[int], norms: Sequence[sb.Norm], adapters: Sequence[sb.Adapter], kind: int = sb.SYMB_NORM_LAYER,
                 eps: float = 1e-5, weight_base: float = 0.0):
        self.h, self.W = handle, W
        d_out, d_in = W.shape
        off = _offsets(lens)
        self.norm, self.linear = sb.NormBatch(d_in, off, norms, kind, eps, weight_base), sb.Batch(d_in, d_out, off, adapters)
        self.T, self.d_in, self.d_out = off[-1], d_in, d_out
        self.N = self.Y = self.dN = self.dX = self.ws = None
        self._streams: Dict[str, int] = {}                             # of each buffer
        self.ws_bytes = max([sb.symb_norm_workspace_bytes(self.norm)] +
                            [sb.symb_workspace_bytes(self.linear, op) for op in (sb.SYMB_OP_FWD, sb.SYMB_OP_BWD_INPUT, sb.SYMB_OP_ADAPTER_GRAD)])

    def _buffers(self, stream: int, **widths) -> None:
        with _on(stream):
            for name, d in widths.items():
                if self._streams.get(name) != stream:
                    setattr(self, name, torch.empty(self.T, d, device="cuda", dtype=BF16))
                    self._streams[name] = stream
            if self._streams.get("ws") != stream:
                self.ws = _workspace(self.ws_bytes)
                self._streams["ws"] = stream

    def forward(self, X: torch.Tensor, bias=None, stream: int = 0) -> torch.Tensor:
        self._buffers(stream, N=self.d_in, Y=self.d_out)
        sb.symb_norm_fwd(self.h, self.norm, X, self.N, stream)
        sb.symb_base_linear_fwd(self.h, self.linear, self.N, self.W, bias, self.Y, None, self.ws, stream)
        return self.Y

    def backward(self, X: torch.Tensor, dY: torch.Tensor, flags: int = sb.SYMB_GRAD_OVERWRITE, stream: int = 0) -> torch.Tensor:
        """dX; the adapters' and norms' gradients go to their own tensors.  Needs the normed rows of the forward pass on the same rows, and their being there in the order of `stream`."""
        if self.N is None:
            raise RuntimeError("backward needs the normed rows of a forward pass")
        self._buffers(stream, dN=self.d_in, dX=self.d_in)
        if self._streams["N"] != stream:
            _also_on(self.N, stream)
        sb.symb_adapter_grad(self.h, self.linear, self.N, dY, None, flags, self.ws, stream)
        sb.symb_base_linear_bwd_input(self.h, self.linear, dY, self.W, self.dN, sb.SYMB_BWD_FULL, self.ws, stream)
        sb.symb_norm_bwd(self.h, self.norm, X, self.dN, self.dX, flags, self.ws, stream)
        return self.dX


@dataclass
class Client:
    """A client's parameters in one block, and its place in the cache."""
    norm: sb.Norm = field(default_factory=sb.Norm)
    adapters: Dict[str, sb.Adapter] = field(default_factory=dict)      # by projection: "q", "k", "v", "o"
    pages: List[int] = field(default_factory=list)
    past: int = 0                                                      # tokens in the cache


class AttentionBlock:
    """norm, query / key / value projections, cache append with rotation, attention, output projection: each for the whole batch, each client with its own norm, adapters and cache
    pages.  The residual is the caller's.  `scale`: what scores are multiplied with, head_dim ** -0.5 unless the model says otherwise; `biases`: bf16, by projection like W, those that it has."""

    def __init__(self, handle, W: Dict[str, torch.Tensor], heads: int, cache: sb.KvCache, rotation=None, kind: int = sb.SYMB_NORM_RMS, eps: float = 1e-6,
                 weight_base: float = 0.0, window: int = 0, cap: float = 0.0, scale: Optional[float] = None, biases: Optional[Dict[str, torch.Tensor]] = None):
        if set(biases or {}) - set(W):
            raise ValueError(f"biases of {sorted(biases)} for projections {sorted(W)}")
        for p, b in (biases or {}).items():
            if b.dtype is not BF16 or b.shape != W[p].shape[:1] or not b.is_contiguous():
                raise ValueError(f"bias of {p}: dense [{W[p].shape[0]}] of bfloat16 expected, got {tuple(b.shape)} of {b.dtype}")
        self.h, self.W, self.heads, self.cache, self.rotation = handle, W, heads, cache, rotation
        self.kind, self.eps, self.weight_base, self.window, self.cap = kind, eps, weight_base, window, cap
        self.scale, self.biases = cache.head_dim ** -0.5 if scale is None else scale, dict(biases or {})
        self.free = list(range(cache.num_pages - 1, -1, -1))           # pages that no client has

    def _reserve(self, c: Client, tokens: int) -> None:
        while len(c.pages) * self.cache.page_tokens < tokens:
            if not self.free:
                raise RuntimeError("the cache has no free page left")
            c.pages.append(self.free.pop())

    def release(self, c: Client) -> None:
        """Gives a client's pages back."""
        self.free += reversed(c.pages)
        c.pages, c.past = [], 0

    def forward(self, X: torch.Tensor, lens: Sequence[int], clients: Sequence[Client], stream: int = 0) -> torch.Tensor:
        """X [T][width]: lens[i] new tokens of clients[i], in order, no client twice.  Returns [T][width], there in the order of `stream`, and moves the clients' places on."""
        if len(lens) != len(clients) or len({id(c) for c in clients}) != len(clients):
            raise ValueError("one length for each client, and each client once")
        if X.shape[0] != sum(lens):
            raise ValueError(f"{X.shape[0]} rows for {sum(lens)} tokens")
        with _on(stream):
            return self._forward(X, lens, clients, stream)

    def _forward(self, X: torch.Tensor, lens: Sequence[int], clients: Sequence[Client], stream: int) -> torch.Tensor:
        T, width = X.shape
        if not T:
            return torch.empty_like(X)
        H, D, off = self.cache.kv_heads, self.cache.head_dim, _offsets(lens)
        for c, n in zip(clients, lens):
            self._reserve(c, c.past + n)
        table = torch.tensor([c.pages + [-1] * (max(len(k.pages) for k in clients) - len(c.pages)) for c in clients], dtype=torch.int32).cuda()
        kv = sb.KvBatch(off, [c.past for c in clients], table)
        rows = {"q": self.heads, "k": H, "v": H}
        batch = {p: sb.Batch(w.shape[1], w.shape[0], off, [c.adapters.get(p, sb.Adapter()) for c in clients]) for p, w in self.W.items()}
        ws = _workspace(max([sb.symb_workspace_bytes(b, sb.SYMB_OP_FWD) for b in batch.values()] + [sb.symb_kv_workspace_bytes(kv, self.cache, self.heads, self.window)]))
        N, out = torch.empty_like(X), torch.empty_like(X)
        heads = {p: torch.empty(T, n, D, device="cuda", dtype=BF16) for p, n in rows.items()}
        sb.symb_norm_fwd(self.h, sb.NormBatch(width, off, [c.norm for c in clients], self.kind, self.eps, self.weight_base), X, N, stream)
        for p in rows:
            sb.symb_base_linear_fwd(self.h, batch[p], N, self.W[p], self.biases.get(p), heads[p], None, ws, stream)
        q = heads["q"]
        sb.symb_kv_append(self.h, kv, self.cache, self.rotation, q, q, heads["k"], heads["v"], stream)
        attended = torch.empty_like(q)
        sb.symb_kv_attention(self.h, kv, self.cache, q, attended, self.scale, self.window, self.cap, ws, stream)
        sb.symb_base_linear_fwd(self.h, batch["o"], attended, self.W["o"], self.biases.get("o"), out, None, ws, stream)
        for c, n in zip(clients, lens):
            c.past += n
        return out


def main() -> None:
    """Four clients with LoRA adapters of their own on a Llama2-7B-shaped block: prompts, 32 decode steps, and a fine-tuning step through a normed projection."""
    import time
    g = torch.Generator(device="cuda").manual_seed(0)
    normal = lambda *s, std=1.0, mean=0.0: (torch.randn(*s, device="cuda", generator=g) * std + mean).to(BF16)  # noqa: E731
    h, width, heads, H, D, r = sb.symb_create(torch.cuda.current_device()), 4096, 32, 32, 128, 16
    W = {p: normal(o, i, std=i ** -0.5) for p, o, i in (("q", heads * D, width), ("k", H * D, width), ("v", H * D, width), ("o", width, heads * D))}

    def lora(p, grads=False):
        d_out, d_in = W[p].shape
        a = sb.Adapter(sb.SYMB_ADAPTER_LORA, r, 2.0, normal(r, d_in, std=d_in ** -0.5), normal(d_out, r, std=r ** -0.5))
        if grads:
            a.dA, a.dB = torch.empty(r, d_in, device="cuda"), torch.empty(d_out, r, device="cuda")
        return a
    lens = [700, 64, 311, 1]
    clients = [Client(sb.Norm(normal(width, std=0.1, mean=1.0)), {p: lora(p) for p in ("q", "v")}) for _ in lens]
    block = AttentionBlock(h, W, heads, sb.KvCache.empty(128, H, D, 64), sb.Rotation(rotation_table(4096, D)))

    def timed(what, f):
        torch.cuda.synchronize()
        t = time.perf_counter()
        f()
        torch.cuda.synchronize()
        print(f"{what}: {(time.perf_counter() - t) * 1e3:.3f} ms", flush=True)
    stream = torch.cuda.current_stream().cuda_stream
    timed("prompts of %s tokens" % lens, lambda: block.forward(normal(sum(lens), width), lens, clients, stream))
    timed("32 decode steps of 4 clients", lambda: [block.forward(normal(4, width), [1] * 4, clients, stream) for _ in range(32)])
    norms = [sb.Norm(c.norm.weight, None, torch.empty(width, device="cuda")) for c in clients]
    step = NormedProjection(h, W["q"], lens, norms, [lora("q", grads=True) for _ in lens], sb.SYMB_NORM_RMS, 1e-6)
    X, dY = normal(sum(lens), width), normal(sum(lens), heads * D)
    timed("fine-tuning step through norm and projection", lambda: (step.forward(X, None, stream), step.backward(X, dY, stream=stream)))
    sb.symb_destroy(h)


if __name__ == "__main__":
    main()
