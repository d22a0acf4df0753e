"""paper_2507_03220_amd/block.py as a model uses it: on streams of its own, with the score scale and the biases that the model has."""
import numpy as np
import pytest
import torch

import gpu_harness as gh
from block_harness import bf16, host, stream
from oracle import block as ob
from paper_2507_03220_amd import binding as sb
from paper_2507_03220_amd import block as blk

pytestmark = pytest.mark.gpu


def _lora(rng, d_in, d_out, r, grads=False):
    a = sb.Adapter(sb.SYMB_ADAPTER_LORA, r, 1.5, bf16(rng, r, d_in, std=d_in ** -0.5), bf16(rng, d_out, r, std=r ** -0.5))
    if grads:
        a.dA, a.dB = torch.empty(r, d_in, device="cuda"), torch.empty(d_out, r, device="cuda")
    return a


def test_a_normed_projection_on_streams_of_its_own():
    """The same bits on torch's current stream, on another, and forward on one with backward on a third; torch's own work between the passes takes what memory it is given."""
    rng = np.random.default_rng(1)
    width, d_out, lens = 256, 384, [70, 3, 0, 129]
    W, X, dY = bf16(rng, d_out, width, std=width ** -0.5), bf16(rng, 202, width, mean=0.3), bf16(rng, 202, d_out)
    weights, ads = [bf16(rng, width, std=0.1, mean=1.0) for _ in lens], [_lora(rng, width, d_out, r, True) for r in (8, 16, 4, 5)]
    grads = [torch.empty(width, device="cuda") for _ in lens]

    def step(first, second):
        run = blk.NormedProjection(gh.handle(), W, lens, [sb.Norm(w, None, g) for w, g in zip(weights, grads)], ads, sb.SYMB_NORM_RMS, 1e-6)
        for g in grads + [t for a in ads for t in (a.dA, a.dB)]:
            g.fill_(float("nan"))
        torch.cuda.synchronize()
        out = []
        for _ in range(3):
            y = run.forward(X, None, first)
            torch.full((202, d_out), float("nan"), device="cuda", dtype=torch.bfloat16)
            if first != second:
                torch.cuda.synchronize()
            d = run.backward(X, dY, stream=second)
            torch.full((202, width), float("nan"), device="cuda", dtype=torch.bfloat16)
            torch.cuda.synchronize()
            out += [y.clone(), d.clone()]
        return out + [t.clone() for a in ads for t in (a.dA, a.dB)] + [g.clone() for g in grads]
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    want = step(stream(), stream())
    assert all(torch.isfinite(t).all() for t in want)
    for first, second in ((a.cuda_stream, a.cuda_stream), (a.cuda_stream, b.cuda_stream), (stream(), a.cuda_stream)):
        for x, y in zip(want, step(first, second)):
            assert torch.equal(x, y)


@pytest.mark.parametrize("scale,biased", [(None, "qkvo"), (3 * 64 ** -0.5, ""), (144 ** -0.5, "qkvo"), (None, "v")])
def test_an_attention_block_with_the_models_scale_and_biases(scale, biased):
    """Prompts and decode steps against 64 bits from the cache that the block wrote, as in test_gpu_block_path.py."""
    rng = np.random.default_rng(2)
    width, heads, H, D, P = 256, 4, 2, 64, 32
    W = {p: bf16(rng, o, i, std=i ** -0.5) for p, o, i in (("q", heads * D, width), ("k", H * D, width), ("v", H * D, width), ("o", width, heads * D))}
    biases = {p: bf16(rng, W[p].shape[0], std=0.7) for p in biased}
    cache, table = sb.KvCache.empty(40, H, D, P), blk.rotation_table(400, D)
    block = blk.AttentionBlock(gh.handle(), W, heads, cache, sb.Rotation(table), scale=scale, biases=biases)
    clients = [blk.Client(sb.Norm(bf16(rng, width, std=0.1, mean=1.0)), {"q": _lora(rng, width, heads * D, 8)}) for _ in range(2)]
    scale = D ** -0.5 if scale is None else scale

    def lin(x, p, c):
        y, a = x @ host(W[p]).T, c.adapters.get(p)
        y = y if a is None else y + a.scale * (x @ host(a.A).T) @ host(a.B).T
        return y + host(biases[p]) if p in biases else y
    for lens in ([70, 33], [1, 1], [40, 1]):
        X = bf16(rng, sum(lens), width)
        out, at = host(block.forward(X, lens, clients, stream())), 0
        for c, n in zip(clients, lens):
            x, pos = host(X[at:at + n]), np.arange(c.past - n, c.past)
            y = ob.norm_fwd([0, n], x, [host(c.norm.weight)], [None], False, 1e-6, 0.0)
            q = ob.turn(lin(y, "q", c).reshape(n, heads, D), host(table), pos, D, False)
            pages = torch.tensor(c.pages[:-(-c.past // P)]).cuda()
            stored = lambda t, s: host(t.view(torch.uint8)[pages].view(torch.float8_e4m3fn)) * 2.0 ** (s.view(torch.uint8)[pages].cpu().numpy()[:, :, None, None].astype(float) - 127)  # noqa: E731
            K = stored(cache.k, cache.k_scale).transpose(0, 2, 1, 3).reshape(-1, H, D)[:c.past]
            V = stored(cache.v, cache.v_scale).transpose(0, 3, 1, 2).reshape(-1, H, D)[:c.past]
            for what, now in (("k", ob.turn(lin(y, "k", c).reshape(n, H, D), host(table), pos, D, False)), ("v", lin(y, "v", c).reshape(n, H, D))):
                # E4M3: 2^-4 of an element at most, of a tensor a fortieth
                assert np.linalg.norm((K if what == "k" else V)[-n:] - now) / np.linalg.norm(now) < 0.04, what
            att, _, _ = ob.attention([0, n], [c.past - n], [K], [V], q, scale, 0, 0.0)
            want = lin(att.reshape(n, -1), "o", c)
            # normed rows, queries and outputs are rounded to bf16 (2^-9 of a tensor), weights too; scores of size 3 or so move by 2^-7
            assert np.linalg.norm(out[at:at + n] - want) / np.linalg.norm(want) < 1.5e-2
            at += n


@pytest.mark.parametrize("name,length,dtype", [("gate", 64, torch.bfloat16), ("q", 32, torch.bfloat16), ("v", 64, torch.float32)])
def test_biases_that_do_not_fit_are_refused(name, length, dtype):
    W = {p: torch.zeros(64, 64, device="cuda", dtype=torch.bfloat16) for p in "qkvo"}
    with pytest.raises(ValueError):
        blk.AttentionBlock(gh.handle(), W, 1, sb.KvCache.empty(2, 1, 64, 32), biases={name: torch.zeros(length, device="cuda", dtype=dtype)})
