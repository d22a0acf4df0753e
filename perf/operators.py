"""What is timed of the operators around the shared projections: what a client of the base executor runs between two of them, for the whole flattened batch.

  norm_fwd    LayerNorm / RMSNorm of every row with its own client's weight (and bias)
  norm_bwd    its input gradient, and every client's weight and bias gradient in fp32
  append      new keys and values, keys and queries turned by their positions, into a paged cache of 8-bit values (E4M3) with one
              power-of-two scale (E8M0) for each page and head
  attention   causal attention of the new rows over that cache: single tokens, prompts, long contexts, grouped heads

A case is one call on one batch of clients: `decode` clients with one new token each come first, `clients` longer ones follow and share `tokens`.
Widths, heads, client counts and lengths are those of `synth` (Llama2-7B-, Granite-20B-, Gemma2-27B-shaped layers, the mixed batch, the tiny
configuration), plus ragged ones.
"""
import functools
import math
import random

import torch

own = False

BF16 = torch.bfloat16
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


# ---- cases ------------------------------------------------------------------------------------------------------------------------
def _norm(op, width, decode=0, clients=0, tokens=0, equal=False, rms=False, bias=False, shared=False, mix=1):
    """rms: no mean taken off, weights stored less one; shared: one weight for all clients (each still gets its own gradient)."""
    return dict(op=op, width=width, decode=decode, clients=clients, tokens=tokens, equal=equal, rms=rms, bias=bias, shared=shared, mix=mix)


def _kv(op, heads, kv_heads, dim, page, decode=0, clients=0, tokens=0, equal=False, past=0, prompt_past=0, turn="halves", turned=0, fused=False,
        window=0, cap=0.0, mix=1):
    """past: the longest context of the one-token clients (the shortest has an eighth); prompt_past: of the others, from none; turn: how the
    elements are paired ("halves", "adjacent", "none"), turned: how many of a head's elements (0 = all); fused: q, k, v are columns of one tensor."""
    return dict(op=op, heads=heads, kv_heads=kv_heads, dim=dim, page=page, decode=decode, clients=clients, tokens=tokens, equal=equal, past=past,
                prompt_past=prompt_past, turn=turn, turned=turned, fused=fused, window=window, cap=cap, mix=mix)


def listed():
    return [
        # the norm before one user's decode step: the smallest call there is
        dict(_norm("norm_fwd", 4096, decode=1, rms=True), name="norm_one"),
        # prompts of sixteen clients through a LayerNorm with bias that they share (Granite-20B's width)
        dict(_norm("norm_fwd", 6144, clients=16, tokens=16384, bias=True, shared=True, mix=2), name="norm_prompts"),
        # training step of the tiny configuration: 4 clients x 64 tokens
        dict(_norm("norm_bwd", 768, clients=4, tokens=256, equal=True, bias=True, mix=3), name="norm_grad_tiny"),
        # training step of twenty clients on Gemma2-27B's width, every client's norm its own, weights stored less one
        dict(_norm("norm_bwd", 4608, clients=20, tokens=20480, equal=True, rms=True, mix=4), name="norm_grad_twenty"),
        # one decode step of the mixed batch's 48 inference clients, as many key heads as query heads (Llama2-7B)
        dict(_kv("append", 32, 32, 128, 64, decode=48, past=4096, mix=5), name="append_decode"),
        # prompts of ragged length with decode steps riding along, two query heads to a key head (Gemma2-27B), q, k and v from one product
        dict(_kv("append", 32, 16, 128, 64, decode=8, clients=6, tokens=6001, past=2000, prompt_past=700, fused=True, mix=6), name="append_prompts"),
        # one user's decode step behind a short context: where latency counts
        dict(_kv("attention", 32, 32, 128, 64, decode=1, past=700, mix=7), name="attend_one"),
        # decode steps of 48 clients, contexts to 8192, sliding window and capped scores as Gemma2 has them
        dict(_kv("attention", 32, 16, 128, 64, decode=48, past=8192, window=4096, cap=50.0, mix=8), name="attend_decode"),
        # a few long contexts, all 48 query heads on one key head (Granite-20B)
        dict(_kv("attention", 48, 1, 128, 128, decode=16, past=131072, mix=9), name="attend_long"),
        # decode steps and ragged prompts in one batch, heads of 64 as the tiny configuration has them, small pages
        dict(_kv("attention", 12, 12, 64, 32, decode=24, clients=3, tokens=389, past=1500, prompt_past=300, mix=10), name="attend_mixed"),
        # prompts of eight clients, some behind a context that is there already, as many key heads as query heads
        dict(_kv("attention", 32, 32, 128, 64, clients=8, tokens=8192, prompt_past=1024, mix=11), name="attend_prompts"),
        # one long prompt, two query heads to a key head: the most work of all
        dict(_kv("attention", 32, 16, 128, 64, clients=1, tokens=8192, mix=12), name="attend_prefill"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _padded(c):
    """Scores that the padded plain form holds: what bounds a drawn case's cost."""
    segs = _segments(c)
    return len(segs) * c["heads"] * max(n for n, _ in segs) * max(n + p for n, p in segs)


def draw(rng):
    """Widths 256..8192, head layouts of the configurations and others, pages of 32 to 128 tokens, 1 to 64 clients, batches of 1 to 20480 rows."""
    while True:
        op = rng.choice(["norm_fwd", "norm_bwd", "append", "attention", "attention"])
        mix, equal = rng.randrange(1 << 20), rng.random() < 0.3
        decode = rng.choice([0, 1, rng.randint(2, 16), rng.randint(17, 48)]) if op != "norm_bwd" else 0
        clients = rng.randint(0 if decode else 1, 16)
        if op in ("norm_fwd", "norm_bwd"):
            width = rng.choice([768, 4096, 4608, 6144, 8 * _spread(rng, 32, 1024)])
            tokens = max(clients, _spread(rng, 16, 20480)) if clients else 0
            if (decode + tokens) * width <= 20480 * 4608:
                return _norm(op, width, decode, clients, tokens, equal, rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.3, mix)
            continue
        heads, kv_heads, dim = rng.choice([(32, 32, 128), (48, 1, 128), (32, 16, 128), (12, 12, 64), (24, 3, 64), (20, 5, 128), (7, 7, 64), (16, 2, 128)])
        page = rng.choice([32, 64, 128])
        past, prompt_past = _spread(rng, 1, 16384), rng.choice([0, _spread(rng, 1, 2048)])
        if op == "append":
            tokens = max(clients, _spread(rng, 16, 8192)) if clients else 0
            turn = rng.choice(["halves", "halves", "adjacent", "none"])
            return _kv(op, heads, kv_heads, dim, page, decode, clients, tokens, equal, past, prompt_past, turn, rng.choice([0, 0, dim // 2]),
                       rng.random() < 0.3, mix=mix)
        tokens = max(clients, _spread(rng, 16, 8192)) if clients else 0
        c = _kv(op, heads, kv_heads, dim, page, decode, clients, tokens, equal, past, prompt_past, window=rng.choice([0, 0, 0, _spread(rng, 16, 4096)]),
                cap=rng.choice([0.0, 0.0, 50.0]), mix=mix)
        if _padded(c) <= 32 * 8192 * 8192:
            return c


def _segments(c):
    """[(new tokens, tokens in the cache before them)] of the batch, from the case alone."""
    r = random.Random(c["mix"])
    lens = []
    if c["clients"]:
        if c["equal"]:
            base, more = divmod(c["tokens"], c["clients"])
            lens = [base + (i < more) for i in range(c["clients"])]
        else:                                     # uneven: exponential shares, at least one token each
            w = [r.expovariate(1.0) + 0.05 for _ in range(c["clients"])]
            left = c["tokens"] - c["clients"]
            lens = [1 + int(left * x / sum(w)) for x in w]
            lens[0] += c["tokens"] - sum(lens)
    past = c.get("past", 0)
    segs = [(1, int(math.exp(r.uniform(math.log(max(past / 8, 1)), math.log(max(past, 1)))))) for _ in range(c["decode"])]
    return segs + [(n, r.randint(0, c.get("prompt_past", 0))) for n in lens]


# ---- states -----------------------------------------------------------------------------------------------------------------------
def _normal(g, *shape, std=1.0, mean=0.0, dtype=BF16):
    return (torch.randn(*shape, device="cuda", generator=g) * std + mean).to(dtype)


def _batch(c):
    """The batch's row maps on the GPU, as a program that runs such batches keeps them."""
    segs = _segments(c)
    off = [0]
    for n, _ in segs:
        off.append(off[-1] + n)
    lens = torch.tensor([n for n, _ in segs], device="cuda")
    past = torch.tensor([p for _, p in segs], device="cuda")
    seg = torch.repeat_interleave(torch.arange(len(segs), device="cuda"), lens)
    index = torch.arange(off[-1], device="cuda") - torch.tensor(off, device="cuda")[seg]
    return dict(c=c, segs=segs, off=off, past=[p for _, p in segs], T=off[-1], S=len(segs), seg=seg, index=index, pos=past[seg] + index, lens=lens, past_t=past)


def _prepare_norm(c, g):
    s = _batch(c)
    d, S, T = c["width"], s["S"], s["T"]
    # activations of a residual stream: a mean that is not zero, rows of different size, a few channels that stand out
    s["X"] = (torch.randn(T, d, device="cuda", generator=g) * torch.exp(0.5 * torch.randn(T, 1, device="cuda", generator=g))
              * (1 + 9 * (torch.rand(1, d, device="cuda", generator=g) < 0.01)) + 0.2).to(BF16)
    s["eps"], s["base"] = (1e-6, 1.0) if c["rms"] else (1e-5, 0.0)
    weights = [_normal(g, d, std=0.1, mean=1.0 - s["base"]) for _ in range(1 if c["shared"] else S)]
    biases = [_normal(g, d, std=0.1) for _ in range(1 if c["shared"] else S)] if c["bias"] else [None]
    s["weights"], s["biases"] = [weights[i % len(weights)] for i in range(S)], [biases[i % len(biases)] for i in range(S)]
    s["Y"] = torch.empty_like(s["X"])
    if c["op"] == "norm_bwd":
        s["dY"] = _normal(g, T, d, std=0.01)
        s["dw"] = torch.empty(S, d, device="cuda")
        s["db"] = torch.empty(S, d, device="cuda") if c["bias"] else None
    if own:
        from paper_2507_03220_amd import binding as sb
        bwd = c["op"] == "norm_bwd"
        s["plan"] = sb.NormBatch(d, s["off"], [sb.Norm(s["weights"][i], s["biases"][i], s["dw"][i] if bwd else None,
                                                       s["db"][i] if bwd and c["bias"] else None) for i in range(S)],
                                 sb.SYMB_NORM_RMS if c["rms"] else sb.SYMB_NORM_LAYER, s["eps"], s["base"])
        s["ws"] = torch.empty(max(sb.symb_norm_workspace_bytes(s["plan"]), 256), device="cuda", dtype=torch.uint8)
    return s


def _prepare_kv(c, g):
    s = _batch(c)
    S, T, P, H, D = s["S"], s["T"], c["page"], c["kv_heads"], c["dim"]
    pages = [-(-(n + p) // P) for n, p in s["segs"]]
    N = sum(pages) + 5
    ids = torch.randperm(N, device="cuda", generator=g, dtype=torch.int32)
    table = torch.full((S, max(pages) + 1), -1, device="cuda", dtype=torch.int32)
    at = 0
    for i, n in enumerate(pages):
        table[i, :n] = ids[at:at + n]
        at += n
    s["table"], s["N"] = table, N
    # what earlier steps left in the cache: pages of different size, a few key channels that stand out
    codes = torch.randn(N, H, P, D, device="cuda", generator=g).mul_(60).mul_(1 + 1.5 * (torch.rand(1, H, 1, D, device="cuda", generator=g) < 0.05))
    s["k"] = codes.clamp_(-448, 448).to(E4M3)
    s["v"] = torch.randn(N, H, D, P, device="cuda", generator=g).mul_(90).clamp_(-448, 448).to(E4M3)
    s["k_scale"], s["v_scale"] = ((127 - 6 + torch.randint(-1, 2, (N, H), device="cuda", generator=g)).to(torch.uint8).view(E8M0) for _ in range(2))
    if c["op"] == "append":
        R = c["turned"] or D
        s["turned"] = 0 if c["turn"] == "none" else R
        most = max(n + p for n, p in s["segs"])
        angle = torch.arange(most, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(R // 2, device="cuda", dtype=torch.float64) * 2 / R)
        s["rotation"] = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous() if s["turned"] else None
        if c["fused"]:
            qkv = _normal(g, T, c["heads"] + 2 * H, D)
            s["q"], s["key"], s["value"] = qkv[:, :c["heads"]], qkv[:, c["heads"]:c["heads"] + H], qkv[:, c["heads"] + H:]
        else:
            s["q"], s["key"], s["value"] = (_normal(g, T, n, D) for n in (c["heads"], H, H))
        s["q_out"] = torch.empty(T, c["heads"], D, device="cuda", dtype=BF16)
        # the pages that the new rows go to: their number in the pool, and which slots are new
        first, last = s["past_t"] // P, (s["past_t"] + s["lens"] - 1) // P
        per = last - first + 1
        unit_seg = torch.repeat_interleave(torch.arange(S, device="cuda"), per)
        start = torch.cumsum(per, 0) - per
        page = first[unit_seg] + torch.arange(unit_seg.numel(), device="cuda") - start[unit_seg]
        s["unit_page"] = table[unit_seg, page].long()
        s["unit_first"] = (s["past_t"][unit_seg] - page * P).clamp(min=0)
        s["unit_end"] = (s["past_t"][unit_seg] + s["lens"][unit_seg] - page * P).clamp(max=P)
        s["row_unit"] = start[s["seg"]] + s["pos"] // P - first[s["seg"]]
    else:
        s["q"] = _normal(g, T, c["heads"], D, std=1.5)
        s["out"] = torch.empty(T, c["heads"], D, device="cuda", dtype=BF16)
        s["scale"] = D ** -0.5
        s["nmax"] = max(n for n, _ in s["segs"])
    if own:
        from paper_2507_03220_amd import binding as sb
        s["plan"] = sb.KvBatch(s["off"], s["past"], table)
        s["cache"] = sb.KvCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
        if c["op"] == "append":
            s["turn"] = sb.Rotation(s["rotation"], sb.SYMB_ROTATE_ADJACENT if c["turn"] == "adjacent" else sb.SYMB_ROTATE_HALVES) if s["turned"] else None
        else:
            s["ws"] = torch.empty(max(sb.symb_kv_workspace_bytes(s["plan"], s["cache"], c["heads"], c["window"]), 256), device="cuda", dtype=torch.uint8)
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 17)
    return (_prepare_norm if case["op"].startswith("norm") else _prepare_kv)(case, g)


# ---- the plain forms --------------------------------------------------------------------------------------------------------------
def _normalised(s):
    """(x-hat, 1 / standard deviation, weight of every row's client)"""
    x = s["X"].float()
    if not s["c"]["rms"]:
        x = x - x.mean(1, keepdim=True)
    r = (x.square().mean(1, keepdim=True) + s["eps"]).rsqrt()
    return x * r, r, (torch.stack(s["weights"]).float() + s["base"])[s["seg"]]


def _plain_norm_fwd(s):
    xh, _, w = _normalised(s)
    y = xh * w
    if s["c"]["bias"]:
        y = y + torch.stack(s["biases"]).float()[s["seg"]]
    s["Y"].copy_(y)
    return s["Y"]


def _plain_norm_bwd(s):
    xh, r, w = _normalised(s)
    dy = s["dY"].float()
    gy = dy * w
    dx = gy - xh * (gy * xh).mean(1, keepdim=True)
    if not s["c"]["rms"]:
        dx = dx - gy.mean(1, keepdim=True)
    s["Y"].copy_(dx * r)
    s["dw"].zero_().index_add_(0, s["seg"], dy * xh)
    if s["c"]["bias"]:
        s["db"].zero_().index_add_(0, s["seg"], dy)
    return {"dx": s["Y"], "dw": s["dw"], "db": s["db"]}


def _turn(s, x):
    """x [T][heads][D] with its first elements turned by the rows' positions."""
    x = x.float()
    R = s["turned"]
    if not R:
        return x
    rows = s["rotation"][s["pos"]][:, None, :]
    cos, sin = rows[..., :R // 2], rows[..., R // 2:]
    if s["c"]["turn"] == "adjacent":
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., R:]], -1)
    a, b = x[..., :R // 2], x[..., R // 2:R]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., R:]], -1)


def _plain_put(s, rows, pool, scale, turned_pool):
    """rows [T][H][D] fp32 into the pool's pages; turned_pool: pages are [H][D][P]."""
    P, U = s["c"]["page"], s["unit_page"].numel()
    codes = pool.view(torch.uint8)[s["unit_page"]]
    old = codes.view(E4M3).float()
    if turned_pool:
        old = old.transpose(2, 3)
    olde = scale.view(torch.uint8)[s["unit_page"]].int() - 127
    old = old * torch.exp2(olde.float())[:, :, None, None]
    new = torch.zeros(U, *old.shape[1:], device="cuda")
    new[s["row_unit"], :, s["pos"] % P] = rows
    slot = torch.arange(P, device="cuda")[None]
    is_new = ((slot >= s["unit_first"][:, None]) & (slot < s["unit_end"][:, None]))[:, None, :, None]
    is_old = (slot < s["unit_first"][:, None])[:, None, :, None]
    # the smallest power of two that brings the largest new value to 448 at most, and no less than the kept tokens have
    m, e = torch.frexp(new.abs().amax((2, 3)))
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(-126, 120)
    e = torch.where(s["unit_first"][:, None] > 0, torch.maximum(e, olde), e)
    put = (torch.where(is_new, new, old) * torch.exp2(-e.float())[:, :, None, None]).to(E4M3).view(torch.uint8)
    keep = is_new | is_old
    if turned_pool:
        put, keep = put.transpose(2, 3), keep.transpose(2, 3)
    pool.view(torch.uint8)[s["unit_page"]] = torch.where(keep, put, codes)
    scale.view(torch.uint8)[s["unit_page"]] = (e + 127).to(torch.uint8)


def _plain_append(s):
    s["q_out"].copy_(_turn(s, s["q"]))
    _plain_put(s, _turn(s, s["key"]), s["k"], s["k_scale"], False)
    _plain_put(s, s["value"].float(), s["v"], s["v_scale"], True)
    return {"q": s["q_out"], "k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _plain_attention(s):
    c = s["c"]
    S, P, H, D, G, n = s["S"], c["page"], c["kv_heads"], c["dim"], c["heads"] // c["kv_heads"], s["nmax"]
    table = s["table"].clamp(min=0).long()
    L = table.shape[1] * P
    k = s["k"].view(torch.uint8)[table].view(E4M3).float() * s["k_scale"].view(torch.uint8)[table].view(E8M0).float()[..., None, None]
    k = k.permute(0, 2, 1, 3, 4).reshape(S, H, L, D)
    v = s["v"].view(torch.uint8)[table].view(E4M3).float() * s["v_scale"].view(torch.uint8)[table].view(E8M0).float()[..., None, None]
    v = v.permute(0, 2, 1, 4, 3).reshape(S, H, L, D)
    q = torch.zeros(S, n, H, G, D, device="cuda")
    q[s["seg"], s["index"]] = s["q"].float().view(s["T"], H, G, D)
    q = q.permute(0, 2, 3, 1, 4).reshape(S, H, G * n, D)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(s["scale"])
    if c["cap"]:
        x = torch.tanh(x.div_(c["cap"])).mul_(c["cap"])
    at = torch.arange(L, device="cuda")
    pos = s["past_t"][:, None] + torch.arange(n, device="cuda")                          # [S][n]
    seen = at[None, None] <= pos[..., None]
    if c["window"]:
        seen &= at[None, None] > pos[..., None] - c["window"]
    x = x.view(S, H, G, n, L).masked_fill_(~seen[:, None, None], float("-inf"))
    x = x.sub_(x.amax(-1, keepdim=True)).exp_()
    x = x.div_(x.sum(-1, keepdim=True)).view(S, H, G * n, L)
    # (a token that no row sees is no part of the sum, whatever its page holds)
    v = v.masked_fill_((at[None] >= (s["past_t"] + s["lens"])[:, None])[:, None, :, None], 0.0)
    o = torch.matmul(x, v).view(S, H, G, n, D).permute(0, 3, 1, 2, 4)
    s["out"].copy_(o[s["seg"], s["index"]].reshape(s["T"], c["heads"], D))
    return s["out"]


# ---- one pass ---------------------------------------------------------------------------------------------------------------------
@functools.lru_cache(maxsize=None)
def _handle():
    from paper_2507_03220_amd import binding as sb
    return sb.symb_create(torch.cuda.current_device())


def _own_pass(s):
    from paper_2507_03220_amd import binding as sb
    c, h, stream = s["c"], _handle(), torch.cuda.current_stream().cuda_stream
    if c["op"] == "norm_fwd":
        sb.symb_norm_fwd(h, s["plan"], s["X"], s["Y"], stream)
        return s["Y"]
    if c["op"] == "norm_bwd":
        sb.symb_norm_bwd(h, s["plan"], s["X"], s["dY"], s["Y"], sb.SYMB_GRAD_OVERWRITE, s["ws"], stream)
        return {"dx": s["Y"], "dw": s["dw"], "db": s["db"]}
    if c["op"] == "append":
        sb.symb_kv_append(h, s["plan"], s["cache"], s["turn"], s["q"], s["q_out"], s["key"], s["value"], stream)
        return {"q": s["q_out"], "k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    sb.symb_kv_attention(h, s["plan"], s["cache"], s["q"], s["out"], s["scale"], c["window"], c["cap"], s["ws"], stream)
    return s["out"]


def run(state):
    if own:
        return _own_pass(state)
    return {"norm_fwd": _plain_norm_fwd, "norm_bwd": _plain_norm_bwd, "append": _plain_append, "attention": _plain_attention}[state["c"]["op"]](state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------------
def work(case):
    c, segs = case, _segments(case)
    T, S = sum(n for n, _ in segs), len(segs)
    if c["op"].startswith("norm"):
        d = c["width"]
        params = (1 if c["shared"] else S) * d * 2
        if c["op"] == "norm_fwd":
            return {"bytes": 2 * T * d * 2 + params * (2 if c["bias"] else 1), "flops": 8 * T * d}
        return {"bytes": 3 * T * d * 2 + params + S * d * 4 * (2 if c["bias"] else 1), "flops": 16 * T * d}
    H, Hq, D, P = c["kv_heads"], c["heads"], c["dim"], c["page"]
    if c["op"] == "append":
        R = 0 if c["turn"] == "none" else c["turned"] or D
        pages = sum((p + n - 1) // P - p // P + 1 for n, p in segs)
        # rows of q, k, v in; q out; the new 8-bit values and the touched pages' scales out; a row's cosines and sines
        return {"bytes": T * ((2 * Hq + 2 * H) * D * 2 + 2 * H * D + R * 4) + pages * 2 * H, "flops": T * ((Hq + H) * R * 3 + 4 * H * D)}
    tokens = pairs = 0
    for n, p in segs:
        w = c["window"] or n + p
        tokens += n + p - max(0, p + 1 - w)
        if p + 1 >= w:                                       # every row sees w tokens, or row j sees p + 1 + j up to w of them
            pairs += n * w
        else:
            grow = min(n, w - p - 1)
            pairs += grow * p + grow * (grow + 1) // 2 + (n - grow) * w
    return {"bytes": 2 * T * Hq * D * 2 + 2 * tokens * H * D + 2 * H * (tokens // P), "flops": 4 * pairs * Hq * D}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------------------
def _exact_norm(s):
    c, d = s["c"], s["c"]["width"]
    ys, dws, dbs = [], [], []
    for i in range(s["S"]):
        x = s["X"][s["off"][i]:s["off"][i + 1]].double()
        w = s["weights"][i].double() + s["base"]
        mu = x.mean(1, keepdim=True) * (0.0 if c["rms"] else 1.0)
        sd = torch.sqrt(((x - mu) ** 2).sum(1, keepdim=True) / d + s["eps"])
        z = (x - mu) / sd
        if c["op"] == "norm_fwd":
            ys.append(z * w + (s["biases"][i].double() if c["bias"] else 0.0))
            continue
        dy = s["dY"][s["off"][i]:s["off"][i + 1]].double()
        t = dy * w
        centre = t.sum(1, keepdim=True) / d * (0.0 if c["rms"] else 1.0)
        ys.append((t - centre - z * ((t * z).sum(1, keepdim=True) / d)) / sd)
        dws.append((dy * z).sum(0))
        dbs.append(dy.sum(0))
    if c["op"] == "norm_fwd":
        return torch.cat(ys)
    return {"dx": torch.cat(ys), "dw": torch.stack(dws), "db": torch.stack(dbs) if c["bias"] else None}


def _e4m3(x):
    """Nearest value of four significant bits (ties to even), steps of 2^-9 below 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_append(s):
    c, P, R = s["c"], s["c"]["page"], s["turned"]
    half = R // 2

    def turned(x):
        x = x.double().clone()
        if R:
            cs = s["rotation"].double()[s["pos"]].unsqueeze(1)
            first, second = (slice(0, R, 2), slice(1, R, 2)) if c["turn"] == "adjacent" else (slice(0, half), slice(half, R))
            z = torch.complex(x[..., first], x[..., second]) * torch.complex(cs[..., :half], cs[..., half:])
            x[..., first], x[..., second] = z.real, z.imag
        return x
    k, v = s["k"].double(), s["v"].double().transpose(2, 3).contiguous()
    ks, vs = s["k_scale"].double(), s["v_scale"].double()
    table = s["table"].cpu()
    for rows, pool, scale in ((turned(s["key"]), k, ks), (s["value"].double(), v, vs)):
        for i, (n, p) in enumerate(s["segs"]):
            for page in range(p // P, (p + n - 1) // P + 1):
                lo, hi = max(p, page * P), min(p + n, page * P + P)
                r = rows[s["off"][i] + lo - p:s["off"][i] + hi - p].transpose(0, 1)                     # [H][tokens][D]
                at, keep = int(table[i, page]), lo - page * P
                need = torch.exp2(torch.ceil(torch.log2(r.abs().amax((1, 2)).clamp(min=2.0 ** -110) / 448)))
                now = torch.maximum(need, scale[at]) if keep else need
                pool[at, :, :keep] = _e4m3(pool[at, :, :keep] * (scale[at] / now)[:, None, None])
                pool[at, :, keep:hi - page * P] = _e4m3(r / now[:, None, None])
                scale[at] = now
    return {"q": turned(s["q"]), "k": k, "v": v.transpose(2, 3).contiguous(), "k_scale": ks, "v_scale": vs}


def _exact_attention(s):
    c, P, G = s["c"], s["c"]["page"], s["c"]["heads"] // s["c"]["kv_heads"]
    out = torch.empty(s["T"], c["heads"], c["dim"], device="cuda", dtype=torch.float64)
    for i, (n, p) in enumerate(s["segs"]):
        pages = s["table"][i, :-(-(n + p) // P)].long()
        K, V = s["k"].view(torch.uint8)[pages].view(E4M3).double(), s["v"].view(torch.uint8)[pages].view(E4M3).double()
        es, vs = s["k_scale"].view(torch.uint8)[pages].double(), s["v_scale"].view(torch.uint8)[pages].double()
        rows = slice(s["off"][i], s["off"][i + 1])
        when = torch.arange(p, p + n, device="cuda")[:, None]
        token = torch.arange(n + p, device="cuda")[None]
        hidden = token > when
        if c["window"]:
            hidden = hidden | (when - token >= c["window"])
        for h in range(c["kv_heads"]):
            kh = (K[:, h] * 2.0 ** (es[:, h] - 127)[:, None, None]).reshape(-1, c["dim"])[:n + p]
            vh = (V[:, h] * 2.0 ** (vs[:, h] - 127)[:, None, None]).transpose(1, 2).reshape(-1, c["dim"])[:n + p]
            for j in range(h * G, h * G + G):
                a = s["q"][rows, j].double() @ kh.t().contiguous() * s["scale"]
                if c["cap"]:
                    a = c["cap"] * torch.tanh(a / c["cap"])
                out[rows, j] = torch.softmax(a.masked_fill(hidden, -math.inf), 1) @ vh
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return (_exact_norm if case["op"].startswith("norm") else _exact_append if case["op"] == "append" else _exact_attention)(s)
