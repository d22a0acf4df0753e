"""What is timed of the losses that a client's training step starts its backward pass from, through the frozen vocabulary matrix that all clients share, for the whole flattened batch.

  ce       softmax cross entropy of every row's label over the vocabulary: losses alone (evaluation, scoring), or with the gradient of the rows
  distill  divergence from a teacher's top logits, at each client's temperature: likewise

A case is one call on one batch: `clients` segments share `rows`; the first `masked` of each segment's rows are prompt and take no part.  Widths, client counts and row counts are those of `synth`
(Llama2-7B-, Granite-20B-, Gemma2-27B-shaped layers, the tiny configuration), vocabularies are of the usual sizes and odd ones.
"""
import functools
import math
import random

import torch

own = False

BF16 = torch.bfloat16


# ---- cases ------------------------------------------------------------------------------------------------------------------------
def _case(op, width, vocab, rows, clients=1, equal=False, masked=0.0, grad=True, cap=0.0, total=False, entries=0, temperature=1.0, ragged=False, mix=1):
    """total: losses are sums, not means; entries: of the teacher for a row, ragged: some rows have fewer; temperature: of the first client, the others' lie around it."""
    return dict(op=op, width=width, vocab=vocab, rows=rows, clients=clients, equal=equal, masked=masked, grad=grad, cap=cap, total=total, entries=entries, temperature=temperature,
                ragged=ragged, mix=mix)


def listed():
    return [
        # scoring one token: the smallest call there is
        dict(_case("ce", 4096, 32000, 1, grad=False, mix=1), name="ce_score_one"),
        # evaluation of eight clients' texts of ragged length
        dict(_case("ce", 6144, 49152, 2001, 8, grad=False, mix=2), name="ce_evaluate"),
        # training step of the tiny configuration: 4 clients x 64 tokens, odd vocabulary
        dict(_case("ce", 768, 50257, 256, 4, equal=True, mix=3), name="ce_grad_tiny"),
        # one client's short text
        dict(_case("ce", 4096, 32000, 37, total=True, mix=4), name="ce_grad_short"),
        # twelve clients answer prompts: half of the rows take no part
        dict(_case("ce", 4096, 32000, 6000, 12, masked=0.5, mix=5), name="ce_grad_answers"),
        # twenty clients on the widest layers, capped logits, the largest vocabulary: the most work of all
        dict(_case("ce", 4608, 256000, 8192, 20, cap=30.0, mix=6), name="ce_grad_large"),
        # how far one row is from its teacher
        dict(_case("distill", 4096, 32000, 1, grad=False, entries=20, temperature=2.0, mix=7), name="distill_one"),
        # evaluation against a teacher
        dict(_case("distill", 4096, 32001, 1500, 6, grad=False, entries=64, ragged=True, mix=8), name="distill_evaluate"),
        # the tiny configuration learns from a teacher
        dict(_case("distill", 768, 50257, 256, 4, equal=True, entries=16, temperature=2.0, mix=9), name="distill_grad_tiny"),
        # eight clients with temperatures of their own
        dict(_case("distill", 4096, 32000, 4096, 8, masked=0.2, entries=64, temperature=2.0, mix=10), name="distill_grad"),
        # many entries, capped logits, the largest vocabulary
        dict(_case("distill", 4608, 256000, 2048, 5, cap=30.0, entries=128, ragged=True, mix=11), name="distill_grad_large"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """1 to 8192 rows of 1 to 20 clients, widths 128 to 8192, vocabularies of 300 to 256000, 1 to 128 entries of a teacher."""
    while True:
        op = rng.choice(["ce", "ce", "distill"])
        width = rng.choice([768, 4096, 4608, 6144, 8 * _spread(rng, 16, 1024)])
        vocab = rng.choice([32000, 49152, _spread(rng, 300, 256000), _spread(rng, 300, 256000)])
        rows = rng.choice([1, _spread(rng, 2, 64), _spread(rng, 64, 8192), _spread(rng, 64, 8192)])
        clients = rng.randint(1, min(rows, 20))
        c = _case(op, width, vocab, rows, clients, rng.random() < 0.3, rng.choice([0.0, 0.0, round(rng.random() * 0.9, 3)]), rng.random() < 0.7, rng.choice([0.0, 0.0, 30.0, 50.0]),
                  rng.random() < 0.3, _spread(rng, 1, 128) if op == "distill" else 0, rng.choice([1.0, 2.0, round(rng.uniform(0.7, 4.0), 2)]), rng.random() < 0.4, rng.randrange(1 << 20))
        if rows * width * vocab <= 8192 * 4608 * 256000 and width * vocab <= 4608 * 256000:
            return c


def _segments(c):
    """[(rows, rows of prompt at their start)] of the batch, from the case alone."""
    r = random.Random(c["mix"])
    if c["equal"]:
        base, more = divmod(c["rows"], c["clients"])
        lens = [base + (i < more) for i in range(c["clients"])]
    else:                                         # uneven: exponential shares, at least one row each
        w = [r.expovariate(1.0) + 0.05 for _ in range(c["clients"])]
        left = c["rows"] - c["clients"]
        lens = [1 + int(left * x / sum(w)) for x in w]
        lens[0] += c["rows"] - sum(lens)
    return [(n, int(n * c["masked"])) for n in lens]


def _temperatures(c):
    r = random.Random(c["mix"] + 1)
    return [c["temperature"]] + [round(c["temperature"] * r.uniform(0.7, 1.4), 3) for _ in range(c["clients"] - 1)]


# ---- states -----------------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 29)
    c, segs = case, _segments(case)
    T, d, V, S = c["rows"], c["width"], c["vocab"], c["clients"]
    off = [0]
    for n, _ in segs:
        off.append(off[-1] + n)
    lens = torch.tensor([n for n, _ in segs], device="cuda")
    prompt = torch.tensor([p for _, p in segs], device="cuda")
    seg = torch.repeat_interleave(torch.arange(S, device="cuda"), lens)
    index = torch.arange(T, device="cuda") - torch.tensor(off, device="cuda")[seg]
    s = dict(c=c, off=off, seg=seg, T=T, S=S)
    s["W"] = (torch.randn(V, d, device="cuda", generator=g) * (3.0 * d ** -0.5)).to(BF16)
    # rows as the last norm leaves them, some sure of their token and some not
    token = torch.randint(0, V, (T,), device="cuda", generator=g)
    sure = 2.5 * torch.rand(T, 1, device="cuda", generator=g)
    s["X"] = (torch.randn(T, d, device="cuda", generator=g) + sure * s["W"][token].float()).to(BF16)
    counts = index >= prompt[seg]
    if c["op"] == "ce":
        s["labels"] = torch.where(counts, token, -100).to(torch.int32)
    else:
        K = c["entries"]
        gaps = torch.randint(1, max((V - 1) // K, 1) + 1, (T, K), device="cuda", generator=g)
        gaps[:, 0] = 0                            # (the top one is the row's token; no token twice)
        ids = (token[:, None] + gaps.cumsum(1)) % V
        fall = -torch.log1p(-torch.rand(T, K, device="cuda", generator=g))
        fall[:, 0] = 0.0
        s["teacher"] = (20.0 + torch.randn(T, 1, device="cuda", generator=g) - fall.cumsum(1) * (8.0 / K)).contiguous()
        keep = torch.full((T, 1), K, device="cuda")
        if c["ragged"]:
            keep = torch.randint(1, K + 1, (T, 1), device="cuda", generator=g)
        here = counts[:, None] & (torch.arange(K, device="cuda")[None] < keep)
        s["ids"] = torch.where(here, ids, -1).to(torch.int32)
    s["scale"] = [round(0.5 + 0.25 * (i % 5), 2) for i in range(S)]
    s["temperature"] = _temperatures(c)
    s["loss"], s["row_loss"] = torch.empty(S, device="cuda"), torch.empty(T, device="cuda")
    s["dX"] = torch.empty_like(s["X"]) if c["grad"] else None
    if own:
        from paper_2507_03220_amd import binding as sb
        s["plan"] = sb.LossBatch(d, V, off, [sb.Loss(a, t) for a, t in zip(s["scale"], s["temperature"])], sb.SYMB_LOSS_SUM if c["total"] else sb.SYMB_LOSS_MEAN, c["cap"])
        s["ws"] = torch.empty(max(sb.symb_loss_workspace_bytes(s["plan"], c["entries"], c["grad"]), 256), device="cuda", dtype=torch.uint8)
    else:
        s["row_scale"] = torch.tensor(s["scale"], device="cuda")[seg][:, None]
        s["row_temperature"] = torch.tensor(s["temperature"], device="cuda")[seg][:, None]
    return s


# ---- the plain forms --------------------------------------------------------------------------------------------------------------
def _plain(s):
    """A thousand rows at a time, whole rows of logits."""
    c = s["c"]
    W = s["W"].float()
    ce = c["op"] == "ce"
    counts = s["labels"] >= 0 if ce else (s["ids"] >= 0).any(1)
    n = torch.zeros(s["S"], device="cuda").index_add_(0, s["seg"], counts.float())
    share = s["row_scale"] * counts[:, None]
    if not c["total"]:
        share = share / n.clamp(min=1.0)[s["seg"]][:, None]
    for at in range(0, s["T"], 1024):
        rows = slice(at, min(at + 1024, s["T"]))
        z = torch.matmul(s["X"][rows].float(), W.t())
        if c["cap"]:
            z = torch.tanh(z.div_(c["cap"])).mul_(c["cap"])
        slope = 1.0 - (z / c["cap"]).square() if c["cap"] and c["grad"] else None
        if ce:
            ids, q = s["labels"][rows].clamp(min=0).long()[:, None], torch.ones(z.shape[0], 1, device="cuda")
            t = torch.ones_like(q)
            # a sure row's loss is what the others' weights are beside the label's: its own score in 64 bits, and no difference of two numbers near each other
            own_z = (s["X"][rows].double() * s["W"][ids[:, 0]].double()).sum(1, keepdim=True)
            if c["cap"]:
                own_z = torch.tanh(own_z / c["cap"]) * c["cap"]
        else:
            t = s["row_temperature"][rows]
            ids, here = s["ids"][rows].clamp(min=0).long(), s["ids"][rows] >= 0
            l = (s["teacher"][rows] / t).masked_fill(~here, float("-inf"))
            l = l - l.amax(1, keepdim=True).clamp(min=-3e38)
            q = l.exp()
            q = q / q.sum(1, keepdim=True).clamp(min=1e-30)
            z = z.div_(t)
        most = z.amax(1, keepdim=True)
        p = (z - most).exp()
        total = p.sum(1, keepdim=True)
        if ce:
            above = (own_z - most).float()
            others = p.scatter(1, ids, 0.0).sum(1, keepdim=True)
            row = torch.where(above > -40.0, torch.log1p(others * torch.exp(-above)), total.log() - above)[:, 0]
        else:
            logq = torch.where(q > 0, q, torch.ones_like(q)).log()
            row = (q * (logq - (z.gather(1, ids) - most - total.log()))).sum(1) * t[:, 0].square()
        s["row_loss"][rows] = torch.where(counts[rows], row, torch.zeros_like(row))
        if not c["grad"]:
            continue
        p = p.div_(total).scatter_add_(1, ids, -q)
        if slope is not None:
            p = p.mul_(slope)
        # (rows that take no part may hold anything)
        s["dX"][rows] = torch.where(counts[rows][:, None], torch.matmul(p.mul_(t * share[rows]), W), 0.0)
    s["loss"].zero_().index_add_(0, s["seg"], s["row_loss"])
    if not c["total"]:
        s["loss"].div_(n.clamp(min=1.0))
    return _outputs(s)


def _outputs(s):
    out = {"loss": s["loss"], "row_loss": s["row_loss"]}
    if s["c"]["grad"]:
        out["dx"] = s["dX"]
    return out


# ---- one pass ---------------------------------------------------------------------------------------------------------------------
@functools.lru_cache(maxsize=None)
def _handle():
    from paper_2507_03220_amd import binding as sb
    return sb.symb_create(torch.cuda.current_device())


def run(state):
    if not own:
        return _plain(state)
    from paper_2507_03220_amd import binding as sb
    s, stream = state, torch.cuda.current_stream().cuda_stream
    if s["c"]["op"] == "ce":
        sb.symb_cross_entropy(_handle(), s["plan"], s["X"], s["W"], s["labels"], s["loss"], s["row_loss"], s["dX"], s["ws"], stream)
    else:
        sb.symb_distillation(_handle(), s["plan"], s["X"], s["W"], s["ids"], s["teacher"], s["loss"], s["row_loss"], s["dX"], s["ws"], stream)
    return _outputs(s)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------------
def work(case):
    c, segs = case, _segments(case)
    n, T, d, V = sum(n - p for n, p in segs), c["rows"], c["width"], c["vocab"]
    # the vocabulary matrix and the rows that take part, labels or teacher in; losses and, of all rows, the gradient out
    moved = V * d * 2 + n * d * 2 + T * (8 * c["entries"] or 4) + T * 4 + c["clients"] * 4 + (T * d * 2 if c["grad"] else 0)
    return {"bytes": moved, "flops": (4 if c["grad"] else 2) * n * d * V}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    c, V = case, case["vocab"]
    rows = torch.zeros(s["T"], device="cuda", dtype=torch.float64)
    dx = torch.zeros(s["T"], c["width"], device="cuda", dtype=torch.float64) if c["grad"] else None
    loss = torch.zeros(s["S"], device="cuda", dtype=torch.float64)
    W = s["W"].double()
    for i in range(s["S"]):
        here = torch.arange(s["off"][i], s["off"][i + 1], device="cuda")
        here = here[(s["labels"][here] >= 0) if c["op"] == "ce" else (s["ids"][here] >= 0).any(1)]
        if not here.numel():
            continue
        T = s["temperature"][i]
        for r in here.split(256):
            x = s["X"][r].double().requires_grad_(c["grad"])
            logits = x @ W.t()
            if c["cap"]:
                logits = c["cap"] * torch.tanh(logits / c["cap"])
            if c["op"] == "ce":
                each = torch.logsumexp(logits, 1) - logits[torch.arange(r.numel(), device="cuda"), s["labels"][r].long()]
            else:
                there = s["ids"][r] >= 0
                logp = torch.log_softmax(logits / T, 1).gather(1, s["ids"][r].long().clamp(0, V - 1))
                logq = torch.log_softmax((s["teacher"][r].double() / T).masked_fill(~there, -math.inf), 1)
                each = T * T * torch.where(there, logq.exp() * (logq - logp), 0.0).sum(1)
            if c["grad"]:
                part = each.sum() * s["scale"][i] / (1 if c["total"] else here.numel())
                dx[r] = torch.autograd.grad(part, x)[0]
            rows[r] = each.detach()
        loss[i] = rows[here].sum() / (1 if c["total"] else here.numel())
    return {"loss": loss, "row_loss": rows, **({"dx": dx} if c["grad"] else {})}
