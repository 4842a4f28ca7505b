"""Cases of the operators that a worker's gradient begins with: a row's top logits as key-value pairs, the
distillation loss on them, and the balance loss of a router, each in its plain form (elementary torch
operations in 32 bits or more) and through the library's calls.

Every case is one pass on inputs that stay on the GPU:

  top       the k largest of each row of logits as (key, value) pairs in descending order, ties to the lower
            index; log sum exp(z / T) of the row and the share of it outside the pairs
  distill   loss of a student's logits against a teacher's top logits, with its gradient (`grad`: none, the
            logits' type, or fp32, as the encoder takes it)
  backward  that gradient alone, times the gradient of each row's loss, from what a forward call kept
  balance   per-expert counts of the selected experts, the balance loss of each segment of tokens and its gradient

Inputs are drawn on the GPU from the seed alone.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
LOG2_KEYS = 32


def listed():
    return [
        # a server's single token: the alternatives and log-probabilities of one row (latency)
        _top("top-one-row", 1, 128_000, 20, "bf16", 1.0),
        # the experts that a router selects for a batch of tokens
        _top("top-router", 8_192, 256, 8, "fp32", 1.0),
        # a teacher's answer to a batch, kept as key-value pairs for distillation
        _top("top-teacher", 2_048, 128_000, 64, "bf16", 2.0),
        # an odd vocabulary (rows start at any element) and many pairs
        _top("top-odd", 509, 50_257, 300, "fp16", 1.0),
        # the smallest distillation step
        _distill("distill-small", 8, 32_000, 32, "fp32", "fp32", 1.0, tail=False, ragged=False),
        # a training batch: loss and gradient in one call, the teacher's tail as one class more
        _distill("distill-train", 4_096, 128_000, 64, "bf16", "bf16", 2.0, tail=True, ragged=False),
        # evaluation: the loss alone, an odd vocabulary, rows with fewer pairs and padded rows
        _distill("distill-eval", 1_023, 50_257, 100, "fp32", "none", 1.5, tail=True, ragged=True),
        # the gradient of an output layer's logits as the encoder takes it, odd rows
        _distill("distill-fp32-gradient", 1_000, 100_003, 50, "bf16", "fp32", 1.0, tail=False, ragged=True),
        # the backward pass by itself
        _distill("distill-backward", 2_048, 32_000, 16, "fp16", "fp16", 4.0, tail=True, ragged=False, backward=True),
        # a few tokens of a small router
        _balance("balance-small", 64, 8, 2, "fp32", 1, ragged=False),
        # a training batch as one segment
        _balance("balance-batch", 65_536, 256, 8, "bf16", 1, ragged=False),
        # sequence by sequence: ragged, with padded tokens, a number of experts that is no power of two
        _balance("balance-sequences", 30_001, 60, 6, "fp16", 37, ragged=True),
    ]


def draw(rng):
    kind = rng.choice(["top", "top", "router", "distill", "distill", "distill", "backward", "balance", "balance"])
    dtype = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    most = 4_096 * 128_000 if dtype != "fp32" else 2_048 * 128_000

    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    if kind == "router":
        experts = size(4, 1_024)
        return _top(None, size(1, 65_536), experts, rng.randint(1, min(experts, 16)), dtype, 1.0)
    if kind == "balance":
        experts, tokens = size(4, 1_024), size(1, 131_072)
        segments = rng.choice([1, 1, size(2, 300)])
        return _balance(None, tokens, experts, rng.randint(1, min(experts, 16)), dtype, segments, ragged=rng.random() < 0.5)
    vocab = size(1_000, 260_000)
    pairs = size(1, 1_000)
    rows = size(1, min(8_192, most // vocab))
    temperature = rng.choice([1.0, 1.0, 2.0, round(rng.uniform(0.5, 5.0), 2)])
    if kind == "top":
        return _top(None, min(rows, most // 2 // vocab), vocab, min(pairs, 512), dtype, temperature)
    backward = kind == "backward"
    grad = rng.choice(["fp32", dtype] if backward else ["none", dtype, dtype, "fp32"])
    if grad == "fp32":
        rows = max(1, rows // 2)
    return _distill(None, rows, vocab, min(pairs, 256), dtype, grad, temperature, tail=rng.random() < 0.5, ragged=rng.random() < 0.5, backward=backward)


def _named(name, case):
    return case if name is None else {"name": name, **case}


def _top(name, rows, vocab, pairs, dtype, temperature):
    return _named(name, {"kind": "top", "rows": rows, "vocab": vocab, "pairs": pairs, "dtype": dtype, "temperature": temperature})


def _distill(name, rows, vocab, pairs, dtype, grad, temperature, tail, ragged, backward=False):
    return _named(name, {"kind": "backward" if backward else "distill", "rows": rows, "vocab": vocab, "pairs": pairs, "dtype": dtype, "grad": grad,
                         "temperature": temperature, "tail": tail, "ragged": ragged})


def _balance(name, tokens, experts, chosen, dtype, segments, ragged):
    return _named(name, {"kind": "balance", "tokens": tokens, "experts": experts, "chosen": chosen, "dtype": dtype, "segments": segments, "ragged": ragged})


def work(case):
    e = {"fp32": 4, "bf16": 2, "fp16": 2, "none": 0}
    if case["kind"] == "balance":
        t, n = case["tokens"], case["tokens"] * case["experts"]
        return {"bytes": 2 * n * e[case["dtype"]] + 4 * t * case["chosen"] + t * case["ragged"], "flops": 8 * n}
    n, pairs = case["rows"] * case["vocab"], case["rows"] * case["pairs"]
    if case["kind"] == "top":
        return {"bytes": n * e[case["dtype"]] + pairs * (4 + e[case["dtype"]]) + 8 * case["rows"], "flops": 4 * n}
    return {"bytes": n * (e[case["dtype"]] + e[case["grad"]]) + 8 * pairs + 8 * case["rows"], "flops": (4 if case["kind"] == "backward" else 8) * n}


# ---- inputs ---------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = TYPES[case["dtype"]]

    def empty(shape, kind):
        return torch.empty(shape, dtype=kind, device="cuda")

    if case["kind"] == "balance":
        t, n, k, s = case["tokens"], case["experts"], case["chosen"], case["segments"]
        x = torch.randn((t, n), generator=gen, device="cuda")
        x += torch.randn((n,), generator=gen, device="cuda")              # some experts are liked more
        x = x.to(dtype)
        chosen = x.float().topk(k, dim=1).indices.to(torch.int32)
        state = dict(case, x=x, chosen=chosen, mask=None, offsets=None, counts=empty((s, n), torch.int32), counted=empty((s,), torch.int32),
                     loss=empty((s,), torch.float32), grad=empty((t, n), dtype))
        if s > 1:
            cuts = torch.randint(0, t + 1, (s - 1,), generator=gen, device="cuda").sort().values
            state["offsets"] = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), t)])
        if case["ragged"]:                                                  # padded tokens, and selections that were dropped
            state["mask"] = torch.rand((t,), generator=gen, device="cuda") < 0.9
            chosen[torch.rand((t, k), generator=gen, device="cuda") < 0.03] = -1
        return state
    rows, vocab, pairs = case["rows"], case["vocab"], case["pairs"]
    z = torch.randn((rows, vocab), generator=gen, device="cuda").mul_(2.0)
    if case["kind"] == "top":
        return dict(case, z=z.to(dtype), keys=empty((rows, pairs), torch.int32), values=empty((rows, pairs), dtype), lse=empty((rows,), torch.float32),
                    tail=empty((rows,), torch.float32))
    # one key from each of `pairs` stretches of the vocabulary: distinct, scattered; the student likes them too
    edge = torch.arange(pairs + 1, device="cuda") * vocab // pairs
    keys = edge[:-1] + (torch.rand((rows, pairs), generator=gen, device="cuda") * (edge[1:] - edge[:-1])).long()
    liked = 6.0 + 2.0 * torch.randn((rows, pairs), generator=gen, device="cuda")
    z.scatter_(1, keys, liked)
    values, order = (liked + torch.randn((rows, pairs), generator=gen, device="cuda")).sort(dim=1, descending=True)
    keys = keys.gather(1, order).to(torch.int32)
    tail = 0.02 + 0.3 * torch.rand((rows,), generator=gen, device="cuda") if case["tail"] else None
    weight = None
    if case["ragged"]:                                                      # fewer pairs in some rows, padded rows
        kept = torch.randint(1, pairs + 1, (rows, 1), generator=gen, device="cuda")
        keys[torch.arange(pairs, device="cuda") >= kept] = -1
        weight = (torch.rand((rows,), generator=gen, device="cuda") < 0.9).float()
    state = dict(case, z=z.to(dtype), keys=keys, values=values, tail=tail, weight=weight, loss=empty((rows,), torch.float32),
                 grad=None if case["grad"] == "none" else empty((rows, vocab), TYPES[case["grad"]]))
    if case["kind"] == "backward":
        state["grad_loss"] = torch.randn((rows,), generator=gen, device="cuda")
        state["kept"] = None                                              # what the forward call keeps: two floats a row
        state["stats"] = _forward_stats(state)
    return state


def _forward_stats(state):
    """What the forward call keeps of a row: the largest logit outside the teacher's keys (of all logits where there is
    no tail) and the sum of exp((z - largest) / T) over the same."""
    z = state["z"].float()
    if state["tail"] is not None:
        keys = state["keys"].long()
        spare = z.new_empty((z.shape[0], 1))
        z = torch.cat([z, spare], 1).scatter_(1, torch.where(keys < 0, z.shape[1], keys), -math.inf)[:, :-1]
    top = z.amax(1)
    return torch.stack([top, ((z - top[:, None]) / state["temperature"]).exp().sum(1)], 1)


# ---- one pass -------------------------------------------------------------------------------

def run(state):
    if own:
        return _run_own(state)
    if state["kind"] == "top":
        return _plain_top(state)
    if state["kind"] == "balance":
        return _plain_balance(state)
    return _plain_distill(state)


def _done(rc):
    if rc != 0:
        raise RuntimeError("the library answers %d" % rc)


_workspace = []


def _run_own(s):
    from paper_2112_04291_b200 import binding
    if s["kind"] == "top":
        _done(binding.top_logits(s["z"], s["keys"], s["values"], temperature=s["temperature"], lse=s["lse"], tail=s["tail"]))
        return {"keys": s["keys"], "values": s["values"], "lse": s["lse"], "tail": s["tail"]}
    if s["kind"] == "distill":
        _done(binding.distill_loss(s["z"], s["keys"], s["values"], loss=s["loss"], grad=s["grad"], temperature=s["temperature"], tail=s["tail"], weight=s["weight"]))
        return {"loss": s["loss"]} if s["grad"] is None else {"loss": s["loss"], "grad": s["grad"]}
    if s["kind"] == "backward":
        _done(binding.distill_loss_backward(s["z"], s["keys"], s["values"], s["stats"], s["grad"], grad_loss=s["grad_loss"], temperature=s["temperature"],
                                            tail=s["tail"], weight=s["weight"]))
        return {"grad": s["grad"]}
    if not _workspace:
        _workspace.append(binding.ensure_workspace(1, binding.params(1.1)))
    _done(binding.expert_counts(s["chosen"], s["counts"], s["counted"], mask=s["mask"], offsets=s["offsets"]))
    _done(binding.balance_loss(s["x"], s["counts"], s["counted"], loss=s["loss"], grad=s["grad"], coef=0.01, mask=s["mask"], offsets=s["offsets"]))
    return {"counts": s["counts"], "counted": s["counted"], "loss": s["loss"], "grad": s["grad"]}


def _plain_top(s):
    z = s["z"].float()
    bits = (z + 0.0).view(torch.int32)
    rank = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long()                       # ascending with the value
    index = torch.arange(z.shape[1], device="cuda")
    best = ((rank << LOG2_KEYS) + (0xFFFFFFFF - index)).topk(s["pairs"], dim=1).values
    keys = 0xFFFFFFFF - (best & 0xFFFFFFFF)
    m = z.amax(1, keepdim=True)
    e = ((z - m) / s["temperature"]).exp()
    total = e.sum(1)
    rest = e.scatter(1, keys, 0.0).sum(1)
    return {"keys": keys.to(torch.int32), "values": s["z"].gather(1, keys), "lse": m[:, 0] / s["temperature"] + total.log(), "tail": rest / total}


def _plain_distill(s):
    z, t = s["z"].float(), s["temperature"]
    rows, vocab = z.shape
    there = s["keys"] >= 0
    at = torch.where(there, s["keys"], 0).long()
    z = z / t
    top = z.amax(1, keepdim=True)
    e = (z - top).exp()
    total = e.sum(1, keepdim=True)
    zk = z.gather(1, at)
    teacher = torch.where(there, s["values"] / t, -math.inf)
    tm = teacher.amax(1, keepdim=True)
    tsum = (teacher - tm).exp().sum(1, keepdim=True)
    tail = s["tail"][:, None] if s["tail"] is not None else torch.zeros_like(tm)
    log_p = teacher - tm - tsum.log() + (1.0 - tail).log()
    p = log_p.exp()
    one_more = torch.where(there, at, vocab)
    per_row = (p * torch.where(there, log_p - (zk - top) + total.log(), 0.0)).sum(1, keepdim=True)
    q = e / total
    target = q.new_zeros((rows, vocab + 1)).scatter_add_(1, one_more, p)[:, :vocab]
    if s["tail"] is not None:
        rest = torch.cat([e, e[:, :1]], 1).scatter_(1, one_more, 0.0)[:, :vocab]
        mass = rest.sum(1, keepdim=True)
        per_row = per_row + tail * (tail.log() - mass.log() + total.log())
        target = target + tail * rest / mass
    scale = torch.ones_like(tm) if s["weight"] is None else s["weight"][:, None]
    grad = None if s["grad"] is None else (q - target) * (scale * t if s["kind"] == "distill" else scale * t * s["grad_loss"][:, None])
    if s["kind"] == "backward":
        return {"grad": grad.to(s["grad"].dtype)}
    loss = (scale * per_row * (t * t))[:, 0]
    return {"loss": loss} if grad is None else {"loss": loss, "grad": grad.to(s["grad"].dtype)}


def _plain_balance(s):
    x = s["x"].float()
    t, n = x.shape
    segments = s["segments"]
    token = torch.arange(t, device="cuda")
    seg = torch.searchsorted(s["offsets"], token, right=True) - 1 if s["offsets"] is not None else torch.zeros_like(token)
    valid = s["mask"] if s["mask"] is not None else torch.ones_like(token, dtype=torch.bool)
    taken = (s["chosen"] >= 0) & valid[:, None]
    cell = torch.where(taken, seg[:, None] * n + s["chosen"], segments * n)
    counts = torch.zeros(segments * n + 1, dtype=torch.int64, device="cuda")
    counts = counts.index_add_(0, cell.reshape(-1), torch.ones_like(cell).reshape(-1))[:-1].view(segments, n)
    counted = torch.zeros(segments, dtype=torch.int64, device="cuda").index_add_(0, seg, valid.long())
    f = counts.float() / counts.sum(1, keepdim=True).clamp(min=1).float()
    e = (x - x.amax(1, keepdim=True)).exp()
    p = e / e.sum(1, keepdim=True)
    fr = f[seg]
    dot = (p * fr).sum(1, keepdim=True)
    scale = torch.where(valid, 0.01 * n / counted.clamp(min=1).float()[seg], 0.0)[:, None]
    grad = scale * p * (fr - dot)
    loss = torch.zeros(segments, dtype=torch.float64, device="cuda").index_add_(0, seg, (scale * dot)[:, 0].double())
    return {"counts": counts.to(torch.int32), "counted": counted.to(torch.int32), "loss": loss.float(), "grad": grad.to(s["grad"].dtype)}


# ---- from the definitions, in 64 bits, a few rows at a time ----------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "balance":
        return _exact_balance(s)
    part = max(1, (1 << 25) // case["vocab"])
    blocks = [(_exact_top if case["kind"] == "top" else _exact_distill)(s, slice(a, a + part)) for a in range(0, case["rows"], part)]
    names = ["lse", "tail"] if case["kind"] == "top" else [n for n in ("loss", "grad") if n in blocks[0]]
    out = {n: torch.cat([b[n] for b in blocks]) for n in names}
    if case["kind"] == "top":
        out.update(keys=None, values=torch.cat([b["values"] for b in blocks]))
    return out


def _exact_top(s, part):
    z = s["z"][part].double()
    ordered = z.sort(dim=1, descending=True).values
    y = ordered / s["temperature"]
    lse = y.logsumexp(1)
    return {"values": ordered[:, :s["pairs"]], "lse": lse, "tail": (y[:, s["pairs"]:].logsumexp(1) - lse).exp()}


def _exact_distill(s, part):
    t = s["temperature"]
    y = s["z"][part].double() / t
    lq = y - y.logsumexp(1, keepdim=True)
    rows, vocab = y.shape
    keys, row = s["keys"][part].long(), torch.arange(rows, device="cuda")[:, None].expand(-1, s["pairs"])
    here = keys >= 0
    row, col = row[here], keys[here]
    is_key = torch.zeros((rows, vocab), dtype=torch.bool, device="cuda")
    is_key[row, col] = True
    # log of the teacher's probability at every class, -inf where it says nothing
    lp = torch.full((rows, vocab), -math.inf, dtype=torch.float64, device="cuda")
    lp[row, col] = s["values"][part].double()[here] / t
    lp = lp - lp.logsumexp(1, keepdim=True)
    if s["tail"] is not None:
        lp = lp + (-s["tail"][part].double()[:, None]).log1p()
    p = lp.exp()
    loss = torch.where(is_key, p * (lp - lq), 0.0).sum(1)
    grad = lq.exp() - p
    if s["tail"] is not None:
        tail = s["tail"][part].double()
        rest = torch.where(is_key, -math.inf, lq)
        log_mass = rest.logsumexp(1)
        loss = loss + tail * (tail.log() - log_mass)
        grad = grad - tail[:, None] * (rest - log_mass[:, None]).exp()
    w = s["weight"][part].double() if s["weight"] is not None else torch.ones_like(loss)
    out = {} if s["kind"] == "backward" else {"loss": w * t * t * loss}
    if s["grad"] is not None:
        out["grad"] = grad * (t * (w * s["grad_loss"][part].double() if s["kind"] == "backward" else w))[:, None]
    return out


def _exact_balance(s):
    x = s["x"].double().cpu()
    n = x.shape[1]
    chosen, ends = s["chosen"].long().cpu(), s["offsets"].tolist() if s["offsets"] is not None else [0, x.shape[0]]
    mask = s["mask"].cpu() if s["mask"] is not None else torch.ones(x.shape[0], dtype=torch.bool)
    grad, losses = torch.zeros_like(x), []
    for a, b in zip(ends[:-1], ends[1:]):
        rows = torch.arange(a, b)[mask[a:b]]
        picks = chosen[rows].reshape(-1)
        f = torch.bincount(picks[picks >= 0], minlength=n).double()
        f = f / f.sum() if f.sum() > 0 else f
        p = x[rows].softmax(1)
        losses.append(0.01 * n * (f * p.mean(0)).sum() if len(rows) else torch.zeros((), dtype=torch.float64))
        if len(rows):
            grad[rows] = 0.01 * n / len(rows) * p * (f - (p @ f)[:, None])
    return {"counts": None, "counted": None, "loss": torch.stack(losses), "grad": grad}
