"""Cases of the operators on rows that are chosen by an id: an embedding's lookup with its gradient by sorted tokens, and
the matrix products of a router's experts, each in its plain form (elementary torch operations in 32 bits or more) and
through the library's calls.

Every case is one pass on inputs that stay on the GPU:

  lookup    rows of a table by token, times a scale, in the table's type or another
  gradient  of that table: tokens put in order, then every row's gradients added up; the whole table's gradient, or
            (`pairs`) the rows that occur as ascending (key, value) pairs, as the encoder takes them
  forward   selections put in order of their experts, then each expert's rows times its weights
  input     the gradient of those rows: the products' gradient times each expert's weights the other way
  weights   the gradient of each expert's weights

Inputs are drawn on the GPU from the seed alone.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
MOST_WEIGHTS = 8 * 14_336 * 4_096
MOST_PRODUCTS = 32_768 * 14_336 * 4_096


def listed():
    return [
        # one step of a server's batch: a few tokens' rows (latency)
        _embed("lookup-small", "lookup", 64, 32_000, 4_096, "bf16", "bf16", ragged=False),
        # a training batch; the table is kept in 32 bits, its rows are used in 16
        _embed("lookup-batch", "lookup", 32_768, 128_000, 4_096, "fp32", "bf16", ragged=False),
        # a training batch's gradient of the whole table in 32 bits, as the dense encoder takes it
        _embed("gradient-dense", "gradient", 16_384, 50_257, 2_048, "bf16", "fp32", ragged=False),
        # the same of an odd width, with padded tokens, in the gradient's own type
        _embed("gradient-odd", "gradient", 30_001, 8_009, 1_001, "fp16", "fp16", ragged=True),
        # the rows that occur alone, as key-value pairs for the encoder
        _embed("gradient-pairs", "pairs", 8_192, 128_000, 1_024, "fp32", "fp32", ragged=False),
        # a server's step: a token each of 16 users, two experts each; bound by the weights
        _experts("experts-decode", "forward", 16, 8, 2, 4_096, 14_336, "bf16", "bf16", ragged=False),
        # a training batch of many small experts, some selections dropped
        _experts("experts-many", "forward", 8_192, 64, 6, 2_048, 1_408, "fp16", "fp16", ragged=True),
        # a training batch of few large experts
        _experts("experts-large", "forward", 16_384, 8, 2, 4_096, 14_336, "bf16", "bf16", ragged=False),
        # the gradients of their inputs
        _experts("input-many", "input", 8_192, 64, 6, 2_048, 1_408, "fp16", "fp16", ragged=True),
        _experts("input-large", "input", 8_192, 8, 2, 4_096, 14_336, "bf16", "bf16", ragged=False),
        # the gradients of their weights in 32 bits, as the encoder takes them, and in their own type
        _experts("weights-many", "weights", 8_192, 64, 6, 2_048, 1_408, "bf16", "fp32", ragged=True),
        _experts("weights-odd", "weights", 1_003, 60, 4, 1_016, 680, "fp16", "fp16", ragged=True),
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["lookup", "gradient", "pairs", "forward", "forward", "input", "weights"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    ragged = rng.random() < 0.5
    if kind in ("lookup", "gradient", "pairs"):
        dtype = rng.choice(["fp32", dtype])
        out = "fp32" if kind == "pairs" else rng.choice([dtype, "fp32"] + (["bf16"] if dtype == "fp32" else []))
        cols = size(8, 8_192)
        vocab = size(2, min(260_000, 300_000_000 // cols))
        return _embed(None, kind, size(1, min(65_536, 200_000_000 // cols)), vocab, cols, dtype, out, ragged)
    experts = size(1, 256)
    ins = 8 * size(8, 1_024)
    outs = 8 * size(8, max(8, min(1_792, MOST_WEIGHTS // experts // ins // 8)))
    chosen = rng.randint(1, min(experts, 8))
    most = min(MOST_PRODUCTS // 2 // (outs * ins * chosen), MOST_WEIGHTS // (max(ins, outs) * chosen), 32_768)
    tokens = size(1, max(1, most))
    return _experts(None, kind, tokens, experts, chosen, ins, outs, dtype, rng.choice([dtype, dtype, "fp32"]), ragged)


def _named(name, case):
    return case if name is None else {"name": name, **case}


def _embed(name, kind, tokens, vocab, cols, dtype, out, ragged):
    return _named(name, {"kind": kind, "tokens": tokens, "vocab": vocab, "cols": cols, "dtype": dtype, "out": out, "ragged": ragged})


def _experts(name, kind, tokens, experts, chosen, ins, outs, dtype, out, ragged):
    return _named(name, {"kind": kind, "tokens": tokens, "experts": experts, "chosen": chosen, "ins": ins, "outs": outs, "dtype": dtype, "out": out,
                         "ragged": ragged})


def _occurring(draws, values):
    """how many of so many values turn up in so many even draws"""
    return int(round(values * -math.expm1(draws * math.log1p(-1.0 / values)))) if values > 1 else 1


def work(case):
    e = {"fp32": 4, "bf16": 2, "fp16": 2}
    ein, eout = e[case["dtype"]], e[case["out"]]
    if "vocab" in case:
        n, cols = case["tokens"], case["cols"]
        rows = _occurring(n, case["vocab"])
        if case["kind"] == "lookup":
            return {"bytes": 4 * n + rows * cols * ein + n * cols * eout, "flops": n * cols}
        if case["kind"] == "gradient":
            return {"bytes": 4 * n + n * cols * ein + case["vocab"] * cols * eout, "flops": n * cols}
        return {"bytes": 4 * n + n * cols * ein + rows * cols * 8, "flops": n * cols}
    rows = case["tokens"] * case["chosen"]
    kept = int(rows * 0.95) if case["ragged"] else rows
    active = _occurring(rows, case["experts"])
    weights, x, y = case["ins"] * case["outs"], case["ins"], case["outs"]
    flops = 2 * kept * weights
    if case["kind"] == "forward":
        return {"bytes": 4 * rows + case["tokens"] * x * ein + active * weights * ein + kept * y * eout, "flops": flops}
    if case["kind"] == "input":
        return {"bytes": kept * y * ein + active * weights * ein + kept * x * eout, "flops": flops}
    return {"bytes": kept * y * ein + case["tokens"] * x * ein + case["experts"] * weights * eout, "flops": flops}


# ---- inputs ---------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype, out = TYPES[case["dtype"]], TYPES[case["out"]]

    def normal(*shape, scale=1.0, kind=dtype):
        a = torch.empty(shape, dtype=kind, device="cuda")
        flat = a.view(-1)
        for i in range(0, flat.numel(), 1 << 26):                          # (in parts: drawn in 32 bits)
            part = flat[i:i + (1 << 26)]
            part.copy_(torch.randn(part.shape, generator=gen, device="cuda").mul_(scale))
        return a

    def full(shape, value, kind=torch.int32):
        return torch.full(shape, value, dtype=kind, device="cuda")

    if "vocab" in case:
        n, vocab, cols = case["tokens"], case["vocab"], case["cols"]
        # words by their rank: the share of the r-th is about 1 / r; ranks lie scattered over the table
        rank = torch.exp(torch.rand((n,), generator=gen, device="cuda", dtype=torch.float64) * math.log(vocab + 1.0)).long() - 1
        place = torch.randperm(vocab, generator=gen, device="cuda")
        ids = place[rank.clamp_(0, vocab - 1)].to(torch.int32)
        if case["ragged"]:                                                  # padded tokens
            ids[torch.rand((n,), generator=gen, device="cuda") < 0.1] = -1
        state = dict(case, ids=ids, scale=math.sqrt(cols) if case["kind"] == "lookup" else 1.0 / 64.0)
        if case["kind"] == "lookup":
            state["table"] = normal(vocab, cols, scale=cols ** -0.5)
            state["rows"] = torch.empty((n, cols), dtype=out, device="cuda")
            return state
        most = min(n, vocab)
        state.update(grad=normal(n, cols), order=full((n,), -1), starts=full((vocab + 1,), -1))
        if case["kind"] == "gradient":
            state["table_grad"] = torch.empty((vocab, cols), dtype=out, device="cuda")
        else:
            state.update(distinct=full((most,), -1), number=full((1,), -1), keys=full((most, cols), -1), values=full((most, cols), 0.0, torch.float32))
        return state

    n, experts, chosen, ins, outs = case["tokens"], case["experts"], case["chosen"], case["ins"], case["outs"]
    scores = torch.randn((n, experts), generator=gen, device="cuda")
    scores += 0.5 * torch.randn((experts,), generator=gen, device="cuda")   # some experts are liked more
    selected = scores.topk(chosen, dim=1).indices.to(torch.int32)
    if case["ragged"]:                                                      # selections that were dropped
        selected[torch.rand((n, chosen), generator=gen, device="cuda") < 0.05] = -1
    flat = selected.reshape(-1)
    where = torch.where(flat < 0, experts, flat).long()
    sizes = torch.bincount(where, minlength=experts + 1)
    state = dict(case, selected=selected, sizes=sizes[:experts].tolist())
    order, starts = _plain_order(flat, experts)
    kept = sum(state["sizes"])
    if case["kind"] == "forward":
        state.update(x=normal(n, ins), w=normal(experts, outs, ins, scale=ins ** -0.5), order=full((n * chosen,), -1), starts=full((experts + 1,), -1),
                     y=full((n * chosen, outs), 0.0, out))
        return state
    state.update(order=order, starts=starts, gy=normal(n * chosen, outs))
    if case["kind"] == "input":
        state.update(w=normal(experts, outs, ins, scale=outs ** -0.5), gx=full((n * chosen, ins), 0.0, out))
    else:
        state.update(x=normal(n, ins), gw=torch.empty((experts, outs, ins), dtype=out, device="cuda"))
    if kept < n * chosen:
        state["gy"][kept:] = math.nan                                       # rows behind the last expert's hold anything
    return state


# ---- one pass -------------------------------------------------------------------------------

def run(state):
    if own:
        return _run_own(state)
    if state["kind"] == "lookup":
        ids = state["ids"].long()
        rows = state["table"][ids.clamp(min=0)].float() * state["scale"]
        return {"rows": torch.where((ids >= 0)[:, None], rows, 0.0).to(state["rows"].dtype)}
    if state["kind"] in ("gradient", "pairs"):
        return _plain_gradient(state)
    return {"forward": _plain_forward, "input": _plain_input, "weights": _plain_weights}[state["kind"]](state)


def _done(rc):
    if rc != 0:
        raise RuntimeError("the library answers %d" % rc)


def _run_own(s):
    from paper_2112_04291_b200 import binding
    if s["kind"] == "lookup":
        _done(binding.embedding(s["table"], s["ids"], s["rows"], scale=s["scale"]))
        return {"rows": s["rows"]}
    if s["kind"] == "gradient":
        binding.ensure_rows_workspace(s["tokens"], s["cols"])
        _done(binding.order_ids(s["ids"], s["order"], s["starts"]))
        _done(binding.embedding_backward(s["grad"], s["ids"], s["order"], s["starts"], s["table_grad"], scale=s["scale"]))
        return {"order": s["order"], "starts": s["starts"], "table_grad": s["table_grad"]}
    if s["kind"] == "pairs":
        binding.ensure_rows_workspace(s["tokens"], s["cols"])
        _done(binding.order_ids(s["ids"], s["order"], s["starts"], distinct=s["distinct"], number=s["number"]))
        _done(binding.embedding_backward_pairs(s["grad"], s["ids"], s["order"], s["starts"], s["distinct"], s["number"], s["keys"], s["values"], scale=s["scale"]))
        return {"order": s["order"], "starts": s["starts"], "distinct": s["distinct"], "number": s["number"], "keys": s["keys"], "values": s["values"]}
    if s["kind"] == "forward":
        binding.ensure_products_workspace(s["tokens"] * s["chosen"], s["ins"])
        _done(binding.order_ids(s["selected"], s["order"], s["starts"]))
        _done(binding.expert_product(s["x"], s["w"], s["starts"], s["y"], order=s["order"], per_row=s["chosen"]))
        return {"order": s["order"], "starts": s["starts"], "y": s["y"]}
    if s["kind"] == "input":
        _done(binding.expert_product_backward_input(s["gy"], s["w"], s["starts"], s["gx"]))
        return {"gx": s["gx"]}
    binding.ensure_products_workspace(s["tokens"] * s["chosen"], s["ins"])
    _done(binding.expert_product_backward_weights(s["gy"], s["x"], s["starts"], s["gw"], order=s["order"], per_row=s["chosen"]))
    return {"gw": s["gw"]}


def _plain_order(ids, span):
    """Positions by (id, position), those of ids outside the span left out (-1 behind the last), and where each id's begin."""
    there = (ids >= 0) & (ids < span)
    key = torch.where(there, ids, span).long()
    counts = torch.zeros(span + 1, dtype=torch.int64, device=ids.device).index_add_(0, key, torch.ones_like(key))
    starts = torch.cat([counts.new_zeros(1), counts[:-1].cumsum(0)])
    position = torch.arange(key.numel(), device=ids.device)
    order = (key * key.numel() + position).sort().values % max(key.numel(), 1)
    order = torch.where(position < starts[-1], order, -1)
    return order.to(torch.int32), starts.to(torch.int32)


def _plain_gradient(s):
    order, starts = _plain_order(s["ids"], s["vocab"])
    vocab, cols = s["vocab"], s["cols"]
    at = torch.where(s["ids"] >= 0, s["ids"], vocab).long()
    total = torch.zeros((vocab + 1, cols), dtype=torch.float64, device="cuda")
    for a in range(0, s["tokens"], 8_192):
        total.index_add_(0, at[a:a + 8_192], s["grad"][a:a + 8_192].double())
    if s["kind"] == "gradient":
        return {"order": order, "starts": starts, "table_grad": (total[:vocab] * s["scale"]).to(s["table_grad"].dtype)}
    occurs = starts[1:] > starts[:-1]
    most = s["distinct"].numel()
    listed_ids = torch.where(occurs, torch.arange(vocab, device="cuda"), vocab).sort().values[:most]
    there = (listed_ids < vocab)[:, None]
    keys = torch.where(there, listed_ids[:, None] * cols + torch.arange(cols, device="cuda"), -1)
    values = torch.where(there, total[listed_ids] * s["scale"], 0.0)
    return {"order": order, "starts": starts, "distinct": torch.where(there[:, 0], listed_ids, -1).to(torch.int32), "number": occurs.sum().to(torch.int32)[None],
            "keys": keys.to(torch.int32), "values": values.float()}


def _groups(sizes):
    at = 0
    for e, size in enumerate(sizes):
        yield e, slice(at, at + size)
        at += size


def _plain_forward(s):
    order, starts = _plain_order(s["selected"].reshape(-1), s["experts"])
    y = torch.zeros((order.numel(), s["outs"]), dtype=s["y"].dtype, device="cuda")
    for e, part in _groups(s["sizes"]):
        y[part] = (s["x"][order[part].long() // s["chosen"]].float() @ s["w"][e].float().t()).to(y.dtype)
    return {"order": order, "starts": starts, "y": y}


def _plain_input(s):
    gx = torch.zeros((s["gy"].shape[0], s["ins"]), dtype=s["gx"].dtype, device="cuda")
    for e, part in _groups(s["sizes"]):
        gx[part] = (s["gy"][part].float() @ s["w"][e].float()).to(gx.dtype)
    return {"gx": gx}


def _plain_weights(s):
    gw = torch.zeros((s["experts"], s["outs"], s["ins"]), dtype=s["gw"].dtype, device="cuda")
    for e, part in _groups(s["sizes"]):
        gw[e] = (s["gy"][part].float().t() @ s["x"][s["order"][part].long() // s["chosen"]].float()).to(gw.dtype)
    return {"gw": gw}


# ---- from the definitions, in 64 bits ---------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "lookup":
        out = torch.zeros((case["tokens"], case["cols"]), dtype=torch.float64, device="cuda")
        there = (s["ids"] >= 0).nonzero()[:, 0]
        out[there] = torch.index_select(s["table"], 0, s["ids"][there]).double() * s["scale"]
        return {"rows": out}
    if "vocab" in case:
        # the rows of each id that occurs, side by side
        there = (s["ids"] >= 0).nonzero()[:, 0]
        words, run, lengths = s["ids"][there].unique(return_inverse=True, return_counts=True)
        by_run = there[run.argsort(stable=True)]
        sums = torch.zeros((0, case["cols"]), dtype=torch.float64, device="cuda")
        if len(words):
            sums = torch.segment_reduce(s["grad"][by_run].double(), "sum", lengths=lengths, axis=0) * s["scale"]
        if case["kind"] == "gradient":
            out = torch.zeros((case["vocab"], case["cols"]), dtype=torch.float64, device="cuda")
            out[words.long()] = sums
            return {"order": None, "starts": None, "table_grad": out}
        values = torch.zeros(s["values"].shape, dtype=torch.float64, device="cuda")
        values[:len(words)] = sums
        return {"order": None, "starts": None, "distinct": None, "number": None, "keys": None, "values": values}
    chosen = s["selected"].reshape(-1)
    picks = [(chosen == e).nonzero()[:, 0] for e in range(case["experts"])]          # ascending: the order within an expert
    tokens = [p // case["chosen"] for p in picks]
    if case["kind"] == "weights":
        out, at = torch.zeros(s["gw"].shape, dtype=torch.float64, device="cuda"), 0
        for e, token in enumerate(tokens):
            out[e] = torch.einsum("rn,rk->nk", s["gy"][at:at + len(token)].double(), s["x"][token].double())
            at += len(token)
        return {"gw": out}
    rows = s["y"] if case["kind"] == "forward" else s["gx"]
    out, at = torch.zeros(rows.shape, dtype=torch.float64, device="cuda"), 0
    for e, token in enumerate(tokens):
        part = slice(at, at + len(token))
        w = s["w"][e].double()
        out[part] = torch.einsum("rk,nk->rn", s["x"][token].double(), w) if case["kind"] == "forward" else torch.einsum("rn,nk->rk", s["gy"][part].double(), w)
        at += len(token)
    return {"order": None, "starts": None, "y": out} if case["kind"] == "forward" else {"gx": out}
