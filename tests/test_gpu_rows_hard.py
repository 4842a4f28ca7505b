"""The operators on rows chosen by an id as they are used together, captured, on several streams, at sizes beyond 2^31 elements, with data that
the calls do not promise anything for, and where their waits run out.

Values are small whole numbers, so that every sum is exact in fp32 and fp16 whatever its order."""
import numpy as np
import pytest
import torch

import rows_ref as ref
from paper_2112_04291_b200 import binding

pytestmark = pytest.mark.gpu
MARK = -77.0


def _whole(shape, most, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda").to(dtype)


def _full(shape, dtype=torch.int32, value=-9):
    return torch.full(shape, value, dtype=dtype, device="cuda")


class Step:
    """Tokens through an embedding, a router's two selected experts of two layers each with a ReLU between, their sum, and back to the gradients of
    both layers' weights and of the embedding as key-value pairs.  Everything is allocated once: the step can be captured."""

    def __init__(self, tokens, vocab, cols, hidden, experts, k, seed):
        h = torch.float16
        self.k, rows, most = k, tokens * k, min(tokens, vocab)
        self.table, self.w1, self.w2 = _whole((vocab, cols), 1, h, seed), _whole((experts, hidden, cols), 1, h, seed + 1), _whole((experts, cols, hidden), 1, h, seed + 2)
        self.ids, self.dout, self.router = _full((tokens,)), _full((tokens, cols), h), _full((tokens, experts), torch.float32)
        self.x, self.y1, self.y2, self.out = _full((tokens, cols), h), _full((rows, hidden), h, 0), _full((rows, cols), h, 0), _full((tokens, cols), h)
        self.selected, self.scores = _full((tokens, k)), _full((tokens, k), torch.float32)
        self.order, self.starts, self.source = _full((rows,)), _full((experts + 1,)), _full((rows,))
        self.by_token, self.token_starts = _full((rows,)), _full((tokens + 1,))
        self.gy2, self.g1, self.gx = _full((rows, cols), h), _full((rows, hidden), h), _full((rows, cols), h)
        self.gw1, self.gw2 = _full(self.w1.shape, torch.float32), _full(self.w2.shape, torch.float32)
        self.dx = _full((tokens, cols), torch.float32)
        self.word_order, self.word_starts, self.distinct, self.number = _full((tokens,)), _full((vocab + 1,)), _full((most,)), _full((1,))
        self.keys, self.values, self.dense = _full((most, cols)), _full((most, cols), torch.float32), _full((vocab, cols), torch.float32)
        binding.ensure_rows_workspace(rows, cols)
        binding.ensure_products_workspace(rows, cols)

    def run(self):
        b = binding
        assert b.embedding(self.table, self.ids, self.x) == 0
        assert b.top_logits(self.router, self.selected, self.scores) == 0
        assert b.order_ids(self.selected, self.order, self.starts) == 0
        torch.div(self.order, self.k, rounding_mode="floor", out=self.source)
        assert b.expert_product(self.x, self.w1, self.starts, self.y1, order=self.order, per_row=self.k) == 0
        h = self.y1.clamp(min=0)
        assert b.expert_product(h, self.w2, self.starts, self.y2) == 0
        assert b.order_ids(self.source, self.by_token, self.token_starts) == 0
        assert b.embedding_backward(self.y2, self.source, self.by_token, self.token_starts, self.out) == 0       # a token's rows added up
        # back
        assert b.embedding(self.dout, self.source, self.gy2) == 0
        assert b.expert_product_backward_weights(self.gy2, h, self.starts, self.gw2) == 0
        assert b.expert_product_backward_input(self.gy2, self.w2, self.starts, self.g1) == 0
        self.g1.mul_(self.y1 > 0)
        assert b.expert_product_backward_weights(self.g1, self.x, self.starts, self.gw1, order=self.order, per_row=self.k) == 0
        assert b.expert_product_backward_input(self.g1, self.w1, self.starts, self.gx) == 0
        assert b.embedding_backward(self.gx, self.source, self.by_token, self.token_starts, self.dx) == 0
        assert b.order_ids(self.ids, self.word_order, self.word_starts, distinct=self.distinct, number=self.number) == 0
        assert b.embedding_backward_pairs(self.dx, self.ids, self.word_order, self.word_starts, self.distinct, self.number, self.keys, self.values) == 0
        assert b.embedding_backward(self.dx, self.ids, self.word_order, self.word_starts, self.dense) == 0

    def draw(self, seed):
        tokens, experts = self.router.shape
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.ids.copy_((torch.rand((tokens,), generator=g, device="cuda") ** 3 * self.table.shape[0]).int())
        self.router.copy_(torch.randn((tokens, experts), generator=g, device="cuda"))
        self.dout.copy_(torch.randint(-1, 2, self.dout.shape, generator=g, device="cuda"))

    def check(self):
        """Against autograd in 64 bits."""
        table, w1, w2 = (t.double().requires_grad_() for t in (self.table, self.w1, self.w2))
        x = table[self.ids.long()]
        picks = self.router.topk(self.k, dim=1).indices
        h = torch.einsum("td,tkhd->tkh", x, w1[picks]).relu()
        out = torch.einsum("tkh,tkdh->td", h, w2[picks])
        (out * self.dout.double()).sum().backward()
        assert torch.equal(self.out.double(), out.detach())
        assert torch.equal(self.gw1.double(), w1.grad) and torch.equal(self.gw2.double(), w2.grad)
        assert torch.equal(self.dense.double(), table.grad)
        n = int(self.number.item())
        words = self.ids.unique().long()
        assert torch.equal(self.distinct[:n].long(), words)
        assert torch.equal(self.keys[:n].long(), words[:, None] * table.shape[1] + torch.arange(table.shape[1], device="cuda"))
        assert torch.equal(self.values[:n], self.dense[words])


def test_a_step_from_tokens_to_the_update():
    """The step's sparse gradient through the encoder, decoder and model update: the same stream as that of the dense gradient."""
    s = Step(tokens=300, vocab=500, cols=24, hidden=40, experts=6, k=2, seed=1)
    s.draw(5)
    s.run()
    s.check()
    n, count = s.dense.numel(), int(s.number.item()) * s.dense.shape[1]
    p = binding.params(1.1)
    binding.ensure_workspace(n, p)
    streams = [torch.zeros(binding.compress_bound(n, p), dtype=torch.uint8, device="cuda") for _ in range(2)]
    assert binding.compress_kv(s.keys.view(-1)[:count], s.values.view(-1)[:count], n, p, streams[0]) == 0
    assert binding.compress(s.dense.view(-1), p, streams[1]) == 0
    size, d, status = binding.stream_info(streams[0])
    assert status == 0 and d > 0 and (size, d, 0) == binding.stream_info(streams[1]) and torch.equal(streams[0][:size], streams[1][:size])
    theta, m, v, scratch = s.table.float().view(-1).clone(), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    hyper = binding.Adam(0.01, 0.9, 0.999, 1e-8)
    assert binding.sparse_adam_update_batch([streams[0]], [size], n, p, hyper, scratch, theta, m, v) == 0 and binding.decode_status() == 0
    moved = theta != s.table.float().view(-1)
    assert int(moved.sum()) == d and (s.dense.view(-1)[moved] != 0).all()
    assert (torch.sign(s.table.float().view(-1) - theta)[moved] == torch.sign(s.dense.view(-1))[moved]).all()


def test_a_step_captured_and_replayed():
    """Two steps captured as graphs of their own share the workspace and are replayed in turn, with inputs that change."""
    steps = [Step(tokens=700, vocab=90, cols=64, hidden=72, experts=5, k=2, seed=3), Step(tokens=130, vocab=2000, cols=40, hidden=24, experts=9, k=3, seed=4)]
    stream, graphs = torch.cuda.Stream(), []
    torch.cuda.synchronize()
    for s in steps:
        s.draw(1)
        with torch.cuda.stream(stream):
            s.run()
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=stream):
                s.run()
        graphs.append(graph)
    for seed in (10, 11, 12):
        for s in steps:
            s.draw(seed)
        torch.cuda.synchronize()
        for graph in graphs:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for s in steps:
            s.check()


def _sorted_case(rows, experts, ins, outs, dtype, seed, most=2):
    starts = torch.linspace(0, rows, experts + 1, device="cuda").int()
    return _whole((rows, ins), most, dtype, seed), _whole((experts, outs, ins), most, dtype, seed + 1), starts, _whole((rows, outs), most, dtype, seed + 2)


def test_calls_without_a_workspace_on_two_streams_at_once():
    cases = []
    for i in range(2):
        x, w, starts, gy = _sorted_case(3000 + 700 * i, 5 + i, 264, 328, torch.bfloat16, i)
        ids = torch.randint(0, 900, (20_000,), dtype=torch.int32, device="cuda")
        cases.append((x, w, starts, gy, ids, _whole((900, 72), 3, torch.float16, i)))

    def run(case):
        x, w, starts, gy, ids, table = case
        y, gx, gw = _full(gy.shape, torch.float32), _full(x.shape, torch.float32), _full(w.shape, torch.float32)
        order, at, rows = _full(ids.shape), _full((901,)), _full((20_000, 72), torch.float32)
        assert binding.expert_product(x, w, starts, y) == 0 and binding.expert_product_backward_input(gy, w, starts, gx) == 0
        assert binding.expert_product_backward_weights(gy, x, starts, gw) == 0
        assert binding.order_ids(ids, order, at) == 0 and binding.embedding(table, ids, rows, scale=2.0) == 0
        return y, gx, gw, order, at, rows
    want = [run(c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(10):
        got = []
        for s, c in zip(streams, cases):
            with torch.cuda.stream(s):
                got.append(run(c))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_products_are_the_same_every_time():
    g = torch.Generator(device="cuda").manual_seed(0)
    x, w, gy = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((5000, 520), (7, 328, 520), (5000, 328)))
    starts = torch.tensor([0, 10, 1200, 1200, 3000, 3300, 4800, 4900], dtype=torch.int32, device="cuda")
    outs = [[_full((5000, 328), torch.float32, 0), _full((5000, 520), torch.bfloat16, 0), _full((7, 328, 520), torch.float32)] for _ in range(2)]
    for i in range(15):
        y, gx, gw = outs[i > 0]
        assert binding.expert_product(x, w, starts, y) == 0 and binding.expert_product_backward_input(gy, w, starts, gx) == 0
        assert binding.expert_product_backward_weights(gy, x, starts, gw) == 0
        assert i == 0 or all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("length", [512, 776, 4_096, 70_016])
def test_long_contractions_lose_no_more_than_short_ones(length):
    """Results of 32 bits against 64: relative, in the 2-norm.  512 values of a contraction are 32 steps of the tensor cores, each of which cuts off at
    most the last bit of the accumulator (2^-23 of it), towards zero; an accumulator that grows evenly is half its last value on average: at most
    32 2^-24 = 1.9e-6 of the sum of 512, and the sums of such pieces, whose signs differ, keep that share."""
    g = torch.Generator(device="cuda").manual_seed(length)
    a, c = (torch.randn((length, 128), generator=g, device="cuda").bfloat16() for _ in range(2))
    gw = _full((1, 128, 128), torch.float32)
    assert binding.expert_product_backward_weights(a, c, torch.tensor([0, length], dtype=torch.int32, device="cuda"), gw) == 0
    want = a.double().t() @ c.double()
    assert (gw[0].double() - want).norm() <= 1.9e-6 * want.norm()
    x, w, y = a.t().contiguous(), c.t().contiguous()[None], _full((128, 128), torch.float32)
    assert binding.expert_product(x, w, torch.tensor([0, 128], dtype=torch.int32, device="cuda"), y) == 0
    assert (y.double() - want).norm() <= 1.9e-6 * want.norm()
    half = _full((128, 128), torch.float16)
    assert binding.expert_product(x.half(), w.half(), torch.tensor([0, 128], dtype=torch.int32, device="cuda"), half) == 0
    want = x.half().double() @ w[0].half().double().t()
    assert (half.double() - want).abs().max() <= ref.rounding(want.abs().max().item(), "fp16") + 1.9e-6 * want.norm()


@pytest.mark.parametrize("rows", [2_000, 40])
def test_products_of_rows_with_infinities_and_nan_elsewhere(rows):
    """What a row holds shows in its own results, and in its own expert's gradient, alone."""
    x, w, starts, gy = _sorted_case(rows, 4, 136, 264, torch.bfloat16, 5)
    s = starts.tolist()
    x[s[1]] = float("inf")
    gy[s[3] - 1] = float("nan")
    y, gx, gw = _full((rows, 264), torch.float32), _full((rows, 136), torch.float32), _full(w.shape, torch.float32)
    assert binding.expert_product(x, w, starts, y) == 0 and binding.expert_product_backward_input(gy, w, starts, gx) == 0
    assert binding.expert_product_backward_weights(gy, x, starts, gw) == 0
    assert not y[s[1]].isfinite().any() and y.isfinite().all(1).sum() == rows - 1
    assert gx[s[3] - 1].isnan().all() and gx.isfinite().all(1).sum() == rows - 1
    for e in range(4):
        part = slice(s[e], s[e + 1])
        want = gy[part].double().t() @ x[part].double()
        assert torch.equal(gw[e].double().nan_to_num(nan=5.0, posinf=6.0, neginf=7.0), want.nan_to_num(nan=5.0, posinf=6.0, neginf=7.0)) or e in (1, 2)
    assert gw[2].isnan().all() and not gw[1].isfinite().any(0).any() and gw[0].isfinite().all() and gw[3].isfinite().all()


def test_no_rows():
    starts, w = torch.zeros(4, dtype=torch.int32, device="cuda"), _whole((3, 72, 40), 1, torch.float16, 1)
    x, gy, gw = torch.empty((0, 40), dtype=torch.float16, device="cuda"), torch.empty((0, 72), dtype=torch.float16, device="cuda"), _full((3, 72, 40), torch.float16)
    for order in (None, torch.empty((0,), dtype=torch.int32, device="cuda")):
        assert binding.expert_product(x, w, starts, gy, order=order) == 0
        gw.fill_(MARK)
        assert binding.expert_product_backward_weights(gy, x, starts, gw, order=order) == 0 and (gw == 0).all()
    assert binding.expert_product_backward_input(gy, w, starts, x) == 0


def test_workspaces_that_are_missing_or_too_small_are_refused():
    keep = binding._workspace_keepalive
    x, w, starts, _ = _sorted_case(4096, 4, 512, 64, torch.bfloat16, 1)
    y, order = _full((4096, 64), torch.bfloat16), torch.arange(4096, dtype=torch.int32, device="cuda")
    ids = torch.zeros(70_000, dtype=torch.int32, device="cuda")
    grad, at = torch.ones((70_000, 64), device="cuda"), _full((11,))
    big, table = _full((70_000,)), _full((10, 64), torch.float32)
    try:
        binding.set_workspace(torch.zeros(2 << 20, dtype=torch.uint8, device="cuda"))
        assert binding.expert_product(x, w, starts, y, order=order) == binding.E_NO_WORKSPACE and (y == -9).all()
        assert binding.expert_product(x, w, starts, y) == 0
        assert binding.order_ids(ids, big, at) == binding.E_NO_WORKSPACE
        assert binding.order_ids(ids[:65_536], big[:65_536], at) == 0
        assert binding.embedding_backward(grad, ids, big, at, table) == binding.E_NO_WORKSPACE
    finally:
        torch.cuda.synchronize()
        binding.set_workspace(keep if keep is not None else torch.zeros(64 << 20, dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()


def test_orders_and_starts_that_nobody_made_touch_nothing_else():
    """Garbage gives unspecified rows, and no access outside the buffers."""
    rows, experts, ins, outs = 600, 5, 72, 136
    x, w, _, gy = _sorted_case(rows, experts, ins, outs, torch.bfloat16, 2)
    store = _full((rows + 64, outs), torch.bfloat16, MARK)
    y = store[32:rows + 32]
    gx_store = _full((rows + 64, ins), torch.bfloat16, MARK)
    binding.ensure_products_workspace(rows, ins)
    order = torch.randint(-2 ** 31, 2 ** 31 - 1, (rows,), dtype=torch.int32, device="cuda")
    for starts in ([5, 3, 900, 2, -1, 100], [-7, 2 ** 31 - 1, 0, 0, 600, 601], [700, 800, 900, 1000, 1100, 1200], [0, 600, 0, 600, 0, 600]):
        at = torch.tensor(starts, dtype=torch.int32, device="cuda")
        gw = _full(w.shape, torch.float32)
        assert binding.expert_product(x, w, at, y, order=order) == 0 and binding.expert_product_backward_input(gy, w, at, gx_store[32:rows + 32]) == 0
        assert binding.expert_product_backward_weights(gy, x, at, gw, order=order) == 0
    torch.cuda.synchronize()
    assert (store[:32] == MARK).all() and (store[rows + 32:] == MARK).all() and (gx_store[:32] == MARK).all() and (gx_store[rows + 32:] == MARK).all()
    ids, starts = torch.randint(-50, 80, (rows,), dtype=torch.int32, device="cuda"), torch.randint(-2 ** 31, 2 ** 31 - 1, (41,), dtype=torch.int32, device="cuda")
    table, keys, values = _full((40 + 64, ins), torch.float32, MARK), _full((40 + 64, ins)), _full((40 + 64, ins), torch.float32, MARK)
    some, number = torch.randint(-2 ** 31, 2 ** 31 - 1, (40,), dtype=torch.int32, device="cuda"), torch.tensor([2 ** 31 - 1], dtype=torch.int32, device="cuda")
    grad = torch.ones((rows, ins), device="cuda")
    binding.ensure_rows_workspace(rows, ins)
    for last in (0, 300, 600, 5000, -1):
        starts[40] = last
        for o in (order, torch.arange(rows, dtype=torch.int32, device="cuda")):
            assert binding.embedding_backward(grad, ids, o, starts, table[32:72]) == 0
            assert binding.embedding_backward_pairs(grad, ids, o, starts, some, number, keys[32:72], values[32:72]) == 0
    alike = torch.full((rows,), 7, dtype=torch.int32, device="cuda")            # a token that goes on over every tile, said to end anywhere
    for end in (-1, 0, 1, 16, 17, 599, 5000):
        starts[7], starts[8], starts[40] = 0, end, rows
        assert binding.embedding_backward(grad, alike, torch.arange(rows, dtype=torch.int32, device="cuda"), starts, table[32:72]) == 0
        assert binding.embedding_backward_pairs(grad, alike, torch.arange(rows, dtype=torch.int32, device="cuda"), starts, some, number, keys[32:72], values[32:72]) == 0
    torch.cuda.synchronize()
    for t, mark in ((table, MARK), (keys, -9), (values, MARK)):
        assert (t[:32] == mark).all() and (t[72:] == mark).all()


def test_lookup_and_gradient_beyond_two_to_the_31_elements():
    vocab, cols = 270_001, 8_200
    ids = torch.tensor([0, vocab - 1, -1, vocab - 2, 262_000, vocab - 1], dtype=torch.int32, device="cuda")
    table = torch.zeros((vocab, cols), dtype=torch.bfloat16, device="cuda")
    for i in ids.unique().tolist():
        if i >= 0:
            table[i] = _whole((cols,), 9, torch.bfloat16, i)
    out = _full((6, cols), torch.float32)
    assert binding.embedding(table, ids, out, scale=2.0) == 0
    assert torch.equal(out, torch.where(ids[:, None] >= 0, table[ids.clamp(min=0).long()].float() * 2.0, 0.0))
    order, starts = _full((6,)), _full((vocab + 1,))
    binding.ensure_rows_workspace(6, cols)
    assert binding.order_ids(ids, order, starts) == 0
    table.fill_(3.0)
    grad = _whole((6, cols), 9, torch.bfloat16, 1)
    assert binding.embedding_backward(grad, ids, order, starts, table) == 0
    assert torch.equal(table[vocab - 1], grad[1] + grad[5]) and torch.equal(table[262_000], grad[4]) and torch.equal(table[0], grad[0]) and torch.equal(table[vocab - 2], grad[3])
    assert int((table != 0).any(1).sum()) == 4


def test_products_beyond_two_to_the_31_elements():
    rows, outs, ins = 70_000, 32_768, 64
    x, starts = _whole((rows, ins), 2, torch.bfloat16, 1), torch.tensor([0, 30_000, 69_990], dtype=torch.int32, device="cuda")
    w = _whole((2, outs, ins), 2, torch.bfloat16, 2)
    y = torch.full((rows, outs), MARK, dtype=torch.bfloat16, device="cuda")
    assert binding.expert_product(x, w, starts, y) == 0
    for r in (0, 29_999, 30_000, 65_535, 65_537, 69_989):
        assert torch.equal(y[r].double(), w[int(r >= 30_000)].double() @ x[r].double())
    assert (y[69_990:] == MARK).all()
    gx = _full((rows, ins), torch.float32, MARK)
    y.copy_((torch.arange(outs, device="cuda") % 3 - 1).expand(rows, outs))
    assert binding.expert_product_backward_input(y, w, starts, gx) == 0
    want = torch.stack([(y[0].double() @ w[e].double()) for e in range(2)]).float()
    assert torch.equal(gx[:30_000], want[0].expand(30_000, ins)) and torch.equal(gx[30_000:69_990], want[1].expand(39_990, ins)) and (gx[69_990:] == MARK).all()
    del y
    experts, outs, ins = 70, 8_192, 4_096                                      # weights of 4.7 GB
    w = torch.zeros((experts, outs, ins), dtype=torch.bfloat16, device="cuda")
    w[69] = _whole((outs, ins), 1, torch.bfloat16, 3)
    x, gy = _whole((40, ins), 1, torch.bfloat16, 4), _whole((40, outs), 1, torch.bfloat16, 5)
    starts = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
    starts[69], starts[70] = 8, 40
    y, gx = _full((40, outs), torch.float32), _full((40, ins), torch.float32)
    assert binding.expert_product(x, w, starts, y) == 0 and binding.expert_product_backward_input(gy, w, starts, gx) == 0
    assert torch.equal(y[8:].double(), x[8:].double() @ w[69].double().t()) and torch.equal(gx[8:].double(), gy[8:].double() @ w[69].double())
    assert (y[:8] == 0).all() and (gx[:8] == 0).all()                          # (expert 68's weights are zero)
    assert binding.expert_product_backward_weights(gy, x, starts, w) == 0
    assert torch.equal(w[69].double(), (gy[8:].double().t() @ x[8:].double()).bfloat16().double()) and torch.equal(w[68].double(), (gy[:8].double().t() @ x[:8].double()))
    assert (w[:68] == 0).all()


@pytest.mark.parametrize("tries", [0xFFFFFFFF, 1, 2, 4, 16])
@pytest.mark.parametrize("rows,experts,ins,outs", [(9_000, 6, 2_056, 1_032), (3_000, 1, 1_032, 520), (1_200, 2, 2_056, 4_104)])
def test_products_whose_waits_run_out_are_not_numbers(tries, rows, experts, ins, outs):
    """From no waits at all to waits of 160 us: each value is as ever or not a number, rows of no expert stay, and the next call is as ever."""
    x, w, starts, gy = _sorted_case(rows, experts, ins, outs, torch.bfloat16, 7, most=1)
    starts[-1] = rows - 100

    def run():
        y, gx, gw = _full((rows, outs), torch.bfloat16, MARK), _full((rows, ins), torch.float32, MARK), _full(w.shape, torch.float32, MARK)
        assert binding.expert_product(x, w, starts, y) == 0 and binding.expert_product_backward_input(gy, w, starts, gx) == 0
        assert binding.expert_product_backward_weights(gy, x, starts, gw) == 0
        torch.cuda.synchronize()
        return y, gx, gw
    want = run()
    try:
        binding.debug_set_wait_limits(copy_tries=tries)
        for _ in range(3):
            for a, b in zip(want, run()):
                lost = b.isnan()
                assert torch.equal(torch.where(lost, a, b), a)
                if tries == 0xFFFFFFFF:
                    assert lost[:rows - 100 if b.shape[0] == rows else None].all()
                if b.shape[0] == rows:
                    assert (b[rows - 100:] == MARK).all()
    finally:
        binding.debug_set_wait_limits()
    assert all(torch.equal(a, b) for a, b in zip(want, run()))


def test_binding_refuses_what_the_library_cannot_see():
    x, w, starts, gy = _sorted_case(32, 4, 64, 64, torch.bfloat16, 1)
    y = _full((32, 64), torch.bfloat16)
    ids = torch.zeros(32, dtype=torch.int32, device="cuda")
    for call in (lambda: binding.expert_product(x, w, starts.long(), y), lambda: binding.expert_product(x, w, starts[:4], y), lambda: binding.expert_product(x, w[0], starts, y),
                 lambda: binding.expert_product(x.cpu(), w, starts, y), lambda: binding.expert_product(x, w.transpose(1, 2), starts, y),
                 lambda: binding.expert_product(x, w, starts, y, order=ids[:5]), lambda: binding.order_ids(ids.long(), ids, starts), lambda: binding.order_ids(ids, ids[:5], starts),
                 lambda: binding.order_ids(ids, ids.clone(), starts, distinct=ids), lambda: binding.embedding(x, ids[:5], y), lambda: binding.embedding(x, ids, y.double()),
                 lambda: binding.embedding_backward(x, ids, ids.clone(), starts, y), lambda: binding.embedding_backward(x, ids.float(), ids.clone(), starts, y[:4])):
        with pytest.raises(AssertionError):
            call()
