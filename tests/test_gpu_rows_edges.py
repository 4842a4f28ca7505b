"""The operators on rows chosen by an id where a part of a warp, a block of a pair, a workspace or a rounding could go wrong.

Values are small whole numbers where nothing else is said, so that every sum is exact in fp32 and fp16 whatever its order."""
import pytest
import torch

from paper_2112_04291_b200 import binding

pytestmark = pytest.mark.gpu
MARK = -77.0


def _whole(shape, most, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda").to(dtype)


def _full(shape, dtype=torch.int32, value=-9):
    return torch.full(shape, value, dtype=dtype, device="cuda")


@pytest.mark.parametrize("ins,outs", [(40, 264), (264, 40), (72, 1000), (8, 8), (136, 488), (776, 520)])
@pytest.mark.parametrize("rows", [129, 200, 256, 700, 5_000])
def test_products_whose_last_lanes_have_nothing_to_write(rows, ins, outs):
    """Outs and ins that are a multiple of 8 but not of 32, in tiles of more than 128 rows: some lanes of a warp write nothing and all of them read the next columns."""
    x, w, gy = _whole((rows, ins), 1, torch.float16, 1), _whole((2, outs, ins), 1, torch.float16, 2), _whole((rows, outs), 1, torch.float16, 3)
    starts = torch.tensor([0, rows // 5, rows], dtype=torch.int32, device="cuda")
    for dtype in (torch.float16, torch.float32):
        y, gx, gw = _full((rows, outs), dtype, MARK), _full((rows, ins), dtype, MARK), _full(w.shape, dtype, MARK)
        assert binding.expert_product(x, w, starts, y) == 0 and binding.expert_product_backward_input(gy, w, starts, gx) == 0
        assert binding.expert_product_backward_weights(gy, x, starts, gw) == 0
        for e, part in enumerate((slice(0, rows // 5), slice(rows // 5, rows))):
            assert torch.equal(y[part].double(), x[part].double() @ w[e].double().t())
            assert torch.equal(gx[part].double(), gy[part].double() @ w[e].double())
            assert torch.equal(gw[e].double(), gy[part].double().t() @ x[part].double())


@pytest.mark.parametrize("experts,ins,outs,most", [(256, 72, 136, 70), (40, 520, 1_032, 300), (9, 2_056, 264, 1_500), (1, 264, 264, 5_000)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_behind_an_experts_last_count_nothing_in_either_block(experts, ins, outs, most, dtype):
    """The last stage of an expert's rows holds the next expert's, or NaN, in both blocks' operands: each gradient is that of its own rows, again and again."""
    g = torch.Generator().manual_seed(experts)
    lengths = torch.randint(0, most, (experts,), generator=g)
    rows = int(lengths.sum())
    starts = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)])
    x, gy = _whole((rows + 70, ins), 1, torch.bfloat16, 1), _whole((rows + 70, outs), 1, torch.bfloat16, 2)
    want = _full((experts, outs, ins), torch.float64, 0.0)
    for e in range(experts):
        part = slice(int(starts[e]), int(starts[e + 1]))
        want[e] = gy[part].double().t() @ x[part].double()
    x[rows:], gy[rows:] = float("nan"), float("inf")
    at = starts.int().cuda()
    for _ in range(20):
        gw = _full((experts, outs, ins), dtype, MARK)
        assert binding.expert_product_backward_weights(gy, x, at, gw) == 0
        assert torch.equal(gw, want.to(gw.dtype))


def test_a_workspace_for_the_largest_batch_serves_every_smaller_one():
    """Tiles become longer at 8193 and 16385 rows of 2048 columns, and at 131073 ids: fewer rows then take more parts of sums, or counts."""
    keep = binding._workspace_keepalive

    def run(tokens, cols, vocab):
        ids, grad = torch.arange(tokens, dtype=torch.int32, device="cuda") % vocab, _full((tokens, cols), torch.bfloat16, 1)
        order, starts, table = _full((tokens,)), _full((vocab + 1,)), _full((vocab, cols), torch.float32)
        assert binding.order_ids(ids, order, starts) == 0 and binding.embedding_backward(grad, ids, order, starts, table) == 0
        assert torch.equal(table, torch.bincount(ids, minlength=vocab).float()[:, None].expand(vocab, cols))
    try:
        for tokens, cols, fewer in ((16_385, 2_048, (16_385, 16_384, 16_383, 8_193, 8_192, 4_100, 17, 1)), (131_073, 8, (131_073, 131_072, 131_071, 65_537, 65_536))):
            torch.cuda.synchronize()
            binding.set_workspace(torch.zeros(binding.rows_workspace_bytes(tokens, cols), dtype=torch.uint8, device="cuda"))
            for n in fewer:
                for c in (cols, cols - 1, cols // 2):
                    run(n, c, 40)
    finally:
        torch.cuda.synchronize()
        binding.set_workspace(keep if keep is not None else torch.zeros(64 << 20, dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()


def test_a_graph_replays_after_its_workspace_was_outgrown():
    """A product by an order lays its rows out in the workspace of its capture, whatever has been registered and allocated since."""
    x, w, ids = _whole((400, 264), 1, torch.float16, 1), _whole((6, 72, 264), 1, torch.float16, 2), _whole((400, 2), 1, torch.int32, 3).abs() * 3
    order, starts, y = _full((800,)), _full((7,)), _full((800, 72), torch.float32)

    def run():
        assert binding.order_ids(ids, order, starts) == 0 and binding.expert_product(x, w, starts, y, order=order, per_row=2) == 0
    binding.ensure_products_workspace(800, 264)
    before = binding._workspace_keepalive
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        run()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            run()
    torch.cuda.synchronize()
    binding.ensure_products_workspace(before.numel() // 512, 264)               # one that is larger
    address, size = before.data_ptr(), before.numel()
    assert binding._workspace_keepalive.data_ptr() != address
    del before
    others = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in range(3)]
    assert all(o.data_ptr() >= address + size or o.data_ptr() + size <= address for o in others)
    for seed in (5, 6):
        x.copy_(_whole(x.shape, 1, torch.float16, seed))
        y.fill_(MARK)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        at = starts.tolist()
        for e in range(6):
            part = slice(at[e], at[e + 1])
            assert torch.equal(y[part].double(), x[order[part].long() // 2].double() @ w[e].double().t())
    assert all((o == 255).all() for o in others)


LENGTHS = [512, 8_192, 8_200, 20_000, 65_536, 65_544, 70_016]


def _losses(got, want):
    """What the sums of positive values lose, on average and at most, of the value."""
    off = want - got.double()
    return (off.mean() / want.mean()).item(), (off.abs() / want).max().item()


@pytest.mark.parametrize("length", LENGTHS)
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_long_sums_of_one_sign_lose_no_more_than_is_said(length, dtype):
    """Values of one sign show best what the tensor cores cut off towards zero.  16 bits: a quarter of half a step just below a power of two, 2^-14 of the
    value in fp16 and 2^-11 in bf16, on average, since roundings of two million results are off by half a step at random (2^-11 / 1000 on average); a
    single one by half a step more (finfo.eps / 2).  32 bits: 2^-18, and half a step for each addition of two sums of 512 values.  More than 28 tiles: no
    contraction is shared."""
    g = torch.Generator(device="cuda").manual_seed(length)
    a = (torch.rand((4_096, length), generator=g, device="cuda") + 0.5).to(dtype)
    c = ((torch.rand((512, length), generator=g, device="cuda") + 0.5) * (1000.0 / length)).to(dtype)
    want = torch.cat([a[i:i + 512].double() @ c.double().t() for i in range(0, 4_096, 512)])
    most = 2.0 ** -14 if dtype == torch.float16 else 2.0 ** -11
    starts, rows = torch.tensor([0, 4_096], dtype=torch.int32, device="cuda"), torch.tensor([0, length], dtype=torch.int32, device="cuda")
    y, wide = _full((4_096, 512), dtype, MARK), _full((4_096, 512), torch.float32, MARK)
    assert binding.expert_product(a, c[None], starts, y) == 0 and binding.expert_product(a, c[None], starts, wide) == 0
    at, ct = a.t().contiguous(), c.t().contiguous()
    gx = _full((4_096, 512), dtype, MARK)
    assert binding.expert_product_backward_input(a, ct[None], starts, gx) == 0
    gw, wide_gw = _full((1, 4_096, 512), dtype, MARK), _full((1, 4_096, 512), torch.float32, MARK)
    assert binding.expert_product_backward_weights(at, ct, rows, gw) == 0 and binding.expert_product_backward_weights(at, ct, rows, wide_gw) == 0
    for got in (y, gx, gw[0]):
        mean, worst = _losses(got, want)
        assert abs(mean) <= most and worst <= most + torch.finfo(dtype).eps / 2
    for got in (wide, wide_gw[0]):
        mean, worst = _losses(got, want)
        assert abs(mean) <= 2.0 ** -18 and worst <= 2.0 ** -18 + (length / 512 + 1) * 2.0 ** -24


@pytest.mark.parametrize("length", [512, 4_096, 4_104, 8_192, 32_768, 32_776])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_sums_whose_first_value_outweighs_the_others_lose_no_more_than_is_said(length, dtype):
    """An accumulator that is large from the first step on cuts off most.  Of the sum: a quarter of half a step (2^-14 fp16, 2^-11 bf16) on average, half of
    it for a single result of 16 bits, and half a step for its rounding; 2^-16 for one of 32 bits, and half a step for each addition of two sums."""
    g = torch.Generator(device="cuda").manual_seed(length)
    a, c = (torch.rand((n, length), generator=g, device="cuda") + 0.5 for n in (4_096, 512))
    a[:, 0] *= 300.0
    c[:, 0] *= length / 3.0
    c *= 10.0 / length
    a, c = a.to(dtype), c.to(dtype)
    want = torch.cat([a[i:i + 512].double() @ c.double().t() for i in range(0, 4_096, 512)])
    assert want.max() < 60_000
    starts, mean_most = torch.tensor([0, 4_096], dtype=torch.int32, device="cuda"), 2.0 ** -14 if dtype == torch.float16 else 2.0 ** -11
    y, wide = _full((4_096, 512), dtype, MARK), _full((4_096, 512), torch.float32, MARK)
    assert binding.expert_product(a, c[None], starts, y) == 0 and binding.expert_product(a, c[None], starts, wide) == 0
    mean, worst = _losses(y, want)
    assert abs(mean) <= mean_most and worst <= 2.0 * mean_most + torch.finfo(dtype).eps / 2
    _, worst = _losses(wide, want)
    assert worst <= 2.0 ** -16 + (length / 512 + 1) * 2.0 ** -24
