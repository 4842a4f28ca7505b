"""Top logits, the distillation loss and the router's counts where their quick ways end: values that mislead the sample of a row, NaN that comes
before any finite value, logits at the border of what the fused exponential takes, segments that no single cluster counts."""
import numpy as np
import pytest
import torch

import loss_ref as ref
from paper_2112_04291_b200 import binding
from test_gpu_losses import MARK, TYPES, _check_distill, _dev, _logits, _run_top, _same

pytestmark = pytest.mark.gpu


def _check_repeated_top(rows, repeats, k, dtype, temperature=1.0):
    """Each of `rows` many times over, in a mixed order: every copy has the pairs, the sum and the tail of the definition."""
    which = np.random.default_rng(k).permutation(np.repeat(np.arange(rows.shape[0]), repeats))
    keys, values, lse, tail = _run_top(_dev(rows, TYPES[dtype])[torch.from_numpy(which).cuda()].contiguous(), k, temperature)
    want_keys, want_values, want_lse, want_tail = ref.top(rows, k, temperature)
    assert np.array_equal(keys.cpu().numpy(), want_keys[which])
    assert np.array_equal(values.double().cpu().numpy(), want_values[which])
    # an exponential is off by EX2 + 3 U |d|, a sum by (cols / 512 + 40) U; m / T, a logarithm and their sum by half a step each
    d = np.minimum((rows.max(1) - rows.min(1)) / temperature, 104.0)
    unit = (ref.EX2 + (3.0 * d + rows.shape[1] / 512.0 + 40.0) * ref.U)[which]
    size = (np.abs(rows.max(1)) / temperature + np.log(rows.shape[1]) + np.abs(want_lse))[which]
    assert np.all(np.abs(lse.double().cpu().numpy() - want_lse[which]) <= unit + 4.0 * ref.U * size)
    assert np.all(np.abs(tail.double().cpu().numpy() - want_tail[which]) <= 2.0 * unit * want_tail[which] + 2.0 ** -126)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("tiles,k", [(2, 300), (2, 700), (3, 300), (4, 60), (6, 40), (4, 300), (4, 1000)])
def test_top_logits_whose_largest_lie_in_the_sample(dtype, tiles, k):
    """Fewer than k values reach the bar that the sample of a row suggests (pieces of 512 bytes, every tiles-th one): the row is gone through again."""
    n = 16 // TYPES[dtype].itemsize
    cols, rng = tiles * 1024 * n, np.random.default_rng([tiles, k])
    vectors = np.arange(tiles * 1024)
    vectors = vectors[vectors // 32 % tiles == 0]
    z = _logits(rng, 12, cols, dtype)
    for r, count in enumerate(np.linspace(k // 5, k - 1, 12).astype(int)):
        chosen = rng.choice(vectors, min(count, len(vectors)), replace=False)
        z[r, chosen * n + rng.integers(0, n, len(chosen))] += 40.0
    _check_repeated_top(torch.from_numpy(z).to(TYPES[dtype]).double().numpy(), 50, k, dtype)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("tailed", [False, True])
@pytest.mark.parametrize("cols,repeats", [(1_000, 40), (5_000, 40), (5_000, 1), (40_000, 40), (128_000, 1)])
def test_no_nan_of_the_students_is_lost(dtype, tailed, cols, repeats):
    """NaN that a thread meets before any finite value, beside -inf or alone; rows without NaN in between."""
    rng = np.random.default_rng(cols)
    n = 16 // TYPES[dtype].itemsize
    z = _logits(rng, 7, cols, dtype)
    z[0, :n - 1], z[0, n - 1] = -np.inf, np.nan                               # the first vector of a thread
    z[1, :n] = np.nan
    z[2, cols - n:] = np.nan                                                  # ... the last
    front = min(4 * 256 * n, cols // 2)
    z[3, :front] = -np.inf                                                    # all of a block's first vectors
    z[3, front // 2 + 3] = np.nan
    z[5, ::n] = np.nan
    z[5, 1:] = np.where(rng.random(cols - 1) < 0.5, -np.inf, z[5, 1:])
    z = np.tile(z, (repeats, 1))
    rows = z.shape[0]
    keys = np.stack([rng.choice(cols, 9, replace=False) for _ in range(rows)]).astype(np.int32)
    values = rng.normal(0, 2, (rows, 9)).astype(np.float32)
    # (keys with finite logits: those that the student rules out have their own test)
    for r in range(rows):
        fine = np.flatnonzero(np.isfinite(z[r]))
        keys[r] = rng.choice(fine, 9, replace=False)
    _check_distill(z, dtype, keys, values, 1.0, rng.uniform(0.05, 0.5, rows).astype(np.float32) if tailed else None)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("tailed", [False, True])
@pytest.mark.parametrize("k", [1, 2, 40])
def test_a_teacher_of_nan_alone_is_no_row_that_counts_for_nothing(dtype, tailed, k):
    rng = np.random.default_rng(k)
    rows, cols = 6, 3_000
    z = _logits(rng, rows, cols, dtype)
    keys = np.stack([rng.choice(cols, k, replace=False) for _ in range(rows)]).astype(np.int32)
    values = rng.normal(0, 2, (rows, k)).astype(np.float32)
    values[0] = np.nan
    values[1, 0], values[1, 1:] = np.nan, -np.inf
    values[2], keys[2] = np.nan, -1                                           # (pairs that are not there may hold anything)
    values[3] = -np.inf
    values[4, -1] = np.nan
    tail = rng.uniform(0.05, 0.5, rows).astype(np.float32) if tailed else None
    if tailed:
        tail[0] = 1.0
    _check_distill(z, dtype, keys, values, 1.0, tail)


@pytest.mark.parametrize("temperature", [1.0, 2.0 ** -20])
@pytest.mark.parametrize("tailed", [False, True])
@pytest.mark.parametrize("rows", [4, 200])
def test_distillation_where_logits_become_far(temperature, tailed, rows):
    """|z| log2(e) / T of 2^26, from where on a fused exponential is not trusted: neighbours of fp32 are 2^5.8 apart there."""
    rng = np.random.default_rng(rows)
    cols = 8_192
    slot, thread = np.arange(cols) // 4 // 256, np.arange(cols) // 4 % 256
    z = np.where(thread < 128, np.where(slot < 4, -46_516_320.0, -46_516_300.0), -46_516_308.0)
    z = np.stack([z, z[::-1], np.where(thread < 128, -46_516_324.0, -46_516_316.0), rng.choice([-46_516_324.0, -46_516_320.0, -46_516_316.0, -46_516_312.0], cols)])
    z = np.tile(z, (rows // 4, 1)) * temperature
    keys = np.stack([rng.choice(cols, 5, replace=False) for _ in range(rows)]).astype(np.int32)
    values = (rng.normal(0, 2, (rows, 5)) * temperature).astype(np.float32)
    _check_distill(z, "fp32", keys, values, temperature, rng.uniform(0.05, 0.5, rows).astype(np.float32) if tailed else None)


@pytest.mark.parametrize("scale", [1.0, 2.0 ** -20])
def test_top_logits_where_logits_become_far(scale):
    """... on the two sides of a bar, which is a value of 16 bits: the pairs are not far, what is below the bar is."""
    rng = np.random.default_rng(1)
    cols, temperature = 8_192, float(np.float32(46_923_774.0 / (2.0 ** 26 / np.log2(np.e)) * scale))
    z = np.full((3, cols), -46_923_776.0)
    z[1, ::3], z[2, ::2] = -46_923_780.0, -46_923_784.0
    for r in range(3):
        z[r, rng.choice(cols, 200, replace=False)] = -46_923_772.0
    _check_repeated_top(z * scale, 100, 64, "fp32", temperature)


NO_WAITS = 0xFFFFFFFF


@pytest.mark.parametrize("dtype,rows,cols", [("bf16", 2_001, 3_000), ("fp32", 9, 6_001), ("fp16", 700, 60_001), ("bf16", 301, 128_000), ("fp32", 3, 262_144), ("fp32", 230, 200_003)])
def test_distillation_rows_whose_waits_run_out_are_nan(dtype, rows, cols):
    """From no wait at all to waits of some tries: a row is what it is with waits of any length, or has no number in it; nothing else is written."""
    gen = torch.Generator(device="cuda").manual_seed(cols)
    kind, k = TYPES[dtype], 20
    z = torch.randn((rows, cols), generator=gen, device="cuda").to(kind)
    keys = torch.randint(0, cols, (rows, k), generator=gen, device="cuda", dtype=torch.int32)
    values = torch.randn((rows, k), generator=gen, device="cuda")
    tail, up = 0.5 * torch.rand(rows, generator=gen, device="cuda"), torch.randn(rows, generator=gen, device="cuda")
    kept = torch.empty((rows, 2), device="cuda")
    assert binding.distill_loss(z, keys, values, stats=kept, tail=tail) == 0

    def loss_alone():
        loss, stats = torch.full((rows,), MARK, device="cuda"), torch.full((rows, 2), MARK, device="cuda")
        assert binding.distill_loss(z, keys, values, loss=loss, stats=stats, tail=tail) == 0
        return torch.cat([loss[:, None], stats], 1)

    def with_gradient():
        loss, stats = torch.full((rows,), MARK, device="cuda"), torch.full((rows, 2), MARK, device="cuda")
        mine = torch.full((rows + 2, cols), MARK, dtype=kind, device="cuda")
        mine[1:-1] = z
        assert binding.distill_loss(mine[1:-1], keys, values, loss=loss, grad=mine[1:-1], stats=stats, tail=tail) == 0
        assert bool((mine[0] == MARK).all()) and bool((mine[-1] == MARK).all())
        return torch.cat([loss[:, None], stats, mine[1:-1].float()], 1)

    def backward():
        grad = torch.full((rows + 2, cols), MARK, device="cuda")
        assert binding.distill_loss_backward(z, keys, values, kept, grad[1:-1], grad_loss=up, tail=tail) == 0
        assert bool((grad[0] == MARK).all()) and bool((grad[-1] == MARK).all())
        return grad[1:-1]

    for call in (loss_alone, with_gradient, backward):
        want = call()
        assert bool(want.isfinite().all())
        for tries in (NO_WAITS, 1, 1, 1, 2, 4, 16):
            try:
                binding.debug_set_wait_limits(copy_tries=tries)
                got = call()
                torch.cuda.synchronize()
            finally:
                binding.debug_set_wait_limits()
            lost = got.isnan()
            assert torch.equal(lost, lost.all(1, keepdim=True).expand_as(lost))
            assert bool((lost | (got == want)).all())
            assert bool(lost.all()) or tries != NO_WAITS
        assert torch.equal(call(), want)


@pytest.mark.parametrize("rows,cols,k", [(1_000, 20_000, 64), (900, 9_000, 700), (448, 3_000, 40), (3, 200_000, 20)])
def test_top_logits_rows_whose_claims_come_late_are_not_there(rows, cols, k):
    z = torch.randn((rows, cols), generator=torch.Generator(device="cuda").manual_seed(k), device="cuda").to(torch.bfloat16)
    want = _run_top(z, k, 1.0)
    for tries in (NO_WAITS, 1, 2):
        try:
            binding.debug_set_wait_limits(copy_tries=tries)
            keys, values, lse, tail = _run_top(z, k, 1.0)
            torch.cuda.synchronize()
        finally:
            binding.debug_set_wait_limits()
        lost = lse.isnan()
        # (a row is lost with the block's wait for it: the blocks that there are at first have their own)
        assert bool(lost.any()) or rows < 900 or tries != NO_WAITS
        assert bool((keys[lost] == -1).all()) and bool(values[lost].isnan().all()) and bool(tail[lost].isnan().all())
        assert all(_same(a[~lost].contiguous(), b[~lost].contiguous()) for a, b in zip((keys, values, lse, tail), want))
    assert all(_same(a, b) for a, b in zip(_run_top(z, k, 1.0), want))


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("tokens,k,experts,segments", [
    (200_003, 8, 60, [5, 5, 6, 70_000, 70_000, 70_001, 199_990]), (131_072, 4, 1024, [0, 65_536, 131_072]), (300_007, 1, 7, [0, 300_007]),
    (90_001, 16, 256, [0, 0, 1_000, 1_000, 90_001, 90_001]),                                        # spread over the GPU
    (100_003, 4, 33, [0] * 3 + [17] * 20 + [99_999] * 20), (100_003, 4, 33, list(range(0, 40)) + [100_003])])      # clusters, of which one has nearly all tokens
def test_counts_of_long_segments(masked, tokens, k, experts, segments):
    """Blocks that meet several segments, segments that several blocks share, empty ones, and tokens outside of all."""
    rng = np.random.default_rng([tokens, k])
    selected = rng.integers(-1, experts + 1, (tokens, k)).astype(np.int32)
    mask = rng.random(tokens) < 0.6 if masked else None
    offsets = np.asarray(segments, np.int64)
    count = len(segments) - 1
    want, want_tokens = np.zeros((count, experts), np.int64), np.zeros(count, np.int64)
    for s in range(count):
        part = slice(segments[s], segments[s + 1])
        kept = selected[part] if mask is None else selected[part][mask[part]]
        want[s], want_tokens[s] = np.bincount(kept[(kept >= 0) & (kept < experts)], minlength=experts), len(kept)
    for _ in range(2):
        counts, counted = torch.full((count, experts), -3, dtype=torch.int32, device="cuda"), torch.full((count,), -3, dtype=torch.int32, device="cuda")
        assert binding.expert_counts(_dev(selected), counts, counted, mask=None if mask is None else _dev(mask), offsets=_dev(offsets)) == 0
        assert np.array_equal(counts.cpu().numpy(), want) and np.array_equal(counted.cpu().numpy(), want_tokens)
