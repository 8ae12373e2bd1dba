"""Attention over a cache whose sequences have mostly ended: places of no keys between those that run."""
import random

import pytest
import torch

from cache_cases import cache
from paper_2202_13538_amd import binding
from test_gpu_cache_attention import BF, HF, biased, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    assert c.check() == 0
    c.close()


def with_gaps(gaps, seed):
    """Lengths of a run of single sequences, each behind a gap of so many places of no keys."""
    rng = random.Random(seed)
    return [x for n in gaps for x in [0] * n + [rng.randint(1, 40)]]


GAPS = [[0, 1, 2, 3] * 5, [63, 64, 65, 62], [255, 256, 257, 254, 0], [1023, 1024, 1025], [4090], [0] * 5 + [4000],
        [64 * i + 63 - i for i in range(10)], [7] * 700, [129, 5, 0, 700, 1] * 7, [4095, 0], [4096, 4100], [0, 5000, 0, 0, 9000, 63]]


@pytest.mark.parametrize("heads", [1, 2, 5, 20])       # of a key head
@pytest.mark.parametrize("gaps", GAPS, ids=lambda g: "-".join(map(str, g[:6])))
def test_sequences_behind_gaps(ctx, gaps, heads):
    lengths = with_gaps(gaps, len(gaps))
    for tail in (0, 300):                               # the last place runs, or has ended long ago
        check(ctx, *cache(lengths + [0] * tail, heads, 1, 16, 8, HF, seed=heads))


@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (2, 1), (6, 1), (40, 2)])
def test_long_sequences_among_thousands_of_places(ctx, heads, kv_heads):
    """Sequences that several workgroups share, where places are counted by lists."""
    lengths = with_gaps([70, 3, 0, 900, 0, 0, 2500, 800, 64], 5) + [0] * 4000
    for place, keys in ((0, 3000), (70, 513), (71, 6000), (1000, 2000), (5000, 1025), (len(lengths) - 1, 4444)):
        lengths[place] = keys
    check(ctx, *cache(lengths, heads, kv_heads, 64, 16, BF, seed=3), how=biased(heads, 128, 16, BF))


def of_two(n, heads, at):
    """A cache of n places, of which the two of `at` have 5 and 90 keys."""
    q, _, _, _, k_pages, v_pages, pages, length = cache([5, 90], heads, 1, 8, 16, BF, seed=4)
    many = torch.randn(n, heads, 8, device="cuda").bfloat16()
    table, lengths = torch.full((n, pages.shape[1]), -1, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    many[at], table[at], lengths[at] = q, pages, length
    return (q, k_pages, v_pages, pages, length), (many, k_pages, v_pages, table, lengths)


@pytest.mark.parametrize("heads", [1, 4])
@pytest.mark.parametrize("n,at", [(1 << 20, (0, (1 << 20) - 1)), (1 << 20, (4097, 600_000)), (300_000, (299_998, 299_999)), ((1 << 24) - 1, (1, (1 << 24) - 3))])
def test_two_of_very_many(ctx, n, at, heads):
    few, many = of_two(n, heads, list(at))
    want, got = binding.cache_attention(ctx, *few), binding.cache_attention(ctx, *many)
    assert ctx.check() == 0
    for x, y in zip(want, got):
        assert torch.equal(x, y[list(at)])
    left = torch.ones(n, dtype=torch.bool, device="cuda")
    left[list(at)] = False
    assert not got[0][left].any() and (got[1][left] == -float("inf")).all()


def least(run, passes=5):
    times = []
    for _ in range(passes):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        run()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b))
    return min(times)


@pytest.mark.parametrize("heads", [1, 4])
@pytest.mark.parametrize("n", [4096, 1 << 20])
def test_ended_sequences_take_no_longer_than_running_ones(ctx, n, heads):
    """Two places that run, the first and the last, against every place with a key; what is launched is the same."""
    _, (q, k_pages, v_pages, pages, length) = of_two(n, heads, [0, n - 1])
    some_page, one = pages.clamp(min=0), torch.ones_like(length)
    few = least(lambda: binding.cache_attention(ctx, q, k_pages, v_pages, pages, length))
    all_ = least(lambda: binding.cache_attention(ctx, q, k_pages, v_pages, some_page, one))
    assert few <= 1.5 * all_ + 0.03, (few, all_)
