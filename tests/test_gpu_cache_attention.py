"""surel_cache_attention on the GPU against attention in 64 bits over the same keys, packed."""
import math
import random

import numpy as np
import pytest
import torch

from attention_cases import reference
from cache_cases import cache
from paper_2202_13538_amd import binding
from test_gpu_attention import bounds, near

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    assert c.check() == 0
    c.close()


def biased(heads, reach, buckets, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    return dict(bias=torch.randn(buckets, heads, generator=g).to(dtype).cuda(),
                bucket=torch.tensor(binding.distance_buckets(reach, buckets, True), dtype=torch.int32).cuda())


def check(ctx, q, k, v, k_off, k_pages, v_pages, pages, length, how=None, scale=None, meant=None):
    how = how or {}
    out, lse = binding.cache_attention(ctx, q, k_pages, v_pages, pages, length, scale=scale, **how)
    one = torch.arange(len(q) + 1)
    r = reference(q, k, v, one, k_off, True, q.shape[2] ** -0.5 if scale is None else scale, **(meant or how))
    b_out, b_lse = bounds(r, q.dtype, q.shape[2], int(length.max()) if len(length) else 0)
    near(lse, r["lse"], b_lse, "lse")
    near(out, r["out"], b_out, "out")
    return out, lse


SHAPES = [  # lengths, heads, kv_heads, dim, rows of a page, heads first
    ([1], 1, 1, 8, 1, False), ([0], 2, 1, 16, 4, True), ([1, 2, 0, 31, 32, 33], 4, 2, 64, 16, False),
    ([64, 63, 65, 5], 3, 1, 40, 5, True), ([255, 256, 257, 1], 8, 8, 32, 16, False), ([300, 7, 0, 0], 6, 2, 96, 24, True),
    ([1000], 16, 1, 128, 64, False), ([2000, 3], 32, 1, 128, 100, True), ([700, 1501], 40, 1, 72, 16, False),
    ([513], 66, 2, 24, 7, True), ([500, 3, 77], 6, 3, 128, 16, False), ([100, 2000], 8, 2, 64, 16, True), ([90, 31], 4, 2, 16, 8, False), ([77, 900], 34, 2, 128, 16, False), ([31, 1, 40], 10, 2, 88, 16, True), ([9] * 200, 4, 4, 80, 8, False), ([40, 0, 17, 5000], 12, 4, 104, 256, True),
    ([128] * 3, 5, 5, 56, 1024, False), ([3001] * 2, 2, 2, 128, 3, True), ([33, 600], 1, 1, 120, 1, False),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("reach", [None, 0, 20, 1024])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_rows_over_their_pages(ctx, shape, reach, dtype):
    lengths, heads, kv_heads, dim, page_rows, heads_first = shape
    args = cache(lengths, heads, kv_heads, dim, page_rows, dtype, seed=len(lengths), heads_first=heads_first)
    check(ctx, *args, how=None if reach is None else biased(heads, reach, min(reach + 1, 12), dtype))


@pytest.mark.parametrize("seqs,most,kv_heads,dim", [(4096, 3, 1, 16), (4097, 70, 1, 8), (9000, 40, 2, 8)])
def test_many_sequences(ctx, seqs, most, kv_heads, dim):
    rng = random.Random(seqs)
    lengths = [rng.choice([0, 1, rng.randint(0, most)]) for _ in range(seqs)]
    args = cache(lengths, 2 * kv_heads, kv_heads, dim, 4, BF, seed=1)
    check(ctx, *args)


def test_one_long_sequence_among_many_short_ones(ctx):
    lengths = [5] * 300
    lengths[100] = 20_000
    lengths[299] = 3000
    args = cache(lengths, 8, 2, 64, 16, HF, seed=2)
    check(ctx, *args, how=biased(8, 128, 16, HF))


def test_queries_that_are_parts_of_a_larger_tensor(ctx):
    _, *rest = cache([40, 300, 0, 9], 4, 2, 32, 16, BF, seed=3)
    qkv = torch.randn(4, 3, 4, 32, device="cuda").bfloat16()
    check(ctx, qkv[:, 0], *rest)
    turned = torch.randn(4, 4, 32, device="cuda").bfloat16()
    check(ctx, turned.transpose(0, 1), *rest)


def test_sequences_that_share_pages(ctx):
    q, k, v, _, k_pages, v_pages, pages, length = cache([90, 64], 4, 2, 64, 16, BF, seed=4)
    pages = torch.cat([pages, pages[:1]])            # a third sequence: the first's beginning
    length = torch.tensor([90, 64, 50], dtype=torch.int32, device="cuda")
    q = torch.cat([q, q[:1]])
    k_all, v_all = (torch.cat([x, x[:50]]) for x in (k, v))
    check(ctx, q, k_all, v_all, torch.tensor([0, 90, 154, 204]), k_pages, v_pages, pages, length)


def test_results_are_the_same_every_time_and_as_packed(ctx):
    args = cache([4000, 1, 77, 2500, 0], 16, 4, 128, 16, BF, seed=5)
    first = check(ctx, *args)
    q, k, v, k_off, k_pages, v_pages, pages, length = args
    for _ in range(5):
        again = binding.cache_attention(ctx, q, k_pages, v_pages, pages, length)
        assert all(torch.equal(x, y) for x, y in zip(first, again))
    # the same rows by attention over packed keys: both within one rounding of the weights and one of the result
    out, lse = binding.attention(ctx, q, k, v, torch.arange(6, device="cuda"), k_off, causal=True)
    assert (out.float() - first[0].float()).abs().max() <= 4 * torch.finfo(BF).eps * v.float().abs().max()
    fine = length > 0
    assert (lse - first[1])[fine].abs().max() < 1e-4 and torch.equal(lse[~fine], first[1][~fine])


def test_scales_and_large_scores(ctx):
    args = cache([500, 40, 3], 4, 1, 64, 16, HF, seed=6)
    for scale in (1e-30, 0.01, 3.0, 50.0):
        check(ctx, *args, scale=scale)
    args = cache([500, 40, 3], 4, 1, 64, 16, BF, seed=7)
    args[0].mul_(1000.0)
    check(ctx, *args)
    for heads, kv_heads in ((2, 2), (8, 1), (20, 1)):         # keys and values below 16-bit floats' normal ones
        q, k, v, k_off, k_pages, v_pages, pages, length = cache([500, 40, 3], heads, kv_heads, 64, 16, HF, seed=8)
        q.mul_(10_000.0)
        for x in (k, v, k_pages, v_pages):
            x.mul_(2.0 ** -18)
        check(ctx, q, k, v, k_off, k_pages, v_pages, pages, length, scale=3.0)


def test_a_bias_that_masks(ctx):
    for dtype, lowest in ((BF, -3e38), (BF, -math.inf), (HF, -65504.0), (HF, -math.inf)):
        args = cache([300, 2, 1, 40], 2, 1, 32, 16, dtype, seed=8)
        how = biased(2, 20, 12, dtype)
        how["bias"][-1] = lowest                     # distances from some on
        # (a bias of -65504 or less is minus infinity by definition: the reference is given that)
        check(ctx, *args, how=how, meant=dict(how, bias=how["bias"].double().masked_fill(how["bias"] <= -65504, -math.inf)))
        how["bias"][:] = lowest                      # all of them: rows that are left nothing
        q, _, _, _, k_pages, v_pages, pages, length = args
        out, lse = binding.cache_attention(ctx, q, k_pages, v_pages, pages, length, **how)
        assert not out.any() and (lse == -math.inf).all()


@pytest.mark.parametrize("group", [2, 5, 20])
def test_what_is_not_finite(ctx, group):
    """A sequence's keys that are not finite are its own affair, and heads' own."""
    lengths = [100, 40, 70, 33]
    args = list(cache(lengths, 2 * group, 2, 80, 16, BF, seed=9))
    q, k, v, k_off, k_pages, v_pages, pages, length = args

    def put(s, j, head, d, x, which):
        page, r = int(pages[s, j // 16]), j % 16
        (k_pages if which == "k" else v_pages)[page, r, head, d] = x
        (k if which == "k" else v)[int(k_off[s]) + j, head, d] = x

    put(0, 99, 1, 3, math.nan, "k")
    put(1, 32, 0, 0, math.inf, "v")                  # the first of a tile that is not full
    q[2, :group] = q[2, :group].abs() + 0.1
    put(2, 64, 0, 7, -math.inf, "k")                 # scores of minus infinity: the key has no weight
    got = binding.cache_attention(ctx, q, k_pages, v_pages, pages, length)
    r = reference(q, k, v, torch.arange(5), k_off, True, 80 ** -0.5)
    out, lse = (x.cpu().double().numpy() for x in got)
    assert np.isnan(out[0, group:]).all() and np.isnan(lse[0, group:]).all() and np.isfinite(out[0, :group]).all()
    assert np.isinf(out[1, :group, 0]).all() and np.isfinite(out[1, :group, 1:]).all() and np.isfinite(out[1, group:]).all()
    b_out, b_lse = bounds(r, BF, 80, 100)
    for s, heads in ((0, slice(0, group)), (1, slice(group, None)), (2, slice(None)), (3, slice(None))):
        # (the score of minus infinity makes its row's largest sum of products infinite, and no bound of it)
        b = np.where(np.isfinite(b_out[s, heads]), b_out[s, heads], 2.25 * 2 ** -8 * r["abs_out"][s, heads] + 1e-4)
        assert (np.abs(out[s, heads] - r["out"][s, heads]) <= b).all(), s
        b = np.where(np.isfinite(b_lse[s, heads]), b_lse[s, heads], 1e-4)
        assert (np.abs(lse[s, heads] - r["lse"][s, heads]) <= b).all(), s


@pytest.mark.parametrize("heads", [4, 16, 50])
def test_lengths_and_pages_that_are_none(ctx, heads):
    args = cache([100, 40, 70], heads, 2, 64, 16, BF, seed=10)
    q, k, v, k_off, k_pages, v_pages, pages, length = args
    whole = binding.cache_attention(ctx, q, k_pages, v_pages, pages, length)
    for bad in (-1, pages.shape[1] * 16 + 1, 2 ** 31 - 1, -2 ** 31):
        wrong = length.clone()
        wrong[1] = bad
        out, lse = binding.cache_attention(ctx, q, k_pages, v_pages, pages, wrong)
        assert ctx.check() == binding.DEV_BAD_LENGTH
        assert not out[1].any() and (lse[1] == -math.inf).all()
        assert torch.equal(out[0], whole[0][0]) and torch.equal(lse[2], whole[1][2])
    for bad in (-1, k_pages.shape[0], 2 ** 31 - 1):
        wrong = pages.clone()
        wrong[0, 2] = bad                            # keys 32 .. 47 of the first sequence
        out, lse = binding.cache_attention(ctx, q, k_pages, v_pages, wrong, length)
        assert ctx.check() == binding.DEV_BAD_PAGE
        assert torch.equal(out[1:], whole[0][1:])
        left = torch.cat([torch.arange(32), torch.arange(48, 100)]).cuda()
        r = reference(q[:1], k[left], v[left], torch.tensor([0, 1]), torch.tensor([0, 84]), True, 64 ** -0.5)
        b_out, b_lse = bounds(r, BF, 64, 84)
        near(out[:1], r["out"], b_out, "out")
        near(lse[:1], r["lse"], b_lse, "lse")


@pytest.mark.parametrize("heads", [2, 8, 300])
def test_a_bucket_that_is_none(ctx, heads):
    q, k, v, k_off, k_pages, v_pages, pages, length = cache([100], heads, 1, 32, 16, BF, seed=11)
    how = biased(heads, 20, 12, BF)
    right = how["bucket"].clone()
    right[5] = 0
    want = binding.cache_attention(ctx, q, k_pages, v_pages, pages, length, bias=how["bias"], bucket=right)
    for bad in (-1, 12, 2 ** 31 - 1):
        wrong = right.clone()
        wrong[5] = bad
        got = binding.cache_attention(ctx, q, k_pages, v_pages, pages, length, bias=how["bias"], bucket=wrong)
        assert ctx.check() == binding.DEV_BAD_BUCKET
        assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_nothing_is_written_behind_the_outputs(ctx):
    q, k, v, k_off, k_pages, v_pages, pages, length = cache([70, 0, 5], 6, 2, 40, 16, HF, seed=12)
    out = torch.full((3 * 6 * 40 + 64,), 7.0, device="cuda").half()
    lse = torch.full((3 * 6 + 64,), 7.0, device="cuda")
    import ctypes
    c = binding._cache(k_pages, v_pages)
    a = binding.CacheAttentionArgs(q.data_ptr(), *q.stride()[:2], pages.data_ptr(), length.data_ptr(), 3, pages.shape[1], 6,
                                   0.2, None, None, 0, 0)
    assert binding.load().surel_cache_attention(ctx.handle, ctypes.byref(c), ctypes.byref(a), out.data_ptr(), lse.data_ptr()) == 0
    assert ctx.check() == 0
    assert (out[720:] == 7).all() and (lse[18:] == 7).all()
    want = binding.cache_attention(ctx, q, k_pages, v_pages, pages, length, scale=0.2)
    assert torch.equal(out[:720].view(3, 6, 40), want[0]) and torch.equal(lse[:18].view(3, 6), want[1])


def test_a_stream_of_its_own_and_a_graph_for_any_lengths(ctx):
    q, k, v, k_off, k_pages, v_pages, pages, length = cache([3000, 0, 77, 2500], 8, 2, 64, 16, BF, seed=13)
    side = torch.cuda.Stream()
    own = binding.Context(0, stream=side)
    side.wait_stream(torch.cuda.current_stream())
    lengths = length.clone()
    with torch.cuda.stream(side):
        binding.cache_attention(own, q, k_pages, v_pages, pages, lengths)   # (grows what it needs)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = binding.cache_attention(own, q, k_pages, v_pages, pages, lengths)
    # an eager call that needs more, in between: the captured one goes on using what it was captured with
    more = cache([6000] * 3, 64, 2, 64, 16, BF, seed=14)
    for now in ([3000, 0, 77, 2500], [1, 0, 0, 2000], [0, 0, 0, 0], [2999, 0, 5, 2500]):
        lengths.copy_(torch.tensor(now, dtype=torch.int32))
        torch.cuda.synchronize()
        binding.cache_attention(own, more[0], *more[4:])
        with torch.cuda.stream(side):    # (calls of one context do not overlap)
            graph.replay()
        torch.cuda.synchronize()
        want = binding.cache_attention(ctx, q, k_pages, v_pages, pages, lengths)
        assert all(torch.equal(x, y) for x, y in zip(got, want)), now
    assert own.check() == 0
    own.close()


def test_two_contexts_at_once(ctx):
    args = cache([5000, 1200, 3], 8, 1, 128, 16, BF, seed=15)
    q, _, _, _, k_pages, v_pages, pages, length = args
    want = binding.cache_attention(ctx, q, k_pages, v_pages, pages, length)
    torch.cuda.synchronize()
    both = [binding.Context(0, stream=torch.cuda.Stream()) for _ in range(2)]
    got = [binding.cache_attention(both[i % 2], q, k_pages, v_pages, pages, length) for i in range(8)]
    torch.cuda.synchronize()
    for c in both:
        assert c.check() == 0
        c.close()
    assert all(torch.equal(x, y) for pair in got for x, y in zip(pair, want))


def test_long_caches_pass_32_bits(ctx):
    """Keys behind more than 4 GiB of pages, and a table of more than 2^16 of them."""
    n_pages, page_rows, kv_heads, dim = 140_000, 16, 8, 128      # 4.3 GiB each of keys and values
    k_pages = torch.zeros((n_pages, page_rows, kv_heads, dim), dtype=BF, device="cuda")
    v_pages = torch.zeros_like(k_pages)
    q = torch.randn(1, 8, dim, device="cuda").to(BF)
    length = torch.tensor([40], dtype=torch.int32, device="cuda")
    pages = torch.tensor([[n_pages - 1, 5, n_pages - 2]], dtype=torch.int32, device="cuda")
    k, v = torch.randn(40, kv_heads, dim, device="cuda").to(BF), torch.randn(40, kv_heads, dim, device="cuda").to(BF)
    slots = (pages[0].long()[torch.arange(40) // 16] * 16 + torch.arange(40, device="cuda") % 16).int()
    binding.cache_store(ctx, k, v, slots, k_pages, v_pages)
    check(ctx, q, k, v, torch.tensor([0, 40]), k_pages, v_pages, pages, length)
