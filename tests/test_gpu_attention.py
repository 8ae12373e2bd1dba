"""surel_attention on the GPU against attention in 64 bits."""
import numpy as np
import pytest
import torch

from attention_cases import UNIT, inputs, offsets, reference
from paper_2202_13538_amd import binding

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    assert c.check() == 0
    c.close()


def near(got, want, bound, what):
    got = got.detach().cpu().double().numpy()
    fine = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), fine), f"{what}: other entries are finite"
    assert np.array_equal(got[~fine], want[~fine], equal_nan=True), f"{what}: infinities and NaN differ"
    off = np.abs(got[fine] - want[fine]) - bound[fine]
    assert off.size == 0 or off.max() <= 0, f"{what}: {off.max():.3g} over its bound"


def bounds(r, dtype, dim, n_keys):
    """Weights are rounded to 16 bits (one unit of sum p|v|), the result is too (one unit of |out| <= sum p|v|); what
    32-bit scores and sums add is far below the quarter unit left over: (dim + n_keys) 2^-24 of |s| and of the
    sum.  lse: a 32-bit dot product of dim terms, a sum of n_keys terms, exp2 and log2 of 2 units."""
    slack = 2.0 ** -24 * (dim + 8) * r["abs_s"] + 2.0 ** -24 * (n_keys + 16)
    finite = np.where(np.isfinite(r["lse"]), np.abs(r["lse"]), 0)
    return 2.25 * UNIT[dtype] * r["abs_out"] + 2 * slack[..., None] * r["abs_out"] + \
        (2.0 ** -25 if dtype == HF else 0), slack + 2.0 ** -22 * (1 + finite)


def check(ctx, q, k, v, q_off, k_off, causal, how, scale=None, want=None):
    out, lse = binding.attention(ctx, q, k, v, q_off, k_off, causal=causal, scale=scale, **how)
    r = want or reference(q, k, v, q_off, k_off, causal, q.shape[2] ** -0.5 if scale is None else scale, **how)
    b_out, b_lse = bounds(r, q.dtype, q.shape[2], k.shape[0])
    near(lse, r["lse"], b_lse, "lse")
    near(out, r["out"], b_out, "out")
    return out, lse


SELF = [  # lengths, heads, kv_heads, dim
    ([1], 1, 1, 8), ([2, 1, 0, 3], 2, 1, 32), ([5] * 40, 4, 4, 16), ([16] * 33, 2, 2, 64),
    ([0, 0, 65, 0, 1, 130], 3, 1, 40), ([127, 128, 129], 4, 2, 128), ([300, 7], 6, 2, 96), ([33, 255, 64], 2, 2, 72),
    ([1] * 200, 2, 1, 24),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("shape", SELF, ids=str)
def test_sequences_that_attend_to_themselves(ctx, shape, biased, causal, dtype):
    lens, heads, kv_heads, dim = shape
    args = inputs(lens, None, heads, kv_heads, dim, dtype, seed=len(lens), causal=causal,
                  **(dict(reach=16, buckets=8) if biased else {}))
    check(ctx, *args[:5], causal, args[5])


CROSS = [  # q lengths, k lengths, heads, kv_heads, dim
    ([1] * 9, [1, 30, 0, 64, 129, 2, 500, 128, 33], 4, 2, 64), ([1], [2000], 8, 1, 128), ([1, 1], [700, 1501], 16, 2, 96),
    ([3, 0, 5], [40, 10, 300], 4, 4, 32), ([40, 7], [2, 600], 2, 1, 64), ([200, 1, 90], [333, 257, 90], 4, 4, 128),
    ([17], [1030], 6, 2, 80), ([4, 9], [0, 3], 2, 2, 16), ([130], [1], 1, 1, 8), ([2] * 50, [3] * 50, 32, 1, 32),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("shape", CROSS, ids=str)
def test_rows_that_attend_to_other_keys(ctx, shape, biased, causal, dtype):
    q_lens, k_lens, heads, kv_heads, dim = shape
    args = inputs(q_lens, k_lens, heads, kv_heads, dim, dtype, seed=sum(k_lens), causal=causal,
                  **(dict(reach=40, buckets=12) if biased else {}))
    check(ctx, *args[:5], causal, args[5])


@pytest.mark.parametrize("reach,buckets", [(0, 1), (1, 3), (128, 32), (1024, 64)])
def test_reaches(ctx, reach, buckets):
    q, k, v, off, _, _ = inputs([700], None, 2, 1, 32, BF, seed=reach)
    g = torch.Generator().manual_seed(reach)
    how = dict(bias=torch.randn(buckets, 2, generator=g).to(BF).cuda(),
               bucket=torch.randint(0, buckets, (2 * reach + 1,), generator=g).int().cuda())
    check(ctx, q, k, v, off, off, False, how)


def test_views_of_one_larger_tensor(ctx):
    g = torch.Generator().manual_seed(5)
    both = torch.randn(90, 4 + 2 + 2, 48, generator=g).to(BF).cuda()
    q, k, v = both[:, :4], both[:, 4:6], both[:, 6:]
    off = offsets([50, 40])
    check(ctx, q, k, v, off, off, True, {})
    heads_first = torch.randn(4, 90, 48, generator=g).to(BF).cuda().transpose(0, 1)   # rows lie inside heads
    check(ctx, heads_first, k, v, off, off, False, {})
    shared = torch.randn(90, 1, 48, generator=g).to(BF).cuda().expand(90, 2, 48)      # one key head, seen as two
    check(ctx, q, shared, shared, off, off, False, {})


def test_large_scores_and_scales(ctx):
    q, k, v, off, _, _ = inputs([200], None, 2, 2, 64, BF, seed=9)
    check(ctx, q * 8, k * 8, v, off, off, True, {})
    check(ctx, q, k, v, off, off, False, {}, scale=3.0)
    check(ctx, q, k, v, off, off, False, {}, scale=1e-3)
    ramp = k * torch.linspace(0.1, 20, 200, device="cuda", dtype=BF)[:, None, None]   # maxima that keep growing
    check(ctx, q, ramp, v, off, off, False, {})


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("lens", [[16] * 20, [70, 150, 90]], ids=str)
def test_what_a_row_does_not_see_has_no_influence(ctx, lens, where, bad):
    """One row of keys or values in the middle is not finite: rows before it and other sequences stay as they are."""
    q, k, v, off, _, _ = inputs(lens, None, 2, 2, 64, BF, seed=4)
    clean, clean_lse = binding.attention(ctx, q, k, v, off, causal=True)
    row = int(off[len(lens) // 2]) + lens[len(lens) // 2] // 2
    (k if where == "k" else v)[row, 0, 3] = bad
    out, lse = binding.attention(ctx, q, k, v, off, causal=True)
    s = len(lens) // 2
    touched = torch.zeros(sum(lens), 2, dtype=torch.bool, device="cuda")
    touched[row:int(off[s + 1]), 0] = True
    r = reference(q, k, v, off, off, True, 0.125)
    want = torch.from_numpy(r["out"]).cuda()
    assert torch.isfinite(out[~touched].float()).all()
    # rows that are gone over once more keep their weights in 32 bits
    assert ((out.double() - want).abs()[~touched] <= (2.25 * UNIT[BF] * torch.from_numpy(r["abs_out"]).cuda())[~touched] + 1e-6).all()
    assert torch.equal(lse[~touched], clean_lse[~touched]) or (lse[~touched] - clean_lse[~touched]).abs().max() < 1e-5
    assert torch.equal(torch.isnan(out[touched]), torch.isnan(want[touched].to(BF)))


def test_results_are_the_same_every_time(ctx):
    q, k, v, q_off, k_off, how = inputs([1, 1, 1], [900, 40, 2000], 8, 2, 64, HF, seed=3, reach=32, buckets=16)
    first = binding.attention(ctx, q, k, v, q_off, k_off, **how)
    for _ in range(3):
        again = binding.attention(ctx, q, k, v, q_off, k_off, **how)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_a_stream_of_its_own_and_a_graph(ctx):
    side = torch.cuda.Stream()
    q, k, v, q_off, k_off, how = inputs([1, 1, 60], [900, 40, 2000], 8, 2, 64, HF, seed=3, reach=32, buckets=16)
    want = binding.attention(ctx, q, k, v, q_off, k_off, causal=True, **how)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        own = binding.Context(0)
        got = binding.attention(own, q, k, v, q_off, k_off, causal=True, **how)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = binding.attention(own, q, k, v, q_off, k_off, causal=True, **how)
    for turn in range(3):
        q.copy_(torch.randn(q.shape, device="cuda"))
        want = binding.attention(ctx, q, k, v, q_off, k_off, causal=True, **how)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), turn
    assert own.check() == 0
    own.close()


def test_offsets_that_do_not_fit_are_reported(ctx):
    own = binding.Context(0)
    q, k, v, off, _, how = inputs([20, 30], None, 2, 2, 32, BF, reach=4, buckets=6)
    for bad in ([0, 60, 50], [0, 20, 49], [1, 20, 50], [0, -5, 50], [0, 2 ** 40, 50], [0, 20, 2 ** 33]):
        binding.attention(own, q, k, v, torch.tensor(bad, device="cuda"))
        assert own.check() == binding.DEV_BAD_OFFSETS, bad
        binding.attention(own, q, k, v, off, torch.tensor(bad, device="cuda"), causal=True)
        assert own.check() == binding.DEV_BAD_OFFSETS, bad
    wrong = how["bucket"].clone()
    wrong[3] = 6
    binding.attention(own, q, k, v, off, bias=how["bias"], bucket=wrong)
    assert own.check() == binding.DEV_BAD_BUCKET
    binding.attention(own, q, k, v, off, **how)
    assert own.check() == 0
    own.close()


def test_nothing_to_do(ctx):
    empty = torch.zeros(0, 2, 32, dtype=BF, device="cuda")
    some = torch.randn(5, 2, 32, device="cuda").to(BF)
    zero, five = offsets([0]), offsets([5])
    out, lse = binding.attention(ctx, empty, some, some, zero, five)
    assert out.shape == (0, 2, 32) and lse.shape == (0, 2)
    out, lse = binding.attention(ctx, some, empty, empty, five, zero)
    assert not out.any() and (lse == -float("inf")).all()


def test_offsets_of_elements_beyond_32_bits(ctx):
    """Keys and values of 2.2e9 elements each: the last sequence lies past 4 GiB."""
    n, dim = 17_200_000, 128
    k = torch.zeros(n, 1, dim, dtype=BF, device="cuda")
    v = torch.zeros(n, 1, dim, dtype=BF, device="cuda")
    g = torch.Generator().manual_seed(1)
    k[-300:] = torch.randn(300, 1, dim, generator=g).to(BF).cuda()
    v[-300:] = torch.randn(300, 1, dim, generator=g).to(BF).cuda()
    q = torch.randn(2, 4, dim, generator=g).to(BF).cuda()
    q_off, k_off = torch.tensor([0, 1, 2], device="cuda"), torch.tensor([0, n - 300, n], device="cuda")
    out, lse = binding.attention(ctx, q, k, v, q_off, k_off)
    r = reference(q[1:], k[-300:], v[-300:], offsets([1]), offsets([300]), False, dim ** -0.5)
    b_out, b_lse = bounds(r, BF, dim, 300)
    near(out[1:], r["out"], b_out, "out")
    near(lse[1:], r["lse"], b_lse, "lse")
    assert not out[0].any() and torch.allclose(lse[0], torch.full((4,), float(np.log(n - 300)), device="cuda"), rtol=1e-5)


MASKED = [  # lengths, keys' lengths or None, heads, kv_heads, dim
    ([1, 16, 0, 16, 5], None, 2, 1, 32), ([300, 7], None, 4, 2, 64), ([200], None, 1, 1, 128), ([9, 2], [700, 3], 4, 2, 64),
    ([1, 1, 1], [900, 2, 3000], 2, 1, 96), ([1] * 40, [3] * 40, 4, 4, 40),
]


def masked_inputs(shape, dtype, value, which):
    """Inputs whose bias masks some distances, and what stands for them in 64 bits: (args, how, bias with -100 for
    the mask, rows that it leaves nothing)."""
    q_lens, k_lens, heads, kv_heads, dim = shape
    q, k, v, q_off, k_off, how = inputs(q_lens, k_lens, heads, kv_heads, dim, dtype, seed=sum(q_lens), reach=16, buckets=9)
    near = torch.arange(-16, 17).abs()
    hidden = {"own": near == 0, "far": near == 16, "all": near >= 0}[which]
    bucket = torch.where(hidden, 8, near % 8).int().cuda()
    bias, stands = how["bias"].clone(), how["bias"].clone()
    bias[8], stands[8] = value, -100.0
    empty = torch.zeros(sum(q_lens), dtype=torch.bool)
    off_q, off_k = q_off.tolist(), k_off.tolist()
    for s in range(len(q_lens)):
        for i in range(off_q[s], off_q[s + 1]):
            at = off_k[s + 1] - (off_q[s + 1] - i)
            seen = torch.arange(off_k[s], min(at + 1, off_k[s + 1]))
            empty[i] = bool(hidden[(seen - at).clamp(-16, 16) + 16].all())
    return (q, k, v, q_off, k_off), dict(bias=bias, bucket=bucket), dict(bias=stands, bucket=bucket), empty


@pytest.mark.parametrize("dtype,value", [(BF, -float("inf")), (BF, torch.finfo(BF).min), (HF, torch.finfo(HF).min)], ids=str)
@pytest.mark.parametrize("which", ["own", "far", "all"])
@pytest.mark.parametrize("shape", MASKED, ids=str)
def test_a_bias_that_masks(ctx, shape, which, dtype, value):
    args, how, stands, empty = masked_inputs(shape, dtype, value, which)
    out, lse = binding.attention(ctx, *args, causal=True, **how)
    assert not out[empty].any() and (lse[empty] == -float("inf")).all()
    r = reference(*args, True, shape[4] ** -0.5, **stands)
    b_out, b_lse = bounds(r, dtype, shape[4], args[1].shape[0])
    some = ~empty.numpy()
    near(out[~empty], r["out"][some], b_out[some], "out")
    near(lse[~empty], r["lse"][some], b_lse[some], "lse")
