"""What fp16 can hold: score gradients of large values and of rows whose gradients are far smaller than others', weights of
values over many keys, and weights far below the largest."""
import numpy as np
import pytest
import torch

from attention_cases import UNIT, inputs, offsets, reference
from paper_2202_13538_amd import binding
from test_gpu_attention import HF, bounds, near

pytestmark = pytest.mark.gpu
U = UNIT[HF]


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    assert c.check() == 0
    c.close()


def gradients(ctx, q, k, v, dout, q_off, k_off, scale, causal=False):
    """Gradients, held to bounds without any step of fp16 but that of the results: weights and score gradients are rounded
    (one unit each), delta comes from a rounded out (2.25), the result is rounded (1); a quarter is for 32-bit scores and sums."""
    out, lse = binding.attention(ctx, q, k, v, q_off, k_off, causal=causal, scale=scale)
    got = binding.attention_grad(ctx, dout, q, k, v, out, lse, q_off, k_off, causal=causal, scale=scale)
    r = reference(q, k, v, q_off, k_off, causal, scale, dout=dout)
    for name, x in zip(("dq", "dk", "dv"), got):
        assert np.abs(r[name]).max() < 60000, "the case itself leaves fp16"
        units = 2.25 if name == "dv" else 4.5
        near(x, r[name], units * U * r["abs_" + name] + 2.0 ** -24, name)
    return got


def test_three_keys_with_one_large_value(ctx):
    """ds is 95,990 and -47,995 twice, dq 3,394."""
    q = torch.zeros(1, 1, 128, dtype=HF, device="cuda")
    k, v = torch.empty(3, 1, 128, dtype=HF, device="cuda"), torch.zeros(3, 1, 128, dtype=HF, device="cuda")
    k[0], k[1:], v[0] = 0.5, 0.1, 3750.0
    dout = torch.full_like(q, 0.9)
    gradients(ctx, q, k, v, dout, offsets([1]), offsets([3]), 128 ** -0.5)


@pytest.mark.parametrize("size", [1e-4, 3000.0])
@pytest.mark.parametrize("lens,k_lens", [([16] * 20, None), ([70, 150, 90], None), ([3, 1], [500, 300])], ids=str)
def test_large_and_small_values(ctx, lens, k_lens, size):
    q, k, v, q_off, k_off, _ = inputs(lens, k_lens, 4, 2, 96, HF, seed=1)
    dout = torch.randn(q.shape, generator=torch.Generator().manual_seed(2)).half().cuda()
    gradients(ctx, (q * 0.5).half(), (k * 0.5).half(), (v * size).half(), dout, q_off, k_off, 96 ** -0.5, causal=k_lens is None)


@pytest.mark.parametrize("n", [2, 600])
def test_subnormal_values_that_cancel(ctx, n):
    """delta is zero, values are below fp16's smallest normal number, score gradients are not zero."""
    sign = torch.ones(n, 1, 1, device="cuda")
    sign[::2] = -1
    q = torch.zeros(3, 1, 128, dtype=HF, device="cuda")
    k, v = (100 * sign).half().expand(n, 1, 128).contiguous(), (4e-5 * sign).half().expand(n, 1, 128).contiguous()
    gradients(ctx, q, k, v, torch.full_like(q, 0.9), offsets([3]), offsets([n]), 128 ** -0.5)


@pytest.mark.parametrize("lens", [[16] * 12, [600]], ids=str)
def test_rows_with_far_smaller_gradients_than_others(ctx, lens):
    q, k, v, off, _, _ = inputs(lens, None, 2, 1, 32, HF, seed=3)
    dout = torch.randn(q.shape, generator=torch.Generator().manual_seed(4)).cuda()
    dout[::2] *= 1e-4
    # (keys in place of queries are large: gradients of queries then are well inside fp16)
    gradients(ctx, (q / 64).half(), (k * 64).half(), v, dout.half(), off, off, 32 ** -0.5)


@pytest.mark.parametrize("lens", [[20] * 12, [300, 280]], ids=str)
def test_sequences_with_far_smaller_gradients_than_others(ctx, lens):
    q, k, v, off, _, _ = inputs(lens, None, 2, 1, 32, HF, seed=5)
    dout = torch.randn(q.shape, generator=torch.Generator().manual_seed(6)).cuda()
    dout[:sum(lens) // 2] *= 1e-4
    dout[sum(lens) // 2:] *= 10
    gradients(ctx, (q * 64).half(), (k / 64).half(), v, dout.half(), off, off, 32 ** -0.5)


def test_values_over_many_keys_seen_alike(ctx):
    """All weights are 1 / n, 100.5 of fp16's smallest steps: rounded as they are, they would be half a percent off."""
    n, rows = 166_937, 64
    g = torch.Generator().manual_seed(7)
    q = torch.zeros(rows, 1, 8, dtype=HF, device="cuda")
    k, v = torch.randn(n, 1, 8, generator=g).half().cuda(), torch.zeros(n, 1, 8, dtype=HF, device="cuda")
    dout = (torch.rand(rows, 1, 8, generator=g) + 0.5).half().cuda()
    offs = offsets([rows]), offsets([n])
    out, lse = binding.attention(ctx, q, k, v, *offs)
    dv = binding.attention_grad(ctx, dout, q, k, v, out, lse, *offs)[2].double()
    want = dout.double().sum(0) / n
    assert ((dv - want).abs() <= 2.25 * U * want).all(), ((dv - want).abs() / want).max().item()


SINKS = [([1], [512], 1), ([1], [512], 300), ([300], [512], 1), ([1] * 600, [512] * 600, 1)]  # few rows, one wave a tile, 128 rows


@pytest.mark.parametrize("q_lens,k_lens,heads", SINKS, ids=lambda x: str(x) if not isinstance(x, list) else f"{len(x)}x{x[0]}")
def test_weights_far_below_the_largest(ctx, q_lens, k_lens, heads):
    """One key of 32 scores 11.75, the others 0: their weights are 132.4 of fp16's smallest steps of the largest."""
    n = sum(k_lens)
    q, k = torch.zeros(sum(q_lens), heads, 8, dtype=HF, device="cuda"), torch.zeros(n, heads, 8, dtype=HF, device="cuda")
    v = torch.ones(n, heads, 8, dtype=HF, device="cuda")
    q[..., 0] = 4.0
    k[7::32, :, 0], v[7::32] = 2.9375, 0.0
    out, lse = binding.attention(ctx, q, k, v, offsets(q_lens), offsets(k_lens), scale=1.0)
    r = reference(q[:1, :1], k[:512, :1], v[:512, :1], offsets([1]), offsets([512]), False, 1.0)
    b_out, b_lse = bounds(r, HF, 8, 512)
    shape = tuple(out.shape)
    near(lse, np.broadcast_to(r["lse"], shape[:2]), np.broadcast_to(b_lse, shape[:2]), "lse")
    near(out, np.broadcast_to(r["out"], shape), np.broadcast_to(b_out, shape), "out")
