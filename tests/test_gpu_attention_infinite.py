"""Infinite elements of keys that are seen: rows whose score is minus infinity leave the key out, whatever the width of a head."""
import numpy as np
import pytest
import torch

from attention_cases import inputs, reference
from paper_2202_13538_amd import binding
from test_gpu_attention import BF, HF, bounds, near
from test_gpu_attention_grad import bounds as grad_bounds
from test_gpu_attention_nonfinite import SHAPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [40, 64, 72, 128])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{sum(s[0])}x{sum(s[1])}x{s[2]}")
def test_scores_of_minus_infinity(shape, dim, dtype):
    q_lens, k_lens, heads, kv_heads, _, causal = shape
    ctx = binding.Context(0)
    q, k, v, q_off, k_off, _ = inputs(q_lens, k_lens, heads, kv_heads, dim, dtype, seed=dim)
    clean = reference(q, k, v, q_off, k_off, causal, dim ** -0.5)
    n = sum(k_lens)
    for row, value in ((5, 0.0), (n // 2, float("nan"))):
        bad_k, bad_v = k.clone(), v.clone()
        bad_k[row, kv_heads - 1, 3] = -float("inf")
        bad_v[row, kv_heads - 1] = value   # (0 times NaN: not a number where the key is seen)
        out, lse = binding.attention(ctx, q, bad_k, bad_v, q_off, k_off, causal=causal)
        r = reference(q, bad_k, bad_v, q_off, k_off, causal, dim ** -0.5)
        b_out, b_lse = bounds(dict(abs_s=clean["abs_s"], lse=r["lse"], abs_out=np.nan_to_num(r["abs_out"])), dtype, dim, n)
        near(lse, r["lse"], b_lse, f"lse, key {row}")
        near(out, r["out"], b_out, f"out, key {row}")
    assert ctx.check() == 0
    ctx.close()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [40, 64, 72, 104])
@pytest.mark.parametrize("lens,k_lens,causal", [([16] * 30, None, True), ([200, 70], None, False), ([3, 5], [300, 400], True)], ids=str)
def test_gradients_of_scores_of_minus_infinity(lens, k_lens, causal, dim, dtype):
    """A weight of zero: only the element of dq that it multiplies infinity in is not a number."""
    ctx = binding.Context(0)
    q, k, v, q_off, k_off, how = inputs(lens, k_lens, 4, 2, dim, dtype, seed=dim, reach=8, buckets=6, causal=causal)
    q[..., 3] = q[..., 3].abs() + 0.1
    dout = torch.randn(q.shape, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    clean = reference(q, k, v, q_off, k_off, causal, dim ** -0.5, dout=dout, **how)
    k[len(k) // 2 + 1, -1, 3] = -float("inf")   # (not the only key of any row: such a row has no weights)
    out, lse = binding.attention(ctx, q, k, v, q_off, k_off, causal=causal, **how)
    got = binding.attention_grad(ctx, dout, q, k, v, out, lse, q_off, k_off, causal=causal, **how)
    r = reference(q, k, v, q_off, k_off, causal, dim ** -0.5, dout=dout, **how)
    for name in ("dq", "dk"):
        # (their bounds' sums multiply the same zeros by infinity: what the other keys give there instead)
        r["abs_" + name] = np.where(np.isfinite(r["abs_" + name]), r["abs_" + name], clean["abs_" + name].max())
    b = grad_bounds(r, q, torch.where(k.isfinite(), k, 0), v, dout, dim ** -0.5)
    for name, x in zip(("dq", "dk", "dv", "dbias"), got):
        near(x, r[name], np.broadcast_to(b[name], r[name].shape), name)
    assert ctx.check() == 0
    ctx.close()
