"""surel_attention where a key or value is not finite: rows that see it get what the formula gives, others stay as they are,
in every kernel that rows are put into (tiles of 128 rows, of 32 with four waves or one, keys in parts)."""
import pytest
import torch

from attention_cases import inputs, reference
from paper_2202_13538_amd import binding
from test_gpu_attention import BF, HF, bounds, near

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    assert c.check() == 0
    c.close()


SHAPES = [  # q lengths, k lengths, heads, kv_heads, dim, causal
    ([1], [200], 1, 1, 64, False), ([1, 1], [130, 64], 4, 1, 64, False), ([3, 0, 5], [40, 10, 300], 4, 4, 32, True),
    ([1, 1], [2000, 700], 8, 2, 96, False), ([7], [1030], 6, 2, 80, True), ([200], [333], 2, 2, 128, True),
    ([1, 2] * 35, [23, 40, 0, 7, 33] * 14, 8, 8, 40, True),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("where,bad", [("k", float("nan")), ("v", float("nan")), ("v", float("inf"))])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{sum(s[0])}x{sum(s[1])}x{s[2]}x{s[4]}")
def test_a_key_that_is_not_finite(ctx, shape, where, bad, dtype):
    """At a place in each of the blocks of 32 keys that a tile of four waves takes, and at the last key."""
    q_lens, k_lens, heads, kv_heads, dim, causal = shape
    q, k, v, q_off, k_off, _ = inputs(q_lens, k_lens, heads, kv_heads, dim, dtype, seed=dim)
    n = sum(k_lens)
    for row in sorted({5, 37, min(70, n - 2), min(101, n - 3), n - 1}):
        bad_k, bad_v = k.clone(), v.clone()
        (bad_k if where == "k" else bad_v)[row, kv_heads - 1, 3] = bad
        out, lse = binding.attention(ctx, q, bad_k, bad_v, q_off, k_off, causal=causal)
        r = reference(q, bad_k, bad_v, q_off, k_off, causal, dim ** -0.5)
        b_out, b_lse = bounds(r, dtype, dim, n)
        near(lse, r["lse"], b_lse, f"lse, key {row}")
        near(out, r["out"], b_out, f"out, key {row}")
