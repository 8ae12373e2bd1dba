"""The kernels that many rows are put into, against 64 bits: one wave a tile of 32 rows (512 tiles and more of few keys, or rows
of more than 64 elements over many), and gradients of 128 keys a workgroup.  Few distinct sequences and heads, repeated."""
import numpy as np
import pytest
import torch

from attention_cases import inputs, offsets, reference
from paper_2202_13538_amd import binding
from test_gpu_attention import BF, HF, bounds, masked_inputs, near
from test_gpu_attention_grad import bounds as grad_bounds

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    assert c.check() == 0
    c.close()


def lengths(lo, hi, n, seed):
    return torch.randint(lo, hi + 1, (n,), generator=torch.Generator().manual_seed(seed)).tolist()


def repeated(x, sequences, heads):
    """Rows [n][heads][...] (or offsets of sequences) that many times over."""
    return x.repeat(sequences, heads, *[1] * (x.dim() - 2))


def expect(r, names, sequences, heads):
    """What a reference and its bounds are for inputs that were repeated."""
    return {n: np.tile(r[n], (sequences, heads, 1)[:r[n].ndim]) for n in names if n in r}


ONE_WAVE = [  # q lengths, k lengths, heads, kv_heads, dim
    ([1] * 13, lengths(0, 40, 13, 1), 2, 2, 24), ([1] * 13, lengths(0, 40, 13, 2), 6, 2, 40),
    (lengths(0, 4, 13, 3), lengths(0, 60, 13, 4), 16, 2, 72), ([1] * 13, lengths(0, 300, 13, 5), 3, 1, 120),
    (lengths(1, 30, 13, 6), lengths(60, 200, 13, 7), 2, 2, 96),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("shape", ONE_WAVE, ids=lambda s: f"{sum(s[0])}x{sum(s[1])}x{s[2]}x{s[4]}")
def test_one_wave_a_tile(ctx, shape, biased, causal, dtype):
    q_lens, k_lens, heads, kv_heads, dim = shape
    q, k, v, q_off, k_off, how = inputs(q_lens, k_lens, heads, kv_heads, dim, dtype, seed=dim, causal=causal,
                                        **(dict(reach=16, buckets=8) if biased else {}))
    r = reference(q, k, v, q_off, k_off, causal, dim ** -0.5, **how)
    r["bound"], r["lse_bound"] = bounds(r, dtype, dim, max(k_lens))
    times, more = 24, 2   # 312 sequences of 2 or 4 key heads
    want = expect(r, ("out", "lse", "bound", "lse_bound"), times, more)
    if biased:
        how["bias"] = how["bias"].repeat(1, more)
    out, lse = binding.attention(ctx, repeated(q, times, more), repeated(k, times, more), repeated(v, times, more),
                                 offsets(q_lens * times), offsets(k_lens * times), causal=causal, **how)
    near(lse, want["lse"], want["lse_bound"], "lse")
    near(out, want["out"], want["bound"], "out")


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("biased", [False, True])
def test_one_wave_a_tile_over_many_keys(ctx, biased, dtype):
    q_lens, k_lens = [1, 1, 2], [30_000, 1, 12_345]
    q, k, v, q_off, k_off, how = inputs(q_lens, k_lens, 6, 2, 72, dtype, seed=1, causal=True,
                                        **(dict(reach=40, buckets=12) if biased else {}))
    r = reference(q, k, v, q_off, k_off, True, 72 ** -0.5, **how)
    out, lse = binding.attention(ctx, q, k, v, q_off, k_off, causal=True, **how)
    b_out, b_lse = bounds(r, dtype, 72, max(k_lens))
    near(lse, r["lse"], b_lse, "lse")
    near(out, r["out"], b_out, "out")


@pytest.mark.parametrize("dtype,value", [(BF, -float("inf")), (HF, torch.finfo(HF).min)], ids=str)
@pytest.mark.parametrize("which", ["own", "far", "all"])
@pytest.mark.parametrize("dim", [40, 128])
def test_one_wave_a_tile_and_a_bias_that_masks(ctx, dim, which, dtype, value):
    q_lens, k_lens = [1, 2, 0, 1], [30, 3, 5, 70]
    shape = (q_lens, k_lens, 6, 2, dim)
    args, how, stands, empty = masked_inputs(shape, dtype, value, which)
    r = reference(*args, True, dim ** -0.5, **stands)
    r["bound"], r["lse_bound"] = bounds(r, dtype, dim, max(k_lens))
    times = 80   # 320 sequences of 2 key heads
    want = expect(r, ("out", "lse", "bound", "lse_bound"), times, 1)
    out, lse = binding.attention(ctx, *(repeated(t, times, 1) for t in args[:3]), offsets(q_lens * times), offsets(k_lens * times),
                                 causal=True, **how)
    none = empty.repeat(times)
    assert not out[none].any() and (lse[none] == -float("inf")).all()
    some = ~none.numpy()
    near(lse[~none], want["lse"][some], want["lse_bound"][some], "lse")
    near(out[~none], want["out"][some], want["bound"][some], "out")


def check_gradients(ctx, q_lens, k_lens, heads, kv_heads, dim, dtype, causal, how_many, times, more):
    q, k, v, q_off, k_off, how = inputs(q_lens, k_lens, heads, kv_heads, dim, dtype, seed=dim, causal=causal, **how_many)
    dout = torch.randn(q.shape, generator=torch.Generator().manual_seed(3)).to(dtype).cuda()
    r = reference(q, k, v, q_off, k_off, causal, dim ** -0.5, dout=dout, **how)
    b = {n: np.broadcast_to(x, r[n].shape) for n, x in grad_bounds(r, q, k, v, dout, dim ** -0.5).items()}
    names = ("dq", "dk", "dv", "dbias")
    want, bound = expect(r, names[:3], times, more), expect(b, names[:3], times, more)
    if how:
        how["bias"] = how["bias"].repeat(1, more)
        want["dbias"], bound["dbias"] = (np.tile(x["dbias"], (1, more)) * times for x in (r, b))
    big_q, big_k, big_v, big_dout = (repeated(t, times, more) for t in (q, k, v, dout))
    off = offsets(q_lens * times)
    offs = (off, off if k_lens is None else offsets(k_lens * times))
    out, lse = binding.attention(ctx, big_q, big_k, big_v, *offs, causal=causal, **how)
    got = binding.attention_grad(ctx, big_dout, big_q, big_k, big_v, out, lse, *offs, causal=causal, **how)
    for name, x in zip(names, got):
        if name in want:
            near(x, want[name], bound[name], name)
        else:
            assert x is None
    return got


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("heads,kv_heads,dim", [(2, 2, 24), (4, 2, 64), (2, 1, 80), (3, 1, 128)])
def test_gradients_of_128_keys_of_short_sequences(ctx, heads, kv_heads, dim, biased, causal, dtype):
    lens = lengths(0, 20, 17, dim)
    lens[3], lens[4], lens[5] = 0, 1, 150   # (sequences that share a tile with others, and one that fills more than one)
    times, more = 40, 8 // kv_heads        # 8 key heads of more than 40 * 150 rows: 375 tiles of 128
    check_gradients(ctx, lens, None, heads, kv_heads, dim, dtype, causal, dict(reach=16, buckets=8) if biased else {}, times, more)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("q_lens,k_lens,heads,kv_heads,dim", [([130, 257], None, 2, 2, 64), ([40, 3], [300, 129], 4, 2, 96),
                                                              ([5], [700], 2, 1, 128)], ids=str)
def test_gradients_of_128_keys_of_longer_sequences(ctx, q_lens, k_lens, heads, kv_heads, dim, biased, causal, dtype):
    times = 16 // len(q_lens)
    more = 128 // kv_heads   # 128 key heads of 16 sequences: over 2,048 tiles of 128
    check_gradients(ctx, q_lens, k_lens, heads, kv_heads, dim, dtype, causal, dict(reach=40, buckets=12) if biased else {}, times, more)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_gradients_of_128_keys_beside_what_is_not_finite(ctx, dtype):
    """One sequence of many holds NaN in keys, values, rows and gradients: the others' gradients stay."""
    lens, times = [16, 9, 20], 400   # 18,000 rows of 4 heads: 562 tiles
    q, k, v, off, _, _ = inputs(lens, None, 4, 4, 64, dtype, seed=4)
    dout = torch.randn(q.shape, generator=torch.Generator().manual_seed(3)).to(dtype).cuda()
    r = reference(q, k, v, off, off, True, 0.125, dout=dout)
    b = grad_bounds(r, q, k, v, dout, 0.125)
    want, bound = expect(r, ("dq", "dk", "dv"), times, 1), expect(b, ("dq", "dk", "dv"), times, 1)
    q, k, v, dout = (repeated(t, times, 1) for t in (q, k, v, dout))
    off = offsets(lens * times)
    s = 200
    row = int(off[s]) + lens[s % 3] // 2
    for t in (q, k, v, dout):
        t[row, :, 3] = float("nan")
    out, lse = binding.attention(ctx, q, k, v, off, causal=True)
    got = binding.attention_grad(ctx, dout, q, k, v, out, lse, off, causal=True)
    keep = torch.ones(len(q), dtype=torch.bool)
    keep[int(off[s]):int(off[s + 1])] = False
    mask = keep.numpy()
    for name, x in zip(("dq", "dk", "dv"), got):
        near(x[keep], want[name][mask], bound[name][mask], name)
        assert torch.isnan(x[row].float()).any()
