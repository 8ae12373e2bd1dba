"""surel_attention_grad on the GPU against the gradients in 64 bits."""
import numpy as np
import pytest
import torch

from attention_cases import UNIT, inputs, offsets, reference
from paper_2202_13538_amd import binding
from test_gpu_attention import BF, CROSS, HF, MASKED, SELF, masked_inputs, near

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    assert c.check() == 0
    c.close()


def bounds(r, q, k, v, dout, scale):
    """In units of the 16-bit type: weights and score gradients are rounded for their products (1 each), delta comes
    from a rounded out (2.25 of p |do| |out|'s sum), results are rounded (1); the quarter on top covers 32-bit
    scores and sums.  fp16 also has a smallest step of 2^-24: of weights, of score gradients (in units of the
    power of two above the largest |dout|) and of results."""
    u, dtype = UNIT[q.dtype], q.dtype
    step = 2.0 ** -24 if dtype == HF else 0.0
    most = lambda t: float(t.double().abs().max()) if t.numel() else 0.0  # noqa: E731
    rows, keys, group = q.shape[0], k.shape[0], q.shape[1] // k.shape[1]
    lift = 2 * most(dout)
    return dict(dq=4.5 * u * r["abs_dq"] + step * (1 + keys * lift * most(k) * scale) + 1e-6 * r["abs_dq"].max(),
                dk=4.5 * u * r["abs_dk"] + step * (1 + rows * group * lift * most(q) * scale) + 1e-6 * r["abs_dk"].max(initial=0),
                dv=2.25 * u * r["abs_dv"] + step * (1 + rows * group * most(dout)) + 1e-6 * r["abs_dv"].max(initial=0),
                **(dict(dbias=3.5 * u * r["abs_dbias"] + step + 1e-6 * r["abs_dbias"].max()) if "dbias" in r else {}))


def check(ctx, q, k, v, q_off, k_off, causal, how, scale=None, std=1.0, dout=None):
    if dout is None:
        g = torch.Generator().manual_seed(77)
        dout = (torch.randn(q.shape, generator=g) * std).to(q.dtype).cuda()
    out, lse = binding.attention(ctx, q, k, v, q_off, k_off, causal=causal, scale=scale, **how)
    got = binding.attention_grad(ctx, dout, q, k, v, out, lse, q_off, k_off, causal=causal, scale=scale, **how)
    scale = q.shape[2] ** -0.5 if scale is None else scale
    r = reference(q, k, v, q_off, k_off, causal, scale, dout=dout, **how)
    b = bounds(r, q, k, v, dout, scale)
    for name, x in zip(("dq", "dk", "dv", "dbias"), got):
        if name in r:
            near(x, r[name], np.broadcast_to(b[name], r[name].shape), name)
        else:
            assert x is None
    return got


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("shape", SELF, ids=str)
def test_sequences_that_attend_to_themselves(ctx, shape, biased, causal, dtype):
    lens, heads, kv_heads, dim = shape
    args = inputs(lens, None, heads, kv_heads, dim, dtype, seed=len(lens), causal=causal,
                  **(dict(reach=16, buckets=8) if biased else {}))
    check(ctx, *args[:5], causal, args[5])


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


def test_many_short_sequences_share_a_bias(ctx):
    args = inputs([16] * 300, None, 2, 2, 32, BF, seed=8, causal=True, reach=15, buckets=16)
    check(ctx, *args[:5], True, args[5])


@pytest.mark.parametrize("std", [1e-4, 64.0])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_small_and_large_gradients(ctx, dtype, std):
    q, k, v, off, _, how = inputs([90, 200], None, 4, 2, 64, dtype, seed=2, reach=16, buckets=8)
    check(ctx, q, k, v, off, off, False, how, std=std)
    check(ctx, q, k, v, off, off, False, how, dout=torch.zeros_like(q))


def test_views_of_one_larger_tensor(ctx):
    g = torch.Generator().manual_seed(5)
    both = torch.randn(90, 4 + 2 + 2, 48, generator=g).to(BF).cuda()
    off = offsets([50, 40])
    check(ctx, both[:, :4], both[:, 4:6], both[:, 6:], off, off, True, {})
    heads_first = torch.randn(4, 90, 48, generator=g).to(BF).cuda().transpose(0, 1)
    check(ctx, heads_first, both[:, 4:6], both[:, 6:], off, off, False, {}, scale=0.7)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("lens", [[16] * 20, [70, 150, 90]], ids=str)
def test_other_sequences_have_no_influence(ctx, lens, bad):
    """One sequence holds what is not finite, in keys, values, rows and gradients: the others' gradients stay."""
    args = inputs(lens, None, 2, 2, 64, BF, seed=4)
    q, k, v, off = (t.clone() for t in args[:4])
    dout = torch.randn(q.shape, device="cuda").to(BF)
    s = len(lens) // 2
    row = int(off[s]) + lens[s] // 2
    for t in (q, k, v, dout):
        t[row, :, 3] = bad
    out, lse = binding.attention(ctx, q, k, v, off, causal=True)
    got = binding.attention_grad(ctx, dout, q, k, v, out, lse, off, causal=True)
    keep = torch.ones(sum(lens), dtype=torch.bool, device="cuda")
    keep[int(off[s]):int(off[s + 1])] = False
    clean_d = torch.where(torch.isfinite(dout), dout, 0)
    r = reference(args[0], args[1], args[2], off, off, True, 0.125, dout=clean_d)
    b = bounds(r, args[0], args[1], args[2], clean_d, 0.125)
    for name, x in zip(("dq", "dk", "dv"), got):
        mask = keep.cpu().numpy()
        near(x[keep], r[name][mask], b[name][mask], name)
        assert not torch.isfinite(x[~keep].float()).all()


def test_results_are_the_same_every_time_and_in_a_graph(ctx):
    q, k, v, off, _, how = inputs([300, 20, 129], None, 8, 2, 64, HF, seed=3, reach=32, buckets=16)
    dout = torch.randn(q.shape, device="cuda").half()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        own = binding.Context(0)
        step = lambda: binding.attention_grad(own, dout, q, k, v, *binding.attention(own, q, k, v, off, **how), off, **how)  # noqa: E731
        first = step()
        for _ in range(3):
            assert all(torch.equal(x, y) for x, y in zip(first, step()))
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step()
    for turn in range(3):
        dout.copy_(torch.randn(q.shape, device="cuda") * 10.0 ** -turn)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), turn
    assert own.check() == 0
    own.close()


def test_nothing_to_do(ctx):
    empty = torch.zeros(0, 2, 32, dtype=BF, device="cuda")
    some = torch.randn(5, 2, 32, device="cuda").to(BF)
    zero, five = offsets([0]), offsets([5])
    for q, k, qo, ko in ((empty, some, zero, five), (some, empty, five, zero), (empty, empty, zero, zero)):
        out, lse = binding.attention(ctx, q, k, k, qo, ko)
        for x in binding.attention_grad(ctx, torch.ones_like(q), q, k, k, out, lse, qo, ko)[:3]:
            assert not x.any()


@pytest.mark.parametrize("dtype,value", [(BF, -float("inf")), (BF, torch.finfo(BF).min), (HF, torch.finfo(HF).min)], ids=str)
@pytest.mark.parametrize("which", ["own", "far", "all"])
@pytest.mark.parametrize("shape", MASKED, ids=str)
def test_a_bias_that_masks(ctx, shape, which, dtype, value):
    """What it hides has no part in any gradient; rows that it leaves nothing have none."""
    args, how, stands, empty = masked_inputs(shape, dtype, value, which)
    dout = torch.randn(args[0].shape, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    out, lse = binding.attention(ctx, *args, causal=True, **how)
    got = binding.attention_grad(ctx, dout, *args[:3], out, lse, *args[3:], causal=True, **how)
    scale = shape[4] ** -0.5
    kept = torch.where(empty[:, None, None].cuda(), 0, dout)
    r = reference(*args, True, scale, dout=kept, **stands)
    b = bounds(r, *args[:3], dout, scale)
    assert not got[0][empty].any() and not got[3][8].any()
    for name, x in zip(("dq", "dk", "dv", "dbias"), got):
        near(x, r[name], np.broadcast_to(b[name], r[name].shape), name)
