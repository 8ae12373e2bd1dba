"""Calls of attention and loss whose workgroups have more than 2^32 threads together."""
import pytest
import torch

from paper_2202_13538_amd import binding

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    assert c.check() == 0
    c.close()
    torch.cuda.empty_cache()


def rows_over_three_keys(n, heads):
    """n single rows over 3 keys each, heads of 8 elements: the longest sums of products are small."""
    g = torch.Generator(device="cuda").manual_seed(n)
    normal = lambda rows: torch.empty(rows, heads, 8, dtype=BF, device="cuda").normal_(generator=g)  # noqa: E731
    one = torch.arange(n + 1, device="cuda")
    return normal(n), normal(3 * n), normal(3 * n), one, 3 * one


def dense(q, k, v, a, b):
    """Scores, weights and values of rows a .. b - 1 in 32 bits: [rows][heads][3], ..., [rows][heads][3][8]."""
    n, heads, dim = q[a:b].shape
    K, V = (x[3 * a:3 * b].float().view(n, 3, heads, dim).transpose(1, 2) for x in (k, v))
    s = (K * q[a:b].float()[:, :, None]).sum(-1) * dim ** -0.5
    return s, s.softmax(-1), K, V


PARTS = 16


def test_many_single_rows(ctx):
    """8.4 million rows of 8 heads: more than 2^26 workgroups of a wave."""
    q, k, v, q_off, k_off = rows_over_three_keys(8_400_001, 8)
    out, lse = binding.attention(ctx, q, k, v, q_off, k_off)
    step = len(q) // PARTS + 1
    for a in range(0, len(q), step):
        s, p, _, V = dense(q, k, v, a, a + step)
        want = (p[..., None] * V).sum(2)
        # weights and results are rounded to 8 bits: 2.25 units of sum p |v| (a quarter for 32 bits)
        assert ((out[a:a + step].float() - want).abs() <= 2.25 * 2.0 ** -8 * (p[..., None] * V.abs()).sum(2) + 1e-6).all()
        assert torch.allclose(lse[a:a + step], s.logsumexp(-1), rtol=1e-5, atol=1e-5)


def test_gradients_of_many_single_rows(ctx):
    """A pooling row for each of 1,048,576 queries with 16 heads: more than 2^24 workgroups of 256 threads."""
    q, k, v, q_off, k_off = rows_over_three_keys(1_048_576, 16)
    dout = torch.empty_like(q).normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    out, lse = binding.attention(ctx, q, k, v, q_off, k_off)
    dq, dk, dv, _ = binding.attention_grad(ctx, dout, q, k, v, out, lse, q_off, k_off)
    step, u = len(q) // PARTS, 2.0 ** -8
    for a in range(0, len(q), step):
        b = a + step
        s, p, K, V = dense(q, k, v, a, b)
        do, Q = dout[a:b].float()[:, :, None], q[a:b].float()[:, :, None]
        dp = (do * V).sum(-1)
        delta = (p * dp).sum(-1, keepdim=True)
        ds = p * (dp - delta)
        size = p * ((do * V).abs().sum(-1) + (p[..., None] * V.abs() * do.abs()).sum((-1, -2))[..., None])
        scale = 8 ** -0.5
        flat = lambda x: x.transpose(1, 2).reshape(-1, 16, 8)  # noqa: E731  [rows][heads][3][8] -> keys
        # (units of bfloat16: weights, score gradients, results 1 each, delta from a rounded out 2.25; a quarter for 32 bits)
        for got, want, bound in ((dq[a:b], (ds[..., None] * K).sum(2) * scale, 4.5 * u * (size[..., None] * K.abs()).sum(2) * scale),
                                 (dk[3 * a:3 * b], flat(ds[..., None] * Q) * scale, 4.5 * u * flat(size[..., None] * Q.abs()) * scale),
                                 (dv[3 * a:3 * b], flat(p[..., None] * do), 2.25 * u * flat(p[..., None] * do.abs()))):
            assert ((got.float() - want).abs() <= bound + 1e-6).all()


def test_a_loss_of_many_rows(ctx):
    """More than 2^26 rows."""
    n, classes, dim = 67_200_003, 5, 8
    g = torch.Generator(device="cuda").manual_seed(2)
    h = torch.empty(n, dim, dtype=BF, device="cuda").normal_(generator=g)
    w = torch.empty(classes, dim, dtype=BF, device="cuda").normal_(generator=g)
    labels = torch.randint(-1, classes, (n,), dtype=torch.int32, device="cuda", generator=g)
    loss, lse = binding.softmax_loss(ctx, h, w, labels)
    step = n // PARTS + 1
    for a in range(0, n, step):
        z = h[a:a + step].float() @ w.float().t()
        want = z.logsumexp(1)
        at = labels[a:a + step].long()
        hit = z.gather(1, at.clamp(min=0)[:, None])[:, 0]
        # 32-bit products of 8 terms, exp2 and log2: some units of 2^-24 of what they are made of
        assert torch.allclose(lse[a:a + step], want, rtol=1e-5, atol=1e-5)
        assert torch.allclose(loss[a:a + step], torch.where(at < 0, 0.0, want - hit), rtol=1e-5, atol=2e-5)
