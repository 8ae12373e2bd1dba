"""surel_softmax_loss and surel_softmax_loss_grad on the GPU against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

from attention_cases import UNIT
from paper_2202_13538_amd import binding
from test_gpu_attention import BF, HF, near

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    assert c.check() == 0
    c.close()


def reference(h, w, labels, dloss):
    """float64 arrays; sums for the bounds: abs_z (the largest sum of |h| |w| of a row), and of every gradient the sum
    of its terms' sizes with the weight p + [label] in front."""
    h, w, dloss = (t.detach().cpu().double().numpy() for t in (h, w, dloss))
    labels = labels.cpu().numpy()
    z = h @ w.T
    top = z.max(1)
    e = np.exp(z - top[:, None])
    lse = top + np.log(e.sum(1))
    counts = (labels >= 0) & (labels < w.shape[0])
    hit = z[np.arange(len(h)), np.where(counts, labels, 0)]
    p = e / e.sum(1)[:, None]
    g, size = p.copy(), p.copy()
    rows = np.arange(len(h))[counts]
    g[rows, labels[counts]] -= 1
    size[rows, labels[counts]] += 1
    d = np.where(counts, dloss, 0)[:, None]
    g, size = g * d, size * np.abs(d)
    abs_h = np.where(counts[:, None], np.abs(h), 0)
    clean = np.where(counts[:, None], h, 0)
    return dict(lse=lse, loss=np.where(counts, lse - hit, 0), abs_z=(np.abs(h) @ np.abs(w).T).max(1),
                dh=g @ w, dw=g.T @ clean, abs_dh=size @ np.abs(w), abs_dw=size.T @ abs_h)


def check(ctx, h, w, labels, dloss=None):
    n, dim = h.shape
    if dloss is None:
        dloss = torch.linspace(-1, 1, n, device="cuda") if n > 1 else torch.ones(n, device="cuda")
    loss, lse = binding.softmax_loss(ctx, h, w, labels)
    dh, dw = binding.softmax_loss_grad(ctx, dloss, h, w, labels, lse)
    r = reference(h, w, labels, dloss)
    # A logit is a 32-bit dot product; the sum over the classes runs in lanes' and parts' sums of at most a few thousand
    # terms each; exp2 and log2 are good to 2 units.
    slack = 2.0 ** -24 * (dim + 8) * r["abs_z"] + 2.0 ** -24 * 4096
    near(lse, r["lse"], slack + 2.0 ** -22 * np.abs(r["lse"]), "lse")
    near(loss, r["loss"], 2 * slack + 2.0 ** -22 * (np.abs(r["lse"]) + np.abs(r["loss"])), "loss")
    # Weights are rounded to 16 bits (one unit), so are results (another); a quarter for 32-bit logits and sums.
    # fp16 has a smallest step: 2^-24 of results, and 2^-24 / 2^11 of weights relative to the largest.
    u, step = UNIT[h.dtype], 2.0 ** -24 if h.dtype == HF else 0.0
    size = lambda t: float(t.double().abs().nan_to_num(0).max())  # noqa: E731
    d = size(dloss)
    z_err = 2.0 ** -24 * (dim + 8) * r["abs_z"].max() * 2 + 1e-6
    near(dh, r["dh"], (2.25 * u + z_err) * r["abs_dh"] + step * (1 + w.shape[0] * 2.0 ** -11 * d * size(w)), "dh")
    near(dw, r["dw"], (2.25 * u + z_err) * r["abs_dw"] + step * (1 + n * 2.0 ** -11 * d * size(h)), "dw")
    return loss, lse, dh, dw


def inputs(n, classes, dim, dtype, seed=0, std=None, ignored=0.1):
    g = torch.Generator().manual_seed(seed)
    h = torch.randn(n, dim, generator=g).to(dtype).cuda()
    w = (torch.randn(classes, dim, generator=g) * (2 * dim ** -0.5 if std is None else std)).to(dtype).cuda()
    labels = torch.randint(0, classes, (n,), generator=g).int()
    labels[torch.rand(n, generator=g) < ignored] = -1
    return h, w, labels.cuda()


SHAPES = [(1, 1, 8), (1, 4096, 64), (7, 33, 16), (32, 1000, 40), (33, 129, 96), (64, 31, 128), (100, 2000, 72), (257, 513, 128),
          (300, 100, 200), (130, 4097, 256), (5, 20_011, 168), (1000, 64, 32), (2, 127, 248)]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("n,classes,dim", SHAPES)
def test_rows_against_classes(ctx, n, classes, dim, dtype):
    check(ctx, *inputs(n, classes, dim, dtype, seed=n + classes))


@pytest.mark.parametrize("dtype", [BF, HF])
def test_parts_of_many_classes_and_of_many_rows(ctx, dtype):
    check(ctx, *inputs(40, 150_001, 64, dtype, seed=1))
    check(ctx, *inputs(9000, 257, 64, dtype, seed=2))


@pytest.mark.parametrize("dtype", [BF, HF])
def test_sharp_and_flat_distributions(ctx, dtype):
    check(ctx, *inputs(70, 600, 64, dtype, seed=3, std=3.0))
    check(ctx, *inputs(70, 600, 64, dtype, seed=4, std=0.0))
    h, w, labels = inputs(70, 600, 64, dtype, seed=5)
    ramp = torch.linspace(0.1, 8, 600, device="cuda", dtype=dtype)[:, None]   # maxima that keep growing
    check(ctx, h, w * ramp, labels)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("scale", [1e-7, 1.0, 65536.0])
def test_scales_of_the_loss(ctx, dtype, scale):
    h, w, labels = inputs(200, 700, 64, dtype, seed=6)
    dloss = torch.rand(200, device="cuda") * (scale / 200)
    check(ctx, h, w, labels, dloss)


def test_labels_at_the_ends_and_shared(ctx):
    h, w, labels = inputs(300, 333, 64, BF, seed=7, ignored=0)
    labels[:100], labels[100:200], labels[200:] = 0, 332, 31
    check(ctx, h, w, labels)
    labels[:] = -1
    loss, lse, dh, dw = check(ctx, h, w, labels)
    assert not loss.any() and not dh.any() and not dw.any()
    labels[:] = -2 ** 31
    check(ctx, h, w, labels)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_rows_that_do_not_count_have_no_influence(ctx, dtype, bad):
    h, w, labels = inputs(90, 400, 64, dtype, seed=8)
    dloss = torch.linspace(-1, 1, 90, device="cuda")
    labels[40] = labels[3] = -1
    lse = binding.softmax_loss(ctx, h, w, labels)[1]
    want = binding.softmax_loss_grad(ctx, dloss, h, w, labels, lse)
    r = reference(h, w, labels, dloss)
    dloss[40] = h[40, 5] = bad
    loss, lse = binding.softmax_loss(ctx, h, w, labels)
    assert loss[40] == 0 and torch.isfinite(loss).all() and not torch.isfinite(lse[40])
    dh, dw = binding.softmax_loss_grad(ctx, dloss, h, w, labels, lse)
    assert torch.equal(dh, want[0])
    near(dw, r["dw"], 2.26 * UNIT[dtype] * r["abs_dw"] + 2.0 ** -13, "dw")


def test_labels_beyond_the_classes_are_reported(ctx):
    own = binding.Context(0)
    h, w, labels = inputs(50, 100, 32, BF, seed=9)
    labels[7] = 100
    loss, lse = binding.softmax_loss(own, h, w, labels)
    assert own.check() == binding.DEV_BAD_LABEL and loss[7] == 0
    dh, dw = binding.softmax_loss_grad(own, torch.ones(50, device="cuda"), h, w, labels, lse)
    assert own.check() == binding.DEV_BAD_LABEL and not dh[7].any()
    labels[7] = -1
    want = binding.softmax_loss_grad(own, torch.ones(50, device="cuda"), h, w, labels, lse)
    assert torch.equal(dh, want[0]) and torch.equal(dw, want[1]) and own.check() == 0
    own.close()


def test_no_rows(ctx):
    h, w, labels = inputs(0, 100, 32, BF)
    loss, lse = binding.softmax_loss(ctx, h, w, labels)
    dh, dw = binding.softmax_loss_grad(ctx, loss, h, w, labels, lse)
    assert loss.shape == (0,) and dh.shape == (0, 32) and not dw.any()


def test_results_are_the_same_every_time_and_in_a_graph(ctx):
    h, w, labels = inputs(500, 9001, 96, HF, seed=10)
    dloss = torch.rand(500, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def step(c):
        loss, lse = binding.softmax_loss(c, h, w, labels)
        return loss, lse, *binding.softmax_loss_grad(c, dloss, h, w, labels, lse)
    with torch.cuda.stream(side):
        own = binding.Context(0)
        first = step(own)
        for _ in range(3):
            assert all(torch.equal(x, y) for x, y in zip(first, step(own)))
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step(own)
    for turn in range(3):
        dloss.copy_(torch.rand(500, device="cuda") * 100.0 ** -turn)
        want = step(ctx)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), turn
    assert own.check() == 0
    own.close()


def test_offsets_of_elements_beyond_32_bits(ctx):
    """A table of 2.2e9 elements whose last rows hold nearly all of the sum."""
    classes, dim = 8_600_000, 256
    w = torch.zeros(classes, dim, dtype=BF, device="cuda")
    g = torch.Generator().manual_seed(1)
    w[-40:] = torch.randn(40, dim, generator=g).to(BF).cuda()
    h = (torch.randn(3, dim, generator=g) * 3).to(BF).cuda()
    labels = torch.tensor([classes - 1, 0, classes - 40], dtype=torch.int32, device="cuda")
    loss, lse = binding.softmax_loss(ctx, h, w, labels)
    z = h.double() @ w[-40:].double().t()
    want = torch.logsumexp(torch.cat([z, torch.full((3, 1), float(np.log(classes - 40)), device="cuda")], 1), 1)
    assert torch.allclose(lse.double(), want, rtol=1e-5)
    assert torch.allclose(loss.double(), want - torch.stack([z[0, 39], z[1, 0] * 0, z[2, 0]]), rtol=1e-4)
    dh, dw = binding.softmax_loss_grad(ctx, torch.ones(3, device="cuda"), h, w, labels, lse)
    p = torch.exp(z - want[:, None])
    p[0, 39] -= 1
    p[2, 0] -= 1
    assert (dh.double() - p @ w[-40:].double()).abs().max() < 2.5 * UNIT[BF] * float((p.abs() @ w[-40:].double().abs()).max())
    assert (dw[-40:].double() - p.t() @ h.double()).abs().max() < 2.5 * UNIT[BF] * float((p.abs().t() @ h.double().abs()).max())
