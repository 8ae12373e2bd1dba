"""surel_sample_classes on the GPU against its definition: rows sorted on the host, sums in 80 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2202_13538_amd import binding

pytestmark = pytest.mark.gpu

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    assert c.check() == 0
    c.close()


def draw(z, u, t=1.0, k=0, p=1.0, floor=0.0):
    """(class, logarithm of its probability) of one row of float64 logits."""
    if np.isnan(z).any() or (z == np.inf).any() or (z == -np.inf).all():
        return -1, -math.inf
    order = np.argsort(-z, kind="stable")
    if t == 0.0:
        return int(order[0]), 0.0
    with np.errstate(over="ignore", under="ignore"):
        w = np.exp((z - z.max()) / t)
    n = len(z) if k < 1 else min(k, len(z))
    if p < 1.0:
        mass = np.cumsum(w[order[:n]].astype(np.longdouble))
        before = np.concatenate([[0], mass[:-1]])
        n = max(1, int((before < np.longdouble(p) * mass[-1]).sum()))
    keep = np.zeros(len(z), bool)
    keep[order[:n]] = True
    keep &= w >= floor
    keep[order[0]] = True
    at = np.flatnonzero(keep & (w > 0))
    mass = np.cumsum(w[at].astype(np.longdouble))
    i = int((mass <= np.longdouble(u) * mass[-1]).sum())
    return int(at[i]), float(np.log(w[at[i]].astype(np.longdouble) / mass[-1]))


def check(ctx, logits, u, temperature=None, top_k=None, top_p=None, min_p=None, flags=0):
    chosen, logp = binding.sample_classes(ctx, logits, u, temperature, top_k, top_p, min_p)
    assert ctx.check() == flags
    z = logits.float().cpu().numpy().astype(np.float64)
    row = lambda x, i, none: none if x is None else x[i].item()  # noqa: E731
    want = [draw(z[i], u[i].item(), row(temperature, i, 1.0), row(top_k, i, 0), row(top_p, i, 1.0), row(min_p, i, 0.0))
            for i in range(len(z))]
    ids = chosen.tolist()
    wrong = [i for i in range(len(z)) if ids[i] != want[i][0]]
    assert not wrong, [(i, ids[i], want[i], row(temperature, i, 1.0), row(top_k, i, 0), row(top_p, i, 1.0), row(min_p, i, 0.0)) for i in wrong[:5]]
    for got, (_, w) in zip(logp.tolist(), want):
        # weights to 2^-45 or so, their sum and logarithm in 64 bits, the result in 32
        assert got == w if w == -math.inf else abs(got - w) <= 2.0 ** -24 * abs(w) + 1e-11, (got, w)
    return chosen, logp


def rows(n, classes, dtype, seed=0, spread=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(n, classes, generator=g, device="cuda") * spread
    few = torch.randint(classes, (n, min(classes, 5)), generator=g, device="cuda")
    z.scatter_add_(1, few, torch.randn(few.shape, generator=g, device="cuda") * 2 + 6)
    uniform = lambda lo, hi: torch.rand(n, generator=g, device="cuda") * (hi - lo) + lo  # noqa: E731
    return z.to(dtype), uniform(0, 1).clamp_(max=1 - 2.0 ** -24), uniform


# classes from one to several chunks and parts; few rows of many classes go in parts, many rows a workgroup each
SHAPES = [(5, 1), (9, 2), (3, 7), (40, 63), (17, 100), (300, 1000), (7, 4096), (600, 4097), (3, 33_000), (300, 40_001), (2, 70_003),
          (5, 235_000), (1, 1_000_003)]


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("n,classes", SHAPES)
def test_plain_draws(ctx, n, classes, dtype):
    z, u, uniform = rows(n, classes, dtype, seed=classes)
    check(ctx, z, u)
    check(ctx, z, u, temperature=uniform(0.3, 2.0))
    check(ctx, z, u, temperature=uniform(0.3, 2.0), min_p=uniform(0.0, 0.3))


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("n,classes", SHAPES)
def test_draws_of_a_row_s_beginning(ctx, n, classes, dtype):
    z, u, uniform = rows(n, classes, dtype, seed=classes + 1)
    t = uniform(0.3, 2.0) * (uniform(0, 1) > 0.1)                # some rows take their largest
    k = torch.randint(-1, min(classes, 500) + 3, (n,), device="cuda", dtype=torch.int32)
    p, floor = uniform(0.0, 1.1), uniform(0.0, 0.1)
    check(ctx, z, u, t, top_k=k)
    check(ctx, z, u, t, top_p=p)
    check(ctx, z, u, t, top_k=k, top_p=p)
    check(ctx, z, u, None, top_k=k, top_p=p, min_p=floor)
    check(ctx, z, u, t, top_k=torch.full_like(k, 2 ** 31 - 1), top_p=torch.full_like(p, 0.999))


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("n,classes", [(50, 37), (300, 5000), (4, 50_000), (6, 150_000)])
def test_ties_go_to_the_lowest_class(ctx, n, classes, dtype):
    """Few distinct logits: classes on the border, more than a list of a bin holds, and all of them."""
    _, u, uniform = rows(n, 1, dtype, seed=classes)
    g = torch.Generator(device="cuda").manual_seed(classes)
    k = torch.randint(1, classes + 1, (n,), device="cuda", dtype=torch.int32, generator=g)
    p = uniform(0.0, 1.0)
    for values in (torch.tensor([0.0]), torch.tensor([1.5, -2.0]), torch.tensor([0.0, -0.0, 1e-3, -1e-3]), torch.arange(8) * 0.5,
                   torch.tensor([3.0, -math.inf])):
        z = values.to("cuda")[torch.randint(len(values), (n, classes), device="cuda", generator=g)].to(dtype)
        z[:, 0] = values[0]
        check(ctx, z, u, top_k=k)
        check(ctx, z, u, top_p=p)
        check(ctx, z, u, uniform(0.5, 2.0), top_k=k, top_p=p)
        check(ctx, z, u, torch.zeros(n, device="cuda"))


@pytest.mark.parametrize("classes", [1000, 60_000])
def test_narrow_wide_and_lopsided_rows(ctx, classes):
    for dtype in (BF, HF, F32):
        for spread, t in ((1e-6, 1.0), (1e-3, 0.01), (0.02, 1.0), (60.0, 1.0), (5000.0, 1.0), (30.0, 0.05), (2.0, 1e-30), (2.0, 100.0)):
            z, u, uniform = rows(6, classes, dtype, seed=3, spread=spread)
            if spread < 1:
                z = (torch.randn(6, classes, device="cuda") * spread).to(dtype)
            temperature = torch.full((6,), t, device="cuda")
            k = torch.tensor([1, 2, 50, classes // 2, classes - 1, classes], dtype=torch.int32, device="cuda")
            check(ctx, z, u, temperature)
            check(ctx, z, u, temperature, top_k=k)
            check(ctx, z, u, temperature, top_p=torch.tensor([0.0, 0.1, 0.5, 0.9, 0.99, 0.999999], device="cuda"))
    # logits that hardly differ from zero, and the largest ones there are
    z = (torch.randn(6, classes, device="cuda").double() * 1e-41).float()
    k = torch.tensor([1, 2, 50, classes // 2, classes - 1, classes], dtype=torch.int32, device="cuda")
    p = torch.tensor([0.0, 0.1, 0.5, 0.9, 0.99, 0.999], device="cuda")
    for t in (1.0, 1e-41, 1e-45):
        check(ctx, z, u, torch.full((6,), t, device="cuda"), top_k=k)
        check(ctx, z, u, torch.full((6,), t, device="cuda"), top_p=p)
    z = torch.where(torch.randn(6, classes, device="cuda") > 0, 3e38, -3e38)
    z[:, 3] = 1e38
    for t in (1.0, 2e38, 3e38):
        check(ctx, z, u, torch.full((6,), t, device="cuda"), top_k=k, top_p=p)
        check(ctx, z, u, torch.full((6,), t, device="cuda"), top_p=p, min_p=torch.full((6,), 0.2, device="cuda"))
    # one class far above all others, and one below
    z = torch.zeros(4, classes, device="cuda")
    z[:, 77] = torch.tensor([40.0, 5.0, -60.0, -1e30], device="cuda")
    for p in (0.5, 0.999):
        check(ctx, z, u[:4].contiguous(), top_p=torch.full((4,), p, device="cuda"))


def test_the_ends_of_u_and_of_the_parameters(ctx):
    z, _, _ = rows(3, 2000, BF, seed=4)
    one = lambda x, kind=torch.float32: torch.full((3,), x, device="cuda", dtype=kind)  # noqa: E731
    for u in (0.0, 2.0 ** -149, 1 - 2.0 ** -24):
        for how in ({}, dict(top_k=one(1, torch.int32)), dict(top_p=one(0.0)), dict(top_p=one(1.0)), dict(top_p=one(math.inf)),
                    dict(min_p=one(1.0)), dict(min_p=one(0.0)), dict(top_k=one(-5, torch.int32)),
                    dict(temperature=one(3e38)), dict(temperature=one(1e-45)), dict(temperature=one(1e-45), top_p=one(0.9))):
            check(ctx, z, one(u), **how)
    # the first class and the last
    z = torch.full((2, 70_000), -math.inf, device="cuda")
    z[0, 0], z[1, -1] = 1.0, -5.0
    chosen, logp = check(ctx, z, torch.tensor([0.3, 0.9], device="cuda"))
    assert chosen.tolist() == [0, 69_999] and logp.tolist() == [0.0, 0.0]


@pytest.mark.parametrize("classes", [300, 100_000])
def test_rows_without_a_class(ctx, classes):
    z, u, uniform = rows(6, classes, F32, seed=5)
    z[1] = -math.inf
    check(ctx, z, u, top_k=torch.full((6,), 5, dtype=torch.int32, device="cuda"))
    for bad in (math.nan, -math.nan, math.inf):
        for at in (0, classes // 2, classes - 1):
            w = z.clone()
            w[4, at] = bad
            if bad != math.inf:
                w[4:5, at:at + 1].view(torch.int32).fill_(0x7FC00000 if math.copysign(1, bad) > 0 else -0x400000)
            check(ctx, w, u, flags=binding.DEV_BAD_CHOICE)
            check(ctx, w, u, top_p=uniform(0.5, 0.9), flags=binding.DEV_BAD_CHOICE)
    one = torch.ones(6, device="cuda")

    def bad_at(x, at=2, of=0.5):
        y = of * one
        y[at] = x
        return y

    for how in (dict(temperature=bad_at(-1.0)), dict(temperature=bad_at(math.nan)), dict(temperature=bad_at(math.inf)),
                dict(top_p=bad_at(-0.1)), dict(top_p=bad_at(math.nan)), dict(min_p=bad_at(-0.1)), dict(min_p=bad_at(1.1)),
                dict(min_p=bad_at(math.nan)), dict(u=bad_at(1.0)), dict(u=bad_at(-1e-3)), dict(u=bad_at(math.nan))):
        chosen, logp = binding.sample_classes(ctx, z, how.pop("u", u), **how)
        assert ctx.check() == binding.DEV_BAD_CHOICE
        assert chosen.tolist()[2] == -1 and logp[2] == -math.inf
        assert (chosen[[0, 3, 4, 5]] >= 0).all() and chosen[1] == -1


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("classes,stride", [(1, 3), (13, 13), (1000, 1001), (1023, 1030), (20_001, 20_007), (120_001, 120_003)])
def test_rows_that_lie_apart_and_start_anywhere(ctx, classes, stride, dtype):
    n = 5
    g = torch.Generator(device="cuda").manual_seed(classes)
    room = torch.full((n * stride + 16,), 50.0, device="cuda").to(dtype)    # what is not a row's would be drawn
    for skip in (0, 1, 3, 7):
        z = room[skip:skip + n * stride].view(n, stride)[:, :classes]
        z.copy_(torch.randn(n, classes, device="cuda", generator=g) * 3)
        u = torch.rand(n, device="cuda", generator=g)
        check(ctx, z, u)
        check(ctx, z, u, top_k=torch.full((n,), 4, dtype=torch.int32, device="cuda"), top_p=torch.full((n,), 0.8, device="cuda"))
    alike = room[:classes].expand(n, classes)
    check(ctx, alike, u)


def test_many_rows_over_three_classes(ctx):
    g = torch.Generator(device="cuda").manual_seed(0)
    z = torch.randn(100_000, 3, device="cuda", generator=g)
    u = torch.rand(100_000, device="cuda", generator=g)
    chosen, logp = binding.sample_classes(ctx, z, u)
    w = torch.exp(z.double() - z.double().amax(1, keepdim=True))
    mass = w.cumsum(1)
    want = (mass <= u[:, None].double() * mass[:, -1:]).sum(1)
    assert torch.equal(chosen.long(), want)
    p = (w / mass[:, -1:]).gather(1, want[:, None])[:, 0].log()
    assert (logp.double() - p).abs().max() < 1e-6


def test_a_row_of_more_classes_than_a_graph_s(ctx):
    """20 million classes: chunks of several slots a thread."""
    classes = 20_000_003
    g = torch.Generator(device="cuda").manual_seed(1)
    z = (torch.randn(1, classes, device="cuda", generator=g) * 2).to(BF)
    for u in (0.1, 0.77):
        check(ctx, z, torch.tensor([u], device="cuda"))
        check(ctx, z, torch.tensor([u], device="cuda"), top_k=torch.tensor([100_000], dtype=torch.int32, device="cuda"),
              top_p=torch.tensor([0.7], device="cuda"))


def test_no_rows(ctx):
    chosen, logp = binding.sample_classes(ctx, torch.empty(0, 5, device="cuda"), torch.empty(0, device="cuda"))
    assert chosen.shape == logp.shape == (0,) and ctx.check() == 0


@pytest.mark.parametrize("n,classes", [(4, 100_000), (300, 700)])
def test_results_are_the_same_every_time_and_in_a_graph(ctx, n, classes):
    z, u, uniform = rows(n, classes, BF, seed=6)
    k = torch.full((n,), 300, dtype=torch.int32, device="cuda")
    how = dict(temperature=uniform(0.5, 1.5), top_k=k, top_p=uniform(0.5, 1.0), min_p=uniform(0, 0.01))
    first = check(ctx, z, u, **how)
    for _ in range(10):
        assert all(torch.equal(x, y) for x, y in zip(first, binding.sample_classes(ctx, z, u, **how)))
    side = torch.cuda.Stream()
    own = binding.Context(0, stream=side)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        binding.sample_classes(own, z, u, **how)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = binding.sample_classes(own, z, u, **how)
    other, more = rows(40, 300_000, F32, seed=7)[:2]
    for turn in range(4):
        z.copy_(torch.randn(n, classes, device="cuda") * 2)
        u.copy_(torch.rand(n, device="cuda"))
        torch.cuda.synchronize()
        binding.sample_classes(own, other, more, top_p=torch.full((40,), 0.9, device="cuda"))   # needs more than what was captured
        with torch.cuda.stream(side):    # (calls of one context do not overlap)
            graph.replay()
        torch.cuda.synchronize()
        want = binding.sample_classes(ctx, z, u, **how)
        assert all(torch.equal(x, y) for x, y in zip(got, want)), turn
    assert own.check() == 0
    own.close()


def test_what_is_drawn_follows_the_probabilities(ctx):
    n = 200_000
    z = torch.tensor([0.0, 1.0, -1.0, 2.0, 0.5], device="cuda").expand(n, 5)
    u = (torch.arange(n, device="cuda", dtype=torch.float64) / n).float().clamp(max=1 - 2.0 ** -24)
    chosen, logp = binding.sample_classes(ctx, z, u, temperature=torch.full((n,), 0.7, device="cuda"))
    p = torch.softmax(z[0].double() / 0.7, 0)
    share = torch.bincount(chosen.long(), minlength=5).double() / n
    assert (share - p).abs().max() < 2 / n + 2.0 ** -23     # u in equal steps: a share is off by a step at each end
    assert (logp.double() - p.log()[chosen.long()]).abs().max() < 1e-6
