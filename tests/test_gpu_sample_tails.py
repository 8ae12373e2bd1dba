"""Nuclei whose border lies far down in a tail of very many classes, each of which weighs next to nothing."""
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


def tail(classes, levels, dtype):
    """(logits [1][classes], their levels by class): class 5 has 0, class 7 -64, the others the levels in turn."""
    z = torch.tensor(levels, dtype=torch.float32, device="cuda").to(dtype).repeat(-(-classes // len(levels)))[:classes]
    z[5], z[7] = 0.0, -64.0
    return z[None]


def expected(z, p, u):
    """(class, logarithm of its probability) by counts of equal logits, in 80 bits.  The border of p and that of u have to be a
    hundredth of a class's weight from a class's end at least: so much is left for sums of 64 bits."""
    z = z[0].double().cpu().numpy()
    L = np.longdouble
    values, counts = np.unique(z, return_counts=True)
    values, counts = values[::-1], counts[::-1]
    w = np.exp(values.astype(L))
    w[values < -64] = 0
    target, kept, before = L(np.float32(p)) * (w * counts).sum(), [], L(0)
    for x, c, v in zip(w, counts, values):
        need = (target - before) / x
        if need <= c:
            assert 0.01 < need % 1 < 0.99
            kept.append((v, int(math.ceil(need)), x))
            break
        kept.append((v, int(c), x))
        before += c * x
    keep = np.full(len(z), -1)
    for i, (v, n, _) in enumerate(kept):
        keep[np.flatnonzero(z == v)[:n]] = i
    total = sum(n * x for _, n, x in kept)
    places = np.flatnonzero(keep >= 0)
    mass = np.cumsum(np.array([x for *_, x in kept], L)[keep[places]])
    i = int((mass <= L(np.float32(u)) * total).sum())
    x = kept[keep[places[i]]][2]
    assert 0.01 < (mass[i] - L(np.float32(u)) * total) / x < 0.99
    return int(places[i]), float(np.log(x / total))


# classes, levels of the tail, top_p: in the list of the border's logits are the largest weight and the tail's
@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("classes,levels,p", [(2_900_000, (-22.564, -22.574), 0.9999), (2_900_000, (-22.5, -22.75, -27.0), 0.9998),
                                              (20_000_003, (-26.25, -26.5, -26.0), 0.999975), (300_000, (-20.0, -19.75), 0.9997)])
def test_a_border_in_a_tail(ctx, classes, levels, p, dtype):
    z = tail(classes, levels, dtype)
    for u in (0.5, 0.99995, 1 - 2.0 ** -23, 1 - 2.0 ** -24):
        chosen, logp = binding.sample_classes(ctx, z, torch.tensor([u], device="cuda"), top_p=torch.tensor([p], device="cuda"))
        assert ctx.check() == 0
        want, of = expected(z, p, u)
        assert chosen.item() == want, (u, chosen.item(), want)
        # sums of weights in 64 bits (their places are worth less than 2^-40 of them), the result in 32
        assert abs(logp.item() - of) <= 2.0 ** -24 * abs(of) + 1e-11, u


@pytest.mark.parametrize("classes,p", [(2_900_000, 0.99993), (20_000_003, 0.9997)])
def test_a_border_among_many_logits_of_a_tail(ctx, classes, p):
    """Levels that differ by some places of their type and by thousands of them: steps of the search that tell some apart only."""
    levels = [-24.0 - 0.001 * (i % 7) - 2.0 ** -19 * i for i in range(301)]
    z = tail(classes, levels, F32)
    for u in (0.99997, 1 - 2.0 ** -23, 1 - 2.0 ** -24):
        chosen, logp = binding.sample_classes(ctx, z, torch.tensor([u], device="cuda"), top_p=torch.tensor([p], device="cuda"))
        assert ctx.check() == 0
        want, of = expected(z, p, u)
        assert chosen.item() == want, (u, chosen.item(), want)
        assert abs(logp.item() - of) <= 2.0 ** -24 * abs(of) + 1e-11, u
