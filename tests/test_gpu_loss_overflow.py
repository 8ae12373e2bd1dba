"""Rows of the softmax loss that are not finite and count: which results are numbers, and how long it takes."""
import pytest
import torch

from paper_2202_13538_amd import binding
from test_gpu_attention import BF, HF
from test_gpu_loss import inputs, reference

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    assert c.check() == 0
    c.close()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("where", ["h", "dloss", "w"])
@pytest.mark.parametrize("n,classes,dim", [(90, 400, 64), (300, 33, 40), (9000, 257, 64)])
def test_which_results_are_numbers(ctx, n, classes, dim, where, dtype):
    h, w, labels = inputs(n, classes, dim, dtype, seed=n)
    labels[5], labels[6] = 3, -1
    dloss = torch.linspace(0.5, 1, n, device="cuda")
    {"h": h, "dloss": dloss, "w": w}[where].view(-1)[(5 if where == "dloss" else 5 * dim + 3)] = NAN
    h[6] = NAN   # (and a row that does not count)
    loss, lse = binding.softmax_loss(ctx, h, w, labels)
    dh, dw = binding.softmax_loss_grad(ctx, dloss, h, w, labels, lse)
    r = reference(h, w, labels, dloss)
    none = (labels < 0).cpu().numpy()   # (rows that do not count have zeros, whatever the formula's 0 NaN is)
    r["loss"][none], r["dh"][none] = 0, 0
    for name, x in (("loss", loss), ("lse", lse), ("dh", dh), ("dw", dw)):
        assert torch.equal(x.isnan().cpu(), torch.from_numpy(r[name]).isnan()), name


def test_a_step_that_overflowed_takes_no_longer(ctx):
    h, w, labels = inputs(8192, 20_000, 128, HF, seed=1)
    dloss = torch.full((8192,), 1e-4, device="cuda")

    def least():
        times = []
        for _ in range(4):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            binding.softmax_loss_grad(ctx, dloss, h, w, labels, binding.softmax_loss(ctx, h, w, labels)[1])
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    clean = least()
    h[-1], labels[-1] = NAN, 7
    spoilt = least()
    assert spoilt < 3 * clean, (clean, spoilt)
