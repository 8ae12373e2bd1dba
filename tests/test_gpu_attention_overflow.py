"""What is not finite and seen (an overflow in a training step): results are not numbers where the formula says so, finite where it
does not, and a call takes about as long as any other."""
import pytest
import torch

from attention_cases import inputs, offsets, reference
from paper_2202_13538_amd import binding
from test_gpu_attention import BF, HF

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    assert c.check() == 0
    c.close()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("where", ["q", "k", "v", "dout"])
@pytest.mark.parametrize("elements", [slice(None), slice(3, 4)], ids=["whole row", "one element"])
@pytest.mark.parametrize("lens,k_lens,causal", [([200, 70], None, True), ([200], None, False), ([16] * 30, None, True),
                                                ([3, 5], [300, 40], True)], ids=str)
def test_which_results_are_numbers(ctx, lens, k_lens, causal, elements, where, dtype):
    """The same elements as in 64 bits, for a row of NaN at several places."""
    q, k, v, q_off, k_off, how = inputs(lens, k_lens, 4, 2, 40, dtype, seed=7, reach=8, buckets=6, causal=causal)
    dout = torch.randn(q.shape, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    what = dict(q=q, k=k, v=v, dout=dout)
    n = len(what[where])
    for row in (0, n // 3, n - 1):
        t = dict(what)
        t[where] = t[where].clone()
        t[where][row, -1, elements] = NAN
        args = t["q"], t["k"], t["v"]
        out, lse = binding.attention(ctx, *args, q_off, k_off, causal=causal, **how)
        dq, dk, dv, _ = binding.attention_grad(ctx, t["dout"], *args, out, lse, q_off, k_off, causal=causal, **how)
        r = reference(*args, q_off, k_off, causal, 40 ** -0.5, dout=t["dout"], **how)
        for name, x in (("out", out), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
            want = torch.from_numpy(r[name]).isnan()
            assert torch.equal(x.isnan().cpu(), want), (name, row)


@pytest.mark.parametrize("where", ["k", "v", "all"])
def test_a_step_that_overflowed_takes_no_longer(ctx, where):
    """4,096 causal rows: with a key or value that all rows see, or everything, not a number at most three times as long.  (Going over
    all keys one by one, as for rows beside one that they do not see, takes 80 to 100 times as long.)"""
    g = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda heads: torch.empty(4096, heads, 128, dtype=HF, device="cuda").normal_(generator=g)  # noqa: E731
    t = dict(q=normal(16), k=normal(2), v=normal(2), dout=normal(16))
    off = offsets([4096])

    def step():
        out, lse = binding.attention(ctx, t["q"], t["k"], t["v"], off, causal=True)
        return binding.attention_grad(ctx, t["dout"], t["q"], t["k"], t["v"], out, lse, off, causal=True)

    def least():
        times = []
        for _ in range(4):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            step()
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    clean = least()
    for name, x in t.items():
        if where == "all":
            x[:] = NAN
        elif name == where:
            x[0] = NAN
    spoilt = least()
    assert spoilt < 3 * clean, (clean, spoilt)
