"""Calls on a context's own stream while torch works on another: the memory of their results."""
import pytest
import torch

from cache_cases import bookkeeping, cache
from paper_2202_13538_amd import binding

pytestmark = pytest.mark.gpu


def calls():
    """Name and call of every operator that makes its results, for two sets of inputs each; a call gives no more than its context."""
    out = []
    for seed in (1, 2):
        plan = bookkeeping([3, 0, 17, 5] * 500, [1, 9, -1, 1] * 500, 4, 6, spare=3, seed=seed)
        q, _, _, _, k_pages, v_pages, pages, length = cache([40, 3, 700] * 20, 8, 2, 64, 16, torch.bfloat16, seed=seed)
        logits = torch.randn(3000, 100, device="cuda", generator=torch.Generator("cuda").manual_seed(seed))
        u = torch.linspace(0, 0.99, 3000, device="cuda")
        out.append(dict(plan=lambda c, p=plan: binding.cache_plan(c, *p, 4, 5600),
                        attend=lambda c, *x, a=(q, k_pages, v_pages, pages, length): binding.cache_attention(c, *a),
                        sample=lambda c, a=(logits, u): binding.sample_classes(c, *a)))
    return out


def places(tensors):
    return {b for t in tensors for b in range(t.data_ptr() // 512, (t.data_ptr() + t.nbytes + 511) // 512)}


@pytest.mark.parametrize("name", ["plan", "attend", "sample"])
def test_results_keep_their_memory(name):
    first, second = (x[name] for x in calls())
    big = torch.randn(8192, 8192, device="cuda").bfloat16()
    room = torch.empty_like(big)
    here, side = torch.cuda.current_stream(), torch.cuda.Stream()
    ctx, own = binding.Context(0), binding.Context(0, stream=side)
    want, want_other = ([x.clone() for x in call(ctx)] for call in (first, second))
    torch.cuda.synchronize()
    # what torch's present stream has given back, and may still write, is not what a call's results get
    passing = [torch.empty_like(x) for x in want]
    was = places(passing)
    del passing
    got = first(own)
    assert not was & places(got)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want, strict=True))
    for _ in range(2):
        for _ in range(60):
            torch.mm(big, big, out=room)
        passing = [torch.empty_like(x).fill_(77) for x in want]
        del passing
        got = first(own)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want, strict=True))
        # nor are results that it has still to read the next call's
        for _ in range(60):
            torch.mm(big, big, out=room)
        read = [x.clone() for x in got]
        was = places(got)
        del got
        other = second(own)
        if not here.query():
            assert not was & places(other)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(read, want, strict=True))
        assert all(torch.equal(x, y) for x, y in zip(other, want_other, strict=True))
    for c in (ctx, own):
        assert c.check() == 0
        c.close()
