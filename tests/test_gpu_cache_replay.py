"""A captured step of a cache's bookkeeping, replayed over sequences that hold pages, fill their last one and end."""
import pytest
import torch

from cache_cases import plan
from paper_2202_13538_amd import binding

pytestmark = pytest.mark.gpu


def state(lengths, page_rows, width, n, turn):
    """(length, pages, ring, turn) on the host: a page is held once or free."""
    order = torch.randperm(n, generator=torch.Generator().manual_seed(sum(lengths))).tolist()
    pages = torch.full((len(lengths), width), -7, dtype=torch.int32)
    for s, x in enumerate(lengths):
        for j in range(-(-x // page_rows)):
            pages[s, j] = order.pop()
    ring = torch.full((n,), -9, dtype=torch.int32)
    for i, page in enumerate(order):
        ring[(turn + i) % n] = page
    return torch.tensor(lengths, dtype=torch.int32), pages, ring, torch.tensor([turn, turn + len(order)])


@pytest.mark.parametrize("seqs,n_rows", [(4, 14), (5000, 5200)])
def test_every_replay_is_the_step_of_its_own_sequences(seqs, n_rows):
    page_rows, width = 4, 6
    n = 4 * seqs
    fill = lambda *x: (list(x) * seqs)[:seqs]  # noqa: E731
    steps = [(fill(3, 0, 17, 5), fill(1, 2, -1, 1), 0), (fill(2, 3, 4, 20), fill(0, 1, 1, -1), 5 * n - 2), (fill(8, 0, 0, 1), fill(-1, 0, 1, 2), n - 1),
             (fill(0), fill(0), 3), (fill(5, 9, 20, 13), fill(-1, -7, -1, -1), 2 * n + 1)]
    side = torch.cuda.Stream()
    ctx = binding.Context(0, stream=side)
    with torch.cuda.stream(side):
        args = [x.cuda() for x in state(steps[0][0], page_rows, width, n, 0)]
        length, pages, ring, turn = args
        added = torch.tensor(steps[0][1], dtype=torch.int32, device="cuda")
        binding.cache_plan(ctx, length, added, pages, ring, turn, page_rows, n_rows)   # (grows what it needs)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = binding.cache_plan(ctx, length, added, pages, ring, turn, page_rows, n_rows)
        assert ctx.check() in (0, binding.DEV_CAPACITY)
        for lengths, adds, at in steps + steps[::-1]:
            now = state(lengths, page_rows, width, n, at)
            for x, y in zip(args, now):
                x.copy_(y)
            added.copy_(torch.tensor(adds, dtype=torch.int32))
            want = plan(now[0], added.cpu(), now[1], now[2], now[3], page_rows, n_rows)
            graph.replay()
            side.synchronize()
            assert ctx.check() == (binding.DEV_CAPACITY if sum(max(a, 0) for a in adds) > n_rows else 0)
            for x, y in zip((*got, pages, ring), want, strict=True):
                assert torch.equal(x.cpu(), torch.tensor(y, dtype=x.dtype).view(x.shape))
    ctx.close()
