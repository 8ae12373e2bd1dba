"""More seeds and queries than one launch of a wavefront each can have (2^26 of them: 2^32 threads)."""
import pytest
import torch

from paper_2202_13538_amd import binding

pytestmark = pytest.mark.gpu

N_NODES, N_SEEDS = 1_000_003, 67_200_001


def test_walks_tables_and_joins_of_more_than_2_to_the_26():
    """Walks of one step on a ring: every block has the seed and a neighbour."""
    ctx = binding.Context(0)
    node = torch.arange(N_NODES, dtype=torch.int32, device="cuda")
    row_ptr = torch.arange(0, 2 * N_NODES + 1, 2, dtype=torch.int32, device="cuda")
    col_idx = torch.stack([(node - 1) % N_NODES, (node + 1) % N_NODES], 1).int().sort(1).values.reshape(-1).contiguous()
    seeds = (torch.arange(N_SEEDS, device="cuda") % N_NODES).int()
    sizes = torch.empty(N_SEEDS, dtype=torch.int32, device="cuda")
    walks = binding.sample_walks(ctx, row_ptr, col_idx, seeds, 1, 1, rng_seed=5, set_sizes=sizes)
    assert torch.equal(walks[:, 0, 0], seeds) and bool((sizes == 2).all())
    step = (walks[:, 0, 1] - seeds) % N_NODES
    assert bool(((step == 1) | (step == N_NODES - 1)).all())
    # a walk is its seed's own: all walks of one node are alike, wherever they stand
    assert torch.equal(walks, walks[seeds.long() % N_NODES])
    off, ids, cnt = binding.build_rpe(ctx, walks, N_NODES)
    assert torch.equal(off, torch.arange(0, 2 * N_SEEDS + 1, 2, device="cuda"))
    assert torch.equal(ids.view(-1, 2), walks[:, 0].sort(1).values)
    first = (walks[:, 0, 0] < walks[:, 0, 1]).to(torch.int16)
    want = torch.stack([first, 1 - first, 1 - first, first], 1).view(-1, 2)
    assert torch.equal(cnt.view(torch.int16), want)
    del want
    fused = binding.sample_walks_rpe(ctx, row_ptr, col_idx, seeds, 1, 1, rng_seed=5)
    for x, y in zip(fused, (walks, off, ids, cnt)):
        assert torch.equal(x.view(torch.int16) if x.dtype == torch.uint16 else x, y.view(torch.int16) if y.dtype == torch.uint16 else y)
    del fused
    # every query names one block twice: its rows once, their counts in both halves
    queries = torch.arange(N_SEEDS, dtype=torch.int32, device="cuda")[:, None].repeat(1, 2)
    join_off, join_ids, join_cnt = binding.join_queries(ctx, off, ids, cnt, queries, max_set=2)
    assert torch.equal(join_off, off) and torch.equal(join_ids, ids)
    for half in range(2):
        assert torch.equal(join_cnt[:, half].view(torch.int16), cnt.view(torch.int16))
    assert ctx.check() == 0
    ctx.close()
    del walks, ids, cnt, join_ids, join_cnt, queries
    torch.cuda.empty_cache()
