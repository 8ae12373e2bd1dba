"""The example: walks, attention with a learned bias and the softmax loss in one training loop, and single rows."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_a_model_of_walks_learns_and_continues_them():
    import walk_model
    from paper_2202_13538_amd import synth

    lib, graph, wl, model, losses = walk_model.train(steps=40, quiet=True)
    assert lib.check() == 0
    # a uniform guess among 4,096 nodes costs 8.3; 40 steps learn at least the nodes' frequencies
    assert losses[0] > 7.5 and sum(losses[-5:]) / 5 < losses[0] - 1.0
    assert all(p.grad is not None and torch.isfinite(p.grad).all() and p.grad.any() for p in model.parameters())
    single, whole = walk_model.continue_walks(lib, graph, model, torch.arange(100, dtype=torch.int32, device="cuda"))
    # the same rows by two ways: weights and results are rounded to 8 bits in different orders
    assert (single.float() - whole.float()).abs().max() <= 4 * torch.finfo(torch.bfloat16).eps * whole.float().abs().max()
    queries = torch.from_numpy(synth.make_queries(wl, *(t.cpu().numpy() for t in graph))).cuda()[:300]
    pooled = walk_model.pool_queries(lib, graph, wl, model, queries)
    assert pooled.shape == (300, 64) and torch.isfinite(pooled.float()).all()
    assert lib.check() == 0
