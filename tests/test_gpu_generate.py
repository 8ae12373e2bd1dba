"""The operators of a paged cache and of sampling together: walks generated by the example's model, against the same steps
with every walk taken in whole."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def trained():
    import walk_model
    return walk_model.train(steps=15, quiet=True)


def logits_of(model, nodes, lengths):
    """Next-node logits behind packed walks, by attention over the whole of them."""
    off = torch.tensor([0, *lengths], device="cuda").cumsum(0)
    return (model(nodes, off)[off[1:] - 1] @ model.table.bfloat16().t()).float()


def test_generated_walks_are_those_of_whole_ones(trained):
    import walk_model
    lib, graph, wl, model, _ = trained
    n, steps = 50, 12
    g = torch.Generator(device="cuda").manual_seed(0)
    lengths = torch.randint(1, 9, (n,), generator=g, device="cuda")       # prompts of 1 to 8 nodes: pages end inside them
    off = torch.nn.functional.pad(lengths.cumsum(0), (1, 0))
    nodes = torch.randint(wl.n_nodes, (int(off[-1]),), generator=g, device="cuda").int()
    u = torch.rand(steps, n, generator=g, device="cuda")
    greedy = walk_model.generate(model, nodes, off, steps, u, temperature=0.0)
    drawn = walk_model.generate(model, nodes, off, steps, u, temperature=0.8, top_k=100, top_p=0.9)
    assert lib.check() == 0
    assert greedy.shape == drawn.shape == (n, steps) and greedy.min() >= 0 and drawn.max() < wl.n_nodes
    assert torch.equal(drawn, walk_model.generate(model, nodes, off, steps, u, temperature=0.8, top_k=100, top_p=0.9))
    walks = [nodes[a:b] for a, b in zip(off[:-1].tolist(), off[1:].tolist())]
    for step in range(steps):
        for got, kind in ((greedy, "greedy"), (drawn, "drawn")):
            whole = [torch.cat([w, got[i, :step]]) for i, w in enumerate(walks)]
            z = logits_of(model, torch.cat(whole), [len(w) for w in whole])
            of = z.gather(1, got[:, step:step + 1].long())[:, 0]
            # The rows come by two ways, rounded to 8 bits in different orders: they differ by a few units of the largest, and
            # so do the logits.
            off_by = 8 * torch.finfo(torch.bfloat16).eps * z.abs().amax(1)
            bar = z.amax(1) if kind == "greedy" else z.topk(100, 1).values[:, -1]
            assert (of >= bar - off_by).all(), (kind, step)


def test_walks_that_come_and_go(trained):
    """A cache of few pages: walks end and others take their pages, and what is attended to is each walk's own."""
    import walk_model
    from attention_cases import UNIT
    from paper_2202_13538_amd import binding
    lib, graph, wl, model, _ = trained
    n, heads, dim, most = 6, model.heads, model.head_dim, 20
    cache = walk_model.Cache(lib, n, most, heads, dim, page_rows=4)
    g = torch.Generator(device="cuda").manual_seed(1)
    kept = [[] for _ in range(n)]                                         # every walk's rows (k, v), on the side
    for step in range(40):
        added = []
        for s in range(n):
            have = sum(len(k) for k, _ in kept[s])
            add = -1 if have > 14 or (have and step % 7 == s) else 5 if have == 0 else 1
            added.append(add)
        total = sum(max(a, 0) for a in added)
        k, v = (torch.randn(total, heads, dim, generator=g, device="cuda").bfloat16() for _ in range(2))
        off = cache.add(torch.tensor(added, dtype=torch.int32, device="cuda"), k, v).tolist()
        for s, a in enumerate(added):
            kept[s] = [] if a < 0 else kept[s] + [(k[off[s]:off[s + 1]], v[off[s]:off[s + 1]])]
        q = torch.randn(n, heads, dim, generator=g, device="cuda").bfloat16()
        out, lse = binding.cache_attention(lib, q, cache.k, cache.v, cache.pages, cache.length)
        rows = [(torch.cat([x for x, _ in w]), torch.cat([y for _, y in w])) if w else (k[:0], v[:0]) for w in kept]
        lengths = [len(x) for x, _ in rows]
        assert cache.length.tolist() == lengths
        k_off = torch.tensor([0, *lengths], device="cuda").cumsum(0)
        want, want_lse = binding.attention(lib, q, torch.cat([x for x, _ in rows]), torch.cat([y for _, y in rows]),
                                           torch.arange(n + 1, device="cuda"), k_off, causal=True)
        # both within 2.25 units of sum p |v| <= max |v| (one for the weights, one for the result, and 32-bit sums)
        assert (out.float() - want.float()).abs().max() <= 4.5 * UNIT[torch.bfloat16] * 5.5
        assert torch.allclose(lse, want_lse, atol=1e-4, rtol=0) or (lse == want_lse).logical_or((lse - want_lse).abs() < 1e-4).all()
    assert lib.check() == 0
