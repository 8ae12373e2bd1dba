"""A model of walks: predict the next node of a walk, then read joined sets and continue walks with it.

    python examples/walk_model.py [--graph rmat4k] [--steps 60]

One attention layer over the steps of sampled walks (a learned bias by step distance), trained with the softmax
loss over all nodes of the graph; the node table is both input and output.  Afterwards

  - walks are continued by one step: a single query row each over the keys and values of the steps so far;
  - every link query is pooled: one query row over the rows of its joined set, packed with join_off as they are.

Needs an MI355X and the built library.  Everything between the walks and the loss runs in this package's kernels;
the projections around attention are torch's.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2202_13538_amd import binding, synth  # noqa: E402


class Attention(torch.autograd.Function):
    """binding.attention with its gradients (of q, k, v and bias)."""

    @staticmethod
    def forward(ctx, lib, q, k, v, q_off, k_off, causal, bias, bucket):
        out, lse = binding.attention(lib, q, k, v, q_off, k_off, causal=causal, bias=bias, bucket=bucket)
        ctx.save_for_backward(q, k, v, out, lse, q_off, k_off, bias, bucket)
        ctx.lib, ctx.causal = lib, causal
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, out, lse, q_off, k_off, bias, bucket = ctx.saved_tensors
        dq, dk, dv, dbias = binding.attention_grad(ctx.lib, dout.contiguous(), q, k, v, out, lse, q_off, k_off,
                                                   causal=ctx.causal, bias=bias, bucket=bucket)
        return None, dq, dk, dv, None, None, None, dbias, None


class SoftmaxLoss(torch.autograd.Function):
    """binding.softmax_loss with its gradients (of rows and table)."""

    @staticmethod
    def forward(ctx, lib, h, w, labels):
        loss, lse = binding.softmax_loss(lib, h, w, labels)
        ctx.save_for_backward(h, w, labels, lse)
        ctx.lib = lib
        return loss

    @staticmethod
    def backward(ctx, dloss):
        h, w, labels, lse = ctx.saved_tensors
        dh, dw = binding.softmax_loss_grad(ctx.lib, dloss.contiguous(), h, w, labels, lse)
        return None, dh, dw, None


class WalkModel(torch.nn.Module):
    def __init__(self, lib: binding.Context, n_nodes: int, dim: int = 64, heads: int = 4, reach: int = 15):
        super().__init__()
        self.lib, self.heads, self.head_dim = lib, heads, dim // heads
        self.table = torch.nn.Parameter(torch.randn(n_nodes, dim) * 0.5)
        self.qkv = torch.nn.Linear(dim, 3 * dim, bias=False)
        self.mix = torch.nn.Linear(dim, dim, bias=False)
        self.bias = torch.nn.Parameter(torch.zeros(reach + 1, heads))
        self.register_buffer("bucket", torch.tensor(binding.distance_buckets(reach, reach + 1, causal=True),
                                                    dtype=torch.int32))

    def project(self, rows: torch.Tensor):
        """(q, k, v) of rows [n][dim]: views of one tensor [n][3][heads][dim of a head]."""
        qkv = torch.nn.functional.linear(rows, self.qkv.weight.bfloat16())
        return qkv.view(len(rows), 3, self.heads, self.head_dim).unbind(1)

    def read(self, rows: torch.Tensor, q, k, v, q_off, k_off) -> torch.Tensor:
        out = Attention.apply(self.lib, q, k, v, q_off, k_off, True, self.bias.bfloat16(), self.bucket)
        return rows + torch.nn.functional.linear(out.reshape(len(rows), -1), self.mix.weight.bfloat16())

    def forward(self, nodes: torch.Tensor, off: torch.Tensor) -> torch.Tensor:
        """Rows [n][dim] behind every step of packed walks (node numbers, int32[n])."""
        rows = self.table.bfloat16()[nodes.long()]
        return self.read(rows, *self.project(rows), off, off)

    def loss(self, nodes: torch.Tensor, off: torch.Tensor) -> torch.Tensor:
        """Mean loss of the next node over all steps but the walks' last ones."""
        labels = torch.cat([nodes[1:], nodes[:1]]).int()
        labels[off[1:] - 1] = -1                              # nothing follows a walk's last step
        each = SoftmaxLoss.apply(self.lib, self(nodes, off), self.table.bfloat16(), labels)
        return each.sum() / (labels >= 0).sum()


def walks_of(lib, graph, seeds, M: int, m: int, rng_seed: int):
    """(nodes int32[n_seeds * M * (m + 1)], off): sampled walks as packed sequences."""
    walks = binding.sample_walks(lib, *graph, seeds, M, m, rng_seed)
    off = torch.arange(seeds.numel() * M + 1, device="cuda") * (m + 1)
    return walks.view(-1), off


def train(graph_name: str = "rmat4k", steps: int = 60, seeds_a_step: int = 256, M: int = 4, m: int = 15,
          quiet: bool = False):
    torch.manual_seed(0)
    wl = synth.WORKLOADS[graph_name]
    row_ptr, col_idx = synth.make_graph(wl)
    graph = (torch.from_numpy(row_ptr).cuda(), torch.from_numpy(col_idx).cuda())
    lib = binding.Context()
    model = WalkModel(lib, wl.n_nodes).cuda()
    adam = torch.optim.Adam(model.parameters(), lr=0.02)
    losses = []
    for step in range(steps):
        seeds = torch.randint(wl.n_nodes, (seeds_a_step,), dtype=torch.int32, device="cuda")
        loss = model.loss(*walks_of(lib, graph, seeds, M, m, rng_seed=step))
        adam.zero_grad()
        loss.backward()
        adam.step()
        losses.append(loss.detach())
        if not quiet and step % 10 == 0:
            print(f"step {step:4d}  loss {losses[-1].item():.3f}", flush=True)
    return lib, graph, wl, model, [x.item() for x in losses]


@torch.no_grad()
def continue_walks(lib, graph, model, seeds, m: int = 8):
    """(rows of the last step by a single query row over kept keys, the same by taking the whole walk in)."""
    nodes, off = walks_of(lib, graph, seeds, 1, m, rng_seed=999)
    whole = model(nodes, off)[off[1:] - 1]
    rows = model.table.bfloat16()[nodes.long()]
    q, k, v = model.project(rows)
    last = off[1:] - 1
    one = torch.arange(seeds.numel() + 1, device="cuda")
    return model.read(rows[last], q[last], k, v, one, off), whole


@torch.no_grad()
def pool_queries(lib, graph, wl, model, queries, M: int = 50, m: int = 4):
    """A row for every query: one query row (the sum of its nodes') over its joined set."""
    seeds = torch.arange(wl.n_nodes, dtype=torch.int32, device="cuda")
    _, rpe_off, rpe_ids, rpe_cnt = binding.sample_walks_rpe(lib, *graph, seeds, M, m)
    join_off, join_ids, _ = binding.join_queries(lib, rpe_off, rpe_ids, rpe_cnt, queries, max_set=1 + M * m)
    table = model.table.bfloat16()
    _, k, v = model.project(table[join_ids.long()])
    q, _, _ = model.project(table[queries.long()].sum(1))
    out, _ = binding.attention(lib, q, k, v, torch.arange(len(queries) + 1, device="cuda"), join_off)
    return out.reshape(len(queries), -1)


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--graph", default="rmat4k", choices=sorted(synth.WORKLOADS))
    p.add_argument("--steps", type=int, default=60)
    a = p.parse_args()
    lib, graph, wl, model, losses = train(a.graph, a.steps)
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f}")
    seeds = torch.arange(32, dtype=torch.int32, device="cuda")
    single, whole = continue_walks(lib, graph, model, seeds)
    print("next nodes of 8 walks:", (single @ model.table.bfloat16().t()).argmax(1)[:8].tolist())
    print("single rows and whole walks differ by", (single - whole).abs().max().item())
    queries = torch.from_numpy(synth.make_queries(wl, *(t.cpu().numpy() for t in graph))).cuda()[:1024]
    print("pooled queries:", tuple(pool_queries(lib, graph, wl, model, queries).shape))
    assert lib.check() == 0


if __name__ == "__main__":
    main()
