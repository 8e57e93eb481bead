"""Curvature-guided walks that train a small mixture of experts, which then answers with walks of its own.

The path: erc_run gives every edge its curvature; walkers draw each next node from the curvature
scores of their node's neighbours (erc_sample_rows over padded neighbour lists); a model learns to
predict the next node of a walk, its nodes routed to experts (erc_route, erc_expert_plan,
erc_expert_gather, erc_expert_combine, with their gradients); at the end nodes are drawn from the
model's scores over all nodes, one row a walker (erc_sample_rows again, as a decoder uses it).

    python examples/walk_experts.py [--steps 60] [--walkers 512]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_27209_gb300 import erc, synth  # noqa: E402


class Route(torch.autograd.Function):
    """(experts, weights) of rows of logits; the weights carry a gradient."""

    @staticmethod
    def forward(ctx, logits, k, score, bias):
        experts, weights = erc.erc_route(logits, k, score=score, bias=bias)
        ctx.save_for_backward(logits, experts)
        ctx.score = score
        ctx.mark_non_differentiable(experts)
        return experts, weights

    @staticmethod
    def backward(ctx, _, dweights):
        logits, experts = ctx.saved_tensors
        return erc.erc_route_backward(logits, experts, dweights.contiguous(), score=ctx.score), None, None, None


class Gather(torch.autograd.Function):
    """Rows in expert order."""

    @staticmethod
    def forward(ctx, x, slot, offsets):
        ctx.save_for_backward(slot)
        return erc.erc_expert_gather(x, slot, offsets)

    @staticmethod
    def backward(ctx, dxs):
        return erc.erc_expert_combine(dxs.contiguous(), ctx.saved_tensors[0]), None, None


class Combine(torch.autograd.Function):
    """The weighted sum of the experts' rows."""

    @staticmethod
    def forward(ctx, y, weights, slot, offsets):
        ctx.save_for_backward(y, weights, slot, offsets)
        return erc.erc_expert_combine(y, slot, weights)

    @staticmethod
    def backward(ctx, dout):
        y, weights, slot, offsets = ctx.saved_tensors
        dy, dweights = erc.erc_expert_combine_backward(dout.contiguous(), y, slot, offsets, weights)
        return dy, dweights, None, None


class Experts(torch.nn.Module):
    """out[t] = sum_j w[t, j] relu(x[t] A_e + b_e), e the j-th expert of row t."""

    def __init__(self, width, n_experts, k, score=erc.ERC_SCORE_SIGMOID):
        super().__init__()
        self.n_experts, self.k, self.score = n_experts, k, score
        self.router = torch.nn.Parameter(torch.randn(width, n_experts) * width**-0.5)
        self.A = torch.nn.Parameter(torch.randn(n_experts, width, width) * width**-0.5)
        self.b = torch.nn.Parameter(torch.zeros(n_experts, width))
        self.register_buffer("bias", torch.zeros(n_experts))  # balances the load, without a gradient

    def forward(self, x):
        experts, weights = Route.apply(x @ self.router, self.k, self.score, self.bias)
        offsets, _, slot = erc.erc_expert_plan(experts, self.n_experts)
        xs = Gather.apply(x, slot, offsets)
        ends = offsets.tolist()
        parts = [torch.relu(xs[ends[e]:ends[e + 1]] @ self.A[e] + self.b[e]) for e in range(self.n_experts)]
        y = torch.cat(parts + [xs[ends[-1]:]])
        if self.training:  # an expert with more than its share is chosen a little less often
            load = (offsets[1:] - offsets[:-1]).float()
            self.bias -= 0.01 * torch.sign(load - load.mean())
        return Combine.apply(y, weights, slot, offsets)


def neighbour_scores(n, src, dst, w, dev):
    """Padded (ids, scores) of every node's neighbours: Eq. 8's edge weight as a logarithm, -inf where
    a node has no more neighbours."""
    out = erc.erc_run(n, *(torch.from_numpy(a).to(dev) for a in (src, dst, w)), erc.Params(K=64, kc=64))
    g = erc.erc_build_laplacian(n, *(torch.from_numpy(a).to(dev) for a in (src, dst, w)))
    q = torch.log(torch.sqrt(torch.clamp(-out["kappa"] + 2 * out["kappa"].max(), min=0)) + 1)
    degree = g.row_ptr[1:] - g.row_ptr[:-1]
    at = g.row_ptr[:-1, None] + torch.arange(int(degree.max()), device=dev)
    some = at < g.row_ptr[1:, None]
    at = torch.where(some, at, 0)
    return g.col[at], torch.where(some, q[g.csr_eid[at].long()], -torch.inf)


def words(rows, generator):
    return torch.randint(-(2**63), 2**63 - 1, (rows,), generator=generator, device=generator.device)


def walk(table, start, steps, generator, temperature=0.7, top_p=0.95):
    """Nodes [walkers, steps + 1] of curvature-guided walks."""
    ids, scores = table
    nodes = [start]
    for _ in range(steps):
        at, _, _ = erc.erc_sample_rows(scores[nodes[-1]], words(start.numel(), generator),
                                       temperature=temperature, top_p=top_p)
        here = nodes[-1]
        nodes.append(torch.where(at >= 0, ids[here, at.clamp(min=0).long()].long(), here))
    return torch.stack(nodes, 1)


def main(steps=60, walkers=512, width=64, n_experts=8, k=2, seed=0, n=400):
    dev = torch.device("cuda:0")
    torch.manual_seed(seed)
    generator = torch.Generator(device=dev).manual_seed(seed)
    table = neighbour_scores(*synth.random_connected(n, 4 * n, seed=seed + 11, weighted=True), dev)
    embed = torch.nn.Embedding(n, width).to(dev)
    model = Experts(width, n_experts, k).to(dev)
    answer = torch.nn.Linear(width, n).to(dev)
    optimiser = torch.optim.Adam([*embed.parameters(), *model.parameters(), *answer.parameters()], lr=1e-2)
    losses = []
    for _ in range(steps):
        start = torch.randint(0, n, (walkers,), generator=generator, device=dev)
        nodes = walk(table, start, 4, generator)
        scores = answer(model(embed(nodes[:, :-1].reshape(-1))))
        loss = torch.nn.functional.cross_entropy(scores, nodes[:, 1:].reshape(-1))
        optimiser.zero_grad()
        loss.backward()
        optimiser.step()
        losses.append(loss.item())
    # the model answers: one draw a walker over all nodes
    model.eval()
    with torch.no_grad():
        ids, logp, kept = erc.erc_sample_rows(answer(model(embed.weight)), words(n, generator),
                                              temperature=0.7, top_k=20, top_p=0.9)
    real = (table[0] == ids[:, None]) & (table[1] > -torch.inf)
    return dict(losses=losses, on_an_edge=real.any(1).float().mean().item(), ids=ids, logp=logp, kept=kept)


if __name__ == "__main__":
    parser = argparse.ArgumentParser()
    parser.add_argument("--steps", type=int, default=60)
    parser.add_argument("--walkers", type=int, default=512)
    args = parser.parse_args()
    r = main(args.steps, args.walkers)
    print(f"loss {r['losses'][0]:.3f} -> {r['losses'][-1]:.3f}; drawn nodes that are neighbours: "
          f"{100 * r['on_an_edge']:.0f}%; kept entries a row: {r['kept'].float().mean().item():.1f}")
