"""A linear projection of a set's vectors, trained in 8 bits so that graph neighbours stay near, and a search in the projection.

    python examples/f8_projection.py [--set gmm10k_d32] [--n N] [--out P] [--steps S] [--batch B]

The neighbours come from a graph of this package.  The projection y = x w^T is a layer whose products run on 8-bit tables: its
input is kept in 8 bits for the backward pass, its weights are quantised once a step and held both ways round, and the gradient of
the weights takes the input as it is held.  The loss asks that a vector be nearer to one of its neighbours than to a vector of
the batch.  Afterwards the set is projected, and its neighbours are looked for among the projections (MXFP4 tables); printed is
the share of the true ones found, before and after training.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1609_07228_amd import efanna, efanna_f8, synth  # noqa: E402


class F8Linear(torch.autograd.Function):
    """x w^T with operands in 8 bits (E4M3 forward, E5M2 for the gradient on its way back); sums in float32.  Gradients have no
    gradients of their own (asking for them is an error)."""

    @staticmethod
    def forward(ctx, x, w):
        kept = efanna_f8.efanna_f8_quantise(x)
        table, turned = efanna_f8.efanna_f8_weights(w)
        ctx.save_for_backward(kept.codes, kept.scales, turned.codes, turned.scales)
        ctx.shape, ctx.types = w.shape, (x.dtype, w.dtype)
        return efanna_f8.efanna_f8_product(kept, table, dtype=x.dtype)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        codes, scales, t_codes, t_scales = ctx.saved_tensors
        n, d = ctx.shape
        dy = dy.contiguous()
        dx = dw = None
        if ctx.needs_input_grad[0]:
            back = efanna_f8.efanna_f8_quantise(dy, torch.float8_e5m2)
            dx = efanna_f8.efanna_f8_product(back, efanna_f8.F8Table(t_codes, t_scales, n), dtype=ctx.types[0])
        if ctx.needs_input_grad[1]:
            dw = efanna_f8.efanna_f8_gradient(dy, efanna_f8.F8Table(codes, scales, d), dtype=ctx.types[1])
        return dx, dw


def neighbours(X, p, k):
    """Graph neighbours of every row (trees, leaves, NN-descent)."""
    perm, leaf_off, n_leaves = efanna.efanna_build_trees(X, p["T"], p["S"], synth.ALGO_SEED)
    graph = efanna.efanna_init_graph(X, perm, leaf_off, n_leaves, p["S"], max(k, p["K"]))
    efanna.efanna_nndescent(X, graph, 4, p["L"], synth.ALGO_SEED)
    return efanna.efanna_get_graph(graph)[0][:, :k].to(torch.int64)


def loss_of(y, k):
    """Of groups of k + 2 projections (a vector, one of its neighbours, k others): cross entropy of the neighbour."""
    y = y.to(torch.float32).view(-1, k + 2, y.shape[1])
    score = -(y[:, :1] - y[:, 1:]).square().sum(dim=2)
    return torch.nn.functional.cross_entropy(score, torch.zeros(len(y), dtype=torch.int64, device=y.device))


def found(X, w, true, k):
    """Share of `true` among the k nearest of the projections."""
    y = efanna_f8.efanna_f8_product(efanna_f8.efanna_f8_quantise(X), efanna_f8.efanna_f8_weights(w)[0], dtype=torch.float32)
    table = efanna.efanna_mx_quantise(y)
    ids, _ = efanna.efanna_mx_nearest(table, table, k, first_self=0)
    return (ids[:, :, None] == true[:, None, :]).any(dim=2).to(torch.float64).mean().item()


def run(name, n, out, steps, batch, k=10, others=6, device="cuda:0"):
    p = synth.params(name)
    X = torch.from_numpy(synth.generate(name, n=n)).to(device)
    X = (X - X.mean(dim=0)) / X.std()
    near = neighbours(X, p, k)
    gen = torch.Generator(device=device).manual_seed(1)
    w = (torch.randn((out, X.shape[1]), generator=gen, device=device) * X.shape[1] ** -0.5).requires_grad_()
    before = found(X, w.detach(), near, k)
    adam = torch.optim.Adam([w], lr=1e-2)
    for _ in range(steps):
        own = torch.randint(0, len(X), (batch,), generator=gen, device=device)
        one = near[own, torch.randint(0, k, (batch,), generator=gen, device=device)]
        rest = torch.randint(0, len(X), (batch, others), generator=gen, device=device)
        rows = torch.cat((own[:, None], one[:, None], rest), dim=1).reshape(-1)
        loss = loss_of(F8Linear.apply(X[rows].to(torch.bfloat16), w), others)
        adam.zero_grad()
        loss.backward()
        adam.step()
    return {"before": before, "after": found(X, w.detach(), near, k)}


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--set", default="gmm10k_d32")
    ap.add_argument("--n", type=int, default=None)
    ap.add_argument("--out", type=int, default=16)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--batch", type=int, default=1024)
    a = ap.parse_args()
    for what, value in run(a.set, a.n, a.out, a.steps, a.batch).items():
        print(f"{what:8s} {value:.4f}")


if __name__ == "__main__":
    main()
