"""A neighbour graph and a search by comparing everything, in MXFP4, with the last word in float32.

    python examples/mx_neighbours.py [--set gmm10k_d32] [--n N] [--k K] [--spare S] [--queries Q]

The set is quantised once.  Every vector's k + spare nearest are taken from the table, the float32 rows decide among
them, and the result is a graph like any other of this package: it is stored with efanna_set_graph and refined by NN-descent,
which finds what the quantisation lost.  Queries go the same way without the graph.  Printed are the recalls against
brute force in float64 on a sample.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1609_07228_amd import efanna, synth  # noqa: E402


def best_of(ids, dists, k):
    """The k first entries of every row in the order (distance, id); empty slots (id -1) come last."""
    dists = torch.where(ids < 0, torch.inf, dists)
    key = (dists.view(torch.int32).to(torch.int64) << 32) | (ids.to(torch.int64) & 0xFFFFFFFF)
    key = key.sort(dim=1).values[:, :k]
    return (key & 0xFFFFFFFF).to(torch.int32), (key >> 32).to(torch.int32).view(torch.float32)


def graph_by_comparison(X, table, k, spare):
    """(ids, dists) of the k nearest among each vector's k + spare nearest of the table, distances of the float32 rows."""
    n = X.shape[0]
    ids, _ = efanna.efanna_mx_nearest(table, table, k + spare, first_self=0)
    own = torch.arange(n, dtype=torch.int32, device=X.device)[:, None].expand_as(ids)
    dists = efanna.efanna_pair_distances(X, own.reshape(-1), torch.where(ids < 0, own, ids).reshape(-1))
    return best_of(ids, dists.view_as(ids), k)


def search_by_comparison(X, table, Q, k, spare):
    """(ids, dists) of the k nearest of every query among its k + spare nearest of the table, likewise."""
    ids, _ = efanna.efanna_mx_nearest(table, efanna.efanna_mx_quantise(Q), k + spare)
    both = torch.cat((X, Q))
    own = torch.arange(X.shape[0], both.shape[0], dtype=torch.int32, device=X.device)[:, None].expand_as(ids)
    dists = efanna.efanna_pair_distances(both, own.reshape(-1), torch.where(ids < 0, own, ids).reshape(-1))
    return best_of(ids, dists.view_as(ids), k)


def recall(ids, X, Q, own=None):
    """Share of the true k nearest (float64) that the rows of ids name; own[i]: the row of X that query i is."""
    dist = torch.cdist(Q.to(torch.float64), X.to(torch.float64))
    if own is not None:
        dist[torch.arange(len(own), device=X.device), own] = torch.inf
    true = dist.topk(ids.shape[1], dim=1, largest=False).indices
    return (ids[:, :, None] == true[:, None, :]).any(dim=2).to(torch.float64).mean().item()


def run(name, n, k, spare, nq, device="cuda:0"):
    p = synth.params(name)
    X = torch.from_numpy(synth.generate(name, n=n)).to(device)
    Q = torch.from_numpy(synth.generate_queries(name, nq)).to(device)
    table = efanna.efanna_mx_quantise(X)
    ids, dists = graph_by_comparison(X, table, k, spare)
    sample = torch.arange(0, X.shape[0], max(1, X.shape[0] // 200), device=device)
    out = {"graph": recall(ids[sample], X, X[sample], sample)}

    graph = efanna.efanna_set_graph(ids, dists)
    efanna.efanna_nndescent(X, graph, 2, p["L"], synth.ALGO_SEED)
    ids, _ = efanna.efanna_get_graph(graph)
    out["refined"] = recall(ids[sample], X, X[sample], sample)

    found, _ = search_by_comparison(X, table, Q, k, spare)
    out["search"] = recall(found, X, Q)

    # a second look at what was found, from the table alone: how the queries' neighbourhoods are spread, and the scores that
    # a linear layer over the whole set would see
    near = efanna.efanna_mx_rows(table, found)
    out["spread"] = (near - near.mean(dim=1, keepdim=True)).square().sum(dim=2).mean().item()
    scores = efanna.efanna_mx_product(efanna.efanna_mx_quantise(Q), table, dtype=torch.bfloat16)
    out["score"] = scores.gather(1, found.to(torch.int64)).to(torch.float32).mean().item()
    return out


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--set", default="gmm10k_d32")
    ap.add_argument("--n", type=int, default=None)
    ap.add_argument("--k", type=int, default=10)
    ap.add_argument("--spare", type=int, default=20)
    ap.add_argument("--queries", type=int, default=100)
    a = ap.parse_args()
    for what, value in run(a.set, a.n, a.k, a.spare, a.queries).items():
        print(f"{what:8s} {value:.4f}")


if __name__ == "__main__":
    main()
