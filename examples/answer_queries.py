"""Which nodes does a node link to?  Embeddings are trained, a head is trained on them, and queries are answered.

    python examples/answer_queries.py [--config tiny] [--steps 60] [--queries 16]

1. the library trains vertex and context rows on a graph of workloads/configs.py, pools walked on the device;
2. a head learns how much each column counts: a node's query row is the norm of its vertex row plus its context row, times
   a gain; dropout on the context row, logistic loss of edges against random pairs (gv_norm_rows, gv_norm_rows_backward);
   edges are scored by the query row against the other node's vertex row, passed through dropout of its own (gv_drop_rows);
3. all vertex rows go into a table of 4 bits (gv_quantize_rows), a seventh of their size; queries are normalised into 8 bits
   and scored against every row of it (gv_norm_rows, gv_score_rows), and the few best are ranked by their full rows.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1903_00757_amd as gv  # noqa: E402
import workloads as W  # noqa: E402


class _Matrix:
    """A matrix of a context as torch sees device memory."""

    def __init__(self, ctx, which, n, dim):
        self.__cuda_array_interface__ = dict(shape=(n, dim), typestr="<f4", version=2, strides=None,
                                             data=(gv.gv_device_embeddings(ctx, which), False))


def train_embeddings(config, samples):
    cfg = W.CONFIGS[config]
    n, src, dst = W.make_graph(config)
    offsets, adj = W.csr_from_edges(n, src, dst)
    pool = min(cfg["pool"], 1 << 19)
    ctx = gv.gv_create(dim=cfg["dim"], num_neg=cfg["num_neg"], neg_weight=cfg["neg_weight"], total_samples=samples,
                       pool_capacity=8)
    gv.gv_set_graph(ctx, n, src, dst)
    gv.gv_set_adjacency(ctx, offsets, adj)
    gv.gv_build_alias(ctx, 0.75)
    gv.gv_init_embeddings(ctx, 1)
    pairs = torch.empty((pool, 2), dtype=torch.int32, device="cuda")
    walk = 0
    for _ in range(-(-samples // pool)):
        walk += gv.gv_augment_device(ctx, pairs.data_ptr(), seed=5, first_walk=walk, count=pool)
        gv.gv_train_device_pool(ctx, pairs.data_ptr(), pool)
    gv.gv_sync(ctx)
    vertex, context = (torch.as_tensor(_Matrix(ctx, which, n, cfg["dim"]), device="cuda") for which in (gv.GV_VERTEX, gv.GV_CONTEXT))
    return ctx, n, src, dst, vertex, context


def train_head(vertex, context, src, dst, steps, batch=4096, drop=0.1, rate=0.05):
    """(gain, first loss, last loss)"""
    n, dim = vertex.shape
    gain = torch.ones(dim, device="cuda")
    moment = torch.zeros(dim, device="cuda")
    src, dst = (torch.from_numpy(e.astype("int64")).cuda() for e in (src, dst))
    gen = torch.Generator(device="cuda").manual_seed(3)
    losses = []
    for step in range(steps):
        edge = torch.randint(src.numel(), (batch // 2,), device="cuda", generator=gen)
        u = torch.cat([src[edge], src[edge]])
        v = torch.cat([dst[edge], torch.randint(n, (batch // 2,), device="cuda", generator=gen)])
        label = (torch.arange(batch, device="cuda") < batch // 2).float()
        at = dict(drop=drop, seed=11, first_row=step * batch)
        q = gv.gv_norm_rows(context[u], gain, vertex[u], keep_rstd=True, **at)
        t = gv.gv_drop_rows(vertex[v], drop, 12, first_row=step * batch)
        score = (q.out * t).sum(1)
        losses.append(torch.nn.functional.softplus(torch.where(label > 0, -score, score)).mean())
        grad = ((torch.sigmoid(score) - label) / batch).unsqueeze(1) * t
        grads = gv.gv_norm_rows_backward(grad, q.sum, gain, q.rstd, keep_residual=False, **at)
        moment.mul_(0.9).addcmul_(grads.gain, grads.gain, value=0.1)
        gain -= rate * grads.gain / (moment.sqrt() + 1e-8)
    return gain, float(torch.stack(losses[:5]).mean()), float(torch.stack(losses[-5:]).mean())


def shortlist(vertex, context, gain, table, nodes, length):
    """The `length` likeliest nodes for each of `nodes`, by 8-bit queries against the 4-bit table."""
    q = gv.gv_norm_rows(context[nodes], gain, vertex[nodes], out_type=torch.int8, keep_sum=False)
    return torch.topk(gv.gv_score_rows(*table, q.out, scale=q.scale), length, dim=1).indices


def answer(vertex, context, gain, table, nodes, best, length):
    """The `best` nodes for each of `nodes`: the shortlist, ranked in full precision."""
    some = shortlist(vertex, context, gain, table, nodes, length)
    q = gv.gv_norm_rows(context[nodes], gain, vertex[nodes]).out
    score = (vertex[some] * q.unsqueeze(1)).sum(2)
    return some.gather(1, torch.topk(score, best, dim=1).indices)


def share_of(got, want):
    """The share of `want` that is in `got`, row by row."""
    return (want.unsqueeze(2) == got.unsqueeze(1)).any(2).float().mean().item()


def run(config="tiny", samples=4_000_000, steps=60, queries=16, best=10, length=100):
    ctx, n, src, dst, vertex, context = train_embeddings(config, samples)
    try:
        gain, first, last = train_head(vertex, context, src, dst, steps)
        table = gv.gv_quantize_rows(vertex, group=32)
        nodes = torch.randint(n, (max(queries, 512),), device="cuda", generator=torch.Generator(device="cuda").manual_seed(9))
        got = answer(vertex, context, gain, table, nodes, best, length)
        plain = shortlist(vertex, context, gain, table, nodes, best)
        exact = torch.topk(gv.gv_norm_rows(context[nodes], gain, vertex[nodes]).out @ vertex.t(), best, dim=1).indices
        torch.cuda.synchronize()
        start = time.perf_counter()
        for _ in range(20):
            answer(vertex, context, gain, table, nodes[:queries], best, length)
        torch.cuda.synchronize()
        each = (time.perf_counter() - start) / 20
        return dict(nodes=n, first_loss=first, last_loss=last, table_alone=share_of(plain, exact), recall=share_of(got, exact),
                    ms=each * 1e3, table_mb=sum(t.nbytes for t in table) / 1e6, rows_mb=vertex.nbytes / 1e6)
    finally:
        del vertex, context
        gv.gv_destroy(ctx)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--config", default="tiny", choices=["tiny", "c2", "c4-small"])
    ap.add_argument("--samples", type=int, default=4_000_000)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--queries", type=int, default=16)
    a = ap.parse_args()
    r = run(a.config, a.samples, a.steps, a.queries)
    print(f"{r['nodes']} nodes; loss of the head {r['first_loss']:.4f} -> {r['last_loss']:.4f}")
    print(f"table {r['table_mb']:.1f} MB instead of {r['rows_mb']:.1f}; of the best ten in full precision its best ten hold "
          f"{100 * r['table_alone']:.1f} %, its best hundred {100 * r['recall']:.1f} %; {a.queries} queries in {r['ms']:.3f} ms")
