"""The exchange plan where layers kept whole lie between split ones: worker processes on CPU (gloo) that hold their own rows below the modulo layer, their
own column shards of split layers and full copies of whole ones, and move data only as sb_exchange_plan says, against the unpartitioned network.  All in 64
bits, so that only a missing, doubled or misplaced block shows."""
import os
import sys

import numpy as np
import pytest
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

import sb_inputs as si

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GATED = 10
ROWS, FEATURES = 3, 12      # of a worker


def binding():
    import __graft_entry__ as ge
    ge.build()
    from paper_2112_15317_b200 import binding as b
    return b


def net():
    # whole, split (behind the modulo layer), whole, whole, split, split, whole, split: every order of neighbours
    return [(si.FC_RELU_WHOLE, 14), (si.FC_RELU, 11), (si.FC_RELU_WHOLE, 9), (si.FC_RELU_WHOLE, 13), (si.FC_RELU, 10), (si.FC_RELU, 12), (si.FC_RELU_WHOLE, 8),
            (si.FC, 7), (si.SOFTMAX_XENT, 7)]


def data(N):
    rng = np.random.default_rng(5)
    widths = [FEATURES] + [o for _, o in net()[:-1]]
    params = [rng.standard_normal((o, i)) / np.sqrt(i) for i, o in zip(widths, widths[1:])]
    return params, rng.standard_normal((N * ROWS, FEATURES)), rng.integers(0, net()[-1][1], N * ROWS)


def loss_gradient(z, y, B):
    p = np.exp(z - z.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    p[np.arange(len(y)), y] -= 1
    return p / B


def reference(N):
    """Weight gradients of the unpartitioned network, and the gradient of its input"""
    params, x, y = data(N)
    acts = [x]
    for (kind, _), w in zip(net(), params):
        z = acts[-1] @ w.T
        acts.append(z if kind == si.FC else np.maximum(z, 0))
    d, grads = loss_gradient(acts[-1], y, len(y)), [None] * len(params)
    for i in range(len(params) - 1, -1, -1):
        grads[i] = d.T @ acts[i]
        d = d @ params[i]
        if i > 0:
            d = d * (acts[i] > 0)
    return grads, d


def run_worker(me, N, K, port, q):
    for p in (ROOT, os.path.join(ROOT, "tests")):
        sys.path.insert(0, p)
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port))
    dist.init_process_group("gloo", rank=me, world_size=N)
    sb = binding()
    layers, (params, x, y) = net(), data(N)
    nodes, plan = sb.partition(layers, 1, 1, FEATURES, K), sb.exchange_plan(layers, 1, 1, FEATURES, ROWS, N, K)
    G, B, gid, off = N // K, N * ROWS, me // K, me % K
    peers = [dist.new_group([g * K + o for g in range(G)]) for o in range(K)]
    own, group = slice(me * ROWS, (me + 1) * ROWS), slice(gid * K * ROWS, (gid + 1) * K * ROWS)

    def messages(kind, layer):
        return [m for m in plan if (m["kind"], m["layer"]) == (kind, layer)]

    def block(M, m):
        return M[m["rows"][0]:m["rows"][1], m["cols"][0]:m["cols"][1]]

    def exchange(msgs, M):
        """{source: block} of what arrives here; M is indexed by rows of the whole batch"""
        got = {m["src"]: (m, torch.empty(block(M, m).shape, dtype=torch.float64)) for m in msgs if m["dst"] == me}
        reqs = [dist.irecv(t, src=s) for s, (_, t) in got.items()]
        reqs += [dist.isend(torch.from_numpy(np.ascontiguousarray(block(M, m))), dst=m["dst"]) for m in msgs if m["src"] == me]
        for r in reqs:
            r.wait()
        return {s: (m, t.numpy()) for s, (m, t) in got.items()}

    def whole(M, cols):
        """M [rows here, cols] in its place of a matrix of the whole batch"""
        full = np.zeros((B, cols))
        full[rows] = M
        return full

    rows, a, gathered, split = own, x[own], False, {}
    inputs, outputs = {}, {}
    for nd in nodes:
        li = nd["layer"]
        if nd["node"] == sb.SB_NODE_MODULO:
            full = whole(a, a.shape[1])
            for m, t in exchange(messages(sb.SB_X_GATHER_ROWS, li), full).values():
                block(full, m)[...] = t
            rows, gathered = group, True
            a = full[rows]
        elif nd["node"] == sb.SB_NODE_SHARD:
            c = si.shard_bounds(nd["dimF"], K)
            full = np.zeros((B, nd["dimF"]))
            full[rows, c[off]:c[off + 1]] = a
            for m, t in exchange(messages(sb.SB_X_GATHER_COLS, li - 1), full).values():
                block(full, m)[...] = t
            a = full[rows]
        elif layers[li][0] != si.SOFTMAX_XENT:
            c = si.shard_bounds(layers[li][1], K)
            split[li] = slice(c[off], c[off + 1]) if nd["shards"] > 1 else slice(0, layers[li][1])
            inputs[li] = a
            z = a @ params[li][split[li]].T
            a = outputs[li] = z if layers[li][0] == si.FC else np.maximum(z, 0)
    d = loss_gradient(a, y[rows], B)
    grads = {}
    last = len(layers) - 2
    d = d[:, split[last]] if d.shape[1] != split[last].stop - split[last].start else d
    for li in range(last, -1, -1):
        if li < last:
            d = d * (outputs[li] > 0)
        grads[li] = d.T @ inputs[li]
        dx = d @ params[li][split[li]]          # gradient of the layer's whole input, a part of the sum where the layer is split
        width = dx.shape[1]
        back = messages(sb.SB_X_REDUCE_ROWS, li) or messages(sb.SB_X_REDUCE_COLS, li - 1)
        if back:
            mine = [m for m in back if m["dst"] == me]
            full = whole(dx, width)
            got = exchange(back, full)
            r, c = (slice(*mine[0]["rows"]), slice(*mine[0]["cols"]))
            assert all((m["rows"], m["cols"]) == (mine[0]["rows"], mine[0]["cols"]) for m in mine)
            total = np.zeros_like(full[r, c])
            for s in range(gid * K, (gid + 1) * K):
                total = total + (full[r, c] if s == me else got[s][1])
            dx = total
            if messages(sb.SB_X_REDUCE_ROWS, li):
                rows = own
        if li > 0 and dx.shape[1] != split[li - 1].stop - split[li - 1].start:
            dx = dx[:, split[li - 1]]           # a whole layer above a split one: the same gradient everywhere, this worker's columns of it
        d = dx
    for m in plan:
        g = None if m["layer"] not in grads else torch.from_numpy(np.ascontiguousarray(grads[m["layer"]]))
        if m["kind"] == sb.SB_X_ALLREDUCE:
            dist.all_reduce(g)
        elif m["kind"] == sb.SB_X_ALLREDUCE_GROUPS and m["src"] in (-1, off):
            dist.all_reduce(g, group=peers[off])
        else:
            continue
        grads[m["layer"]] = g.numpy()
    q.put((me, grads, {li: (s.start, s.stop) for li, s in split.items()}, d))
    dist.barrier()
    dist.destroy_process_group()


@pytest.mark.parametrize("N,K", [(2, 2), (4, 4), (4, 2), (2, 1)])
def test_workers_that_follow_the_plan_have_the_gradients_of_the_whole_network(N, K):
    binding()
    ctx = mp.get_context("spawn")
    q = ctx.Queue()
    port = 27000 + (os.getpid() * 7 + N * 5 + K) % 4000
    procs = [ctx.Process(target=run_worker, args=(r, N, K, port, q)) for r in range(N)]
    for p in procs:
        p.start()
    results = [q.get(timeout=300) for _ in procs]
    for p in procs:
        p.join(timeout=60)
        assert p.exitcode == 0
    ref, ref_dx = reference(N)
    for me, grads, split, dx in results:
        for li, g in grads.items():
            assert np.allclose(g, ref[li][slice(*split[li])], rtol=1e-10, atol=1e-13), (me, li)
        assert np.allclose(dx, ref_dx[me * ROWS:(me + 1) * ROWS], rtol=1e-10, atol=1e-13), me


@pytest.mark.parametrize("N,K", [(2, 2), (4, 2), (6, 3)])
def test_split_layer_on_a_gated_block_returns_the_sum_of_the_partial_gradients(N, K):
    """The split layer above the last block holds a part of that block's output gradient on every worker of a group: everyone needs the parts of all others,
    full width, before the block's backward pass.  Nothing of the kind between the blocks, or below the first."""
    b = binding()
    layers = [(si.CONV3X3_RELU, 8), (si.MAXPOOL2, 0), (si.FC_RELU, 64), (GATED, 96), (GATED, 40), (si.FC_RELU, 32), (si.FC, 10), (si.SOFTMAX_XENT, 10)]
    msgs = b.exchange_plan(layers, 8, 8, 8, 4, N, K)
    back = [m for m in msgs if m["kind"] == b.SB_X_REDUCE_COLS and m["layer"] == 4]
    assert sorted((m["src"], m["dst"]) for m in back) == [(s, d) for s in range(N) for d in range(N) if s != d and s // K == d // K]
    assert all(m["backward"] == 1 and m["cols"] == (0, 64) and m["width"] == 64 for m in back)
    assert all(m["rows"] == (m["dst"] // K * K * 4, (m["dst"] // K + 1) * K * 4) for m in back)
    assert not [m for m in msgs if m["layer"] in (2, 3) and m["kind"] == b.SB_X_REDUCE_COLS]
    assert not [m for m in msgs if m["layer"] == 4 and m["kind"] == b.SB_X_GATHER_COLS]
    at = [k for k, m in enumerate(msgs) if m in back]
    above = max(k for k, m in enumerate(msgs) if m["kind"] == b.SB_X_REDUCE_COLS and m["layer"] == 5)
    below = min(k for k, m in enumerate(msgs) if m["kind"] == b.SB_X_REDUCE_ROWS)
    assert above < min(at) and max(at) < below
