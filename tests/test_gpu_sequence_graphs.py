"""Captured calls of the page pool, of the admission to sequences and of projections staged in a memory: each replay, on new
inputs, against the same calls made eagerly elsewhere."""
import pytest
import torch

from test_gpu_sequences import World, gen, rand

pytestmark = pytest.mark.gpu

D = 64


@pytest.fixture(scope="module")
def rv():
    from paper_2609_23286_amd import rv as _rv
    _rv.init()
    return _rv


def capture(run):
    """A graph of run(), and what it returned."""
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = run()
    return g, out


def replays(g, inputs, refill, eager, outputs):
    for i in range(3):
        for t in inputs:
            t.copy_(refill(t))
        g.replay()
        torch.cuda.synchronize()
        want = eager()
        torch.cuda.synchronize()
        for n, (a, b) in enumerate(zip(outputs, want)):
            assert torch.equal(a, b), (i, n)


def test_fork_append_attend_gather(rv):
    """Children forked inside a page, which each appends to (its copy is in the graph), attended and read."""
    H, g = 3, gen(21)
    worlds = [World(rv, H, 80, 12, 900, seed=4) for _ in range(2)]
    parents = []
    for w in worlds:
        a = w.open()
        w.append([a], [300])
        parents.append(a)
    n = [5, 70, 0, 130]
    K, V = rand(g, sum(n), H, D), rand(g, sum(n), H, D)
    Q = rand(g, 8, H, D)

    def step(w, parent, fill=None):
        kids = w.pool.fork(parent, 290, 4)
        w.pool.append(kids, K, V, n)
        out, lse = torch.empty_like(Q), torch.empty(8 * H, device="cuda")
        rv.attend_seqs(Q, None, None, w.pool, kids, [2] * 4, out, lse)
        rows = [290 + r for r in n]
        k, v = (torch.empty(sum(rows) * H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        w.pool.gather(kids, k, v, rows)
        return kids, (out, lse, k, v)

    graph, (kids, outs) = capture(lambda: step(worlds[0], parents[0]))

    def eager():
        kids, outs = step(worlds[1], parents[1])
        worlds[1].pool.release(kids)
        return outs

    replays(graph, (K, V, Q), lambda t: rand(g, *t.shape), eager, outs)
    worlds[0].verify([parents[0]])
    assert [worlds[0].pool.len(k) for k in kids] == [290 + r for r in n]


def test_compact_gather(rv):
    H, g = 2, gen(22)
    w = World(rv, H, 60, 4, 900, seed=5)
    a, b = w.open(), w.open()
    w.append([a, b], [500, 200])
    rows = {s: w.rows[s] for s in (a, b)}
    n, first = [170, 40], [100, 64]
    keep = torch.zeros(H * sum(n), dtype=torch.int32, device="cuda")

    def refill(t):
        parts = [torch.randint(f, w.rows[s][0].shape[1], (H * k,), generator=g, device="cuda", dtype=torch.int32)
                 for s, k, f in zip((a, b), n, first)]
        return torch.cat(parts)

    keep.copy_(refill(keep))

    def step():
        w.pool.compact([a, b], keep, n, first)
        out = torch.empty(H * (sum(n) + sum(first)), D, dtype=torch.bfloat16, device="cuda")
        w.pool.gather([a, b], out, None, [f + k for f, k in zip(first, n)])
        return (out,)

    def model():
        out, at = [], 0
        for s, k, f in zip((a, b), n, first):
            idx = keep[at:at + H * k].view(H, k).long()[..., None].expand(-1, -1, D)
            out.append(torch.cat((rows[s][0][:, :f], rows[s][0].gather(1, idx)), dim=1).reshape(-1, D))
            at += H * k
        return (torch.cat(out),)

    graph, outs = capture(step)
    replays(graph, (keep,), refill, model, outs)


def test_attend_admit_gather(rv):
    H, N, k, n, g = 4, 45, 6, 3, gen(23)
    worlds = [World(rv, H, 60, 8, 400, seed=6) for _ in range(2)]
    seqs = []
    for w in worlds:
        seqs.append([w.open() for _ in range(n)])
        w.append(seqs[-1], [70, 0, 128])
    Q, K, V = (rand(g, n, N, H, D) for _ in range(3))

    def step(w, seqs):
        flat = [t.view(-1, H, D) for t in (Q, K, V)]
        out, lse = torch.empty_like(flat[0]), torch.empty(n, H, N, device="cuda")
        rv.attend_seqs(*flat, w.pool, seqs, [N] * n, out, lse)
        sal, idx = torch.empty_like(lse), torch.empty(n, H, k, dtype=torch.int32, device="cuda")
        rv.admit_seqs(Q, K, V, lse, (6, 7, 3, 2), k, w.pool, seqs, sal, idx)
        rows = [r + k for r in (70, 0, 128)]
        got = torch.empty(sum(rows) * H, D, dtype=torch.bfloat16, device="cuda")
        w.pool.gather(seqs, None, got, rows)
        return out, lse, sal, idx, got

    graph, outs = capture(lambda: step(worlds[0], seqs[0]))

    def eager():
        outs = step(worlds[1], seqs[1])
        for s, r in zip(seqs[1], (70, 0, 128)):
            worlds[1].pool.truncate(s, r)
        return outs

    replays(graph, (Q, K, V), lambda t: rand(g, *t.shape), eager, outs)


def test_stage_attend_staged(rv):
    H, N, g = 4, 75, gen(24)
    prep = rv.QKVPrep(H, H, norm="rms", axes=1, base=10000.0)
    x = rand(g, N, 3 * H * D)
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    old = rand(g, H, 90, D)
    mems = [rv.Memory(H, reserve_tokens=400, max_tokens=400) for _ in range(2)]
    for m in mems:
        m.write(old, old)

    def step(m):
        Q = torch.empty(N, H, D, dtype=torch.bfloat16, device="cuda")
        rv.stage_qkv(prep, *x.split(H * D, dim=1), pos, Q, m)
        out, lse = torch.empty_like(Q), torch.empty(H, N, device="cuda")
        rv.attend_staged(Q, m, out, lse)
        return Q, out, lse

    graph, outs = capture(lambda: step(mems[0]))
    replays(graph, (x,), lambda t: rand(g, *t.shape), lambda: step(mems[1]), outs)
