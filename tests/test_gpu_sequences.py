"""Paged sequences and the attention over them on the GPU: rows bit for bit against a plain model,
attention against the definition in 64 bits.

The attention's bound is util.out_error_bound (probabilities, partial outputs and the output are each
rounded to bf16), the log-sum-exp's LSE_ATOL."""
import math

import numpy as np
import pytest
import torch

from util import LSE_ATOL, out_error_bound

pytestmark = pytest.mark.gpu

D = 64


@pytest.fixture(scope="module")
def rv():
    from paper_2609_23286_amd import rv as _rv
    _rv.init()
    return _rv


def rand(gen, *shape, scale=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale).bfloat16()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


class World:
    """A pool and, per open sequence, its K and V rows [H, n, 64]."""

    def __init__(self, rv, H, pages, seqs, max_rows, seed=0):
        self.rv, self.H, self.g = rv, H, gen(seed)
        self.pool = rv.Pool(H, pages, seqs, max_rows)
        self.rows = {}

    def open(self):
        s = self.pool.open()
        self.rows[s] = (torch.empty(self.H, 0, D, dtype=torch.bfloat16, device="cuda"),) * 2
        return s

    def append(self, seqs, n):
        K, V = rand(self.g, sum(n), self.H, D), rand(self.g, sum(n), self.H, D)
        self.pool.append(seqs, K, V, n)
        at = 0
        for s, r in zip(seqs, n):
            self.rows[s] = tuple(torch.cat((old, new[at:at + r].transpose(0, 1)), dim=1)
                                 for old, new in zip(self.rows[s], (K, V)))
            at += r

    def fork(self, s, n_rows=None, n=1):
        out = self.pool.fork(s, n_rows, n)
        for c in out:
            self.rows[c] = tuple(t[:, :n_rows] if n_rows is not None else t for t in self.rows[s])
        return out

    def release(self, seqs):
        self.pool.release(seqs)
        for s in seqs:
            del self.rows[s]

    def compact(self, seqs, n_keep, first):
        keeps = []
        for s, k, f in zip(seqs, n_keep, first):
            n = self.rows[s][0].shape[1]
            keep = torch.randint(f, n, (self.H, k), generator=self.g, device="cuda", dtype=torch.int32)
            keeps.append(keep.flatten())
            idx = keep.long()[..., None].expand(-1, -1, D)
            self.rows[s] = tuple(torch.cat((t[:, :f], t.gather(1, idx)), dim=1) for t in self.rows[s])
        self.pool.compact(seqs, torch.cat(keeps), n_keep, first)

    def verify(self, seqs=None):
        seqs = sorted(self.rows) if seqs is None else seqs
        n = [self.rows[s][0].shape[1] for s in seqs]
        assert [self.pool.len(s) for s in seqs] == n
        K = torch.full((sum(n) * self.H + 1, D), 7.0, dtype=torch.bfloat16, device="cuda")
        V = K.clone()
        self.pool.gather(seqs, K[:-1], V[:-1], n)
        for got, i in ((K, 0), (V, 1)):
            want = torch.cat([self.rows[s][i].reshape(-1, D) for s in seqs]) if seqs else K[:0]
            assert torch.equal(got[:-1], want)
            assert bool((got[-1] == 7).all()), "a row behind the last was written"

    def check_attention(self, seqs, n_tokens, group=1, frame=True, scale=1.0, sampled=None, out_lse=None):
        H, Hq, total = self.H, self.H * group, sum(n_tokens)
        Q = rand(self.g, total, Hq, D, scale=scale)
        K, V = (rand(self.g, total, H, D) if frame else None for _ in range(2))
        out = torch.full((total + 1, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((total * Hq + 1,), 7.0, device="cuda")
        self.rv.attend_seqs(Q, K, V, self.pool, seqs, n_tokens, out[:total], lse[:-1])
        assert bool((out[total] == 7).all()) and float(lse[-1]) == 7
        at = 0
        for s, n in zip(seqs, n_tokens):
            k, v = self.rows[s]
            if frame:
                k, v = (torch.cat((t, f[at:at + n].transpose(0, 1)), dim=1) for t, f in ((k, K), (v, V)))
            got_lse = lse[at * Hq:(at + n) * Hq].reshape(Hq, n)
            if n:
                self.check_one(Q[at:at + n], k, v, out[at:at + n], got_lse, group)
            at += n
        return Q, K, V, out[:total], lse[:-1]

    @staticmethod
    def check_one(q, k, v, out, lse, group):
        for hq in range(q.shape[1]):
            kk, vv = k[hq // group].double(), v[hq // group].double()
            if len(kk) == 0:
                assert bool((out[:, hq] == 0).all()) and bool((lse[hq] == -math.inf).all())
                continue
            z = q[:, hq].double() @ kk.t() / 8
            ref = torch.softmax(z, 1) @ vv
            bound = out_error_bound(ref.cpu().numpy(), float(vv.abs().max()))
            err = float((out[:, hq].double() - ref).abs().max())
            assert err <= bound, (hq, err, bound)
            err = float((lse[hq].double() - torch.logsumexp(z, 1)).abs().max())
            assert err <= LSE_ATOL, (hq, err)


# ---- rows ---------------------------------------------------------------------------------

@pytest.mark.parametrize("H", [1, 3, 16])
def test_append_in_parts_and_at_page_borders(rv, H):
    w = World(rv, H, 40, 4, 700)
    s = [w.open() for _ in range(3)]
    for n in ([1, 63, 64], [63, 1, 65], [0, 130, 1], [64, 0, 0], [200, 2, 127]):
        w.append(s, n)
        w.verify()
    assert w.pool.free_pages == 40 - sum(-(-w.pool.len(q) // 64) for q in s)


def test_forks_share_pages_and_copy_on_append(rv):
    w = World(rv, 4, 30, 12, 1000)
    a = w.open()
    w.append([a], [300])  # 5 pages, the last with 44 rows
    free = w.pool.free_pages
    kids = w.fork(a, n=3) + w.fork(a, 280) + w.fork(a, 256) + w.fork(a, 0)
    assert w.pool.free_pages == free
    w.verify()
    w.append([a] + kids, [1, 20, 0, 64, 5, 1, 2])
    w.verify()
    w.append([kids[1]], [3])  # the only one left on the first page 4
    w.verify()
    w.release([a, kids[0]])
    w.append(kids[1:], [70] * 5)
    w.verify()
    w.release(kids[1:])
    assert w.pool.free_pages == 30


def test_a_longer_fork_is_copied_while_a_shorter_one_is_written(rv):
    """Both share a page; one call appends to both: the longer one's rows are read whole."""
    for order in (0, 1):
        w = World(rv, 2, 20, 4, 400, seed=order)
        a = w.open()
        w.append([a], [120])
        b = w.fork(a, 100)[0]
        w.append([a, b] if order else [b, a], [30, 30])
        w.verify()


@pytest.mark.parametrize("seed", range(4))
def test_random_operations(rv, seed):
    r = np.random.RandomState(seed)
    w = World(rv, int(r.choice([1, 2, 5])), 60, 12, 900, seed)
    w.open()
    for step in range(60):
        seqs = list(w.rows)
        what = r.randint(6)
        some = [int(s) for s in r.permutation(seqs)[:r.randint(1, 5)]]
        try:
            if what == 0:
                w.open()
            elif what == 1:
                s = some[0]
                w.fork(s, r.randint(w.pool.len(s) + 1), r.randint(1, 3))
            elif what in (2, 3):
                w.append(some, [int(x) for x in r.randint(0, 150, len(some))])
            elif what == 4:
                some = [s for s in some if w.pool.len(s) > 0]
                first = [int(r.randint(w.pool.len(s))) for s in some]
                if some:
                    w.compact(some, [int(x) for x in r.randint(1, 200, len(some))], first)
            elif len(seqs) > 3:
                w.release(some[:1])
        except rv.RVError as e:
            assert e.status == rv.RV_ERR_CAPACITY
            if what == 4:  # (the model went ahead)
                break
        if step % 6 == 5:
            w.verify()


def test_batches_of_many_sequences(rv):
    """More sequences, pages and runs than one launch's arguments hold."""
    w = World(rv, 2, 1200, 300, 40000)
    a = w.open()
    w.append([a], [100])
    kids = w.fork(a, n=290)
    w.append(kids, [(i * 37) % 150 for i in range(290)])
    w.verify()
    w.compact(kids[:150], [1 + i % 90 for i in range(150)], [i % 101 for i in range(150)])
    w.verify()
    w.release(kids)
    w.append([a], [30000])  # 470 pages, out of order after the releases
    w.verify()
    w.compact([a], [20000], [70])
    w.verify()


def test_compaction_picks_rows_per_head(rv):
    w = World(rv, 3, 60, 4, 2000)
    a = w.open()
    w.append([a], [700])
    b = w.fork(a)[0]
    w.compact([b], [1], [0])
    w.verify()
    w.compact([a], [650], [130])  # repeats allowed
    w.verify()
    # numbers outside [first, length) give rows of zeros
    n = w.pool.len(a)
    keep = torch.tensor([[0, 64, n, -1, 65], [n - 1, 2 ** 31 - 1, 63, 64, 64], [64, 64, 64, 64, -2 ** 31]],
                        dtype=torch.int32, device="cuda")
    ok = (keep >= 64) & (keep < n)
    w.rows[a] = tuple(torch.cat((t[:, :64], t.gather(1, keep.long().clamp(0, n - 1)[..., None].expand(-1, -1, D)) *
                                 ok[..., None]), dim=1) for t in w.rows[a])
    w.pool.compact([a], keep, [5], [64])
    w.verify()
    w.pool.compact([a], None, [0], [65])  # nothing kept behind row 65: a truncation
    w.rows[a] = tuple(t[:, :65] for t in w.rows[a])
    w.verify()


def test_gather_ranges(rv):
    w = World(rv, 5, 20, 4, 900)
    a = w.open()
    w.append([a], [500])
    first, n = [0, 63, 64, 100, 499, 500], [1, 2, 64, 400, 1, 0]
    K = torch.empty(sum(n) * 5, D, dtype=torch.bfloat16, device="cuda")
    w.pool.gather([a] * 6, K, None, n, first)
    want = torch.cat([w.rows[a][0][:, f:f + r].reshape(-1, D) for f, r in zip(first, n)])
    assert torch.equal(K, want)


# ---- attention ------------------------------------------------------------------------------

@pytest.mark.parametrize("rows", [0, 1, 63, 64, 65, 1000])
@pytest.mark.parametrize("tokens", [1, 33, 130])
@pytest.mark.parametrize("frame", [False, True])
def test_one_sequence(rv, rows, tokens, frame):
    w = World(rv, 2, 20, 2, 1100, seed=rows + tokens)
    s = w.open()
    w.append([s], [rows])
    w.check_attention([s], [tokens], frame=frame)


@pytest.mark.parametrize("H,group", [(1, 1), (4, 4), (2, 8), (3, 5), (16, 1)])
@pytest.mark.parametrize("tokens", [1, 5, 40])
def test_forks_of_a_long_prefix(rv, H, group, tokens):
    w = World(rv, H, 200, 20, 3000, seed=H + tokens)
    a = w.open()
    w.append([a], [2100])
    kids = w.fork(a, n=9)
    w.append(kids, [0, 1, 28, 44, 64, 100, 300, 7, 500])
    w.check_attention(kids, [tokens] * 9, group, frame=tokens > 1)


def test_a_tree_of_forks_and_strangers(rv):
    w = World(rv, 4, 300, 30, 3000)
    a, z = w.open(), w.open()
    w.append([a, z], [1000, 130])
    b = w.fork(a, 900, 2)
    w.append(b, [500, 620])
    c = w.fork(b[0], n=3) + w.fork(b[1], n=4)
    w.append(c, [10, 200, 0, 64, 1, 1, 333])
    empty = w.open()
    order = [z] + c[:3] + [b[0], empty] + c[3:] + [b[1], a, a, z]
    tokens = [3, 1, 2, 0, 5, 4, 1, 1, 70, 2, 1, 200, 1, 9]
    for frame in (False, True):
        w.check_attention(order, tokens, group=2, frame=frame)


def test_whole_frames_over_a_shared_prefix(rv):
    w = World(rv, 8, 100, 8, 2000)
    a = w.open()
    w.append([a], [1500])
    kids = w.fork(a, n=3)
    w.append(kids, [100, 3, 0])
    w.check_attention(kids, [1041, 700, 129], frame=True)
    w.check_attention([a], [1374], frame=True, scale=3.0)


@pytest.mark.parametrize("H,lengths,tokens", [
    (16, [130] * 8, 513),               # more query tiles than workgroups at a time: some are dealt out whole
    (16, [130, 200, 129, 250] * 2, 513),  # and of different lengths
    (16, [64] * 7, 640),                # 560 tiles: a round and a small rest
    (2, [3000], 300),                   # six tiles, each in equal pieces
    (2, [3000, 3000], 129),
    (1, [40], 300),                     # short: whole tiles
    (2, [5000, 2000], 300),             # different lengths: chunks that run from one tile into the next
    (16, [1500], 1041),
], ids=str)
def test_strangers_with_many_queries(rv, H, lengths, tokens):
    w = World(rv, H, sum(n // 64 + 2 for n in lengths), len(lengths), max(lengths) + 64)
    seqs = [w.open() for _ in lengths]
    w.append(seqs, lengths)
    w.check_attention(seqs, [tokens] * len(seqs), frame=True)


def test_more_sequences_than_a_launch_takes(rv):
    w = World(rv, 2, 700, 200, 600)
    a = w.open()
    w.append([a], [200])
    kids = w.fork(a, n=150)
    w.append(kids, [i % 97 for i in range(150)])
    pairs = [c for k in kids for c in (k, w.fork(k)[0] if k < 40 else k)]
    w.check_attention(pairs, [1 + i % 3 for i in range(len(pairs))], frame=False)


def test_long_memory(rv):
    w = World(rv, 2, 1700, 8, 53041)
    a = w.open()
    w.append([a], [52000])
    kids = w.fork(a, n=5)
    w.append(kids, [1041, 0, 64, 3, 500])
    w.check_attention(kids, [1, 5, 2, 1, 17], group=2, frame=True)


def test_rows_past_a_sequences_end_are_never_used(rv):
    """The pages first hold NaN and infinities everywhere."""
    w = World(rv, 2, 12, 4, 700)
    s = w.open()
    bad = torch.full((700, 2, D), math.nan, dtype=torch.bfloat16, device="cuda")
    bad[::2] = math.inf
    w.pool.append([s], bad, bad, [700])
    w.pool.release([s])
    s = w.open()
    w.append([s], [65])
    t = w.fork(s, 3)[0]
    for tokens in (1, 40, 140):
        w.check_attention([s, t], [tokens, tokens], frame=False)
        w.check_attention([s, t], [tokens, tokens], frame=True)


def test_large_logits_and_late_maxima(rv):
    """Scores rise over the pages, so that the softmax's reference has to follow."""
    w = World(rv, 1, 80, 4, 3000)
    s = w.open()
    n = 2000
    K = rand(w.g, n, 1, D) * torch.linspace(0.01, 12, n, device="cuda").bfloat16()[:, None, None]
    V = rand(w.g, n, 1, D)
    w.pool.append([s], K, V, [n])
    w.rows[s] = (K.transpose(0, 1), V.transpose(0, 1))
    k = w.fork(s, 1990, 3)
    # |z| reaches a few hundred: 2^-24 of it, 64 products and the base-2 factor, stays below 1e-4
    w.check_attention([s] + k, [1, 2, 40, 1], frame=False, scale=2.0)


def test_results_repeat_and_do_not_depend_on_the_stream(rv):
    w = World(rv, 4, 100, 8, 2000)
    a = w.open()
    w.append([a], [1000])
    kids = w.fork(a, n=4)
    w.append(kids, [10, 20, 30, 40])
    Q, K, V, out, lse = w.check_attention(kids, [1, 3, 60, 2], frame=True)
    out2, lse2 = torch.zeros_like(out), torch.zeros_like(lse)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    rv.attend_seqs(Q, K, V, w.pool, kids, [1, 3, 60, 2], out2, lse2, stream=s)
    s.synchronize()
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


def test_captured_step(rv):
    """append, attend and truncate as one captured step, replayed on new inputs."""
    w = World(rv, 4, 100, 8, 2000)
    a = w.open()
    w.append([a], [1000])
    kids = w.fork(a, n=4)
    w.append(kids, [10] * 4)
    Q, K, V = (rand(w.g, 8, 4, D) for _ in range(3))
    out, lse = torch.empty_like(Q), torch.empty(4, 4, 2, device="cuda")
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        w.pool.append(kids, K, V, [2] * 4)
        rv.attend_seqs(Q, None, None, w.pool, kids, [2] * 4, out, lse)
    for i in range(3):
        for t in (Q, K, V):
            t.copy_(rand(w.g, 8, 4, D))
        g.replay()
        torch.cuda.synchronize()
        for j, s in enumerate(kids):
            k, v = (torch.cat((t, n[2 * j:2 * j + 2].transpose(0, 1)), dim=1) for t, n in zip(w.rows[s], (K, V)))
            w.check_one(Q[2 * j:2 * j + 2], k, v, out[2 * j:2 * j + 2], lse[j], 1)


# ---- with the path that is there --------------------------------------------------------------

def test_a_stream_in_pages_equals_a_stream_in_memories(rv):
    """Projections to admitted rows, frame by frame, for several streams at once in a pool and one by
    one in memories: the same selections and the same rows."""
    H, grid, k, n = 4, (6, 7, 3, 2), 5, 3
    N = 6 * 7 + 3
    g = gen(5)
    prep = rv.QKVPrep(H, H, norm="layer", axes=2)
    t = torch.arange(N, device="cuda") - 3
    pos = torch.where(t[:, None] >= 0, torch.stack((t // 7 + 1, t % 7 + 1), 1), 0).to(torch.int32)
    pool = rv.Pool(H, 40, 8, 400)
    seqs = [pool.open() for _ in range(n)]
    mems = [rv.Memory(H, reserve_tokens=64, max_tokens=400) for _ in range(n)]

    def frame(seqs, mems, budget, frame_id):
        n = len(seqs)
        x = torch.randn(n * N, 3 * H * D, generator=g, device="cuda").bfloat16()
        q, kk, v = x.split(H * D, dim=1)
        Q, K, V = (torch.empty(n * N, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(3))
        rv.prepare_qkv(prep, q, kk, v, pos.repeat(n, 1), Q, K, V)
        out, lse = torch.empty_like(Q), torch.empty(n, H, N, device="cuda")
        rv.attend_seqs(Q, K, V, pool, seqs, [N] * n, out, lse)
        sal = torch.empty(n, H, N, device="cuda")
        idx = torch.empty(n, H, budget, dtype=torch.int32, device="cuda")
        four = [t.view(n, N, H, D) for t in (Q, K, V)]
        rv.admit_seqs(*four, lse, grid, budget, pool, seqs, sal, idx)
        for i, m in enumerate(mems):
            o, l = torch.empty(N, H, D, dtype=torch.bfloat16, device="cuda"), torch.empty(H, N, device="cuda")
            rv.attend_frame(four[0][i], four[1][i], four[2][i], m, o, l)
            assert float((l - lse[i]).abs().max()) <= LSE_ATOL
            s2, i2 = torch.empty_like(sal[i]), torch.empty_like(idx[i])
            # the pool's own log-sum-exp: the selection and the rows are then the same to the bit
            rv.admit_layers([four[0][i]], [four[1][i]], [four[2][i]], [lse[i]], grid, budget, [m], frame_id, [s2], [i2])
            assert torch.equal(s2, sal[i]) and torch.equal(i2, idx[i])
        for s, m in zip(seqs, mems):
            rows = m.len
            assert pool.len(s) == rows
            gk, gv = (torch.empty(H * rows, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            pool.gather([s], gk, gv, [rows])
            mk, mv, _ = m.read()
            assert torch.equal(gk.view(torch.int16).cpu(), mk.view(-1, D))
            assert torch.equal(gv.view(torch.int16).cpu(), mv.view(-1, D))

    frame(seqs, mems, N, 0)  # the anchor frame: every row
    for f in range(1, 5):
        frame(seqs, mems, k, f)
    # continuations of the first stream
    kids = pool.fork(seqs[0], n=3)
    copies = []
    for _ in kids:
        m = rv.Memory(H, reserve_tokens=400, max_tokens=400)
        rows = [t.contiguous() for t in mems[0].read()[:2]]
        m.write(*rows)
        copies.append(m)
    frame(kids, copies, k, 5)


def test_admission_of_more_sequences_than_a_launch_takes(rv):
    H, N, k, n = 2, 30, 3, 53
    g = gen(6)
    pool = rv.Pool(H, 120, 60, 100)
    seqs = [pool.open() for _ in range(n)]
    Q, K, V = (rand(g, n, N, H, D) for _ in range(3))
    out, lse = torch.empty(n * N, H, D, dtype=torch.bfloat16, device="cuda"), torch.empty(n, H, N, device="cuda")
    rv.attend_seqs(Q.view(-1, H, D), K.view(-1, H, D), V.view(-1, H, D), pool, seqs, [N] * n, out, lse)
    sal = torch.empty(n, H, N, device="cuda")
    idx = torch.empty(n, H, k, dtype=torch.int32, device="cuda")
    rv.admit_seqs(Q, K, V, lse, (5, 6, 0, 2), k, pool, seqs, sal, idx)
    gk = torch.empty(n, H, k, D, dtype=torch.bfloat16, device="cuda")
    pool.gather(seqs, gk, None, [k] * n)
    want = K.transpose(1, 2).gather(2, idx.long()[..., None].expand(-1, -1, -1, D))
    assert torch.equal(gk, want)
    assert torch.equal(sal.topk(k, dim=2).indices.sort(2).values.int(), idx)


# ---- refusals, bindings, graphs, sizes -----------------------------------------------------------

def refused(rv, status, words, call, *args, **kw):
    with pytest.raises(rv.RVError, match=words) as e:
        call(*args, **kw)
    assert e.value.status == status


def test_refusals_change_nothing(rv):
    w = World(rv, 2, 10, 5, 300)  # 3 pages taken below; the appends refused for pages need 8, the compaction 10
    pool = w.pool
    a, b = w.open(), w.open()
    w.append([a, b], [100, 64])
    c = w.fork(a, 90)[0]
    free = pool.free_pages
    K = rand(w.g, 400, 2, D)
    INV, CAP = rv.RV_ERR_INVALID, rv.RV_ERR_CAPACITY
    gone = w.open()
    w.release([gone])
    refused(rv, INV, "named twice", pool.append, [a, a], K[:2], K[:2], [1, 1])
    refused(rv, INV, "not open", pool.append, [gone], K[:1], K[:1], [1])
    refused(rv, INV, "not open", pool.append, [-1], K[:1], K[:1], [1])
    refused(rv, INV, "not open", pool.append, [5], K[:1], K[:1], [1])
    refused(rv, CAP, "max_rows", pool.append, [a, b], K[:202], K[:202], [1, 201][::-1])
    refused(rv, INV, "K and V are required", pool.append, [a], None, K[:1], [1])
    refused(rv, CAP, "pages", pool.append, [a, b, c], K, K, [150, 100, 150])
    with pytest.raises(ValueError, match="shape"):
        pool.append([a], K[:2], K[:2], [1])
    with pytest.raises(ValueError, match="contiguous"):
        pool.append([a], K[:2, :, :].transpose(0, 1).contiguous().transpose(0, 1), K[:2], [2])
    refused(rv, INV, "n_rows", pool.fork, a, 101)
    refused(rv, INV, "n_rows", pool.fork, a, -1)
    refused(rv, INV, "not open", pool.fork, gone, 0)
    refused(rv, CAP, "can be opened", pool.fork, a, 10, 3)
    refused(rv, INV, "n_rows", pool.truncate, a, 101)
    refused(rv, INV, "named twice", pool.release, [b, b])
    refused(rv, INV, "rows", pool.gather, [a], K[:2].view(4, D), None, [2], [99])
    refused(rv, INV, "rows", pool.gather, [a], K[:2].view(4, D), None, [2], [-1])
    keep = torch.zeros(2 * 500, dtype=torch.int32, device="cuda")
    refused(rv, INV, "first", pool.compact, [a], keep[:2], [1], [101])
    refused(rv, CAP, "max_rows", pool.compact, [a], keep[:2 * 250], [250], [64])
    refused(rv, CAP, "pages", pool.compact, [a, b, c], keep, [200, 140, 160], [0, 0, 0])
    refused(rv, INV, "keep is NULL", pool.compact, [a], None, [1], [0])
    with pytest.raises(ValueError, match="keep"):
        pool.compact([a], keep[:3], [1], [0])
    Q, lse = rand(w.g, 3, 2, D), torch.empty(6, device="cuda")
    out = torch.empty_like(Q)
    refused(rv, INV, "not open", rv.attend_seqs, Q, None, None, pool, [gone], [3], out, lse)
    refused(rv, INV, "both", rv.attend_seqs, Q, Q, None, pool, [a], [3], out, lse)
    refused(rv, INV, "multiple of 2", rv.attend_seqs, Q[:, :1].contiguous(), None, None, pool, [a], [3],
            out[:, :1].contiguous(), lse[:3])
    with pytest.raises(ValueError, match="lse"):
        rv.attend_seqs(Q, None, None, pool, [a], [3], out, lse[:5])
    with pytest.raises(ValueError, match="shape"):
        rv.attend_seqs(Q, None, None, pool, [a], [2], out, lse[:4])
    with pytest.raises(ValueError, match="sequences"):
        rv.attend_seqs(Q, None, None, pool, [a, b], [3], out, lse)
    four = Q[None].expand(2, -1, -1, -1).contiguous()
    sal, idx = torch.empty(2, 2, 3, device="cuda"), torch.empty(2, 2, 1, dtype=torch.int32, device="cuda")
    refused(rv, INV, "named twice", rv.admit_seqs, four, four, four, sal, (1, 3, 0, 2), 1, pool, [a, a], sal, idx)
    refused(rv, INV, "does not describe", rv.admit_seqs, four, four, four, sal, (1, 2, 0, 2), 1, pool, [a, b], sal, idx)
    refused(rv, INV, "budget", rv.admit_seqs, four, four, four, sal, (1, 3, 0, 2), 4, pool, [a, b], sal,
            torch.empty(2, 2, 4, dtype=torch.int32, device="cuda"))
    assert pool.free_pages == free
    w.verify()
    for _ in range(2):  # what is left can still be opened and filled
        w.open()
    refused(rv, CAP, "open", pool.open)
    w.append([a, b, c], [10, 10, 10])
    w.verify()


def test_a_pool_too_large_for_the_device(rv):
    free = torch.cuda.mem_get_info()[0]
    refused(rv, rv.RV_ERR_OOM, "pool allocation", rv.Pool, 1024, 1 << 30, 4, 1000)
    assert abs(torch.cuda.mem_get_info()[0] - free) < 1 << 28
    World(rv, 1, 2, 1, 10).open()


def test_a_refused_stage_leaves_the_memory_alone(rv):
    mem = rv.Memory(2, reserve_tokens=4, max_tokens=8)
    prep = rv.QKVPrep(2, 2, norm="rms", axes=0)
    x = torch.zeros(9, 128, dtype=torch.bfloat16, device="cuda")
    Q = torch.zeros(9, 2, D, dtype=torch.bfloat16, device="cuda")
    refused(rv, rv.RV_ERR_CAPACITY, "max_tokens", rv.stage_qkv, prep, x, x, x, None, Q, mem)
    refused(rv, rv.RV_ERR_INVALID, "kv heads", rv.stage_qkv, rv.QKVPrep(2, 1, axes=0, norm=None), x, x[:, :64], x[:, :64],
            None, Q, mem)
    assert mem.len == 0 and mem.capacity == 4


def test_tensors_of_another_device_are_refused(rv, monkeypatch):
    w = World(rv, 2, 12, 5, 300)
    a = w.open()
    K = rand(w.g, 2, 2, D)
    monkeypatch.setattr(rv, "_where", lambda stream: (1, 0))
    with pytest.raises(ValueError, match="device 0 while device 1"):
        w.pool.append([a], K, K, [2])
    with pytest.raises(ValueError, match="device 0 while device 1"):
        rv.attend_seqs(K, None, None, w.pool, [a], [2], K, torch.empty(4, device="cuda"))
    prep = rv.QKVPrep(2, 2, norm=None, axes=0)
    x = K.view(2, 128)
    with pytest.raises(ValueError, match="device 0 while device 1"):
        rv.prepare_qkv(prep, x, x, x, None, K, K, K)
    assert w.pool.len(a) == 0


class Index(int):
    pass


def test_plain_and_other_arguments_give_the_same(rv):
    """What _rv_bind does not take (other integer types, bit views, subclasses) goes through ctypes."""
    outs = []
    for way in range(2):
        w = World(rv, 2, 20, 6, 300, seed=3)
        K, V = rand(w.g, 90, 2, D), rand(w.g, 90, 2, D)
        if way:
            class Sub(torch.Tensor):
                pass
            K, V = K.view(torch.int16), V.as_subclass(Sub)
        num = Index if way else int
        a = w.pool.open()
        w.pool.append([num(a)], K, V, [num(90)])
        kids = w.pool.fork(num(a), num(80), num(2))
        w.pool.append(tuple(num(k) for k in kids), K[:5], V[:5], (num(2), num(3)))
        Q = rand(gen(9), 4, 4, D)
        out, lse = torch.empty_like(Q), torch.empty(16, device="cuda")
        rv.attend_seqs(Q.view(torch.int16) if way else Q, None, None, w.pool, [num(k) for k in kids], [num(1), num(3)], out, lse)
        keep = torch.tensor([[70, 1], [5, 5]], dtype=torch.int32, device="cuda")
        w.pool.compact([num(kids[0])], keep, [num(2)], [num(1)])
        got = torch.empty(6 + 166, D, dtype=torch.bfloat16, device="cuda")
        w.pool.gather([num(k) for k in kids], got, None, [num(3), num(83)])
        w.pool.release([num(kids[1])])
        outs.append((out, lse, got, torch.tensor([w.pool.free_pages, *kids])))
        prep = rv.QKVPrep(2, 1, norm="rms", axes=1, base=10000.0)
        q, k, v = (rand(gen(s), 3, h * D) for s, h in ((1, 2), (2, 1), (3, 1)))
        if way:
            q, k, v = (t.view(torch.int16) for t in (q, k, v))
        res = [torch.empty(3, h, D, dtype=torch.bfloat16, device="cuda") for h in (2, 1, 1)]
        pos = torch.arange(3, dtype=torch.int32, device="cuda")
        rv.prepare_qkv(prep, q, k, v, pos if way else pos[:, None], *res)
        outs[-1] += tuple(res)
    assert all(torch.equal(x, y) for x, y in zip(*outs))


def test_two_graphs_share_the_workspace(rv):
    w = World(rv, 2, 200, 20, 4000)
    a = w.open()
    w.append([a], [3000])
    kids = w.fork(a, n=8)
    w.append(kids, [5 * i for i in range(8)])
    cases = []
    for tokens in ([1] * 8, [40, 3, 0, 1, 1, 1, 1, 130]):
        n = sum(tokens)
        Q, K, V = (rand(w.g, n, 2, D) for _ in range(3))
        out, lse = torch.empty_like(Q), torch.empty(2 * n, device="cuda")
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            rv.attend_seqs(Q, K, V, w.pool, kids, tokens, out, lse)
        cases.append((g, tokens, Q, K, V, out, lse))
    for rep in range(3):
        for g, tokens, Q, K, V, out, lse in cases:
            for t in (Q, K, V):
                t.copy_(rand(w.g, *t.shape))
            g.replay()
            o2, l2 = torch.empty_like(out), torch.empty_like(lse)
            rv.attend_seqs(Q, K, V, w.pool, kids, tokens, o2, l2)
            torch.cuda.synchronize()
            assert torch.equal(out, o2) and torch.equal(lse, l2)


def test_rows_past_four_gigabytes(rv):
    """2.5 million rows of 16 heads: 5.1 GB of keys, page offsets past 2^32 bytes."""
    H, part, parts = 16, 500_000, 5
    pool = rv.Pool(H, part * parts // 64 + 40, 4, part * parts + 64)
    s = pool.open()
    g = gen(11)
    last = None
    for i in range(parts):
        K = torch.empty(part, H, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        V = torch.empty(part, H, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        pool.append([s], K, V, [part])
        if i == parts - 1:
            last = K, V
        del K, V
    n = part * parts
    got = torch.empty(H, 100, D, dtype=torch.bfloat16, device="cuda")
    pool.gather([s], None, got, [100], [n - 100])
    assert torch.equal(got, last[1][-100:].transpose(0, 1))
    keep = torch.randint(n - 5000, n, (H, 70), generator=g, device="cuda", dtype=torch.int32)
    c = pool.fork(s, n)[0]
    Q = rand(g, 2, H, D)
    out, lse = torch.empty_like(Q), torch.empty(H, 2, device="cuda")
    rv.attend_seqs(Q, None, None, pool, [c], [2], out, lse)
    for h in (0, H - 1):
        k, v = torch.empty(1, n, D, dtype=torch.bfloat16, device="cuda"), None
        K = torch.empty(H, n, D, dtype=torch.bfloat16, device="cuda")
        pool.gather([c], K, None, [n])
        k = K[h].clone()
        pool.gather([c], None, K, [n])
        v = K[h].clone()
        del K
        z = Q[:, h].double() @ k.double().t() / 8
        ref = torch.softmax(z, 1) @ v.double()
        assert float((out[:, h].double() - ref).abs().max()) <= out_error_bound(ref.cpu().numpy(), float(v.abs().max()))
        assert float((lse[h].double() - torch.logsumexp(z, 1)).abs().max()) <= LSE_ATOL
    pool.compact([c], keep, [70])
    got = torch.empty(H, 70, D, dtype=torch.bfloat16, device="cuda")
    pool.gather([c], got, None, [70])
    rows = (keep.long() - (n - part))[..., None].expand(-1, -1, D)
    assert torch.equal(got, last[0].transpose(0, 1).gather(1, rows))
    pool.close()
