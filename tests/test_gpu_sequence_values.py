"""Attention over sequences on the GPU, each element against its own bound and each head as a whole (attention_bounds):
over long contexts an output is far smaller than the values it is made of."""
import math

import pytest
import torch

from attention_bounds import check_rows
from test_gpu_sequences import World, gen, rand
from util import LSE_ATOL

pytestmark = pytest.mark.gpu

D = 64


@pytest.fixture(scope="module")
def rv():
    from paper_2609_23286_amd import rv as _rv
    _rv.init()
    return _rv


class Checked(World):
    """Checks every head of every sequence by attention_bounds."""

    @staticmethod
    def check_one(q, k, v, out, lse, group):
        for hq in range(q.shape[1]):
            kk, vv = k[hq // group].double(), v[hq // group].double()
            if len(kk) == 0:
                assert bool((out[:, hq] == 0).all()) and bool((lse[hq] == -math.inf).all())
                continue
            z = q[:, hq].double() @ kk.t() / 8
            check_rows(out[:, hq].double(), z, vv)
            assert float((lse[hq].double() - torch.logsumexp(z, 1)).abs().max()) <= LSE_ATOL

    def truncate(self, s, n_rows):
        self.pool.truncate(s, n_rows)
        self.rows[s] = tuple(t[:, :n_rows] for t in self.rows[s])


@pytest.mark.parametrize("rows", [1, 63, 65, 1000])
@pytest.mark.parametrize("tokens", [1, 33, 130])
@pytest.mark.parametrize("frame", [False, True])
def test_one_sequence(rv, rows, tokens, frame):
    w = Checked(rv, 2, 20, 2, 1100, seed=rows + tokens)
    s = w.open()
    w.append([s], [rows])
    w.check_attention([s], [tokens], frame=frame)


@pytest.mark.parametrize("H,group", [(1, 1), (4, 4), (3, 5), (16, 1)])
@pytest.mark.parametrize("tokens", [1, 5, 40])
def test_forks_of_a_long_prefix(rv, H, group, tokens):
    w = Checked(rv, H, 200, 20, 3000, seed=H + tokens)
    a = w.open()
    w.append([a], [2100])
    kids = w.fork(a, n=9)
    w.append(kids, [0, 1, 28, 44, 64, 100, 300, 7, 500])
    w.check_attention(kids, [tokens] * 9, group, frame=tokens > 1)


@pytest.mark.parametrize("root", [64, 128, 320, 640, 1280])
@pytest.mark.parametrize("tokens", [1, 5, 150])
def test_branches_below_a_short_root(rv, root, tokens):
    """What all share is not worth a pass of its own (but few tokens over the longest root): the branches' passes begin with it."""
    w = Checked(rv, 2, 300, 40, 5000, seed=root + tokens)
    a = w.open()
    w.append([a], [root])
    leaves = []
    for trunk in w.fork(a, n=3):
        w.append([trunk], [2500 + 100 * len(leaves)])
        kids = w.fork(trunk, n=5)
        w.append(kids, [0, 1, 64, 30, 200])
        leaves += kids
    w.check_attention(leaves, [tokens] * len(leaves), group=2, frame=tokens != 1)
    w.check_attention(leaves + [a], [1 + i % 3 for i in range(len(leaves))] + [2], frame=False)


@pytest.mark.parametrize("H,lengths,tokens", [
    (16, [130] * 8, 513), (16, [130, 200, 129, 250] * 2, 513), (2, [3000], 300), (2, [3000, 3000], 129),
    (2, [5000, 2000], 300), (16, [1500], 1041)], ids=str)
def test_strangers_with_many_queries(rv, H, lengths, tokens):
    w = Checked(rv, H, sum(n // 64 + 2 for n in lengths), len(lengths), max(lengths) + 64)
    seqs = [w.open() for _ in lengths]
    w.append(seqs, lengths)
    w.check_attention(seqs, [tokens] * len(seqs), frame=True)


def test_whole_frames_over_a_shared_prefix(rv):
    w = Checked(rv, 8, 100, 8, 2000)
    a = w.open()
    w.append([a], [1500])
    kids = w.fork(a, n=3)
    w.append(kids, [100, 3, 0])
    w.check_attention(kids, [1041, 700, 129], frame=True)
    w.check_attention([a], [1374], frame=True, scale=3.0)


@pytest.mark.parametrize("tokens", [[1, 5, 2, 1, 17], [300, 1, 1, 129, 64]], ids=str)
def test_long_memory(rv, tokens):
    w = Checked(rv, 2, 1700, 8, 53041)
    a = w.open()
    w.append([a], [52000])
    kids = w.fork(a, n=5)
    w.append(kids, [1041, 0, 64, 3, 500])
    w.check_attention(kids, tokens, group=2, frame=True)
    w.check_attention([a], [700], frame=True)


def test_rows_past_four_gigabytes(rv):
    """2.5 million rows of 16 heads, 5.1 GB of keys.  A few dozen rows, all over each head's, hold a token's query as
    their key, so that the outputs are made of just their values."""
    H, part, parts, each = 16, 500_000, 5, 8
    pool = rv.Pool(H, part * parts // 64 + 40, 4, part * parts + 64)
    s = pool.open()
    g = gen(12)
    Q = rand(g, 2, H, D)
    kept = []
    for i in range(parts):
        K = torch.empty(part, H, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        V = torch.empty(part, H, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        at = torch.randperm(part, generator=g, device="cuda")[:2 * each]
        at[0], at[each] = part - 1, 0
        for t in range(2):  # z = c |q|^2 / 8 = 25, beside log(2.5e6) = 14.7 and the others' spread
            q = Q[t].float()
            K[at[t * each:(t + 1) * each]] = (q * 200 / q.square().sum(-1, keepdim=True)).bfloat16()
        pool.append([s], K, V, [part])
        kept.append(V[at])
        del K, V
    n = part * parts
    c = pool.fork(s, n)[0]
    out, lse = torch.empty_like(Q), torch.empty(H, 2, device="cuda")
    rv.attend_seqs(Q, None, None, pool, [c], [2], out, lse)
    for t in range(2):  # most of each output is its own rows' mean value
        mean = torch.cat([v[t * each:(t + 1) * each] for v in kept]).double().mean(0)
        assert float((out[t].double() - mean).norm() / mean.norm()) < 0.2
    rows = torch.empty(H, n, D, dtype=torch.bfloat16, device="cuda")
    for h in (0, 7, H - 1):
        pool.gather([c], rows, None, [n])
        k = rows[h].clone()
        pool.gather([c], None, rows, [n])
        v = rows[h].double()
        z = Q[:, h].double() @ k.double().t() / 8
        check_rows(out[:, h].double(), z, v)
        assert float((lse[h].double() - torch.logsumexp(z, 1)).abs().max()) <= LSE_ATOL
    pool.close()


# ---- truncation ------------------------------------------------------------------------------

@pytest.mark.parametrize("cut", [0, 1, 63, 64, 65, 128, 190, 200, 256, 299, 300])
@pytest.mark.parametrize("shared", [None, "longer", "shorter", "cut"])
def test_append_truncate_append(rv, cut, shared):
    """The cut inside a page and at its border; a fork that shares the cut page, of all rows, of fewer and of as many
    rows as are left, keeps its own."""
    w = Checked(rv, 2, 40, 8, 800, seed=cut)
    a = w.open()
    w.append([a], [300])
    if shared:
        w.fork(a, {"longer": 300, "shorter": max(cut - 5, 0), "cut": cut}[shared])
    w.truncate(a, cut)
    w.verify()
    w.append([a], [77])
    w.verify()
    w.append(sorted(w.rows), [70] * len(w.rows))
    w.verify()
    w.check_attention(sorted(w.rows), [3] * len(w.rows), frame=True)
    w.truncate(a, 0)
    w.append([a], [130])
    w.verify()
    w.check_attention(sorted(w.rows), [1] * len(w.rows), frame=False)
    w.release(sorted(w.rows))
    assert w.pool.free_pages == 40


def test_truncated_pages_go_to_others(rv):
    """Pages that a truncation frees are another sequence's next ones, while the first goes on."""
    w = Checked(rv, 3, 12, 4, 700)
    a, b = w.open(), w.open()
    w.append([a, b], [500, 100])  # 8 and 2 pages
    for cut, more, other in ((100, 0, 380), (64, 30, 0), (30, 200, 0)):
        w.truncate(a, cut)
        w.append([b, a], [other, more])
        w.verify()
        w.check_attention([a, b], [2, 140], frame=True)


def test_a_truncated_step_is_captured_again(rv):
    """A step is captured, replayed and taken back; the next step's pages are the same ones, and a graph of it holds."""
    w = Checked(rv, 4, 60, 4, 2000)
    a = w.open()
    w.append([a], [700])
    kids = w.fork(a, n=3)
    w.append(kids, [60, 3, 64])
    for tokens in (2, 70):
        total = tokens * 3
        Q, K, V = (rand(w.g, total, 4, D) for _ in range(3))
        out, lse = torch.empty_like(Q), torch.empty(3, 4, tokens, device="cuda")
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            w.pool.append(kids, K, V, [tokens] * 3)
            rv.attend_seqs(Q, None, None, w.pool, kids, [tokens] * 3, out, lse)
        for i in range(3):
            for t in (Q, K, V):
                t.copy_(rand(w.g, total, 4, D))
            g.replay()
            torch.cuda.synchronize()
            for j, s in enumerate(kids):
                mine = slice(tokens * j, tokens * (j + 1))
                k, v = (torch.cat((t, n[mine].transpose(0, 1)), dim=1) for t, n in zip(w.rows[s], (K, V)))
                w.check_one(Q[mine], k, v, out[mine], lse[j], 1)
        for s in kids:
            w.pool.truncate(s, w.rows[s][0].shape[1])
        w.verify()
        w.check_attention(kids, [1, 2, 3], frame=True)
