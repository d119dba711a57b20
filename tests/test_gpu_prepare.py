"""prepare_qkv, its gradients and the staged form against the definition in 64 bits.

Error bounds.  A head's 64 elements are summed as 16 terms a lane and two exchanges, in fp32: a
relative error of 18 x 2^-24 of the sum of magnitudes, in the mean, in the mean square (halved by
the root) and, backward, in the two sums; a handful of further fp32 roundings (root, quotient,
weight, sine and cosine, two products and a sum) come to less than 14 x 2^-24.  Together below 2^-18 of the
row's largest magnitude forward and 2^-17 backward (three sums), for rows whose mean is no larger than
their deviation.  bf16 outputs are then rounded once: 2^-8 of the value."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

D = 64


@pytest.fixture(scope="module")
def rv():
    from paper_2609_23286_amd import rv as _rv
    _rv.init()
    return _rv


def definition(x, heads, norm, eps, axes, base, weight, bias, pos):
    """[N, heads, 64] in 64 bits, from the formulas, pair by pair."""
    y = x.double().reshape(x.shape[0], heads, D)
    if norm:
        g = y - y.mean(-1, keepdim=True) if norm == "layer" else y
        y = g / torch.sqrt((g * g).mean(-1, keepdim=True) + eps)
        if weight is not None:
            y = y * weight.double()
        if bias is not None:
            y = y + bias.double()
    if axes == 0:
        return y
    block = D // axes
    out = torch.empty_like(y)
    pos = pos.double().reshape(-1, axes)
    for a in range(axes):
        for i in range(block // 2):
            t = (pos[:, a] * base ** (-2.0 * i / block))[:, None]
            p, q = y[..., a * block + i], y[..., a * block + block // 2 + i]
            out[..., a * block + i] = p * t.cos() - q * t.sin()
            out[..., a * block + block // 2 + i] = q * t.cos() + p * t.sin()
    return out


class Case:
    def __init__(self, rv, N, Hq, Hk, norm="layer", axes=2, dtype=torch.bfloat16, base=100.0, eps=1e-5, fused=False,
                 vectors="all", pos=None, scale=1.0, seed=0):
        g = torch.Generator(device="cuda").manual_seed(1000 + seed)
        self.N, self.Hq, self.Hk, self.norm, self.axes, self.base, self.eps = N, Hq, Hk, norm, axes, base, eps

        def normal(*shape):
            return torch.randn(*shape, generator=g, device="cuda")

        widths = [Hq * D, Hk * D, Hk * D]
        if fused:
            wide = (normal(N, sum(widths) + 64) * scale).to(dtype)
            self.q, self.k, self.v, _ = wide.split(widths + [64], dim=1)
        else:
            self.q, self.k, self.v = ((normal(N, w) * scale).to(dtype) for w in widths)
        self.qw = self.qb = self.kw = self.kb = None
        if norm and vectors != "none":
            self.qw, self.kw = 1 + 0.2 * normal(D), 1 + 0.2 * normal(D)
            if vectors == "all":
                self.qb, self.kb = 0.1 * normal(D), 0.1 * normal(D)
        self.pos = None
        if axes:
            self.pos = pos if pos is not None else torch.randint(0, 60, (N, axes), generator=g, device="cuda",
                                                                 dtype=torch.int32)
        self.prep = rv.QKVPrep(Hq, Hk, norm=norm, eps=eps, axes=axes, base=base, q_weight=self.qw, q_bias=self.qb,
                               k_weight=self.kw, k_bias=self.kb)
        self.dQ, self.dK, self.dV = (normal(N, h, D).bfloat16() for h in (Hq, Hk, Hk))

    def expect(self, name):
        x, heads, w, b = {"Q": (self.q, self.Hq, self.qw, self.qb), "K": (self.k, self.Hk, self.kw, self.kb)}[name]
        return definition(x, heads, self.norm, self.eps, self.axes, self.base, w, b, self.pos)

    def empty(self):
        return [torch.full((self.N + 1, h, D), 7.0, dtype=torch.bfloat16, device="cuda")
                for h in (self.Hq, self.Hk, self.Hk)]


def check(got, ref, bits, round_to=2.0 ** -8):
    scale = ref.abs().amax(dim=-1, keepdim=True).clamp_min(1e-30)
    err = (got.double() - ref).abs() - round_to * ref.abs() - 2.0 ** -bits * scale
    assert float(err.max()) <= 0, f"past the bound by {float(err.max())}"


CASES = [
    dict(N=1, Hq=1, Hk=1),
    dict(N=1, Hq=12, Hk=12, norm="rms", axes=1, base=10000.0, fused=True),
    dict(N=2, Hq=16, Hk=4, norm="rms", axes=2, vectors="weights"),
    dict(N=7, Hq=3, Hk=3, norm="layer", axes=1, vectors="none"),
    dict(N=63, Hq=5, Hk=1, norm=None, axes=2),
    dict(N=130, Hq=16, Hk=16, norm="layer", axes=0),
    dict(N=33, Hq=2, Hk=2, norm=None, axes=0, fused=True),
    dict(N=1041, Hq=16, Hk=16),
    dict(N=1041, Hq=16, Hk=8, dtype=torch.float32, fused=True),
    dict(N=257, Hq=12, Hk=3, dtype=torch.float32, norm="rms", axes=1, base=500000.0),
    dict(N=20011, Hq=4, Hk=2, norm="rms", axes=2, fused=True),
    dict(N=9001, Hq=1, Hk=1, dtype=torch.float32),
]
IDS = [f"N{c['N']}-H{c['Hq']}.{c['Hk']}-{c.get('norm', 'layer')}-{c.get('axes', 2)}ax" for c in CASES]


@pytest.mark.parametrize("c", CASES, ids=IDS)
def test_forward(rv, c):
    x = Case(rv, **c)
    Q, K, V = x.empty()
    N = x.N
    rv.prepare_qkv(x.prep, x.q, x.k, x.v, x.pos, Q[:N], K[:N], V[:N])
    for name, got in (("Q", Q), ("K", K)):
        check(got[:N], x.expect(name), 18)
    assert torch.equal(V[:N], x.v.reshape(N, x.Hk, D).bfloat16())
    for t in (Q, K, V):
        assert bool((t[N:] == 7).all()), "a row behind the last token was written"


@pytest.mark.parametrize("axes", [1, 2])
def test_far_and_negative_positions(rv, axes):
    far = [0, 1, -1, 65535, 123456789, 2 ** 31 - 1, -2 ** 31, 1000003]
    pos = torch.tensor(far, dtype=torch.int32, device="cuda")[:, None]
    if axes == 2:
        pos = torch.cat((pos, pos.flip(0)), dim=1)
    # (64-bit angles of 2^31 steps carry 2^31 x 2^-53 = 2^-22 of their own)
    x = Case(rv, 8, 2, 2, norm=None, axes=axes, base=10000.0, pos=pos.contiguous())
    Q, K, _ = x.empty()
    rv.prepare_qkv(x.prep, x.q, x.k, None, x.pos, Q[:8], K[:8], None)
    check(Q[:8], x.expect("Q"), 18)
    check(K[:8], x.expect("K"), 18)


def test_small_and_large_values(rv):
    for scale, dtype in ((1e-12, torch.float32), (1e15, torch.float32), (3e4, torch.bfloat16)):
        x = Case(rv, 5, 2, 2, norm="layer", dtype=dtype, scale=scale)
        Q, K, V = x.empty()
        rv.prepare_qkv(x.prep, x.q, x.k, x.v, x.pos, Q[:5], K[:5], V[:5])
        check(Q[:5], x.expect("Q"), 18)
    x = Case(rv, 3, 1, 1, norm="rms")
    x.q.zero_()  # eps alone keeps the root from zero
    Q, K, V = x.empty()
    rv.prepare_qkv(x.prep, x.q, x.k, x.v, x.pos, Q[:3], K[:3], V[:3])
    check(Q[:3], x.expect("Q"), 18)


def test_no_tokens(rv):
    x = Case(rv, 0, 2, 2)
    Q, K, V = x.empty()
    rv.prepare_qkv(x.prep, x.q, x.k, x.v, x.pos, Q[:0], K[:0], V[:0])
    sums = [torch.ones(D, device="cuda") for _ in range(4)]
    e = torch.empty(0, 2 * D, dtype=torch.bfloat16, device="cuda")
    rv.prepare_qkv_bwd(x.prep, x.q, x.k, x.pos, x.dQ, x.dK, x.dV, e, e, e, *sums)
    assert all(bool((t == 0).all()) for t in sums)
    assert all(bool((t == 7).all()) for t in (Q, K, V))


def backward(rv, x, sums=True):
    N = x.N
    wide = torch.full((N + 1, (x.Hq + 2 * x.Hk) * D + 64), 7.0, dtype=x.q.dtype, device="cuda")
    dq, dk, dv, rest = wide.split([x.Hq * D, x.Hk * D, x.Hk * D, 64], dim=1)
    vecs = {"dq_weight": x.qw, "dq_bias": x.qb, "dk_weight": x.kw, "dk_bias": x.kb}
    out = {n: torch.empty(D, device="cuda") for n, v in vecs.items() if v is not None and sums}
    rv.prepare_qkv_bwd(x.prep, x.q, x.k, x.pos, x.dQ, x.dK, x.dV, dq[:N], dk[:N], dv[:N], **out)
    assert bool((wide[N:] == 7).all()) and bool((rest == 7).all()), "elements beside the gradients were written"
    return dict(out, dq=dq[:N], dk=dk[:N], dv=dv[:N])


@pytest.mark.parametrize("c", CASES, ids=IDS)
def test_backward(rv, c):
    x = Case(rv, **c)
    got = backward(rv, x)
    round_to = 2.0 ** -8 if x.q.dtype == torch.bfloat16 else 2.0 ** -24
    assert torch.equal(got["dv"], x.dV.reshape(x.N, -1).to(x.q.dtype))
    for n, heads, src, w, b, grad in (("q", x.Hq, x.q, x.qw, x.qb, x.dQ), ("k", x.Hk, x.k, x.kw, x.kb, x.dK)):
        leaves = {m: t.double().requires_grad_() for m, t in (("x", src), ("w", w), ("b", b)) if t is not None}
        y = definition(leaves["x"], heads, x.norm, x.eps, x.axes, x.base, leaves.get("w"), leaves.get("b"), x.pos)
        ref = dict(zip(leaves, torch.autograd.grad(y, list(leaves.values()), grad.double())))
        # the scale of a row's gradient: r times the largest incoming element
        xs = src.double().reshape(x.N, heads, D)
        r = 1.0 if not x.norm else 1 / torch.sqrt(
            (xs - (xs.mean(-1, keepdim=True) if x.norm == "layer" else 0)).square().mean(-1, keepdim=True) + x.eps)
        scale = grad.double().abs().amax(-1, keepdim=True) * r * (1.0 if w is None else float(w.abs().max())) * 2
        rows = ref["x"].reshape(x.N, heads, D)
        err = (got["d" + n].double().reshape(rows.shape) - rows).abs() - round_to * rows.abs() - 2.0 ** -17 * scale
        assert float(err.max()) <= 0, f"d{n}: past the bound by {float(err.max())}"
        # sums over all rows: each term as above, the additions rows x 2^-24 of the sum of magnitudes at most
        turned = definition(grad.double(), heads, None, 0, x.axes, x.base, None, None,
                            None if x.pos is None else -x.pos)
        normed = definition(src, heads, x.norm, x.eps, 0, x.base, None, None, None)
        per = 2.0 ** -17 + x.N * heads * 2.0 ** -24
        for m, terms in (("w", turned * normed), ("b", turned)):
            if m in ref:
                # (a turned element's error is relative to its pair, so to the row's largest)
                size = (terms.abs() + turned.abs().amax(-1, keepdim=True) * (normed.abs() if m == "w" else 1)).sum((0, 1))
                e = (got[f"d{n}_{'weight' if m == 'w' else 'bias'}"].double() - ref[m]).abs() - per * size
                assert float(e.max()) <= 0, f"d{n} {m}: past the bound by {float(e.max())}"


def test_backward_against_differences(rv):
    x = Case(rv, 9, 3, 2, dtype=torch.float32)
    got = backward(rv, x)
    g = torch.Generator(device="cuda").manual_seed(3)
    for n, heads, src, w, b, grad in (("q", 3, x.q, x.qw, x.qb, x.dQ), ("k", 2, x.k, x.kw, x.kb, x.dK)):
        for m, base in (("", src), ("_weight", w), ("_bias", b)):
            d = torch.randn(base.shape, generator=g, device="cuda").double()
            h = 1e-5

            def loss(step):
                a = {"": src.double(), "_weight": w.double(), "_bias": b.double()}
                a[m] = a[m] + step * d
                y = definition(a[""], heads, x.norm, x.eps, x.axes, x.base, a["_weight"], a["_bias"], x.pos)
                return float((y * grad.double()).sum())

            slope = (loss(h) - loss(-h)) / (2 * h)
            mine = float((got[f"d{n}{m}"].double() * d).sum())
            size = float((got[f"d{n}{m}"].double() * d).abs().sum())
            assert abs(mine - slope) <= 2.0 ** -17 * size + 1e-6 * (1 + abs(slope)), (n, m, mine, slope)


def test_same_inputs_same_bits(rv):
    x = Case(rv, 4001, 16, 4)
    a, b = backward(rv, x), backward(rv, x)
    assert all(torch.equal(a[n], b[n]) for n in a)


def test_staged_form_writes_the_frame_into_the_arena(rv):
    x = Case(rv, 75, 16, 4, fused=True)
    Q, K, V = (t[:75].clone() for t in x.empty())
    rv.prepare_qkv(x.prep, x.q, x.k, x.v, x.pos, Q, K, V)
    mem = rv.Memory(4, reserve_tokens=10, max_tokens=400)
    old = torch.randn(4, 90, D, device="cuda").bfloat16()
    mem.write(old, old)
    Q2 = torch.zeros_like(Q)
    rv.stage_qkv(x.prep, x.q, x.k, x.v, x.pos, Q2, mem)  # (grows the arena)
    assert torch.equal(Q, Q2) and mem.len == 90
    sal = torch.rand(4, 75, device="cuda")
    rv.admit(sal, 75, K, V, mem, 1)  # every row of the frame, by the other way
    a = mem.read()
    mem.truncate(90)
    rv.stage_qkv(x.prep, x.q, x.k, x.v, x.pos, Q2, mem)
    qs = rv.qsub(0, 0, 75, 1)
    lse = torch.zeros(4, 75, device="cuda")
    rv.admit_staged_layers([torch.zeros(75, 4, D, dtype=torch.bfloat16, device="cuda")], [lse], qs, 75, [mem], 1,
                           [sal], None)
    b = mem.read()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_captured_and_on_another_stream(rv):
    x = Case(rv, 300, 16, 16)
    outs = [t[:300].clone() for t in x.empty()]
    eager = [t[:300].clone() for t in x.empty()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    vecs = [torch.empty(D, device="cuda") for _ in range(4)]
    grads = [torch.empty_like(t) for t in (x.q, x.k, x.v)]
    with torch.cuda.graph(g, stream=s):
        rv.prepare_qkv(x.prep, x.q, x.k, x.v, x.pos, *outs)
        rv.prepare_qkv_bwd(x.prep, x.q, x.k, x.pos, x.dQ, x.dK, x.dV, *grads, *vecs)
    for seed in range(3):
        y = Case(rv, 300, 16, 16, seed=seed)
        for n in ("q", "k", "v", "dQ", "dK", "dV"):
            getattr(x, n).copy_(getattr(y, n))
        g.replay()
        torch.cuda.synchronize()
        rv.prepare_qkv(x.prep, x.q, x.k, x.v, x.pos, *eager)
        assert all(torch.equal(a, b) for a, b in zip(outs, eager))
        got = backward(rv, x)
        names = ("dq", "dk", "dv", "dq_weight", "dq_bias", "dk_weight", "dk_bias")
        assert all(torch.equal(got[n], t) for n, t in zip(names, grads + vecs))


def test_rows_far_apart(rv):
    """Element offsets past 2^31."""
    N, stride = 9000, 300_000
    wide = torch.empty(N * stride, dtype=torch.bfloat16, device="cuda").view(N, stride)
    x = Case(rv, N, 2, 1, norm="rms")
    q, k, v = wide[:, 128:256], wide[:, 512:576], wide[:, 299_904:299_968]
    for far, near in ((q, x.q), (k, x.k), (v, x.v)):
        far.copy_(near)
    Q, K, V = (t[:N] for t in x.empty())
    rv.prepare_qkv(x.prep, q, k, v, x.pos, Q, K, V)
    near = [torch.empty_like(t) for t in (Q, K, V)]
    rv.prepare_qkv(x.prep, x.q, x.k, x.v, x.pos, *near)
    assert all(torch.equal(a, b) for a, b in zip((Q, K, V), near))
    want = backward(rv, x)
    sums = {n: torch.empty(D, device="cuda") for n in ("dq_weight", "dq_bias", "dk_weight", "dk_bias")}
    grads = wide[:, 1024:1152], wide[:, 2048:2112], wide[:, 4096:4160]
    rv.prepare_qkv_bwd(x.prep, q, k, x.pos, x.dQ, x.dK, x.dV, *grads, **sums)
    assert all(torch.equal(a, want[n]) for a, n in zip(grads, ("dq", "dk", "dv")))
    assert all(torch.equal(sums[n], want[n]) for n in sums)


def test_the_binding_refuses_before_the_launch(rv):
    x = Case(rv, 5, 2, 1)
    Q, K, V = (t[:5] for t in x.empty())
    for call, words in (
            (lambda: rv.prepare_qkv(x.prep, x.q[:, :64], x.k, x.v, x.pos, Q, K, V), "q: shape"),
            (lambda: rv.prepare_qkv(x.prep, x.q, x.k[:4], x.v, x.pos, Q, K, V), "4 rows, expected 5"),
            (lambda: rv.prepare_qkv(x.prep, x.q, x.k.float(), x.v, x.pos, Q, K, V), "another dtype"),
            (lambda: rv.prepare_qkv(x.prep, x.q.half(), x.k, x.v, x.pos, Q, K, V), "dtype"),
            (lambda: rv.prepare_qkv(x.prep, x.q.t().contiguous().t(), x.k, x.v, x.pos, Q, K, V), "contiguous"),
            (lambda: rv.prepare_qkv(x.prep, x.q, x.k, x.v, x.pos.long(), Q, K, V), "pos: dtype"),
            (lambda: rv.prepare_qkv(x.prep, x.q, x.k, x.v, x.pos[:, :1], Q, K, V), "pos"),
            (lambda: rv.prepare_qkv(x.prep, x.q, x.k, x.v, None, Q, K, V), "pos is required"),
            (lambda: rv.prepare_qkv(x.prep, x.q, x.k, x.v, x.pos, Q[:, :1], K, V), "Q"),
            (lambda: rv.prepare_qkv(x.prep, x.q, x.k, x.v, x.pos, Q, K, None), "both"),
            (lambda: rv.prepare_qkv(x.prep, x.q.cpu(), x.k, x.v, x.pos, Q, K, V), "device tensor"),
            (lambda: rv.prepare_qkv(x.prep, x.q[:1].expand(5, -1), x.k, x.v, x.pos, Q, K, V), "row stride"),
            (lambda: backward(rv, Case(rv, 5, 2, 1, norm=None), True) and rv.prepare_qkv_bwd(
                x.prep, x.q, x.k, x.pos, x.dQ, x.dK, x.dV, x.q.float(), x.k, x.v), "another dtype")):
        with pytest.raises((rv.RVError, ValueError, TypeError), match=words):
            call()
    assert all(bool((t == 7).all()) for t in (Q, K, V))
