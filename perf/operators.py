"""The calls that surround the attention of a frame, with their inputs, plain forms and references.

  prepare      rv.prepare_qkv: per-head norm of queries and keys and the position rotation
  prepare_bwd  rv.prepare_qkv_bwd: the gradients of the same step
  branch       Pool.fork, Pool.append, Pool.gather: children of one sequence go on by themselves
  compact      Pool.compact: a sequence keeps the listed rows of every head
  attend       rv.attend_seqs: several sequences' queries over their pages, shared ones read once

`own` chooses what `run` does: False, the plain form (elementary torch operations in 32 bits); True,
the framework's calls.  Heads hold 64 elements.  Inputs are bf16 unless a case says otherwise.
"""
import math

import torch

own = False

D = 64
PAGE = 64  # rows of a page
KINDS = ("prepare", "prepare_bwd", "branch", "compact", "attend")


def _prep(name, kind, tokens, q_heads=16, kv_heads=16, norm="layer", axes=2, base=100.0, dtype="bf16", fused=False,
          first=0):
    """tokens of `first`, first + 1, ... (one axis) or of frames of 28 x 37 patches after 5 special tokens
    (two); fused: q, k, v are column ranges of one projection's output."""
    c = {"kind": kind, "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "norm": norm, "axes": axes,
         "base": base, "dtype": dtype, "fused": fused, "first": first}
    return dict(c, name=name) if name else c


def _branch(name, parent, at, children, rows, step=0, heads=16):
    """children of a sequence of `parent` rows, forked after row `at`; child i appends rows - i step rows."""
    c = {"kind": "branch", "parent": parent, "at": at, "children": children, "rows": rows, "step": step,
         "heads": heads}
    return dict(c, name=name) if name else c


def _compact(name, seqs, rows, first, keep, heads=16):
    """Each of `seqs` sequences of `rows` rows keeps its first `first` rows and `keep` of the others."""
    c = {"kind": "compact", "seqs": seqs, "rows": rows, "first": first, "keep": keep, "heads": heads}
    return dict(c, name=name) if name else c


def _attend(name, seqs, tokens, prefix, own_rows, step=0, q_heads=16, kv_heads=16, frame=False, sigma=1.0):
    """`seqs` sequences with `prefix` rows in common; sequence i has own_rows - i step rows of its own (0 at
    least) and `tokens` queries; frame: the queries' own keys and values are attended too."""
    c = {"kind": "attend", "seqs": seqs, "tokens": tokens, "prefix": prefix, "own": own_rows, "step": step,
         "q_heads": q_heads, "kv_heads": kv_heads, "frame": frame, "sigma": sigma}
    return dict(c, name=name) if name else c


def listed():
    return [
        # One token at a far position, a fused projection, root-mean-square norm: a decoding step.
        _prep("prepare_token", "prepare", 1, 12, 12, "rms", 1, 10000.0, fused=True, first=123457),
        # Eight ViT-L frames of 1041 tokens (layer norm, rotation by patch row and column).
        _prep("prepare_frames", "prepare", 8 * 1041),
        # Training: one frame of a fused bf16 projection with shared key heads ...
        _prep("prepare_bwd_frame", "prepare_bwd", 1041, 16, 8, "rms", fused=True),
        # ... and eight frames in 32 bits.
        _prep("prepare_bwd_frames", "prepare_bwd", 8 * 1041, dtype="f32"),
        # Four continuations of a stream take one row each; the page they share is half full.
        _branch("branch_tokens", parent=2000, at=2000, children=4, rows=1),
        # Eight continuations from a point inside the stream, a whole anchor frame or less each.
        _branch("branch_frames", parent=5000, at=4321, children=8, rows=1041, step=37),
        # One percent of a frame's rows stay behind the anchor frame.
        _compact("compact_frame", seqs=1, rows=2082, first=1041, keep=10),
        # Two long memories are halved, row by row and head by head.
        _compact("compact_long", seqs=2, rows=52000, first=1041, keep=25000),
        # The smallest batch: launches and host calls.
        _attend("attend_tiny", seqs=2, tokens=1, prefix=70, own_rows=7, q_heads=2, kv_heads=2),
        # Single tokens of 16 continuations over a stream's memory, four query heads to a key head.
        _attend("attend_tokens", seqs=16, tokens=1, prefix=9990, own_rows=643, step=37, q_heads=16, kv_heads=4),
        # Camera and register tokens of 48 continuations over the long memory.
        _attend("attend_long", seqs=48, tokens=5, prefix=52000, own_rows=1041, step=17),
        # Whole frames of four continuations of a stream, their own keys included.
        _attend("attend_frames", seqs=4, tokens=1041, prefix=5000, own_rows=430, step=110, frame=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(KINDS)
    heads = rng.choice((1, 2, 3, 4, 8, 12, 16, 16))
    if kind.startswith("prepare"):
        group = rng.choice((1, 1, 2, 4))
        axes = rng.choice((0, 1, 2, 2))
        c = _prep(None, kind, _log_int(rng, 1, 8 * 1041), heads * group if heads * group <= 16 else heads, heads,
                  rng.choice((None, "rms", "layer", "layer")), axes, rng.choice((100.0, 10000.0, 500000.0)),
                  rng.choice(("bf16", "bf16", "f32")), rng.random() < 0.5,
                  _log_int(rng, 1, 1000000) if axes == 1 else 0)
    elif kind == "branch":
        at, n = _log_int(rng, 1, 5000), _log_int(rng, 1, 8)
        rows = _log_int(rng, 1, 1041)
        c = _branch(None, at + rng.choice((0, 0, 1, 100)), at, n, rows, rng.randint(0, rows // n), heads)
    elif kind == "compact":
        rows = _log_int(rng, 2, 52000)
        first = rng.choice((0, rng.randint(0, rows // 2)))
        c = _compact(None, rng.choice((1, 1, 2)), rows, first, _log_int(rng, 1, max(1, (rows - first) // 2)), heads)
    else:
        frame = rng.random() < 0.5
        group = rng.choice((1, 1, 2, 4))
        c = _attend(None, _log_int(rng, 1, 48), _log_int(rng, 1, 1041), rng.choice((0, 63, 64, 1041,
                    _log_int(rng, 1, 52000), _log_int(rng, 1, 52000))), _log_int(rng, 1, 1041), rng.randint(0, 40),
                    heads * group if heads * group <= 16 else heads, heads, frame, rng.choice((0.5, 1.0, 1.0, 2.0)))
        while work(c)["flops"] > 1.2e11 or work(c)["bytes"] > 4e8:  # about the largest listed ones
            if c["tokens"] > 5:
                c["tokens"] = c["tokens"] * 3 // 4
            else:
                c["seqs"] = max(1, c["seqs"] * 3 // 4)
                c["prefix"] = c["prefix"] * 3 // 4
    return c


def _rows_of(c):
    """Rows each child appends (branch), or each sequence's own rows (attend)."""
    if c["kind"] == "branch":
        return [max(0, c["rows"] - i * c["step"]) for i in range(c["children"])]
    return [max(0, c["own"] - i * c["step"]) for i in range(c["seqs"])]


def work(c):
    flops, row = 0.0, D * 2
    if c["kind"].startswith("prepare"):
        size = 2 if c["dtype"] == "bf16" else 4
        elems = c["tokens"] * (c["q_heads"] + 2 * c["kv_heads"]) * D
        pos = 4 * c["tokens"] * c["axes"]
        if c["kind"] == "prepare":
            nbytes, flops = elems * (size + 2) + pos, 10.0 * elems
        else:  # q and k again, the incoming gradients, the outgoing ones
            qk = c["tokens"] * (c["q_heads"] + c["kv_heads"]) * D
            nbytes, flops = qk * size + elems * (2 + size) + pos, 25.0 * qk
    elif c["kind"] == "branch":  # the rows that the children do not share, in and out
        n = sum(c["at"] % PAGE + r for r in _rows_of(c))
        nbytes = 2 * 2 * n * c["heads"] * row
    elif c["kind"] == "compact":
        nbytes = c["seqs"] * c["heads"] * (2 * 2 * (c["first"] + c["keep"]) * row + 4 * c["keep"])
    else:
        q, rows = c["tokens"] * c["seqs"], _rows_of(c)
        keys = c["prefix"] + sum(rows) + (q if c["frame"] else 0)
        nbytes = 2 * q * c["q_heads"] * row + 4 * q * c["q_heads"] + 2 * keys * c["kv_heads"] * row
        context = sum(c["prefix"] + r + (c["tokens"] if c["frame"] else 0) for r in rows)
        flops = 4.0 * D * c["q_heads"] * c["tokens"] * context
    return {"bytes": float(nbytes), "flops": float(flops)}


# ---- inputs ---------------------------------------------------------------------------

def _inputs(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape, scale=1.0, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=g).mul_(scale).to(dtype)

    if c["kind"].startswith("prepare"):
        N, Hq, Hk = c["tokens"], c["q_heads"], c["kv_heads"]
        dtype = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
        widths = (Hq * D, Hk * D, Hk * D)
        if c["fused"]:
            q, k, v = normal(N, sum(widths), dtype=dtype).split(widths, dim=1)
        else:
            q, k, v = (normal(N, w, dtype=dtype) for w in widths)
        x = {"q": q, "k": k, "v": v}
        if c["norm"]:
            x["q_weight"], x["k_weight"] = (1.0 + normal(D, scale=0.2, dtype=torch.float32) for _ in range(2))
            if c["norm"] == "layer":
                x["q_bias"], x["k_bias"] = (normal(D, scale=0.1, dtype=torch.float32) for _ in range(2))
        if c["axes"] == 1:
            x["pos"] = (c["first"] + torch.arange(N, device="cuda", dtype=torch.int32))[:, None].contiguous()
        elif c["axes"] == 2:
            t = torch.arange(N, device="cuda") % 1041 - 5
            pos = torch.stack((t // 37 + 1, t % 37 + 1), dim=1)
            x["pos"] = torch.where(t[:, None] >= 0, pos, 0).to(torch.int32)
        if c["kind"] == "prepare_bwd":
            x["dQ"], x["dK"], x["dV"] = normal(N, Hq, D), normal(N, Hk, D), normal(N, Hk, D)
        return x
    if c["kind"] == "branch":
        H, n = c["heads"], sum(_rows_of(c))
        return {"K": normal(c["parent"], H, D), "V": normal(c["parent"], H, D), "new_K": normal(n, H, D),
                "new_V": normal(n, H, D)}
    if c["kind"] == "compact":
        S, H, M, first, keep = c["seqs"], c["heads"], c["rows"], c["first"], c["keep"]
        order = torch.empty((S, H, M - first), device="cuda").uniform_(generator=g).argsort(dim=2)
        return {"K": normal(S, M, H, D), "V": normal(S, M, H, D),
                "keep": (order[:, :, :keep].sort(dim=2).values + first).to(torch.int32).contiguous()}
    Hq, Hk, q, r = c["q_heads"], c["kv_heads"], c["seqs"] * c["tokens"], sum(_rows_of(c))
    x = {"Q": normal(q, Hq, D, scale=c["sigma"])}
    for t in ("K", "V"):
        x["prefix_" + t], x["own_" + t] = normal(c["prefix"], Hk, D), normal(r, Hk, D)
        if c["frame"]:
            x[t] = normal(q, Hk, D)
    return x


def prepare(c, seed):
    x = _inputs(c, seed)
    s = {"c": c, "x": x}
    if not own:
        return s
    from paper_2609_23286_amd import rv
    rv.init()
    bf16 = {"dtype": torch.bfloat16, "device": "cuda"}
    if c["kind"].startswith("prepare"):
        N, Hq, Hk = c["tokens"], c["q_heads"], c["kv_heads"]
        s["prep"] = rv.QKVPrep(Hq, Hk, norm=c["norm"], axes=c["axes"], base=c["base"],
                               **{n: x.get(n) for n in ("q_weight", "q_bias", "k_weight", "k_bias")})
        if c["kind"] == "prepare":
            s["out"] = {"Q": torch.empty((N, Hq, D), **bf16), "K": torch.empty((N, Hk, D), **bf16),
                        "V": torch.empty((N, Hk, D), **bf16)}
        else:
            s["out"] = {n: torch.empty(x[n[1:]].shape, dtype=x["q"].dtype, device="cuda") for n in ("dq", "dk", "dv")}
            s["out"].update({"d" + n: torch.empty(D, dtype=torch.float32, device="cuda")
                             for n in ("q_weight", "q_bias", "k_weight", "k_bias") if n in x})
    elif c["kind"] == "branch":
        H, rows = c["heads"], _rows_of(c)
        pages = -(-c["parent"] // PAGE) + sum(2 + r // PAGE for r in rows)
        s["pool"] = rv.Pool(H, pages, max_seqs=1 + len(rows), max_rows=c["parent"] + c["rows"])
        s["seq"] = s["pool"].open()
        s["pool"].append([s["seq"]], x["K"], x["V"], [c["parent"]])
        s["rows"] = rows
        s["first"] = c["at"] // PAGE * PAGE
        n = sum(c["at"] - s["first"] + r for r in rows)
        s["out"] = [torch.empty((n * H, D), **bf16) for _ in range(2)]
    elif c["kind"] == "compact":
        S, H, M, n = c["seqs"], c["heads"], c["rows"], c["first"] + c["keep"]
        s["pool"] = rv.Pool(H, S * (-(-M // PAGE) + n // PAGE + 2), max_seqs=2 * S, max_rows=M)
        s["seqs"] = [s["pool"].open() for _ in range(S)]
        s["pool"].append(s["seqs"], x["K"].flatten(0, 1), x["V"].flatten(0, 1), [M] * S)
        s["out"] = [torch.empty((S, H, n, D), **bf16) for _ in range(2)]
    else:
        H, rows, S, n = c["kv_heads"], _rows_of(c), c["seqs"], c["tokens"]
        pages = -(-c["prefix"] // PAGE) + sum(2 + r // PAGE for r in rows)
        s["pool"] = rv.Pool(H, pages, max_seqs=1 + S, max_rows=c["prefix"] + c["own"])
        parent = s["pool"].open()
        s["pool"].append([parent], x["prefix_K"], x["prefix_V"], [c["prefix"]])
        s["seqs"] = s["pool"].fork(parent, n=S)
        s["pool"].release([parent])
        s["pool"].append(s["seqs"], x["own_K"], x["own_V"], rows)
        s["tokens"] = [n] * S
        s["out"] = {"out": torch.empty((S * n, c["q_heads"], D), **bf16),
                    "lse": torch.empty((S, c["q_heads"], n), dtype=torch.float32, device="cuda")}
    return s


# ---- one pass -------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2609_23286_amd import rv
    c, x, out = s["c"], s["x"], s["out"]
    if c["kind"] == "prepare":
        rv.prepare_qkv(s["prep"], x["q"], x["k"], x["v"], x.get("pos"), out["Q"], out["K"], out["V"])
    elif c["kind"] == "prepare_bwd":
        rv.prepare_qkv_bwd(s["prep"], x["q"], x["k"], x.get("pos"), x["dQ"], x["dK"], x["dV"], **out)
    elif c["kind"] == "branch":
        pool, rows, first = s["pool"], s["rows"], s["first"]
        seqs = pool.fork(s["seq"], c["at"], len(rows))
        pool.append(seqs, x["new_K"], x["new_V"], rows)
        pool.gather(seqs, *out, first=[first] * len(rows), n_rows=[c["at"] - first + r for r in rows])
        pool.release(seqs)
    elif c["kind"] == "compact":
        pool, n = s["pool"], c["first"] + c["keep"]
        seqs = [pool.fork(q)[0] for q in s["seqs"]]
        pool.compact(seqs, x["keep"], [c["keep"]] * len(seqs), first=[c["first"]] * len(seqs))
        pool.gather(seqs, *out, n_rows=[n] * len(seqs))
        pool.release(seqs)
    else:
        rv.attend_seqs(x["Q"], x.get("K"), x.get("V"), s["pool"], s["seqs"], s["tokens"], out["out"], out["lse"])
    return out


def _angles(c, x):
    """cos, sin [tokens, 1, 64] of every element's angle, 64-bit angles rounded to 32."""
    half = D // c["axes"] // 2
    freq = c["base"] ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    angle = x["pos"].double()[:, :, None] * freq  # [tokens, axes, half]
    angle = torch.cat((angle, angle), dim=2).flatten(1)[:, None]
    return angle.cos().float(), angle.sin().float()


def _partners(c, y):
    """Element i of every axis block's first half becomes minus its partner, of the second half plus."""
    y = y.unflatten(-1, (c["axes"], 2, D // c["axes"] // 2))
    return torch.stack((-y[..., 1, :], y[..., 0, :]), dim=-2).flatten(-3)


def _normed(c, t):
    """(t - its mean, for a layer norm) / its deviation, and 1 / the deviation."""
    if c["norm"] == "layer":
        t = t - t.mean(dim=-1, keepdim=True)
    r = 1.0 / (t.square().mean(dim=-1, keepdim=True) + 1e-5).sqrt()
    return t * r, r


def _run_plain(s):
    c, x = s["c"], s["x"]
    if c["kind"].startswith("prepare"):
        out = {}
        cos, sin = _angles(c, x) if c["axes"] else (None, None)
        for n in ("q", "k"):
            t = x[n].float().unflatten(1, (-1, D))
            if c["kind"] == "prepare":
                if c["norm"]:
                    t = _normed(c, t)[0] * x[n + "_weight"] + x.get(n + "_bias", 0.0)
                if c["axes"]:
                    t = t * cos + _partners(c, t) * sin
                out[n.upper()] = t.bfloat16()
                continue
            dy = x["d" + n.upper()].float()
            if c["axes"]:
                dy = dy * cos - _partners(c, dy) * sin
            if c["norm"]:
                t, r = _normed(c, t)
                out[f"d{n}_weight"] = (dy * t).sum(dim=(0, 1))
                if c["norm"] == "layer":
                    out[f"d{n}_bias"] = dy.sum(dim=(0, 1))
                dy = dy * x[n + "_weight"]
                dy = dy - t * (dy * t).mean(dim=-1, keepdim=True) - (
                    dy.mean(dim=-1, keepdim=True) if c["norm"] == "layer" else 0.0)
                dy = dy * r
            out["d" + n] = dy.flatten(1).to(x[n].dtype)
        if c["kind"] == "prepare":
            out["V"] = x["v"].unflatten(1, (-1, D)).bfloat16()
        else:
            out["dv"] = x["dV"].flatten(1).to(x["q"].dtype)
            order = ("dq", "dk", "dv", "dq_weight", "dq_bias", "dk_weight", "dk_bias")
            out = {n: out[n] for n in order if n in out}
        return out
    if c["kind"] == "branch":
        first = c["at"] // PAGE * PAGE
        got = []
        for t in ("K", "V"):
            parts, at = [], 0
            for r in _rows_of(c):
                child = torch.cat((x[t][first:c["at"]], x["new_" + t][at:at + r]))
                parts.append(child.transpose(0, 1).reshape(-1, D))
                at += r
            got.append(torch.cat(parts))
        return got
    if c["kind"] == "compact":
        index = x["keep"].long()[..., None].expand(-1, -1, -1, D)
        return [torch.cat((x[t].transpose(1, 2)[:, :, :c["first"]], x[t].transpose(1, 2).gather(2, index)), dim=2)
                for t in ("K", "V")]
    n, Hk, rows = c["tokens"], c["kv_heads"], _rows_of(c)
    outs, lses, at = [], [], 0
    for i, r in enumerate(rows):
        k, v = ([x["prefix_" + t], x["own_" + t][at:at + r]] + ([x[t][i * n:(i + 1) * n]] if c["frame"] else [])
                for t in ("K", "V"))
        k, v = (torch.cat(t).float().transpose(0, 1).contiguous() for t in (k, v))  # [Hk, context, 64]
        at += r
        q = x["Q"][i * n:(i + 1) * n].float().unflatten(1, (Hk, -1))  # [n, Hk, group, 64]
        q = q.permute(1, 2, 0, 3).reshape(Hk, -1, D)
        if k.shape[1] == 0:
            outs.append(torch.zeros((n, c["q_heads"], D), device="cuda"))
            lses.append(torch.full((c["q_heads"], n), -math.inf, device="cuda"))
            continue
        z = torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(D)
        top = z.amax(dim=2, keepdim=True)
        z = (z - top).exp()
        total = z.sum(dim=2, keepdim=True)
        o = torch.bmm(z, v) / total
        outs.append(o.reshape(c["q_heads"], n, D).transpose(0, 1))
        lses.append((top + total.log()).reshape(c["q_heads"], n))
    return {"out": torch.cat(outs).bfloat16(), "lse": torch.stack(lses)}


# ---- the definition, in 64 bits -------------------------------------------------------

def _rotate_exact(c, y, pos):
    """Every pair of y [tokens, heads, 64] as a complex number times exp(i angle)."""
    if not c["axes"]:
        return y
    blocks = y.reshape(*y.shape[:2], c["axes"], 2, -1)
    z = torch.complex(blocks[:, :, :, 0], blocks[:, :, :, 1])
    half = z.shape[-1]
    freq = torch.tensor([c["base"] ** (-i / half) for i in range(half)], dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos.double()[:, None, :, None] * freq)
    z = z * turn
    return torch.stack((z.real, z.imag), dim=3).reshape(y.shape)


def _prepared_exact(c, t, weight, bias, pos):
    y = t.reshape(t.shape[0], -1, D)
    if c["norm"] == "layer":
        var, mean = torch.var_mean(y, dim=-1, correction=0, keepdim=True)
        y = (y - mean) / torch.sqrt(var + 1e-5)
    elif c["norm"] == "rms":
        y = y / torch.sqrt(torch.linalg.vector_norm(y, dim=-1, keepdim=True) ** 2 / D + 1e-5)
    if weight is not None:
        y = y * weight
    if bias is not None:
        y = y + bias
    return _rotate_exact(c, y, pos)


def exact(c, seed):
    x = _inputs(c, seed)
    if c["kind"].startswith("prepare"):
        out, grads = {}, {}
        for n in ("q", "k"):
            ins = {m: x[m].double().requires_grad_() for m in (n, n + "_weight", n + "_bias") if m in x}
            with torch.enable_grad():
                y = _prepared_exact(c, ins[n], ins.get(n + "_weight"), ins.get(n + "_bias"), x.get("pos"))
            out[n.upper()] = y.detach()
            if c["kind"] == "prepare_bwd":
                got = torch.autograd.grad(y, list(ins.values()), x["d" + n.upper()].double())
                grads.update(("d" + m, t) for m, t in zip(ins, got))
        if c["kind"] == "prepare":
            return dict(out, V=x["v"].reshape(c["tokens"], -1, D).double())
        grads["dv"] = x["dV"].reshape(c["tokens"], -1).double()
        order = ("dq", "dk", "dv", "dq_weight", "dq_bias", "dk_weight", "dk_bias")
        return {n: grads[n] for n in order if n in grads}
    if c["kind"] == "branch":
        new = [torch.split(x["new_" + t], _rows_of(c)) for t in ("K", "V")]
        first = c["at"] - c["at"] % PAGE
        return [torch.cat([torch.cat((x[t][first:c["at"]], r)).permute(1, 0, 2).reshape(-1, D) for r in parts]).double()
                for t, parts in zip(("K", "V"), new)]
    if c["kind"] == "compact":
        S, H = c["seqs"], c["heads"]
        got = [torch.empty((S, H, c["first"] + c["keep"], D), dtype=torch.float64, device="cuda") for _ in range(2)]
        head_rows = torch.arange(c["first"], device="cuda")
        for b in range(S):
            for h in range(H):
                rows = torch.cat((head_rows, x["keep"][b, h].long()))
                got[0][b, h] = x["K"][b, rows, h].double()
                got[1][b, h] = x["V"][b, rows, h].double()
        return got
    n, S, group = c["tokens"], c["seqs"], c["q_heads"] // c["kv_heads"]
    out = torch.zeros((S * n, c["q_heads"], D), dtype=torch.float64, device="cuda")
    lse = torch.full((S, c["q_heads"], n), -math.inf, dtype=torch.float64, device="cuda")
    own_k, own_v = (torch.split(x["own_" + t], _rows_of(c)) for t in ("K", "V"))
    for kv in range(c["kv_heads"]):
        pk, pv = x["prefix_K"][:, kv].double(), x["prefix_V"][:, kv].double()
        for b in range(S):
            mine = slice(b * n, (b + 1) * n)
            k, v = [pk, own_k[b][:, kv].double()], [pv, own_v[b][:, kv].double()]
            if c["frame"]:
                k.append(x["K"][mine, kv].double())
                v.append(x["V"][mine, kv].double())
            k, v = torch.cat(k), torch.cat(v)
            if not len(k):
                continue
            for h in range(kv * group, (kv + 1) * group):
                z = x["Q"][mine, h].double() @ k.t() / 8.0
                lse[b, h] = torch.logsumexp(z, dim=1)
                out[mine, h] = torch.softmax(z, dim=1) @ v
    return {"out": out, "lse": lse}
