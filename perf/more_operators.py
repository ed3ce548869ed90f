"""Operators of a block over packed sequences, as measurable cases.

`rotary`: rotary positions on the heads of a projection (query and key heads side by side), and the transposed rotation of their gradient.
`attn_fwd`, `attn_bwd`: attention over sequences of different lengths packed behind one another, with fewer key and value heads than query heads.
`norm_fwd`, `norm_bwd`: what joins a branch to the residual stream: the norm behind the branch, its gate, the scaled residual sum and the norm in front
of the next branch.

Where `own` is false they are computed in plain torch operations, where it is true by the framework's entry points.  Sizes are those of the
framework's workloads (`synth.CONFIGS`) or generic.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


# ---------------------------------------------------------------------- cases
def _rotary(tokens, heads, others, head_dim, rot, layout, dtype, far=0, scaled=1.0, transpose=False):
    """`others`: value heads that share the rows of the projection and are not turned; `far`: where positions begin at most."""
    return {"kind": "rotary", "tokens": tokens, "heads": heads, "others": others, "head_dim": head_dim, "rot": rot, "layout": layout, "dtype": dtype,
            "far": far, "scaled": scaled, "transpose": transpose}


def _attn(kind, tokens, seqs, heads, kv_heads, head_dim, dtype, causal=True, mix=1, tail=0):
    """`mix`: which lengths the sequences have; `tail`: rows behind the last sequence."""
    return {"kind": kind, "tokens": tokens, "seqs": seqs, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "causal": causal,
            "mix": mix, "tail": tail}


def _norm(kind, rows, cols, post, pre, gates, dtype, stream, add=False):
    """`post`, `pre`: kind of the norm behind the branch and in front of the next; `gates`: rows of the gate (0: none), `stream`: type of the residual."""
    return {"kind": kind, "rows": rows, "cols": cols, "post": post, "pre": pre, "gates": gates, "dtype": dtype, "stream": stream, "add": add}


def listed():
    return [
        # a small float model's micro-batch, queries and keys of 4 heads: latency
        dict(_rotary(128, 8, 4, 32, 32, "half", "f32"), name="rotary-small-f32"),
        # 8192 packed tokens of 16 query and 2 key heads
        dict(_rotary(8192, 18, 2, 128, 128, "half", "bf16"), name="rotary-bf16"),
        # part of the head, far positions of a context that has been extended, and the gradient's way back
        dict(_rotary(16384, 30, 5, 64, 48, "interleaved", "bf16", far=150000, scaled=8.0, transpose=True), name="rotary-back-part"),
        # a few short samples of a small model: latency
        dict(_attn("attn_fwd", 200, 5, 8, 4, 64, "bf16", mix=2), name="attn-small"),
        # a packed row of documents at the default workload's width
        dict(_attn("attn_fwd", 8192, 21, 25, 5, 64, "bf16", mix=3, tail=13), name="attn-packed"),
        # long documents
        dict(_attn("attn_fwd", 16384, 3, 16, 8, 128, "bf16", mix=4), name="attn-long"),
        # training on few tokens of a float model, odd head size, no mask
        dict(_attn("attn_bwd", 632, 3, 8, 4, 80, "f32", causal=False, mix=5), name="attn-grad-f32"),
        # gradients of the packed row
        dict(_attn("attn_bwd", 8192, 21, 25, 5, 64, "bf16", mix=3, tail=13), name="attn-grad-packed"),
        # of longer documents, two key and value heads
        dict(_attn("attn_bwd", 8192, 2, 16, 2, 128, "bf16", mix=6), name="attn-grad-long"),
        # norm behind the branch, gate per channel, norm in front of the next one; the stream in float, as a stage keeps it
        dict(_norm("norm_fwd", 8192, 2048, "rms", "rms", 1, "bf16", "f32"), name="norm-join"),
        # its gradients, LayerNorm and a gate for each sequence, at the default workload's width
        dict(_norm("norm_bwd", 8192, 1600, "layer", "layer", 8, "bf16", "bf16"), name="norm-join-back"),
        # a short sequence of a small model: latency
        dict(_norm("norm_bwd", 60, 512, "none", "rms", 0, "bf16", "f32", add=True), name="norm-back-small"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rotary", "attn_fwd", "attn_fwd", "attn_bwd", "attn_bwd", "norm_fwd", "norm_bwd"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    if kind == "rotary":
        head_dim = 8 * rng.choice((2, 4, 8, 8, 10, 12, 16, 16, 24, 32))
        rot = head_dim if rng.random() < 0.5 else 2 * rng.randint(1, head_dim // 2)
        while True:
            tokens, heads, others = _spread(rng, 1, 32768), rng.randint(1, 40), rng.choice((0, 1, 2, 5, 8))
            if tokens * (heads + others) * head_dim <= 16384 * 35 * 64:
                break
        return _rotary(tokens, heads, others, head_dim, rot, rng.choice(("half", "interleaved")), dtype, far=rng.choice((0, 1000, 1000000)),
                       scaled=rng.choice((1.0, 4.0, 32.0)), transpose=rng.random() < 0.5)
    if kind.startswith("attn"):
        most = 16384 * 16384 * 16 * 128 // 4 / (1 if dtype == "bf16" else 24)
        while True:
            kv_heads, group = rng.choice((1, 2, 4, 5, 8, 16)), rng.choice((1, 1, 2, 4, 5, 8))
            head_dim = rng.choice((64, 64, 128, 128, 8 * rng.randint(1, 16)))
            tokens = _spread(rng, 1, 16384)
            c = _attn(kind, tokens, min(tokens, _spread(rng, 1, 64)), kv_heads * group, kv_heads, head_dim, dtype, causal=rng.random() < 0.75,
                      mix=rng.randint(1, 10 ** 6), tail=rng.choice((0, 0, rng.randint(1, 100))))
            if kv_heads * group <= 40 and _pairs(c) * kv_heads * group * head_dim * (1 if kind == "attn_fwd" else 2.5) <= most:
                return c
    cols = 8 * _spread(rng, 8, 512)
    rows = _spread(rng, 1, min(32768, 8192 * 2048 // cols))
    gates = rng.choice((0, 0, 1, 1, rng.choice([g for g in range(1, rows + 1) if rows % g == 0][:8])))
    post, pre = rng.choice((("none", "layer"), ("none", "rms"), ("rms", "rms"), ("layer", "layer"), ("rms", "none"), ("layer", "none"), ("rms", "layer")))
    return _norm(kind, rows, cols, post, pre, gates, dtype, rng.choice(("f32", dtype)), add=rng.random() < 0.5)


def _lengths(case):
    """Lengths of the sequences: spread over their logarithm, in any order, one of them empty where there are many."""
    rng = random.Random(case["mix"])
    n, total = case["seqs"], case["tokens"]
    share = [math.exp(rng.uniform(0, 3)) for _ in range(n)]
    if n > 8:
        share[rng.randrange(n)] = 0.0
    at, done, out = 0.0, 0, []
    for s in share:
        at += s
        end = int(round(total * min(1.0, at / sum(share))))
        out.append(end - done)
        done = end
    out[max(range(n), key=lambda i: share[i])] += total - done
    return out


def _pairs(case):
    """Pairs of a query and a key that it sees, of one head."""
    return sum(n * (n + 1) // 2 if case["causal"] else n * n for n in _lengths(case))


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "rotary":
        n = case["tokens"] * case["heads"]
        return {"bytes": 2 * e * n * case["head_dim"] + 4 * case["tokens"], "flops": 3 * n * case["rot"]}
    if case["kind"].startswith("attn"):
        t, h, kv, d = case["tokens"], case["heads"], case["kv_heads"], case["head_dim"]
        if case["kind"] == "attn_fwd":
            return {"bytes": e * t * d * 2 * (h + kv) + 4 * t * h, "flops": 4 * _pairs(case) * h * d}
        return {"bytes": e * t * d * 4 * (h + kv) + 4 * t * h, "flops": 10 * _pairs(case) * h * d}
    es = 4 if case["stream"] == "f32" else 2
    n, two = case["rows"] * case["cols"], case["pre"] != "none"
    if case["kind"] == "norm_fwd":
        return {"bytes": n * (2 * es + e + (e if two else 0)), "flops": 16 * n}
    return {"bytes": n * (2 * es + 2 * e + (es + e if two else 0)), "flops": 32 * n}


# --------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    rnd = lambda *shape: torch.randn(shape, device=DEV, generator=gen)  # noqa: E731
    return {"rotary": _prepare_rotary, "attn_fwd": _prepare_attn, "attn_bwd": _prepare_attn, "norm_fwd": _prepare_norm,
            "norm_bwd": _prepare_norm}[case["kind"]](case, gen, rnd)


def _prepare_rotary(case, gen, rnd):
    t, h, d, rot = case["tokens"], case["heads"], case["head_dim"], case["rot"]
    rows = rnd(t, h + case["others"], d).to(DTYPE[case["dtype"]])
    # documents of some hundred tokens, each from a position of its own on where contexts are long
    new = torch.rand(t, device=DEV, generator=gen) < 1 / 300
    new[0] = True
    number = new.long().cumsum(0) - 1
    first = torch.nonzero(new)[:, 0]
    begin = torch.randint(0, case["far"] + 1, (t,), device=DEV, generator=gen)[number]
    positions = (torch.arange(t, device=DEV) - first[number] + begin).to(torch.int32)
    # a pair's angle per position; the slow ones of an extended context are slower by its factor
    freq = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    slow = freq * 2048 < 2 * math.pi
    freq = torch.where(slow, freq / case["scaled"], freq)
    return {"case": dict(case), "x": rows[:, :h], "y": torch.empty((t, h, d), device=DEV, dtype=rows.dtype), "positions": positions, "freq": freq,
            "magnitude": 1.0 + 0.1 * math.log(case["scaled"])}


def _prepare_attn(case, gen, rnd):
    t, tail, h, kv, d, dt = case["tokens"], case["tail"], case["heads"], case["kv_heads"], case["head_dim"], DTYPE[case["dtype"]]
    lengths = _lengths(case)
    # one projection's rows: query, key and value heads side by side; scores of standard deviation 1.5
    rows = rnd(t + tail, h + 2 * kv, d)
    rows[:, :h] *= 1.5
    rows = rows.to(dt)
    ends = torch.tensor([0] + lengths).cumsum(0).to(torch.int32).to(DEV)
    s = {"case": dict(case), "q": rows[:, :h], "k": rows[:, h:h + kv], "v": rows[:, h + kv:], "offsets": ends, "lengths": lengths,
         "ctx": torch.zeros((t + tail, h, d), device=DEV, dtype=dt), "lse": torch.zeros((h, t + tail), device=DEV)}
    if case["kind"] == "attn_bwd":
        _attend(s)                                                         # what the forward left
        s["dctx"] = rnd(t + tail, h, d).to(dt)
        grad = torch.zeros((t + tail, h + 2 * kv, d), device=DEV, dtype=dt)
        s["dq"], s["dk"], s["dv"] = grad[:, :h], grad[:, h:h + kv], grad[:, h + kv:]
    return s


def _prepare_norm(case, gen, rnd):
    r, c, dt, st = case["rows"], case["cols"], DTYPE[case["dtype"]], DTYPE[case["stream"]]
    gain = lambda kind: (1 + 0.1 * rnd(c)).to(dt) if kind != "none" else None  # noqa: E731
    bias = lambda kind: (0.1 * rnd(c)).to(dt) if kind == "layer" else None  # noqa: E731
    # a stream that has grown over the blocks, with channels larger than others; a branch's result around it
    size = torch.exp(0.5 * rnd(c))
    s = {"case": dict(case), "x": (2.0 * rnd(r, c) * size).to(st), "f": (rnd(r, c) * size + 0.2).to(dt), "post_gain": gain(case["post"]),
         "post_bias": bias(case["post"]), "pre_gain": gain(case["pre"]), "pre_bias": bias(case["pre"]),
         "gate": (0.5 + 0.3 * rnd(case["gates"], c)).to(dt) if case["gates"] else None, "alpha": 1.0 if case["gates"] else 0.9, "beta": 0.7,
         "y": torch.empty((r, c), device=DEV, dtype=st), "h": torch.empty((r, c), device=DEV, dtype=dt) if case["pre"] != "none" else None,
         "stats": torch.zeros((4, r), device=DEV)}
    if case["kind"] == "norm_bwd":
        _join(s)                                                           # what the forward left
        s["dy"], s["dh"] = rnd(r, c).to(st), rnd(r, c).to(dt) if case["pre"] != "none" else None
        s["dx"], s["df"] = torch.empty((r, c), device=DEV, dtype=st), torch.empty((r, c), device=DEV, dtype=dt)
        for name in ("post_gain", "post_bias", "pre_gain", "pre_bias", "gate"):
            s["d" + name] = None if s[name] is None else rnd(*s[name].shape)
    return s


# ------------------------------------------------------------------------ run
def run(state):
    return {"rotary": _run_rotary, "attn_fwd": _run_attn_fwd, "attn_bwd": _run_attn_bwd, "norm_fwd": _run_norm_fwd,
            "norm_bwd": _run_norm_bwd}[state["case"]["kind"]](state)


def _run_rotary(s):
    case = s["case"]
    if own:
        from paper_2107_06925_amd import binding as b
        b.chimera_op_rotary(s["x"], s["y"], s["freq"], positions=s["positions"], layout=b.ROTARY_HALF if case["layout"] == "half" else b.ROTARY_INTERLEAVED,
                            magnitude=s["magnitude"], transpose=case["transpose"])
        return s["y"]
    rot = case["rot"]
    angle = s["positions"].double()[:, None] * s["freq"][None, :]
    cos, sin = (angle.cos() * s["magnitude"]).float()[:, None], (angle.sin() * s["magnitude"]).float()[:, None]
    if case["transpose"]:
        sin = -sin
    x, y = s["x"].float(), s["y"]
    if case["layout"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, a * sin + b * cos
    y[..., rot:] = s["x"][..., rot:]
    return y


def _sequences(s):
    """Of each sequence: its rows, and the key and value heads taken at a time, so that scores stay below 2 GB."""
    case, at = s["case"], 0
    group = case["heads"] // case["kv_heads"]
    for n in s["lengths"]:
        if n:
            step = max(1, min(case["kv_heads"], (1 << 29) // (group * n * n)))
            for j in range(0, case["kv_heads"], step):
                yield slice(at, at + n), n, group, slice(j, min(j + step, case["kv_heads"]))
        at += n


def _of_group(x, rows, kv, group):
    """Rows of the query heads that share key and value heads: [heads, group * rows, dim]."""
    part = x[rows, kv.start * group:kv.stop * group].float()
    n, _, d = part.shape
    return part.reshape(n, -1, group, d).permute(1, 2, 0, 3).reshape(-1, group * n, d)


def _back(x, n, group):
    """The other way round: [rows, heads, dim]."""
    return x.reshape(x.shape[0], group, n, -1).permute(2, 0, 1, 3).reshape(n, x.shape[0] * group, -1)


def _scores(s, q, k, n, group):
    z = torch.matmul(q, k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(s["case"]["head_dim"]))
    if s["case"]["causal"]:
        place = torch.arange(n, device=DEV)
        z.view(-1, group, n, n).masked_fill_(place[None, :] > place[:, None], float("-inf"))
    return z


def _attend(s):
    for rows, n, group, kv in _sequences(s):
        q, k, v = _of_group(s["q"], rows, kv, group), _of_group(s["k"], rows, kv, 1), _of_group(s["v"], rows, kv, 1)
        z = _scores(s, q, k, n, group)
        top = z.amax(2, keepdim=True)
        p = torch.exp(z - top)
        total = p.sum(2, keepdim=True)
        heads = slice(kv.start * group, kv.stop * group)
        s["ctx"][rows, heads] = _back(torch.matmul(p, v) / total, n, group).to(s["ctx"].dtype)
        s["lse"][heads, rows] = (top + torch.log(total)).reshape(-1, n)


def _run_attn_fwd(s):
    if own:
        from paper_2107_06925_amd import binding as b
        b.chimera_op_attention_packed_fwd(s["q"], s["k"], s["v"], s["offsets"], s["ctx"], s["lse"], causal=s["case"]["causal"])
    else:
        _attend(s)
    return {"ctx": s["ctx"], "lse": s["lse"]}


def _run_attn_bwd(s):
    if own:
        from paper_2107_06925_amd import binding as b
        b.chimera_op_attention_packed_bwd(s["q"], s["k"], s["v"], s["offsets"], s["ctx"], s["lse"], s["dctx"], s["dq"], s["dk"], s["dv"],
                                          causal=s["case"]["causal"])
    else:
        scale = 1.0 / math.sqrt(s["case"]["head_dim"])
        for rows, n, group, kv in _sequences(s):
            q, k, v = _of_group(s["q"], rows, kv, group), _of_group(s["k"], rows, kv, 1), _of_group(s["v"], rows, kv, 1)
            o, do = _of_group(s["ctx"], rows, kv, group), _of_group(s["dctx"], rows, kv, group)
            heads = slice(kv.start * group, kv.stop * group)
            p = torch.exp(_scores(s, q, k, n, group) - s["lse"][heads, rows].reshape(-1, group * n, 1))
            s["dv"][rows, kv] = _back(torch.matmul(p.transpose(1, 2).contiguous(), do), n, 1).to(s["dv"].dtype)
            ds = p * (torch.matmul(do, v.transpose(1, 2).contiguous()) - (do * o).sum(2, keepdim=True)) * scale
            s["dq"][rows, heads] = _back(torch.matmul(ds, k), n, group).to(s["dq"].dtype)
            s["dk"][rows, kv] = _back(torch.matmul(ds.transpose(1, 2).contiguous(), q), n, 1).to(s["dk"].dtype)
    return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


def _normalised(x, kind):
    """x hat, and the mean and the reciprocal deviation that make it."""
    mean = x.mean(1) if kind == "layer" else torch.zeros_like(x[:, 0])
    centred = x - mean[:, None]
    rstd = 1 / torch.sqrt(centred.square().mean(1) + EPS)
    return centred * rstd[:, None], mean, rstd


def _per_row(s):
    """The gate of each row."""
    g = s["gate"].float()
    return g.repeat_interleave(s["case"]["rows"] // g.shape[0], 0) if g.shape[0] > 1 else g


def _join(s):
    case, u = s["case"], s["f"].float()
    if case["post"] != "none":
        u, s["stats"][0], s["stats"][1] = _normalised(u, case["post"])
        u = u * s["post_gain"].float()
        if s["post_bias"] is not None:
            u = u + s["post_bias"].float()
    if s["gate"] is not None:
        u = u * _per_row(s)
    y = s["alpha"] * s["x"].float() + s["beta"] * u
    s["y"].copy_(y)
    if case["pre"] != "none":
        h, s["stats"][2], s["stats"][3] = _normalised(y, case["pre"])
        h = h * s["pre_gain"].float()
        s["h"].copy_(h if s["pre_bias"] is None else h + s["pre_bias"].float())


def _norms(s):
    from paper_2107_06925_amd import binding as b
    kind = {"none": b.NORM_NONE, "layer": b.NORM_LAYER, "rms": b.NORM_RMS}
    return dict(post=kind[s["case"]["post"]], post_gain=s["post_gain"], post_bias=s["post_bias"], pre=kind[s["case"]["pre"]], pre_gain=s["pre_gain"],
                gate=s["gate"], alpha=s["alpha"], beta=s["beta"])


def _run_norm_fwd(s):
    if own:
        from paper_2107_06925_amd import binding as b
        b.chimera_op_branch_norm_fwd(s["f"], s["x"], s["y"], s["h"], s["stats"], pre_bias=s["pre_bias"], eps=EPS, **_norms(s))
    else:
        _join(s)
    out = {"y": s["y"]}
    if s["case"]["post"] != "none":
        out["post_stats"] = s["stats"][:2]
    if s["h"] is not None:
        out |= {"h": s["h"], "pre_stats": s["stats"][2:]}
    return out


def _run_norm_bwd(s):
    case = s["case"]
    names = [n for n in ("post_gain", "post_bias", "pre_gain", "pre_bias", "gate") if s[n] is not None]
    if own:
        from paper_2107_06925_amd import binding as b
        b.chimera_op_branch_norm_bwd(s["f"], s["y"], s["stats"], s["dy"], s["dh"], s["dx"], s["df"], overwrite=not case["add"],
                                     **_norms(s), **{"d" + n: s["d" + n] for n in names})
    else:
        grads = {}
        dy = s["dy"].float()
        if case["pre"] != "none":
            hat = (s["y"].float() - s["stats"][2][:, None]) * s["stats"][3][:, None]
            dh = s["dh"].float()
            grads["pre_gain"], grads["pre_bias"] = (dh * hat).sum(0), dh.sum(0)
            dhat = dh * s["pre_gain"].float()
            mean = dhat.mean(1, keepdim=True) if case["pre"] == "layer" else 0.0
            dy = dy + s["stats"][3][:, None] * (dhat - mean - hat * (dhat * hat).mean(1, keepdim=True))
        s["dx"].copy_(s["alpha"] * dy)
        du = s["beta"] * dy
        u = s["f"].float()
        if case["post"] != "none":
            hat = (u - s["stats"][0][:, None]) * s["stats"][1][:, None]
            u = hat * s["post_gain"].float()
            if s["post_bias"] is not None:
                u = u + s["post_bias"].float()
        if s["gate"] is not None:
            grads["gate"] = (du * u).view(case["gates"], -1, case["cols"]).sum(1)
            du = du * _per_row(s)
        if case["post"] != "none":
            grads["post_gain"], grads["post_bias"] = (du * hat).sum(0), du.sum(0)
            dhat = du * s["post_gain"].float()
            mean = dhat.mean(1, keepdim=True) if case["post"] == "layer" else 0.0
            du = s["stats"][1][:, None] * (dhat - mean - hat * (dhat * hat).mean(1, keepdim=True))
        s["df"].copy_(du)
        for n in names:
            if case["add"]:
                s["d" + n] += grads[n]
            else:
                s["d" + n].copy_(grads[n])
    return {"dx": s["dx"], "df": s["df"]} | {"d" + n: s["d" + n] for n in names}


# ---------------------------------------------------------------------- exact
def exact(case, seed):
    """What run() gives on these inputs, from the definitions in 64 bits."""
    s = prepare(case, seed)
    if case["kind"] == "rotary":
        return _exact_rotary(case, s)
    if case["kind"].startswith("attn"):
        return _exact_attn(case, s)
    return _exact_norm(case, s)


def _exact_rotary(case, s):
    """Pairs as complex numbers, turned by a unit number."""
    rot = case["rot"]
    y = s["x"].double().clone()
    theta = s["positions"].double().outer(s["freq"]) * (-1.0 if case["transpose"] else 1.0)
    turn = torch.polar(torch.full_like(theta, s["magnitude"]), theta)[:, None]
    if case["layout"] == "half":
        z = torch.complex(y[..., :rot // 2].contiguous(), y[..., rot // 2:rot].contiguous()) * turn
        y[..., :rot] = torch.cat((z.real, z.imag), -1)
    else:
        z = torch.view_as_complex(y[..., :rot].reshape(*y.shape[:2], rot // 2, 2)) * turn
        y[..., :rot] = torch.view_as_real(z).flatten(-2)
    return y


def _exact_attn(case, s):
    """Head by head and sequence by sequence."""
    back, ratio = case["kind"] == "attn_bwd", case["heads"] // case["kv_heads"]
    out = {n: torch.zeros(s[n].shape, device=DEV, dtype=torch.float64) for n in (("dq", "dk", "dv") if back else ("ctx", "lse"))}
    ends = s["offsets"].tolist()
    for lo, hi in zip(ends, ends[1:]):
        if hi == lo:
            continue
        hidden = torch.ones((hi - lo, hi - lo), device=DEV, dtype=torch.bool).triu(1) if case["causal"] else None
        for h in range(case["heads"]):
            q, k, v = s["q"][lo:hi, h].double(), s["k"][lo:hi, h // ratio].double(), s["v"][lo:hi, h // ratio].double()
            z = (q @ k.t()).div_(math.sqrt(case["head_dim"]))
            if hidden is not None:
                z.masked_fill_(hidden, -math.inf)
            if not back:
                out["ctx"][lo:hi, h], out["lse"][h, lo:hi] = torch.softmax(z, 1) @ v, torch.logsumexp(z, 1)
                continue
            p = z.sub_(s["lse"][h, lo:hi].double()[:, None]).exp_()
            do = s["dctx"][lo:hi, h].double()
            out["dv"][lo:hi, h // ratio] += p.t() @ do
            ds = p * ((do @ v.t()) - torch.linalg.vecdot(do, s["ctx"][lo:hi, h].double())[:, None]) / math.sqrt(case["head_dim"])
            out["dq"][lo:hi, h] = ds @ k
            out["dk"][lo:hi, h // ratio] += ds.t() @ q
    return out


def _exact_norm(case, s):
    """The forward from its definition; the gradients by the chain rule, norm by norm, from the statistics that the forward left."""
    f64 = lambda n: None if s[n] is None else s[n].double()  # noqa: E731
    rows = torch.arange(case["rows"], device=DEV)
    gate = f64("gate")[rows * case["gates"] // case["rows"]] if case["gates"] else torch.ones((1, 1), device=DEV, dtype=torch.float64)

    def norm(x, kind, gain, bias):
        mean = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
        rstd = ((x - mean).pow(2).mean(1, keepdim=True) + EPS).rsqrt()
        h = (x - mean) * rstd * gain
        return (h if bias is None else h + bias), torch.cat((mean, rstd), 1).t()

    def norm_back(x, kind, gain, stats, dh):
        hat = (x - stats[0].double()[:, None]) * stats[1].double()[:, None]
        d = dh * gain
        c = x.shape[1]
        dx = d - hat * (torch.linalg.vecdot(d, hat) / c)[:, None]
        if kind == "layer":
            dx = dx - (d.sum(1) / c)[:, None]
        return dx * stats[1].double()[:, None], torch.linalg.vecdot(dh, hat, dim=0), dh.sum(0)

    f = f64("f")
    if case["kind"] == "norm_fwd":
        out, u = {}, f
        if case["post"] != "none":
            u, out["post_stats"] = norm(f, case["post"], f64("post_gain"), f64("post_bias"))
        out["y"] = s["alpha"] * f64("x") + s["beta"] * gate * u
        if case["pre"] != "none":
            out["h"], out["pre_stats"] = norm(out["y"], case["pre"], f64("pre_gain"), f64("pre_bias"))
        return out
    dy, grads = f64("dy"), {}
    if case["pre"] != "none":
        dx, grads["pre_gain"], grads["pre_bias"] = norm_back(f64("y"), case["pre"], f64("pre_gain"), s["stats"][2:], f64("dh"))
        dy = dy + dx
    du, u = s["beta"] * gate * dy, f
    df = du
    if case["post"] != "none":
        u = (f - s["stats"][0].double()[:, None]) * s["stats"][1].double()[:, None] * f64("post_gain")
        u = u if s["post_bias"] is None else u + f64("post_bias")
        df, grads["post_gain"], grads["post_bias"] = norm_back(f, case["post"], f64("post_gain"), s["stats"][:2], du)
    if case["gates"]:
        grads["gate"] = (s["beta"] * dy * u).unflatten(0, (case["gates"], -1)).sum(1)
    out = {"dx": s["alpha"] * dy, "df": df}
    for n in ("post_gain", "post_bias", "pre_gain", "pre_bias", "gate"):
        if s[n] is not None:
            out["d" + n] = grads[n] + s["d" + n].double() if case["add"] else grads[n]
    return out
