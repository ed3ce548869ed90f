"""The operators at the end of a training iteration, as measurable cases.

`xent_fwd`, `xent_bwd`: vocabulary projection and softmax cross-entropy of the last stage without its logits, the loss alone and its
gradients.  `adamw`: the step over all of a stage's tensors, moments in 32 or in 8 bits.  `grad_norm`: the norm over the gradients of a worker's
stages, and the factor that clips them.

Where `own` is false they are computed in plain torch operations, where it is true by the framework's entry points.  Sizes are those
of the framework's workloads (`synth.CONFIGS`, the vocabulary of `bench.py`) or generic.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 256                     # values that share a scale in 8-bit moments
BETA1, BETA2, EPS, LR, DECAY, STEP, SEED = 0.9, 0.95, 1e-8, 3e-4, 0.1, 7, 1234


# ---------------------------------------------------------------------- cases
def _xent(kind, tokens, hidden, vocab, ld, dtype, **more):
    return dict({"kind": kind, "tokens": tokens, "hidden": hidden, "vocab": vocab, "ld": ld, "dtype": dtype}, **more)


def _adamw(bits, dtype, blocks, hidden, odd=0, clip=True):
    return {"kind": "adamw", "bits": bits, "dtype": dtype, "blocks": blocks, "hidden": hidden, "odd": odd, "clip": clip}


def listed():
    return [
        # evaluation of a handful of tokens by a small float model
        dict(_xent("xent_fwd", 24, 256, 1000, 1000, "f32"), name="loss-small-f32"),
        # evaluation at the default workload's width; a vocabulary that is no multiple of 8, stored padded
        dict(_xent("xent_fwd", 2048, 1600, 50257, 50304, "bf16"), name="loss-bf16"),
        # fine-tuning on one short sequence: latency
        dict(_xent("xent_bwd", 60, 512, 8000, 8000, "bf16", weighted=True, add=False), name="grad-small"),
        # the last stage's micro-batch of the default workload, gradients added to those of earlier micro-batches
        dict(_xent("xent_bwd", 2048, 1600, 50257, 50304, "bf16", weighted=False, add=True), name="grad-bf16"),
        # the largest: logits of 1 GB that are never there
        dict(_xent("xent_bwd", 8192, 2048, 65536, 65536, "bf16", weighted=True, add=False), name="grad-large"),
        # float, odd sizes
        dict(_xent("xent_bwd", 632, 320, 30001, 30008, "f32", weighted=True, add=True), name="grad-f32"),
        # the smallest workload's stage: 24 tensors, launch latency
        dict(_adamw(32, "f32", 2, 128), name="adamw-small-f32"),
        # the default workload's stage, float master weights
        dict(_adamw(32, "bf16", 6, 1600), name="adamw-bf16"),
        # 8-bit moments: a small model with an odd tensor (a table of odd length), and a stage of the deep workload
        dict(_adamw(8, "bf16", 1, 256, odd=12345), name="adamw8-small"),
        dict(_adamw(8, "bf16", 2, 2048), name="adamw8-bf16"),
        # both stages' gradients of the smallest and of the default workload
        {"kind": "grad_norm", "tensors": 2, "n": 396544, "name": "norm-small"},
        {"kind": "grad_norm", "tensors": 2, "n": 184425600, "name": "norm-large"},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("xent_fwd", "xent_bwd", "xent_bwd", "adamw", "adamw", "grad_norm"))
    if kind.startswith("xent"):
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        # float costs several times as much: a range of its own
        most = 8192 * 2048 * 65536 / (1 if dtype == "bf16" else 16)
        while True:
            tokens, hidden, vocab = _spread(rng, 1, 8192), 8 * _spread(rng, 8, 256), _spread(rng, 100, 65536)
            if rng.random() < 0.3:
                tokens = max(1, tokens // 64 * 64)
            if tokens * hidden * vocab <= most:
                break
        ld = (vocab + 7) // 8 * 8 if rng.random() < 0.5 else (vocab + 127) // 128 * 128
        if kind == "xent_fwd":
            return _xent(kind, tokens, hidden, vocab, ld, dtype)
        return _xent(kind, tokens, hidden, vocab, ld, dtype, weighted=rng.random() < 0.5, add=rng.random() < 0.5)
    if kind == "adamw":
        hidden = 8 * _spread(rng, 8, 256)
        blocks = rng.randint(1, max(1, min(6, 180_000_000 // (12 * hidden * hidden + 13 * hidden))))
        return _adamw(rng.choice((8, 32)), rng.choice(("bf16", "bf16", "f32")), blocks, hidden, odd=rng.choice((0, _spread(rng, 1, 100000))),
                      clip=rng.random() < 0.7)
    tensors = rng.randint(1, 8)
    return {"kind": "grad_norm", "tensors": tensors, "n": _spread(rng, 1000, 300_000_000 // tensors)}


def _sizes(case):
    """Element counts of the step's tensors and which of them decay: a stage's blocks, and one more tensor."""
    h = case["hidden"]
    block = [(h, 0), (h, 0), (3 * h * h, 1), (3 * h, 0), (h * h, 1), (h, 0), (h, 0), (h, 0), (4 * h * h, 1), (4 * h, 0), (4 * h * h, 1), (h, 0)]
    every = block * case["blocks"] + ([(case["odd"], 1)] if case["odd"] else [])
    return [n for n, _ in every], [bool(d) for _, d in every]


def _pad(n):
    return -(-n // BLOCK) * BLOCK


def work(case):
    if case["kind"].startswith("xent"):
        t, h, v, e = case["tokens"], case["hidden"], case["vocab"], 4 if case["dtype"] == "f32" else 2
        if case["kind"] == "xent_fwd":
            return {"bytes": e * (t * h + h * v) + 4 * t + 8 * t, "flops": 2 * t * h * v}
        return {"bytes": e * (2 * t * h + h * v) + (8 if case["add"] else 4) * h * v + 4 * t * (3 if case["weighted"] else 2), "flops": 6 * t * h * v}
    if case["kind"] == "adamw":
        n = sum(_sizes(case)[0])
        weights = 8 if case["dtype"] == "f32" else 10                      # read, written; bf16: the float one, and the bf16 one written
        states = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
        return {"bytes": n * (4 + weights + states), "flops": 15 * n}
    return {"bytes": 4 * case["tensors"] * case["n"], "flops": 2 * case["tensors"] * case["n"]}


# --------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    return {"xent_fwd": _prepare_xent, "xent_bwd": _prepare_xent, "adamw": _prepare_adamw, "grad_norm": _prepare_norm}[case["kind"]](case, gen)


def _prepare_xent(case, gen):
    t, h, v, ld, dt = case["tokens"], case["hidden"], case["vocab"], case["ld"], DTYPE[case["dtype"]]
    # normalised hidden states, logits of standard deviation 2, targets spread as words are; every tenth token is padding
    hid = torch.randn((t, h), device=DEV, generator=gen).to(dt)
    w = (torch.randn((h, ld), device=DEV, generator=gen) * (2.0 / math.sqrt(h))).to(dt)
    targets = (torch.exp(torch.rand(t, device=DEV, generator=gen) * math.log(v)) - 1).long().clamp(0, v - 1).to(torch.int32)
    targets[torch.rand(t, device=DEV, generator=gen) < 0.1] = -1
    s = {"case": dict(case), "h": hid, "w": w[:, :v], "targets": targets, "scale": 1.0 / t}
    if case["kind"] == "xent_fwd":
        s["loss_rows"], s["lse"], s["loss"] = torch.empty(t, device=DEV), torch.empty(t, device=DEV), torch.zeros(1, device=DEV)
        return s
    s["lse"] = torch.logsumexp(hid.float() @ s["w"].float(), 1)            # what the forward left
    s["dloss"] = torch.rand(t, device=DEV, generator=gen) + 0.5 if case["weighted"] else None
    s["dh"] = torch.empty((t, h), device=DEV, dtype=dt)
    s["dw"] = (torch.randn((h, ld), device=DEV, generator=gen) * 1e-3)[:, :v]
    return s


def _random_bits(n, step, seed):
    """32 bits for each value, from its number, the step and the seed: what the 8-bit moments are rounded by."""
    mask = 0xFFFFFFFF
    key = (seed * 0x243F6A89 + step * 0xB7E15163) & mask
    x = (torch.arange(n, device=DEV) * 0x9E3779B1 + key) & mask
    x = (x ^ (x >> 15)) * 0x6A09E667 & mask
    x = (x ^ (x >> 13)) * 0xBB67AE85 & mask
    return x ^ (x >> 16)


def _encode(x, bits16, floor):
    """[blocks, BLOCK] floats -> e4m3 codes and the blocks' scales; `floor`: what is not zero stays above it."""
    top = x.abs().amax(1, keepdim=True)
    some = top > 1e-30
    inv = torch.where(some, 448.0 / top, torch.zeros_like(top))
    y = x.abs() * inv
    code = (((y * 2.0 ** -120).view(torch.int32) + bits16 * 16 + 8) >> 20).clamp(max=126)
    if floor:
        code = torch.where(y > 0, code.clamp(min=1), code)
    code = torch.where(y > 0, code, torch.zeros_like(code))
    code = torch.where(x < 0, code | 128, code)
    return code.to(torch.uint8).view(torch.float8_e4m3fn), torch.where(some, top / 448.0, torch.zeros_like(top)).reshape(-1)


def _prepare_adamw(case, gen):
    sizes, decays = _sizes(case)
    at = [0]
    for n in sizes:
        at.append(at[-1] + _pad(n))                                       # tensors begin at multiples of a block of moments
    total = at[-1]
    rnd = lambda: torch.randn(total, device=DEV, generator=gen)  # noqa: E731
    used = torch.zeros(total, device=DEV)
    decay = torch.zeros(total, device=DEV)
    for n, d, a in zip(sizes, decays, at):
        used[a:a + n] = 1
        decay[a:a + n] = DECAY * d
    # gradients whose size differs from row to row and moments that fit them
    size = torch.exp(torch.randn(total // BLOCK, device=DEV, generator=gen)).repeat_interleave(BLOCK) * 1e-3
    master, grad = rnd() * 0.02 * used, rnd() * size * used
    m, v = rnd() * size * 0.3 * used, (rnd() * size).square() * used
    s = {"case": dict(case), "at": at, "sizes": sizes, "decays": decays, "decay": decay, "grad": grad, "param": master.to(DTYPE[case["dtype"]]),
         "master": master if case["dtype"] == "bf16" else None, "factor": torch.full((1,), 0.37, device=DEV) if case["clip"] else None}
    if case["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        half = torch.full((total // BLOCK, BLOCK), 0x7FFF, device=DEV, dtype=torch.int32)
        s["m"], ms = _encode(m.view(-1, BLOCK), half, False)
        s["v"], vs = _encode(v.sqrt().view(-1, BLOCK), half, True)
        s["scales"] = torch.stack((ms, vs), 1).contiguous()                # a pair for each block
    if own:
        # the handle that a training program keeps for its tensors
        from paper_2107_06925_amd import binding as b
        part = lambda x: [x.view(-1)[a:a + n] for a, n in zip(at, sizes)]  # noqa: E731
        s["optimizer"] = b.AdamW(part(s["param"]), part(grad), part(s["m"]), part(s["v"]), masters=part(master) if case["dtype"] == "bf16" else None,
                                 scales=None if case["bits"] == 32 else [s["scales"][a // BLOCK:(a + _pad(n)) // BLOCK] for a, n in zip(at, sizes)],
                                 decay=[DECAY * d for d in decays], beta1=BETA1, beta2=BETA2, eps=EPS)
    return s


def _prepare_norm(case, gen):
    grads = torch.randn(case["tensors"] * case["n"], device=DEV, generator=gen) * 1e-3
    return {"case": dict(case), "grads": grads, "out": torch.empty(2, device=DEV)}


# ------------------------------------------------------------------------ run
def run(state):
    return {"xent_fwd": _run_xent_fwd, "xent_bwd": _run_xent_bwd, "adamw": _run_adamw, "grad_norm": _run_norm}[state["case"]["kind"]](state)


def _run_xent_fwd(s):
    if own:
        from paper_2107_06925_amd import binding as b
        b.chimera_op_linear_xent_fwd(s["h"], s["w"], s["targets"], s["scale"], s["loss_rows"], s["lse"], s["loss"])
    else:
        z = s["h"].float() @ s["w"].float()
        top = z.amax(1)
        s["lse"].copy_(top + torch.log(torch.exp(z - top[:, None]).sum(1)))
        t, valid = s["targets"].long(), s["targets"] >= 0
        at = z.gather(1, t.clamp(min=0)[:, None])[:, 0]
        s["loss_rows"].copy_(torch.where(valid, s["scale"] * (s["lse"] - at), torch.zeros_like(at)))
        s["loss"] += s["loss_rows"].sum()
    return {"loss_rows": s["loss_rows"], "lse": s["lse"], "loss": s["loss"]}


def _run_xent_bwd(s):
    add = s["case"]["add"]
    if own:
        from paper_2107_06925_amd import binding as b
        b.chimera_op_linear_xent_bwd(s["h"], s["w"], s["targets"], s["lse"], s["scale"], s["dh"], s["dw"], dloss=s["dloss"], overwrite=not add)
    else:
        h, w = s["h"].float(), s["w"].float()
        dz = torch.exp(h @ w - s["lse"][:, None])
        t, valid = s["targets"].long(), s["targets"] >= 0
        rows = torch.arange(t.numel(), device=DEV)
        dz[rows, t.clamp(min=0)] -= 1
        coef = s["scale"] * valid.float()
        if s["dloss"] is not None:
            coef = coef * s["dloss"]
        dz *= coef[:, None]
        s["dh"].copy_(dz @ w.t())
        dw = h.t() @ dz
        if add:
            s["dw"] += dw
        else:
            s["dw"].copy_(dw)
    return {"dh": s["dh"], "dw": s["dw"]}


def _run_adamw(s):
    eight = s["case"]["bits"] == 8
    if own:
        s["optimizer"].step(lr=LR, step=STEP, seed=SEED, grad_scale=s["factor"])
    else:
        g = s["grad"] * s["factor"] if s["factor"] is not None else s["grad"]
        if eight:
            m = s["m"].float() * s["scales"][:, :1]
            r = s["v"].float() * s["scales"][:, 1:]
            g = g.view(-1, BLOCK)
            v = r * r
        else:
            m, v = s["m"], s["v"]
        m = m * BETA1 + g * (1 - BETA1)
        v = v * BETA2 + (g * g) * (1 - BETA2)
        r = v.sqrt()
        p = s["param"] if s["master"] is None else s["master"]
        keep = 1 - s["decay"] * LR
        step = (m * (LR / (1 - BETA1 ** STEP))) / (r * (1 / math.sqrt(1 - BETA2 ** STEP)) + EPS)
        p.copy_(p * keep - step.view(-1))
        if s["master"] is not None:
            s["param"].copy_(p)
        if eight:
            bits = _random_bits(m.numel(), STEP, SEED).view(-1, BLOCK)
            codes, ms = _encode(m, (bits & 0xFFFF).int(), False)
            s["m"].view(torch.uint8).copy_(codes.view(torch.uint8))
            codes, vs = _encode(r, (bits >> 16).int(), True)
            s["v"].view(torch.uint8).copy_(codes.view(torch.uint8))
            s["scales"].copy_(torch.stack((ms, vs), 1))
        else:
            s["m"].copy_(m)
            s["v"].copy_(v)
    out = {"param": s["param"], "m": s["m"], "v": s["v"]}
    if s["master"] is not None:
        out["master"] = s["master"]
    if eight:
        out["scales"] = s["scales"]
    return out


def _run_norm(s):
    if own:
        from paper_2107_06925_amd import binding as b
        b.chimera_op_grad_norm(list(s["grads"].chunk(s["case"]["tensors"])), 1.0, s["out"])
    else:
        norm = s["grads"].square().sum(dtype=torch.float64).sqrt()
        s["out"][0] = norm
        s["out"][1] = torch.clamp(1.0 / norm, max=1.0)
    return s["out"]


# ---------------------------------------------------------------------- exact
def exact(case, seed):
    """What run() gives on these inputs, from the definitions in 64 bits."""
    s = prepare(case, seed)
    if case["kind"] == "grad_norm":
        norm = float(torch.linalg.vector_norm(s["grads"], dtype=torch.float64))
        return torch.tensor([norm, min(1.0, 1.0 / norm)], dtype=torch.float64)
    if case["kind"] == "adamw":
        g = s["grad"].double() * (float(s["factor"]) if case["clip"] else 1.0)
        if case["bits"] == 8:
            spread = s["scales"].double().repeat_interleave(BLOCK, 0)
            m, v = s["m"].to(torch.float64).view(-1) * spread[:, 0], (s["v"].to(torch.float64).view(-1) * spread[:, 1]).square()
        else:
            m, v = s["m"].double(), s["v"].double()
        m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g.square()
        p = (s["param"] if s["master"] is None else s["master"]).double()
        p = p - LR * s["decay"].double() * p - LR * (m / (1 - BETA1 ** STEP)) / ((v / (1 - BETA2 ** STEP)).sqrt() + EPS)
        out = {"param": p, "m": m, "v": v}
        if s["master"] is not None:
            out["master"] = p
        if case["bits"] == 8:                                             # codes are rounded at random; their scales are not
            top = torch.stack((m.abs().view(-1, BLOCK).amax(1), v.sqrt().view(-1, BLOCK).amax(1)), 1)
            out |= {"m": None, "v": None, "scales": torch.where(top > 1e-30, top / 448, torch.zeros_like(top))}
        return out
    h, w, t = s["h"].double(), s["w"].double(), s["targets"].long()
    z = torch.matmul(h, w)
    valid = (t >= 0).double()
    if case["kind"] == "xent_fwd":
        lse = torch.logsumexp(z, dim=1)
        rows = valid * s["scale"] * (lse - z[torch.arange(t.numel(), device=DEV), t.clamp(min=0)])
        return {"loss_rows": rows, "lse": lse, "loss": rows.sum().reshape(1)}
    z.sub_(s["lse"].double()[:, None]).exp_()
    z[torch.arange(t.numel(), device=DEV), t.clamp(min=0)] -= 1.0
    z.mul_((valid * s["scale"] * (s["dloss"].double() if case["weighted"] else 1.0))[:, None])
    dw = torch.matmul(h.t(), z)
    return {"dh": torch.matmul(z, w.t()), "dw": s["dw"].double() + dw if case["add"] else dw}
