"""GPU parity of the loss without logits, the gradient norm and AdamW against plain 64-bit arithmetic (torch float64).

Tolerances are per element and count roundings.  A sum of K products in floats, in any order, is off by at most K 2^-24 of the sum of the products'
magnitudes (float operands, held as three bf16 numbers, leave out 2^-24 of each product more); the hardware's exp2 by 2^-22 relative, its argument,
rounded, by 2^-23 |x| more; a result in bf16 by 2^-8, half a step."""
import math

import pytest

from paper_2107_06925_amd import binding as b

pytestmark = pytest.mark.gpu

E24, E23, E22 = 2.0 ** -24, 2.0 ** -23, 2.0 ** -22


def _torch():
    import torch
    return torch


def _dtype(dtype):
    torch = _torch()
    return torch.float32 if dtype == b.F32 else torch.bfloat16


def _case(dtype, tokens, hidden, vocab, ldw=None, ldh=None, ignore=0.2, seed=0, peak=2.0, poison=True):
    """h, w, targets on views whose rows lie further apart than they are long; NaN wherever the operators must not look."""
    torch = _torch()
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ldw, ldh = ldw or (vocab + 7) // 8 * 8, ldh or hidden
    t = _dtype(dtype)
    w = torch.full((hidden, ldw), float("nan") if poison else 0.0, device="cuda", dtype=t)
    w[:, :vocab] = (torch.randn((hidden, vocab), device="cuda", generator=gen) * (peak / math.sqrt(hidden))).to(t)
    h = torch.full((tokens, ldh), float("nan") if poison else 0.0, device="cuda", dtype=t)
    h[:, :hidden] = torch.randn((tokens, hidden), device="cuda", generator=gen).to(t)
    targets = torch.randint(0, vocab, (tokens,), device="cuda", generator=gen, dtype=torch.int32)
    drop = torch.rand(tokens, device="cuda", generator=gen) < ignore
    if ignore and tokens > 2:
        drop[tokens // 2] = True
    targets[drop] = torch.tensor([-1, -100, vocab, 2 ** 31 - 1, -2 ** 31], device="cuda", dtype=torch.int64).to(torch.int32)[torch.arange(int(drop.sum())).cuda() % 5]
    return h[:, :hidden], w[:, :vocab], targets


def _logits(h, w, dtype):
    """z in 64 bits and how far a float z may be from it."""
    z = h.double() @ w.double()
    k = h.shape[1]
    off = (k + 8 + (16 if dtype == b.F32 else 0)) * E24 * (h.double().abs() @ w.double().abs())
    return z, off


def _forward(h, w, targets, scale, loss0=0.5, workspace=None):
    torch = _torch()
    tokens = h.shape[0]
    rows, lse = torch.full((tokens,), float("nan"), device="cuda"), torch.full((tokens,), float("nan"), device="cuda")
    loss = torch.full((1,), loss0, device="cuda")
    b.chimera_op_linear_xent_fwd(h, w, targets, scale, rows, lse, loss, workspace=workspace)
    return rows, lse, loss


def _check_forward(dtype, h, w, targets, scale, rows, lse, loss, loss0=0.5):
    torch = _torch()
    z, off = _logits(h, w, dtype)
    want = torch.logsumexp(z, 1)
    # a shift of all logits by `off`, and sums of exponentials off by (V + 64) 2^-24 + 2^-22 + what the arguments lose (x 2^-23 weighted with e^-x: below 2^-23)
    lse_off = off.amax(1) + (w.shape[1] * E24 if w.shape[1] < 4096 else 4096 * E24) + 4 * E22 + want.abs() * E23
    assert ((lse.double() - want).abs() <= lse_off).all(), float(((lse.double() - want).abs() / lse_off).max())
    valid = (targets >= 0) & (targets < w.shape[1])
    at = z.gather(1, targets.clamp(0, w.shape[1] - 1).long()[:, None])[:, 0]
    per = torch.where(valid, scale * (want - at), torch.zeros_like(at))
    per_off = torch.where(valid, abs(scale) * (lse_off + off.amax(1) + 2 * E24 * (want.abs() + at.abs())), torch.zeros_like(at))
    assert ((rows.double() - per).abs() <= per_off).all()
    total = float(rows.double().sum()) + loss0
    assert abs(float(loss) - total) <= (rows.numel() + 8) * E24 * (float(rows.double().abs().sum()) + abs(loss0))


# tiles of 256x256 need 144 of them (1024 x 9300), more 128x128 tiles than CUs 2200 tokens x 2000; both ends of a tile, one token, one word
FWD = [(1, 8, 1, 8, 8), (1, 64, 7, 16, 64), (2, 8, 8, 8, 16), (24, 256, 1000, 1000, 256), (33, 72, 257, 264, 80), (130, 136, 513, 576, 136), (128, 64, 384, 384, 64),
       (1, 1600, 50257, 50304, 1600), (1024, 64, 9300, 9304, 64), (1000, 192, 9473, 9480, 200), (2200, 128, 2001, 2008, 128), (70, 128, 30011, 30016, 128)]


@pytest.mark.parametrize("dtype", [b.F32, b.BF16])
@pytest.mark.parametrize("tokens,hidden,vocab,ldw,ldh", FWD)
def test_linear_xent_fwd(dtype, tokens, hidden, vocab, ldw, ldh):
    print("linear xent fwd", dtype, tokens, hidden, vocab, ldw, ldh, flush=True)
    h, w, targets = _case(dtype, tokens, hidden, vocab, ldw, ldh, seed=tokens + vocab)
    rows, lse, loss = _forward(h, w, targets, 0.25)
    _check_forward(dtype, h, w, targets, 0.25, rows, lse, loss)


@pytest.mark.parametrize("dtype", [b.F32, b.BF16])
def test_linear_xent_fwd_extreme_logits(dtype):
    # one word holds all of the probability; all logits equal; logits of +-80 000; every token ignored
    torch = _torch()
    h, w, targets = _case(dtype, 40, 64, 3001, ignore=0.0, seed=5)
    h[:10] *= 40
    h[10:20] = 0
    h[20:30] *= 20000
    targets[30:] = -1
    rows, lse, loss = _forward(h, w, targets, 1.0)
    _check_forward(dtype, h, w, targets, 1.0, rows, lse, loss)
    assert (lse[10:20] - math.log(3001)).abs().max() <= 1e-5
    targets.fill_(-1)
    rows, _, loss = _forward(h, w, targets, 1.0)
    assert torch.equal(rows, torch.zeros_like(rows)) and float(loss) == 0.5


def _backward(dtype, h, w, targets, lse, scale, dloss=None, overwrite=False, piece=0, want=("dh", "dw"), lddw=None, lddh=None, seed=9, workspace=None):
    torch = _torch()
    (tokens, hidden), vocab = h.shape, w.shape[1]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dh = torch.full((tokens, lddh or hidden), 7.0, device="cuda", dtype=_dtype(dtype))
    dw0 = torch.randn((hidden, lddw or (vocab + 7) // 8 * 8), device="cuda", generator=gen) * 1e-3
    dw = dw0.clone()
    if overwrite:
        dw[:, :vocab] = float("nan")
    b.chimera_op_linear_xent_bwd(h, w, targets, lse, scale, dh[:, :hidden] if "dh" in want else None, dw[:, :vocab] if "dw" in want else None, dloss=dloss,
                                 overwrite=overwrite, piece=piece, workspace=workspace)
    assert torch.equal(dw[:, vocab:], dw0[:, vocab:]), "columns behind the vocabulary are left as they are"
    assert (dh[:, hidden:] == 7.0).all()
    return dh[:, :hidden], dw[:, :vocab], dw0[:, :vocab]


def _check_backward(dtype, h, w, targets, lse, scale, dloss, dh, dw, dw0):
    torch = _torch()
    tokens, vocab = h.shape[0], w.shape[1]
    valid = (targets >= 0) & (targets < vocab)
    h = torch.where(valid[:, None], h, torch.zeros_like(h))                # (a token that does not count may hold anything)
    lse = torch.where(valid, lse, torch.zeros_like(lse))
    z, off = _logits(h, w, dtype)
    x = z - lse.double()[:, None]
    p = x.exp()
    # p: z is off by `off`, z - lse and its product with log2 e are rounded, exp2; one rounding of p - 1, one of its product with coef
    p_off = p * (off + 3 * E24 * (x.abs() + z.abs()) + E22) + E23 * (p + 1)
    coef = scale * (valid.double() if dloss is None else torch.where(valid, dloss.double(), torch.zeros_like(dloss).double()))
    dz = p.clone()
    rows = torch.arange(tokens, device="cuda")
    dz[rows, targets.clamp(0, vocab - 1).long()] -= 1
    dz *= coef[:, None]
    dz_off = coef.abs()[:, None] * p_off + 2 * E24 * dz.abs()
    hd, wd = h.double(), w.double()
    if dh is not None:
        want = dz @ wd.t()
        mag = dz.abs() @ wd.abs().t()
        rounding = 2.0 ** -11 if dtype == b.BF16 else 3 * E24          # dz as one fp16 number
        tol = dz_off @ wd.abs().t() + (rounding + (vocab + 64 + 80) * E24) * mag + (2.0 ** -8 if dtype == b.BF16 else E24) * want.abs() + 1e-38
        assert ((dh.double() - want).abs() <= tol).all(), float(((dh.double() - want).abs() / tol).max())
        assert (dh[~valid] == 0).all()
    if dw is not None:
        want = hd.t() @ dz
        mag = hd.abs().t() @ dz.abs()
        # dz in two fp16 numbers: 2^-22 of it, and 2^-25 2^-14 of the largest there is (below fp16's smallest numbers)
        top = float((coef.abs() * hd.abs().amax(1)).max())
        tol = hd.abs().t() @ dz_off + (E22 + (2 * tokens + 80) * E24) * mag + tokens * 2.0 ** -36 * top + E24 * (want + dw0.double()).abs() + 1e-38
        got = dw.double() - dw0.double()
        assert ((got - want).abs() <= tol + E24 * dw0.double().abs()).all(), float(((got - want).abs() / tol).max())


# (tokens, hidden, vocab, ldw, piece): one piece and several, the last a few columns or ending inside a group of 8; dW cut along the tokens, on
# 256x256 tiles (3000 x 256 x 30001, 9000 x 136 x 2051) and on 128x128 ones (6100 x 72 x 1100); uncut on 256x256 tiles: BWD_LARGE, below
BWD = [(1, 8, 1, 8, 0), (1, 64, 7, 16, 0), (2, 8, 8, 8, 0), (3, 16, 9, 24, 0), (24, 256, 1000, 1000, 0), (33, 72, 257, 264, 256), (130, 136, 1027, 1088, 256),
       (260, 264, 771, 776, 512), (60, 512, 8000, 8000, 0), (1024, 64, 9300, 9304, 0), (40, 1000, 9473, 9480, 4864), (2200, 128, 2001, 2008, 0),
       (4100, 2304, 1031, 1032, 512), (3000, 256, 30001, 30008, 0), (100, 320, 20011, 20024, 4608),
       (6100, 72, 1100, 1104, 512), (9000, 136, 2051, 2056, 0)]


@pytest.mark.parametrize("dtype", [b.F32, b.BF16])
@pytest.mark.parametrize("tokens,hidden,vocab,ldw,piece", BWD)
def test_linear_xent_bwd(dtype, tokens, hidden, vocab, ldw, piece):
    torch = _torch()
    print("linear xent bwd", dtype, tokens, hidden, vocab, ldw, piece, flush=True)
    h, w, targets = _case(dtype, tokens, hidden, vocab, ldw, hidden + 8, seed=tokens + vocab)
    lse = torch.logsumexp(h.double() @ w.double(), 1).float()
    valid = (targets >= 0) & (targets < vocab)
    h[~valid] = float("nan")
    lse[~valid] = float("nan")
    gen = torch.Generator(device="cuda").manual_seed(3)
    dloss = torch.randn(tokens, device="cuda", generator=gen) * torch.exp(3 * torch.randn(tokens, device="cuda", generator=gen))
    for weights, overwrite in ((None, True), (dloss, False)):
        dh, dw, dw0 = _backward(dtype, h, w, targets, lse, 0.01, weights, overwrite, piece, lddw=ldw + 8, lddh=hidden + 16)
        _check_backward(dtype, h, w, targets, lse, 0.01, weights, dh, dw, torch.zeros_like(dw0) if overwrite else dw0)


@pytest.mark.parametrize("dtype", [b.F32, b.BF16])
def test_linear_xent_bwd_one_gradient_alone_and_bit_for_bit(dtype):
    torch = _torch()
    h, w, targets = _case(dtype, 150, 136, 1027, seed=2)
    _, lse, _ = _forward(h, w, targets, 1.0)
    both = _backward(dtype, h, w, targets, lse, 0.1, piece=512)
    again = _backward(dtype, h, w, targets, lse, 0.1, piece=512)
    assert torch.equal(both[0], again[0]) and torch.equal(both[1], again[1])
    dh, dw, dw0 = _backward(dtype, h, w, targets, lse, 0.1, piece=512, want=("dh",))
    assert torch.equal(dh, both[0]) and torch.equal(dw, dw0)
    dh, dw, _ = _backward(dtype, h, w, targets, lse, 0.1, piece=512, want=("dw",))
    assert torch.equal(dw, both[1]) and (dh == 7.0).all()


@pytest.mark.parametrize("dtype", [b.F32, b.BF16])
def test_linear_xent_bwd_ranges(dtype):
    # rows of h and weights of very different size: fp16 holds 2^-24 .. 65504, the operands here span 2^-100 .. 2^40
    torch = _torch()
    h, w, targets = _case(dtype, 64, 64, 500, ignore=0.0, seed=11)
    for i, e in enumerate((-100, -60, -30, -20, -10, 0, 10, 16)):
        h[i * 8:i * 8 + 8] *= 2.0 ** e
    w *= 2.0 ** -14                                                         # logits of at most a few
    lse = torch.logsumexp(h.double() @ w.double(), 1).float()
    for dloss in (None, torch.exp2(torch.linspace(-60, 40, 64, device="cuda")), torch.zeros(64, device="cuda")):
        dh, dw, dw0 = _backward(dtype, h, w, targets, lse, 2.0 ** -10, dloss, overwrite=True)
        _check_backward(dtype, h, w, targets, lse, 2.0 ** -10, dloss, dh, dw, torch.zeros_like(dw0))
    targets.fill_(500)                                                      # nothing counts
    dh, dw, _ = _backward(dtype, h, w, targets, lse, 1.0, None, overwrite=True)
    assert (dh == 0).all() and (dw == 0).all()
    dh, dw, dw0 = _backward(dtype, h, w, targets, lse, 1.0, None)
    assert torch.equal(dw, dw0)


def test_linear_xent_gradient_against_differences():
    # the gradients the backward leaves are those of the loss the forward leaves (float, central differences along random directions)
    torch = _torch()
    h, w, targets = _case(b.F32, 30, 40, 203, seed=4, poison=False)
    h, w = h.contiguous(), w
    _, lse, _ = _forward(h, w, targets, 0.1)
    dh, dw, _ = _backward(b.F32, h, w, targets, lse, 0.1, overwrite=True)
    gen = torch.Generator(device="cuda").manual_seed(8)
    for k in range(4):
        u, v = torch.randn(h.shape, device="cuda", generator=gen), torch.randn(w.shape, device="cuda", generator=gen)
        u, v = u / u.norm(), v / v.norm()
        step = 2.0 ** -4
        f = []
        for s in (step, -step):
            wide = torch.zeros((40, 208), device="cuda")
            wide[:, :203] = w + s * v
            f.append(float(_forward(h + s * u, wide[:, :203], targets, 0.1)[0].double().sum()))
        slope = float((dh.double() * u).sum() + (dw.double() * v).sum())
        assert abs((f[0] - f[1]) / (2 * step) - slope) <= 2e-3 * max(1.0, abs(slope))      # step^2/6 of the third derivative, 2^-24 of a loss of 50 / step


def test_linear_xent_captured_and_on_another_stream():
    torch = _torch()
    h, w, targets = _case(b.BF16, 200, 128, 3001, seed=6)
    rows, lse, loss = _forward(h, w, targets, 0.1)
    want = _backward(b.BF16, h, w, targets, lse, 0.1, piece=1024, overwrite=True)
    side = torch.cuda.Stream()
    ws_f = torch.empty(b.lib().chimera_op_linear_xent_fwd_workspace_bytes(b.BF16, 200, 128, 3001), dtype=torch.uint8, device="cuda")
    ws_b = torch.empty(b.lib().chimera_op_linear_xent_bwd_workspace_bytes(b.BF16, 200, 128, 3001, 1024), dtype=torch.uint8, device="cuda")
    rows2, lse2, loss2 = torch.zeros(200, device="cuda"), torch.zeros(200, device="cuda"), torch.zeros(1, device="cuda")
    dh2, dw2 = torch.zeros((200, 128), device="cuda", dtype=torch.bfloat16), torch.zeros((128, 3008), device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()

    def both():
        b.chimera_op_linear_xent_fwd(h, w, targets, 0.1, rows2, lse2, loss2, workspace=ws_f)
        b.chimera_op_linear_xent_bwd(h, w, targets, lse2, 0.1, dh2, dw2[:, :3001], overwrite=True, piece=1024, workspace=ws_b)
    with torch.cuda.stream(side):
        both()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            both()
    for _ in range(3):
        for t in (rows2, lse2, loss2, dh2, dw2):
            t.fill_(-3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(rows2, rows) and torch.equal(lse2, lse) and torch.equal(dh2, want[0]) and torch.equal(dw2[:, :3001], want[1])
        assert abs(float(loss2) + 3.0 - (float(loss) - 0.5)) <= 1e-5


def test_linear_xent_two_calls_at_once():
    torch = _torch()
    cases = [_case(b.BF16, 700, 256, 5003, seed=s) for s in (1, 2)]
    alone, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for h, w, targets in cases:
        rows, lse, _ = _forward(h, w, targets, 0.1)
        alone.append((rows, lse) + _backward(b.BF16, h, w, targets, lse, 0.1, piece=2048, overwrite=True)[:2])
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(3):
        for i, (h, w, targets) in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                rows, lse, _ = _forward(h, w, targets, 0.1)
                dh, dw = torch.empty_like(h, memory_format=torch.contiguous_format), torch.empty((256, 5008), device="cuda")
                ws = b.chimera_op_linear_xent_bwd(h, w, targets, lse, 0.1, dh, dw[:, :5003], overwrite=True, piece=2048)
                got[i] = (rows, lse, dh, dw[:, :5003], ws)
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(x, y) for x, y in zip(got[i], alone[i]))


@pytest.mark.parametrize("dtype", [b.F32, b.BF16])
@pytest.mark.parametrize("tokens,hidden,vocab,ldw,piece", [(96, 64, 504, 504, 256), (130, 256, 1001, 1016, 0)])
def test_head_loss_pieces_against_head_loss(dtype, tokens, hidden, vocab, ldw, piece):
    torch = _torch()
    print("head pieces", dtype, tokens, hidden, vocab, flush=True)
    t = _dtype(dtype)
    gen = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    y, g, be = rnd(tokens, hidden).to(t), (1 + 0.1 * rnd(hidden)).to(t), (0.1 * rnd(hidden)).to(t)
    w = torch.zeros((hidden, ldw), device="cuda", dtype=t)
    w[:, :vocab] = (0.2 * rnd(hidden, vocab)).to(t)
    targets = torch.randint(0, vocab, (tokens,), device="cuda", generator=gen, dtype=torch.int32)

    def outputs(ld):
        return [torch.zeros((tokens, hidden), device="cuda", dtype=t), torch.full((hidden,), 0.5, device="cuda"), torch.full((hidden,), -0.5, device="cuda"),
                torch.full((hidden, ld), 0.25, device="cuda"), torch.full((1,), 2.0, device="cuda")]
    got = outputs(ldw)
    b.chimera_head_loss_pieces(y, targets, g, be, w[:, :vocab], 1.0 / tokens, *got, piece=piece)
    # 64 bits, through autograd
    p = [x.double().requires_grad_() for x in (y, g, be, w[:, :vocab])]
    h = torch.nn.functional.layer_norm(p[0], (hidden,), p[1], p[2], 1e-5)
    loss = torch.nn.functional.cross_entropy(h @ p[3], targets.long())
    loss.backward()
    tol = 2e-2 if dtype == b.BF16 else 1e-4                                   # the head's bars: h is rounded to the type between the kernels
    want = [p[0].grad, p[1].grad + 0.5, p[2].grad - 0.5, p[3].grad + 0.25]
    for name, a, q in zip(("dy", "dg", "db", "dw"), [got[0], got[1], got[2], got[3][:, :vocab]], want):
        base = {"dy": 0.0, "dg": 0.5, "db": -0.5, "dw": 0.25}[name]
        err = float((a.double() - q).abs().max() / (q - base).abs().max())
        assert err <= tol, (name, err)
    assert (got[3][:, vocab:] == 0.25).all()
    assert abs(float(got[4]) - 2.0 - float(loss)) <= tol * float(loss)
    if vocab % 8 == 0:                                                        # and the head that keeps its logits agrees
        kept = outputs(vocab)
        b.chimera_head_loss(y, targets, g, be, w, 1.0 / tokens, *kept)
        for a, q in zip(got, kept):
            assert float((a.double() - q.double()).abs().max()) <= 2 * tol * max(1e-3, float(q.double().abs().max()))
    # tokens that do not count: as if they were not there
    targets[::3] = -1
    few = outputs(ldw)
    b.chimera_head_loss_pieces(y, targets, g, be, w[:, :vocab], 1.0 / tokens, *few, piece=piece)
    assert (few[0][::3].float() == 0).all()


# ---------------------------------------------------------------- gradient norm
@pytest.mark.parametrize("sizes", [[1], [3], [4095, 1, 0, 4097], [100003] * 5, [7] * 150, [5_000_001, 20_000_003], [70_000_000]])
def test_grad_norm(sizes):
    torch = _torch()
    print("grad norm", len(sizes), sum(sizes), flush=True)
    gen = torch.Generator(device="cuda").manual_seed(2)
    grads = [torch.randn(n + 1, device="cuda", generator=gen)[1:] * 1e-3 for n in sizes]       # 4-byte aligned only
    out = torch.empty(2, device="cuda")
    want = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    for max_norm in (want * 0.5, want * 2, 1e-20):
        b.chimera_op_grad_norm(grads, max_norm, out)
        norm, factor = (float(x) for x in out)
        assert abs(norm - want) <= 2 * E24 * want                                 # one rounding: the sum is in double
        assert abs(factor - min(1.0, max_norm / want)) <= 3 * E24 * factor
    b.chimera_op_grad_norm(grads, want * 2, out)
    assert float(out[1]) == 1.0


def test_grad_norm_ranges():
    torch = _torch()
    out = torch.empty(2, device="cuda")
    for values, norm, factor in (([0.0, 0.0], 0.0, 1.0), ([3e30, 4e30], 5e30, 2e-31), ([3e-30, -4e-30], 5e-30, 1.0), ([3.4e38, 1.0], 3.4e38, 1 / 3.4e38)):
        b.chimera_op_grad_norm([torch.tensor(values, device="cuda")], 1.0, out)
        assert abs(float(out[0]) - norm) <= 4 * E24 * norm and abs(float(out[1]) - factor) <= 4 * E24 * factor + 2.0 ** -149
    for bad in (float("inf"), float("nan"), -float("inf")):
        b.chimera_op_grad_norm([torch.tensor([1.0, bad, 2.0], device="cuda")], 1.0, out)
        assert not math.isfinite(float(out[0])) and math.isnan(float(out[1]))
    b.chimera_op_grad_norm([torch.full((2000,), 3e38, device="cuda")], 1.0, out)          # the norm itself overflows
    assert math.isinf(float(out[0])) and math.isnan(float(out[1]))


# ------------------------------------------------------------------------ AdamW
def _tensors(dtype, sizes, bits, seed=0, shift=0):
    """Weights, gradients and moments of tensors that lie in one buffer, `shift` elements from an aligned place."""
    torch = _torch()
    gen = torch.Generator(device="cuda").manual_seed(seed)
    total = sum(sizes) + shift
    cut = lambda x: [p for p in x[shift:].split(sizes)]  # noqa: E731
    size = torch.exp(torch.randn(total, device="cuda", generator=gen))
    master, grad = torch.randn(total, device="cuda", generator=gen) * 0.02, torch.randn(total, device="cuda", generator=gen) * size * 1e-3
    s = dict(grads=cut(grad), params=cut(master.to(_dtype(dtype))), masters=cut(master) if dtype == b.BF16 else None, scales=None)
    if dtype == b.F32:
        s["params"] = cut(master)
    if bits == 32:
        s["ms"], s["vs"] = cut(torch.randn(total, device="cuda", generator=gen) * size * 3e-4), cut((torch.randn(total, device="cuda", generator=gen) * size * 1e-3) ** 2)
    else:
        s["ms"], s["vs"] = (cut(torch.randint(0, 127, (total,), device="cuda", generator=gen, dtype=torch.uint8).view(torch.float8_e4m3fn)) for _ in range(2))
        s["scales"] = [torch.rand(2 * ((n + 255) // 256), device="cuda", generator=gen) * 1e-5 for n in sizes]
    return s


def _moments(s, i):
    """m and v of tensor i in 64 bits."""
    torch = _torch()
    if s["scales"] is None:
        return s["ms"][i].double(), s["vs"][i].double()
    n = s["ms"][i].numel()
    scale = s["scales"][i].double().view(-1, 2).repeat_interleave(256, 0)[:n]
    return s["ms"][i].to(torch.float64) * scale[:, 0], (s["vs"][i].to(torch.float64) * scale[:, 1]) ** 2


def _clone(s):
    return {k: None if x is None else [t.clone() for t in x] for k, x in s.items()}


H = dict(beta1=0.9, beta2=0.95, eps=1e-8)
SIZES = [[15_000_003], [1], [255, 1, 257], [4096, 4095, 0, 4097, 3], [64] * 120, [300_001, 12], [2_000_003]]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [b.F32, b.BF16])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "%dx%d" % (len(s), max(s)))
@pytest.mark.parametrize("shift", [0, 3])
def test_adamw(dtype, bits, sizes, shift):
    torch = _torch()
    print("adamw", dtype, bits, len(sizes), shift, flush=True)
    s = _tensors(dtype, sizes, bits, shift=shift)
    old = _clone(s)
    decay = [0.1 * (i % 3) for i in range(len(sizes))]
    factor = torch.tensor([0.4], device="cuda")
    b.AdamW(decay=decay, **H, **s).step(lr=2e-3, step=5, seed=77, grad_scale=factor)
    for i, n in enumerate(sizes):
        g = old["grads"][i].double() * float(factor)
        m0, v0 = _moments(old, i)
        m, v = 0.9 * m0 + (1 - 0.9) * g, 0.95 * v0 + (1 - 0.95) * g * g
        p0 = (old["masters"] or old["params"])[i].double()
        update = 2e-3 / (1 - 0.9 ** 5) * m / (v.sqrt() / math.sqrt(1 - 0.95 ** 5) + 1e-8)
        p = p0 * (1 - 2e-3 * decay[i]) - update
        new = (s["masters"] or s["params"])[i].double()
        # m: three roundings of terms that may cancel; v, its root, the quotient: some ten of 2^-24
        m_off = 4 * E24 * (0.9 * m0.abs() + 0.1 * g.abs())
        rel = 2e-3 / (1 - 0.9 ** 5) / (v.sqrt() / math.sqrt(1 - 0.95 ** 5) + 1e-8)
        off = rel * m_off + 12 * E24 * update.abs() + 3 * E24 * p0.abs() + E24 * p.abs()
        assert ((new - p).abs() <= off).all(), float(((new - p).abs() / off).max())
        if dtype == b.BF16:
            assert torch.equal(s["params"][i], s["masters"][i].to(torch.bfloat16))
        assert torch.equal(s["grads"][i], old["grads"][i])
        if bits == 32:
            assert ((s["ms"][i].double() - m).abs() <= m_off).all()
            assert ((s["vs"][i].double() - v).abs() <= 6 * E24 * v).all()
            continue
        got_m, got_v = _moments(s, i)
        pad = (n + 255) // 256 * 256 - n
        blocks = lambda x: torch.nn.functional.pad(x, (0, pad)).view(-1, 256)  # noqa: E731
        top = torch.stack((blocks(m.abs()).amax(1), blocks(v.sqrt()).amax(1)), 1) if n else torch.zeros((0, 2), device="cuda").double()
        top_off = 8 * E24 * top
        if n:
            top_off[:, 0] += blocks(m_off).amax(1)
        assert ((s["scales"][i].double().view(-1, 2) - top / 448).abs() <= top_off / 448 + 1e-33).all()
        for got, want, big, off in ((got_m, m, top[:, 0], m_off), (got_v.sqrt(), v.sqrt(), top[:, 1], 8 * E24 * v.sqrt())):
            # rounded to one of the two codes beside it: a step of e4m3 is 2^-3 of the power of two below, at least 2^-9 of 448ths
            unit = big.repeat_interleave(256)[:n] / 448
            step = unit * torch.exp2(torch.floor(torch.log2((want.abs() / unit).clamp(min=2.0 ** -6))) - 3)
            assert ((got - want).abs() <= step * (1 + 1e-5) + off + 8 * E24 * want.abs()).all()
        assert ((got_v > 0) == (v > 0)).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_is_a_function_of_its_arguments(bits):
    torch = _torch()
    runs = []
    for seed, step in ((1, 3), (1, 3), (2, 3), (1, 4)):
        s = _tensors(b.BF16, [5000, 333], bits)
        b.AdamW(**H, **s).step(lr=1e-3, step=step, seed=seed)
        runs.append(s)
    same = lambda x, y: all(torch.equal(a.view(torch.uint8), c.view(torch.uint8)) for a, c in zip(x["ms"] + x["vs"], y["ms"] + y["vs"]))  # noqa: E731
    assert same(runs[0], runs[1]) and torch.equal(runs[0]["masters"][0], runs[1]["masters"][0])
    if bits == 8:
        assert not same(runs[0], runs[2]) and not same(runs[0], runs[3])
    # tensors that are stepped together round as tensors of one call whose blocks are counted on: the second one alone starts at block 0
    s = _tensors(b.BF16, [5120, 333], bits)
    t = _clone(s)
    b.AdamW(**H, **s).step(lr=1e-3, step=3, seed=1)
    flat = {k: None if x is None else [torch.cat(x)] for k, x in t.items()}                   # 5120 = 20 blocks: the same numbers
    b.AdamW(**H, **flat).step(lr=1e-3, step=3, seed=1)
    assert torch.equal(flat["masters"][0], torch.cat(s["masters"])) and torch.equal(flat["ms"][0].view(torch.uint8), torch.cat(s["ms"]).view(torch.uint8))


def test_adamw_eight_bit_rounding_is_unbiased():
    # v decays by 0.999 a step while gradients are zero: rounding to nearest would never move it.  After 1000 steps sqrt(v) is
    # 0.6063 of what it was on average; a value takes random steps of 6 to 12 %, its standard deviation is below 0.4, the mean of 65536 below 0.0016
    torch = _torch()
    n = 65536
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    m = torch.zeros(n, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn)
    v = torch.full((n,), 64.0, device="cuda").to(torch.float8_e4m3fn)
    scale = torch.ones(2 * n // 256, device="cuda")
    scale[0::2] = 0
    v[::256], g[::256] = 448.0, 448.0                         # the block's largest stays, and its scale with it
    opt = b.AdamW([p], [g], [m], [v], scales=[scale], beta1=0.9, beta2=0.999)
    for step in range(1, 1001):
        opt.step(lr=0.0, step=step, seed=5)
    r = v.float() * scale.view(-1, 2)[:, 1].repeat_interleave(256)
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[::256] = False
    assert abs(float(r[keep].mean()) / 64.0 - 0.999 ** 500) <= 0.008
    assert abs(float(scale[1]) - 1) <= 1e-3
    # one step's bits: the mean of many values that lie between two codes, and both moments rounded independently
    g = torch.full((n,), 1.0, device="cuda")
    g[::256] = 3.3
    m.view(torch.uint8).zero_(), v.view(torch.uint8).zero_(), scale.zero_()
    opt = b.AdamW([p], [g], [m], [v], scales=[scale], beta1=0.0, beta2=0.5)
    opt.step(lr=0.0, step=1, seed=9)
    x, y = m.float()[keep] / (448 / 3.3), v.float()[keep] / (448 / 3.3)
    assert abs(float(x.mean()) - 1) <= 5 * 0.06 / math.sqrt(n) and abs(float(y.mean()) - 1) <= 5 * 0.06 / math.sqrt(n)
    a, c = (x > x.mean()).float(), (y > y.mean()).float()
    assert abs(float(((a - a.mean()) * (c - c.mean())).mean())) <= 5 * 0.25 / math.sqrt(n)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_left_out_and_poisoned(bits):
    torch = _torch()
    s = _tensors(b.BF16, [1000, 300], bits)
    old = _clone(s)
    for bad in (float("nan"), float("inf"), -float("inf")):
        b.AdamW(**H, **s).step(lr=1e-3, step=2, grad_scale=torch.tensor([bad], device="cuda"))
        for k in s:
            for x, y in zip(s[k] or [], old[k] or []):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), k
    # a gradient that is not a number stays in its value (in 8 bits an infinite one in its block)
    s["grads"][0][7] = float("nan")
    b.AdamW(**H, **s).step(lr=1e-3, step=2)
    assert torch.isnan(s["masters"][0][7]) and torch.isfinite(s["masters"][0][8:]).all() and torch.isfinite(s["masters"][1]).all()
    m, v = _moments(s, 0)
    assert torch.isnan(m[7]) and torch.isnan(v[7]) and torch.isfinite(m[8:]).all() and torch.isfinite(v[8:]).all()
    # tiny and huge gradients
    s = _tensors(b.F32, [512], bits)
    s["grads"][0][:256] = 1e-40
    s["grads"][0][256:] = 1e15
    if bits == 8:
        s["ms"][0].view(torch.uint8).zero_(), s["vs"][0].view(torch.uint8).zero_(), s["scales"][0].zero_()
    else:
        s["ms"][0].zero_(), s["vs"][0].zero_()
    b.AdamW(**H, **s).step(lr=1e-3, step=1)
    assert torch.isfinite(s["params"][0]).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_recorded_steps_follow_device_hyperparameters(bits):
    torch = _torch()
    import ctypes as C
    import numpy as np
    want, got = _tensors(b.BF16, [3000, 77], bits), _tensors(b.BF16, [3000, 77], bits)
    opt = b.AdamW(**H, **got)
    hyper = torch.zeros(b.ADAMW_HYPER_BYTES, dtype=torch.uint8, device="cuda")

    def tell(lr, step, seed):
        h = b.AdamWHyper(lr, 0.9, 0.95, 1e-8, step, seed)
        raw = np.frombuffer(bytes(C.string_at(C.addressof(h), C.sizeof(h))), dtype=np.uint8).copy()
        hyper[:raw.size].copy_(torch.from_numpy(raw))
    start = _clone(got)
    tell(1e-3, 1, 4)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        opt.step(lr=0, step=0, d_hyper=hyper)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            opt.step(lr=0, step=0, d_hyper=hyper)
    for k in got:
        for x, y in zip(got[k] or [], start[k] or []):
            x.copy_(y)
    ref = b.AdamW(**H, **want)
    for step in range(1, 5):
        ref.step(lr=1e-3 / step, step=step, seed=step * 10)
        tell(1e-3 / step, step, step * 10)
        graph.replay()
        torch.cuda.synchronize()
        for k in got:
            for x, y in zip(got[k] or [], want[k] or []):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), (step, k)


# ----------------------------------------------------------- together, in a stage
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [b.F32, b.BF16])
def test_stage_steps(dtype, bits):
    """Forward, loss in pieces, backward, norm, step, three times over: every step's weights against 64 bits from the gradients the library left."""
    torch = _torch()
    from paper_2107_06925_amd import synth
    from gpu_util import make_stage
    print("stage steps", dtype, bits, flush=True)
    L, hidden, seq, mb, vocab = 2, 72, 24, 3, 1003
    tokens = seq * mb
    st, _ = make_stage(L, hidden, 4, seq, mb, dtype, 0)
    t = _dtype(dtype)
    gen = torch.Generator(device="cuda").manual_seed(6)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    x, targets = rnd(tokens, hidden).to(t), torch.randint(-1, vocab, (tokens,), device="cuda", generator=gen, dtype=torch.int32)
    g, be = torch.ones(hidden, device="cuda", dtype=t), torch.zeros(hidden, device="cuda", dtype=t)
    w = torch.zeros((hidden, 1008), device="cuda", dtype=t)
    w[:, :vocab] = (0.1 * rnd(hidden, vocab)).to(t)
    dy = torch.empty((tokens, hidden), device="cuda", dtype=t)
    y, _ = st.set_io(0, x, dy)
    wm = w.float().clone()
    dg, db, dw = torch.zeros(hidden, device="cuda"), torch.zeros(hidden, device="cuda"), torch.zeros((hidden, 1008), device="cuda")
    moments = dict(ms=[torch.zeros_like(dw)], vs=[torch.zeros_like(dw)], scales=None)
    head = b.AdamW([w if dtype == b.BF16 else wm], [dw], masters=[wm] if dtype == b.BF16 else None, **moments, decay=[0.01])
    st.adamw_init(bits)
    norm, loss = torch.empty(2, device="cuda"), torch.zeros(1, device="cuda")
    params = st.grads.numel()
    sizes = [int(math.prod(s)) for _ in range(L) for s in synth.param_shapes(hidden).values()]
    matrix = torch.cat([torch.full((n,), float(len(s) == 2)) for (n, s) in zip(sizes, list(synth.param_shapes(hidden).values()) * L)]).double().cuda()
    m = v = torch.zeros(params, device="cuda", dtype=torch.float64)
    p = st.weights.double().clone()
    for step in range(1, 4):
        st.zero_grads()
        st.fwd(0)
        for a in (dg, db, dw, loss):
            a.zero_()
        b.chimera_head_loss_pieces(y, targets, g, be, (w if dtype == b.BF16 else wm.to(t))[:, :vocab], 1.0 / tokens, dy, dg, db, dw, loss, piece=256)
        with pytest.raises(b.ChimeraError) as e:
            st.adamw_step(1e-3, step)                          # a micro-batch is in flight
        assert e.value.code == b.ESTATE
        st.bwd(0)
        b.chimera_op_grad_norm([st.grads, dw], 0.05, norm)
        st.adamw_step(3e-3, step, decay=0.1, seed=3, grad_scale=norm[1:])
        head.step(3e-3, step, grad_scale=norm[1:])
        assert math.isfinite(float(loss)) and 0 < float(norm[1]) <= 1
        grad = st.grads.double() * float(norm[1])
        want = math.sqrt(float(st.grads.double().square().sum() + dw.double().square().sum()))
        assert abs(float(norm[0]) - want) <= 2 * E24 * want
        m, v = 0.9 * m + 0.1 * grad, 0.95 * v + 0.05 * grad * grad
        update = 3e-3 / (1 - 0.9 ** step) * m / ((v / (1 - 0.95 ** step)).sqrt() + 1e-8)
        p = p * (1 - 3e-3 * 0.1 * matrix) - update
        got = st.weights.double()
        if bits == 32:
            off = 1e-4 * update.abs().amax() * step + 1e-6 * p.abs() + (2.0 ** -8 * p.abs() if dtype == b.BF16 else 0)
            assert ((got - p).abs() <= off).all()
        else:
            # m and sqrt(v) to 12.5 % each a step at the worst: a quarter of an update, once a moment has been rounded (after the first step), on
            # top of what the smallest codes of a block lose; seen over all weights
            err = float((got - p).norm() / (3e-3 * math.sqrt(params)))
            assert err <= (0.01 if step == 1 else 0.3 * step) + (2.0 ** -9 * float(p.norm()) / (3e-3 * math.sqrt(params)) if dtype == b.BF16 else 0), err
        p = st.weights.double().clone() if dtype == b.F32 else p


def test_tensors_elsewhere_are_refused():
    torch = _torch()
    z = lambda *s, d=torch.float32, at="cuda": torch.zeros(s, dtype=d, device=at)  # noqa: E731
    i32 = torch.int32
    good = dict(h=z(3, 16), w=z(16, 24), targets=z(3, d=i32), scale=1.0, loss_rows=z(3), lse=z(3), loss=z(1))
    for bad in (dict(h=z(3, 16, at="cpu")), dict(w=z(16, 24, at="cpu")), dict(targets=z(3, d=i32, at="cpu")), dict(lse=z(3, at="cpu")), dict(loss=z(1, at="cpu"))):
        with pytest.raises(ValueError, match="current GPU"):
            b.chimera_op_linear_xent_fwd(**dict(good, **bad))
    with pytest.raises(ValueError, match="current GPU"):
        b.chimera_op_grad_norm([z(4), z(4, at="cpu")], 1.0, z(2))
    with pytest.raises(ValueError, match="current GPU"):
        b.AdamW([z(4)], [z(4, at="cpu")], [z(4)], [z(4)])
    step = b.AdamW([z(4)], [z(4)], [z(4)], [z(4)])
    with pytest.raises(ValueError, match="current GPU"):
        step.step(1e-3, 1, grad_scale=z(1, at="cpu"))


# ------------------------------------------------- 8-bit moments, bit for bit
def _random_bits(number, step, seed):
    """32 bits for each value, from its number in the call (CPU, integers modulo 2^32)."""
    mask = 0xFFFFFFFF
    key = (seed & mask) * 0x243F6A89 + (step & mask) * 0xB7E15163
    x = ((number & mask) * 0x9E3779B1 + (number >> 32) * 0x6A09E667 + (key & mask)) & mask
    x = ((x ^ (x >> 15)) * 0x6A09E667) & mask
    x = ((x ^ (x >> 13)) * 0xBB67AE85) & mask
    return x ^ (x >> 16)


def _codes(x, bits16, stays):
    """[blocks, 256] floats -> e4m3 codes and scales, from the formula: up or down by 16 random bits; what `stays` does not fall to zero.  Each operation rounded by itself."""
    torch = _torch()
    top = x.abs().amax(1, keepdim=True)
    some = top > 1e-30
    y = x.abs() * torch.where(some, (1.0 / top) * 448.0, torch.zeros_like(top))
    code = (((y * 2.0 ** -120).view(torch.int32) + bits16.to(torch.int32) * 16 + 8) >> 20).clamp(max=126)
    if stays:
        code = torch.where((x > 0) & some, code.clamp(min=1), code)
    code = torch.where(x < 0, code | 128, code).to(torch.uint8)
    return code, torch.where(some, top * (torch.ones(1) / 448.0), torch.zeros_like(top))


def _eight_bit_step(s, factor, step, seed):
    """Codes and scales of all tensors after a step, on the CPU."""
    torch = _torch()
    out, block = [], 0
    for i, g in enumerate(s["grads"]):
        n = g.numel()
        blocks = (n + 255) // 256
        if not n:
            out.append(None)
            continue
        pad = lambda x: torch.nn.functional.pad(x.cpu(), (0, blocks * 256 - n)).view(blocks, 256)  # noqa: E731
        scale = s["scales"][i].cpu().view(-1, 2)
        m, r = pad(s["ms"][i].float()) * scale[:, :1], pad(s["vs"][i].float()) * scale[:, 1:]
        x = pad(g) * factor
        m, v = m * H["beta1"] + x * (1.0 - H["beta1"]), (r * r) * H["beta2"] + (x * x) * (1.0 - H["beta2"])
        bits = _random_bits(torch.arange(blocks * 256) + block * 256, step, seed).view(blocks, 256)
        root = v.double().sqrt().float()              # correctly rounded (53 bits hold a float's root to twice its bits and more); torch's own float root is not, everywhere
        (cm, sm), (cv, sv) = _codes(m, bits & 0xFFFF, False), _codes(root, bits >> 16, True)
        out.append((cm.view(-1)[:n], cv.view(-1)[:n], torch.cat((sm, sv), 1).view(-1)))
        block += blocks
    return out


@pytest.mark.parametrize("sizes", [[1], [255, 1, 257], [4096, 4095, 0, 4097, 3], [64, 300, 1] * 40, [300_001, 12, 0, 70_000]], ids=lambda s: "%dx%d" % (len(s), max(s)))
@pytest.mark.parametrize("dtype", [b.F32, b.BF16])
def test_adamw_eight_bit_codes_bit_for_bit(dtype, sizes):
    torch = _torch()
    print("adamw codes", dtype, len(sizes), max(sizes), flush=True)
    s = _tensors(dtype, sizes, 8, seed=len(sizes))
    handle = b.AdamW(**H, **s)
    factor = torch.tensor([0.4])
    for step, seed in ((1, 0), (2, 77), (70_000, 2 ** 32 - 1)):
        want = _eight_bit_step(s, factor, step, seed)
        handle.step(lr=1e-3, step=step, seed=seed, grad_scale=factor.cuda())
        for i, w in enumerate(want):
            if w is not None:
                assert torch.equal(s["ms"][i].view(torch.uint8).cpu(), w[0]) and torch.equal(s["vs"][i].view(torch.uint8).cpu(), w[1]), (i, step)
                assert torch.equal(s["scales"][i].cpu(), w[2]), (i, step)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [b.F32, b.BF16])
def test_stage_steps_as_its_tensors_do(dtype, bits):
    """A stage's step and the step over the same tensors leave the same bits, master weights among them."""
    torch = _torch()
    from paper_2107_06925_amd import synth
    from gpu_util import make_stage
    print("stage as tensors", dtype, bits, flush=True)
    L, hidden, seq, mb = 2, 72, 24, 3
    st, _ = make_stage(L, hidden, 4, seq, mb, dtype, 0)
    gen = torch.Generator(device="cuda").manual_seed(6)
    x, dy = (torch.randn((seq * mb, hidden), device="cuda", generator=gen).to(_dtype(dtype)) for _ in range(2))
    st.set_io(0, x, dy)
    shapes = list(synth.param_shapes(hidden).values()) * L
    sizes = [math.prod(q) for q in shapes]
    params = [t.clone() for t in st.weights.split(sizes)]
    masters = [t.float() for t in params] if dtype == b.BF16 else None
    moment = lambda: [torch.zeros(n, device="cuda", dtype=torch.float32 if bits == 32 else torch.uint8) for n in sizes]  # noqa: E731
    scales = None if bits == 32 else [torch.zeros(2 * ((n + 255) // 256), device="cuda") for n in sizes]
    handle = b.AdamW(params, list(st.grads.split(sizes)), moment(), moment(), masters=masters, scales=scales, decay=[0.1 if len(q) == 2 else 0.0 for q in shapes])
    st.adamw_init(bits)
    norm = torch.empty(2, device="cuda")
    start = st.weights.clone()
    for step in range(1, 4):
        st.zero_grads()
        st.fwd(0)
        st.bwd(0)
        b.chimera_op_grad_norm([st.grads], 0.05, norm)
        handle.step(3e-3, step, seed=5, grad_scale=norm[1:])
        st.adamw_step(3e-3, step, decay=0.1, seed=5, grad_scale=norm[1:])
        assert torch.equal(st.weights, torch.cat(params)), step
        if masters:
            assert torch.equal(st.adamw_state[:4 * st.weights.numel()].view(torch.float32), torch.cat(masters)), step
    assert not torch.equal(st.weights, start)


def test_adamw_rounds_by_all_of_the_seed_and_the_step():
    # workers that take rank << 32 | seed must not round alike; numbers below 2^32 keep the bits of the formula above
    torch = _torch()
    seen = []
    for seed, step in ((9, 3), (1 << 32 | 9, 3), (2 << 32 | 9, 3), (9, 1 << 32 | 3), (1 << 63 | 9, 3)):
        s = _tensors(b.BF16, [5000, 333], 8)
        b.AdamW(**H, **s).step(lr=1e-3, step=step, seed=seed)
        seen.append(torch.cat([t.view(torch.uint8) for t in s["ms"] + s["vs"]]))
    for i in range(len(seen)):
        for j in range(i):
            assert float((seen[i] != seen[j]).float().mean()) > 0.2, (i, j)


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), 1e25, float("nan")])
def test_adamw_eight_bit_infinities_stay_in_their_value(bad):
    """1e25 is finite and its square is not: v alone becomes infinite.  The block's other values step as if the gradient were zero there."""
    torch = _torch()
    s, calm = _tensors(b.BF16, [600], 8, seed=2), _tensors(b.BF16, [600], 8, seed=2)
    at = 300                                                              # in the second block
    for q in (s, calm):                                                   # not its largest, whatever the gradient
        q["ms"][0].view(torch.uint8)[at] = 0
        q["vs"][0].view(torch.uint8)[at] = 8
    s["grads"][0][at], calm["grads"][0][at] = bad, 0.0
    others = torch.arange(600, device="cuda") != at
    if bad == 1e25:                                                       # its m is finite, and the block's largest
        others &= (torch.arange(600, device="cuda") < 256) | (torch.arange(600, device="cuda") >= 512)
    handles = [b.AdamW(**H, **q) for q in (s, calm)]
    for step in (1, 2):
        for h in handles:
            h.step(lr=1e-3, step=step, seed=4)
        for k in ("params", "masters", "ms", "vs"):
            x, y = (q[k][0].view(torch.uint8).view(600, -1)[others] for q in (s, calm))
            assert torch.equal(x, y), (step, k)
        m, v = _moments(s, 0)
        assert torch.isnan(v[at]) and (bad == 1e25 or torch.isnan(m[at]))
        keep = torch.arange(600, device="cuda") != at
        assert torch.isfinite(m[keep]).all() and torch.isfinite(v[keep]).all() and torch.isfinite(s["masters"][0][keep]).all()
        if bad != 1e25:
            assert torch.equal(s["scales"][0], calm["scales"][0])
        s["grads"][0][at] = 0.0                                           # once


# ------------------------------------------------------------- shared memory
@pytest.mark.parametrize("dtype", [b.F32, b.BF16])
@pytest.mark.parametrize("tokens,hidden,vocab,piece", [(150, 136, 1027, 512), (40, 64, 300, 0)])
def test_linear_xent_dh_in_the_place_of_h_and_beside_it(dtype, tokens, hidden, vocab, piece):
    torch = _torch()
    h, w, targets = _case(dtype, tokens, hidden, vocab, seed=2)
    _, lse, _ = _forward(h, w, targets, 1.0)
    dh, dw, _ = _backward(dtype, h, w, targets, lse, 0.1, piece=piece, overwrite=True)
    place = h.clone()                                                     # on h
    dw2 = torch.zeros((hidden, (vocab + 7) // 8 * 8), device="cuda")
    b.chimera_op_linear_xent_bwd(place, w, targets, lse, 0.1, place, dw2[:, :vocab], overwrite=True, piece=piece)
    assert torch.equal(place, dh) and torch.equal(dw2[:, :vocab], dw)
    both = torch.cat((h, torch.zeros_like(h)), 1)                         # rows of dh between those of h
    b.chimera_op_linear_xent_bwd(both[:, :hidden], w, targets, lse, 0.1, both[:, hidden:], dw2[:, :vocab], overwrite=True, piece=piece)
    assert torch.equal(both[:, hidden:], dh) and torch.equal(both[:, :hidden], h) and torch.equal(dw2[:, :vocab], dw)


@pytest.mark.parametrize("dtype", [b.F32, b.BF16])
@pytest.mark.parametrize("tokens,hidden", [(130, 256), (67, 1600)])
def test_head_in_pieces_dy_in_the_place_of_y(dtype, tokens, hidden):
    torch = _torch()
    vocab, t = 1001, _dtype(dtype)
    gen = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    y, g, be = rnd(tokens, hidden).to(t), (1 + 0.1 * rnd(hidden)).to(t), (0.1 * rnd(hidden)).to(t)
    w = (rnd(hidden, 1008) / math.sqrt(hidden)).to(t)
    targets = torch.randint(0, vocab, (tokens,), device="cuda", generator=gen, dtype=torch.int32)
    runs = []
    for place in (False, True):
        x = y.clone()
        dy = x if place else torch.zeros_like(y)
        rest = [torch.zeros(hidden, device="cuda"), torch.zeros(hidden, device="cuda"), torch.zeros((hidden, 1008), device="cuda"), torch.zeros(1, device="cuda")]
        b.chimera_head_loss_pieces(x, targets, g, be, w[:, :vocab], 1.0 / tokens, dy, *rest)
        runs.append([dy] + rest)
    for a, c in zip(*runs):
        assert torch.equal(a, c)


# ------------------------------------------------ logsumexps of other rows
@pytest.mark.parametrize("dtype", [b.F32, b.BF16])
def test_linear_xent_bwd_with_other_logsumexps(dtype):
    torch = _torch()
    h, w, targets = _case(dtype, 70, 64, 1001, seed=3)
    z = h.double() @ w.double()
    gen = torch.Generator(device="cuda").manual_seed(3)
    dloss = torch.rand(70, device="cuda", generator=gen) + 0.5
    # over twice as many words; much larger; as small as bf16 takes: the largest probability 3.9
    for lse in ((torch.logsumexp(z, 1) + math.log(2)).float(), (torch.logsumexp(z, 1) + 30).float(), (z.amax(1) - math.log(3.9)).float()):
        dh, dw, dw0 = _backward(dtype, h, w, targets, lse, 0.01, dloss, overwrite=True, piece=512)
        _check_backward(dtype, h, w, targets, lse, 0.01, dloss, dh, dw, torch.zeros_like(dw0))
    # smaller than that for some tokens: float follows the formula, bf16 leaves no finite number, and the other tokens' rows as they are
    less = lse.clone()
    less[::7] -= 3.0
    valid = (targets >= 0) & (targets < 1001)
    dh2, dw, dw0 = _backward(dtype, h, w, targets, less, 0.01, dloss, overwrite=True, piece=512)
    if dtype == b.F32:
        _check_backward(dtype, h, w, targets, less, 0.01, dloss, dh2, dw, torch.zeros_like(dw0))
    else:
        low = torch.zeros(70, dtype=torch.bool, device="cuda")
        low[::7] = True
        assert not torch.isfinite(dh2[low & valid]).any() and torch.equal(dh2[~low], dh[~low])


# ------------------------------------------------------ the dispatch of large calls
def _wide(tokens, hidden, vocab):
    """Columns of a bf16 forward on 256x256 tiles, from its workspace: a (maximum, sum) pair for each token and tile column, and a float a token."""
    need = b.lib().chimera_op_linear_xent_fwd_workspace_bytes(b.BF16, tokens, hidden, vocab)
    columns = (need - (4 * tokens + 255) // 256 * 256) // (8 * tokens)
    return 256 * ((vocab + 127) // 128 - columns)                         # each 256 wide tile is one column fewer


# whole rounds of 256x256 tiles and 128x128 ones behind them: a few of those and many, one round and several, in bands where W (164 MB) does not stay in the
# memory-side cache, rows that end inside a tile; and 256x256 tiles alone, several rounds of them
@pytest.mark.parametrize("tokens,hidden,vocab,ldw,mixed", [(400, 512, 33001, 33008, True), (300, 256, 33001, 33064, True), (2048, 72, 50257, 50264, True),
                                                           (1100, 192, 20001, 20008, True), (700, 320, 45001, 45008, True), (2100, 2048, 40001, 40008, True), (2048, 256, 32765, 32768, False)])
def test_linear_xent_fwd_of_two_tile_sizes(tokens, hidden, vocab, ldw, mixed):
    _torch()
    print("linear xent fwd, large", tokens, hidden, vocab, ldw, flush=True)
    wide = _wide(tokens, hidden, vocab)
    assert (0 < wide < vocab) if mixed else wide >= vocab
    h, w, targets = _case(b.BF16, tokens, hidden, vocab, ldw, hidden + 8, seed=tokens + vocab)
    ends = [0, 255, 256, vocab - 1] + ([wide - 1, wide, wide + 127, wide + 128] if mixed else [])       # words beside the seams
    for i, word in enumerate(ends):
        targets[i], targets[tokens - 1 - i] = min(word, vocab - 1), min(word, vocab - 1)
    rows, lse, loss = _forward(h, w, targets, 0.25)
    _check_forward(b.BF16, h, w, targets, 0.25, rows, lse, loss)


# bf16, dW in 256x256 tiles (from 128 of them on) over an undivided contraction, straight into the caller's matrix: rows of tokens beside them of 256 (more
# than 128 tokens) or of 128; several pieces, the last one of a few columns, several rounds of tiles
BWD_LARGE = [(300, 2048, 20001, 20008, 0), (300, 1024, 20003, 20016, 9984), (130, 1600, 21001, 21008, 20992), (1500, 1600, 12007, 12008, 0),
             (100, 2048, 32001, 32008, 0), (16, 1024, 50257, 50264, 0), (1, 1600, 50257, 50304, 0), (128, 2048, 20485, 20488, 10240)]


@pytest.mark.parametrize("tokens,hidden,vocab,ldw,piece", BWD_LARGE)
def test_linear_xent_bwd_large(tokens, hidden, vocab, ldw, piece):
    test_linear_xent_bwd(b.BF16, tokens, hidden, vocab, ldw, piece)


@pytest.mark.parametrize("dtype", [b.F32, b.BF16])
@pytest.mark.parametrize("tokens,hidden,vocab,ldw,piece", [(700, 512, 20001, 20008, 0), (2100, 256, 5003, 5008, 1024), (160, 2048, 16400, 16400, 0)])
def test_head_in_pieces_large(dtype, tokens, hidden, vocab, ldw, piece):
    """Several tiles of every product, against 64 bits through autograd.  Logits of deviation 1, whose rounded operands move dy and dW by less than the
    rounding of h and of dh to the type, half of the bar each; a quarter of the tokens does not count."""
    torch = _torch()
    print("head pieces, large", dtype, tokens, hidden, vocab, flush=True)
    t = _dtype(dtype)
    gen = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    y, g, be = rnd(tokens, hidden).to(t), (1 + 0.1 * rnd(hidden)).to(t), (0.1 * rnd(hidden)).to(t)
    w = torch.full((hidden, ldw), float("nan"), device="cuda", dtype=t)
    w[:, :vocab] = (rnd(hidden, vocab) / math.sqrt(hidden)).to(t)
    targets = torch.randint(0, vocab, (tokens,), device="cuda", generator=gen, dtype=torch.int32)
    targets[::4] = -1
    got = [torch.full((tokens, hidden), 9.0, device="cuda", dtype=t), torch.full((hidden,), 0.5, device="cuda"), torch.full((hidden,), -0.5, device="cuda"),
           torch.full((hidden, ldw), 0.25, device="cuda"), torch.full((1,), 2.0, device="cuda")]
    b.chimera_head_loss_pieces(y, targets, g, be, w[:, :vocab], 1.0 / tokens, *got, piece=piece)
    p = [x.double().requires_grad_() for x in (y, g, be, w[:, :vocab])]
    h = torch.nn.functional.layer_norm(p[0], (hidden,), p[1], p[2], 1e-5)
    loss = torch.nn.functional.cross_entropy(h @ p[3], targets.long(), ignore_index=-1, reduction="sum") / tokens
    loss.backward()
    tol = 2e-2 if dtype == b.BF16 else 1e-4
    for name, a, q in zip(("dy", "dg", "db", "dw"), [got[0].double(), got[1].double() - 0.5, got[2].double() + 0.5, got[3][:, :vocab].double() - 0.25], [x.grad for x in p]):
        err = float((a - q).abs().max() / q.abs().max())
        assert err <= tol, (name, err)
    assert (got[3][:, vocab:] == 0.25).all() and (got[0][::4] == 0).all()
    assert abs(float(got[4]) - 2.0 - float(loss.detach())) <= tol * float(loss.detach())


@pytest.mark.parametrize("dtype,piece", [(b.F32, 0), (b.BF16, 0), (b.BF16, 65536)])
def test_linear_xent_beyond_2_31_logits(dtype, piece):
    """40000 x 65536: rows and columns at both ends and on both sides of the 2^31st logit, against 64 bits."""
    torch = _torch()
    print("linear xent, 2.6e9 logits", dtype, piece, flush=True)
    tokens, hidden, vocab, scale = 40000, 64, 65536, 0.01
    h, w, targets = _case(dtype, tokens, hidden, vocab, seed=1)
    few = torch.cat([torch.arange(a, a + 12) for a in (0, 16378, 32762, 39988)]).cuda()
    targets[few[::3]] = (few[::3] * 331 % vocab).to(torch.int32)
    rows, lse, loss = _forward(h, w, targets, scale)
    _check_forward(dtype, h[few], w, targets[few], scale, rows[few], lse[few], float(rows[few].double().sum()) + 0.5)
    total = float(rows.double().sum()) + 0.5
    assert abs(float(loss) - total) <= (tokens + 8) * E24 * (float(rows.double().abs().sum()) + 0.5)
    dh, dw, _ = _backward(dtype, h, w, targets, lse, scale, overwrite=True, piece=piece)
    _check_backward(dtype, h[few], w, targets[few], lse[few], scale, None, dh[few], None, None)
    cols = torch.cat([torch.arange(0, 8).cuda(), targets[few[::3]].long(), torch.arange(vocab - 8, vocab).cuda(), torch.arange(32764, 32772).cuda()])
    wc = w[:, cols]
    z, off = _logits(h, wc, dtype)
    x = z - lse.double()[:, None]
    p = x.exp()
    p_off = p * (off + 3 * E24 * (x.abs() + z.abs()) + E22) + E23 * (p + 1)
    valid = ((targets >= 0) & (targets < vocab)).double()
    dz = scale * valid[:, None] * (p - (targets.long()[:, None] == cols[None, :]).double())
    dz_off = scale * valid[:, None] * p_off + 2 * E24 * dz.abs()
    hd = h.double()
    want, mag = hd.t() @ dz, hd.abs().t() @ dz.abs()
    top = scale * float(hd.abs().max())
    tol = hd.abs().t() @ dz_off + (E22 + (2 * tokens + 80) * E24) * mag + tokens * 2.0 ** -36 * top + E24 * want.abs() + 1e-38
    assert ((dw[:, cols].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", [b.F32, b.BF16])
@pytest.mark.parametrize("tokens,hidden,first,vocab,piece", [(40, 64, 4, 1012, 256), (33, 72, 12, 1001, 0), (130, 136, 8, 1008, 512), (9, 16, 4, 3, 0)])
def test_linear_xent_of_the_last_columns_of_a_matrix(dtype, tokens, hidden, first, vocab, piece):
    """W and dW as the columns behind `first` of wider matrices: nothing behind the last row is there, nor asked for."""
    torch = _torch()
    first = first if dtype == b.F32 else (first + 7) // 8 * 8                 # 16 bytes
    wide = (first + vocab + 7) // 8 * 8
    print("linear xent, last columns", dtype, tokens, hidden, first, vocab, wide, flush=True)
    h, w, targets = _case(dtype, tokens, hidden, vocab, seed=7)
    full = torch.full((hidden, wide), float("nan"), device="cuda", dtype=_dtype(dtype))
    full[:, first:first + vocab] = w
    part = full[:, first:first + vocab]
    rows, lse, loss = _forward(h, part, targets, 0.25)
    _check_forward(dtype, h, w, targets, 0.25, rows, lse, loss)
    dfull = torch.full((hidden, wide), 0.5, device="cuda")
    dpart, dh = dfull[:, first:first + vocab], torch.zeros_like(h)
    for overwrite in (True, False):
        b.chimera_op_linear_xent_bwd(h, part, targets, lse, 0.25, dh, dpart, overwrite=overwrite, piece=piece)
        _check_backward(dtype, h, w, targets, lse, 0.25, None, dh, dpart, torch.zeros_like(dpart) if overwrite else before)
        before = dpart.clone()
    assert (dfull[:, :first] == 0.5).all() and (dfull[:, first + vocab:] == 0.5).all()


# ------------------------------------------------ beyond 2^31 values in a tensor
def test_grad_norm_beyond_2_31_values():
    torch = _torch()
    n = 2 ** 31 + 4099
    print("grad norm", n, flush=True)
    g = torch.zeros(n, device="cuda")
    at = torch.tensor([0, 2 ** 30, 2 ** 31 - 1, 2 ** 31, 2 ** 31 + 1, n - 1], device="cuda")
    g[at] = torch.tensor([1.0, 2.0, 4.0, 8.0, 16.0, 32.0], device="cuda")
    out = torch.empty(2, device="cuda")
    b.chimera_op_grad_norm([g, g[n - 1:]], 1e9, out)
    assert abs(float(out[0]) - math.sqrt(1365 + 1024)) <= 2 * E24 * float(out[0]) and float(out[1]) == 1.0


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_beyond_2_31_values(bits):
    """Windows at both ends and across the 2^31st value: the weights are those of a step over the window alone, codes those of the formula."""
    torch = _torch()
    n = 2 ** 31 + 70_003
    print("adamw", bits, n, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(5)
    long = lambda d=torch.float32, m=n: torch.zeros(m, device="cuda", dtype=d)  # noqa: E731
    p, g, small = long(), long(), torch.float32 if bits == 32 else torch.uint8
    m, v, scale = long(small), long(small), None if bits == 32 else long(m=2 * ((n + 255) // 256))
    windows = [(0, 5000), (2 ** 31 - 2560, 2 ** 31 + 2560), (n // 256 * 256 - 2560, n)]
    for a, z in windows:
        p[a:z], g[a:z] = torch.randn(z - a, device="cuda", generator=gen), torch.randn(z - a, device="cuda", generator=gen)
    parts = [dict(params=[p[a:z].clone()], grads=[g[a:z]], ms=[torch.zeros(z - a, device="cuda", dtype=small)], vs=[torch.zeros(z - a, device="cuda", dtype=small)],
                  scales=None if bits == 32 else [torch.zeros(2 * ((z - a + 255) // 256), device="cuda")]) for a, z in windows]
    b.AdamW([p], [g], [m], [v], scales=None if bits == 32 else [scale], decay=[0.1], **H).step(lr=1e-2, step=1, seed=3)
    for (a, z), q in zip(windows, parts):
        b.AdamW(decay=[0.1], **q, **H).step(lr=1e-2, step=1, seed=3)
        assert torch.equal(p[a:z], q["params"][0]), a
        if bits == 32:
            assert torch.equal(m[a:z], q["ms"][0]) and torch.equal(v[a:z], q["vs"][0]), a
            continue
        assert torch.equal(scale[a // 256 * 2:(z + 255) // 256 * 2][:q["scales"][0].numel() - 2], q["scales"][0][:-2]), a
        blocks = (z - a) // 256                                           # (windows begin at a block; a last one that is not whole is left out)
        x = g[a:a + blocks * 256].cpu().view(blocks, 256)
        r = _random_bits(torch.arange(blocks * 256) + a, 1, 3).view(blocks, 256)
        cm, _ = _codes(x * (1.0 - H["beta1"]), r & 0xFFFF, False)
        cv, _ = _codes(((x * x) * (1.0 - H["beta2"])).double().sqrt().float(), r >> 16, True)
        assert torch.equal(m[a:a + blocks * 256].cpu(), cm.view(-1)) and torch.equal(v[a:a + blocks * 256].cpu(), cv.view(-1)), a
    assert not p[6000:2 ** 31 - 3000].any() and not m[6000:2 ** 31 - 3000].any()
