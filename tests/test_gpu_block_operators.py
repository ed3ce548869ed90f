"""GPU parity of rotary positions, attention over packed sequences and the norms around a branch against plain 64-bit arithmetic (torch float64).

Tolerances are per element and count roundings: half a step of a float is 2^-24 of the value, of bf16 2^-8; a sum of K floats, in any order, is off by at most
K 2^-24 of the sum of magnitudes; the hardware's exp2 by 2^-22 relative, its argument, rounded, by 2^-23 |x| more."""
import math

import pytest

from paper_2107_06925_amd import binding as b

from gpu_util import TOL, rel_err

pytestmark = pytest.mark.gpu

E24, E23, E22 = 2.0 ** -24, 2.0 ** -23, 2.0 ** -22
HALF = {b.F32: 2.0 ** -24, b.BF16: 2.0 ** -8}           # half a step of a result, relative


def _torch():
    import torch
    return torch


def _type(dtype):
    torch = _torch()
    return torch.float32 if dtype == b.F32 else torch.bfloat16


def _gen(seed):
    return _torch().Generator(device="cuda").manual_seed(seed)


def _randn(gen, *shape):
    return _torch().randn(shape, device="cuda", generator=gen)


def _within(got, want, tol, what):
    torch = _torch()
    off = (got.double() - want).abs()
    assert torch.isfinite(got.float()).all(), what + ": not finite"
    assert (off <= tol).all(), "%s: %.3g of the tolerance" % (what, float((off / tol.clamp(min=1e-300)).max()))


def _gapped(gen, dtype, rows, heads, dim, gap, fill=float("nan")):
    """[rows, heads, dim] whose rows lie heads * dim + gap apart, `fill` between them."""
    torch = _torch()
    whole = torch.full((rows, heads * dim + gap), fill, device="cuda", dtype=_type(dtype))
    view = whole[:, :heads * dim].unflatten(1, (heads, dim))
    view.copy_(_randn(gen, rows, heads, dim))
    return whole, view


# -------------------------------------------------------------------------- rotary
def _turned(x, theta, magnitude, layout, transpose):
    """In 64 bits, and how far a float computation may be off: angles by 2^-50 of themselves and 2^-23, four roundings and sine and cosine to two steps."""
    torch = _torch()
    rot = 2 * theta.shape[1]
    y, tol = x.double().clone(), torch.zeros(x.shape, device="cuda", dtype=torch.float64)
    at = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == b.ROTARY_HALF else (slice(0, rot, 2), slice(1, rot, 2))
    p, q = x.double()[..., at[0]], x.double()[..., at[1]]
    c, s = torch.cos(theta)[:, None], torch.sin(theta)[:, None] * (-1 if transpose else 1)
    y[..., at[0]], y[..., at[1]] = magnitude * (p * c - q * s), magnitude * (p * s + q * c)
    e = abs(magnitude) * (p.abs() + q.abs()) * (theta.abs()[:, None] * 2.0 ** -50 + E23 + 8 * E24)
    tol[..., at[0]], tol[..., at[1]] = e, e
    return y, tol


@pytest.mark.parametrize("dtype", [b.F32, b.BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("layout", [b.ROTARY_HALF, b.ROTARY_INTERLEAVED], ids=["half", "interleaved"])
@pytest.mark.parametrize("tokens,heads,dim,rot,gap", [(1, 1, 2, 2, 0), (1, 4, 64, 64, 0), (3, 5, 64, 50, 7), (33, 18, 128, 128, 256), (130, 3, 80, 22, 0), (7, 40, 256, 256, 0), (65, 2, 9, 6, 3),
                                                      (1025, 6, 32, 16, 64), (515, 1, 8, 8, 0), (2, 4096, 16, 8, 0)])
def test_rotary(dtype, layout, tokens, heads, dim, rot, gap):
    torch = _torch()
    gen = _gen(tokens * 7 + rot)
    whole, x = _gapped(gen, dtype, tokens, heads, dim, gap)
    positions = torch.randint(0, 2 ** 31 - 1, (tokens,), device="cuda", generator=gen, dtype=torch.int32)
    positions[tokens // 2:] %= 4096
    positions[0] = 0
    freq = b.chimera_rotary_frequencies(rot, 10000.0).cuda()
    for transpose, magnitude, where in ((False, 1.0, positions), (True, 1.25, positions), (False, -0.5, None)):
        theta = (torch.arange(tokens, device="cuda") if where is None else where).double()[:, None] * freq
        want, tol = _turned(x, theta, magnitude, layout, transpose)
        tol = torch.where(tol > 0, tol + HALF[dtype] * want.abs(), tol)
        out, y = _gapped(gen, dtype, tokens, heads, dim, gap + 5, fill=3.0)
        b.chimera_op_rotary(x, y, freq, positions=where, layout=layout, magnitude=magnitude, transpose=transpose)
        _within(y, want, tol, "y")                                       # (columns from rot on: equal)
        assert (out[:, heads * dim:] == 3.0).all()
        kept = whole.clone()
        view = kept[:, :heads * dim].unflatten(1, (heads, dim))
        b.chimera_op_rotary(view, view, freq, positions=where, layout=layout, magnitude=magnitude, transpose=transpose)
        assert torch.equal(view, y) and kept[:, heads * dim:].isnan().all()


def test_rotary_leaves_masked_columns_and_rows_alone():
    """A number that is not finite stays in its pair."""
    torch = _torch()
    x = torch.ones((4, 2, 64), device="cuda")
    x[1, 0, 3], x[2, 1, 40], x[3, 0, 63] = float("nan"), float("inf"), -float("inf")
    y = torch.empty_like(x)
    b.chimera_op_rotary(x, y, b.chimera_rotary_frequencies(32).cuda())
    bad = ~torch.isfinite(y)
    assert bad.sum() == 4 and bad[1, 0, [3, 19]].all() and bad[2, 1, 40] and bad[3, 0, 63]


def test_rotary_offsets_beyond_32_bits():
    torch = _torch()
    tokens, ld = 40000, 65536
    whole = torch.empty(tokens * ld, device="cuda", dtype=torch.bfloat16)
    x = whole.as_strided((tokens, 2, 64), (ld, 64, 1), 0)
    x.copy_(_randn(_gen(3), tokens, 2, 64))
    y = torch.empty((tokens, 2, 64), device="cuda", dtype=torch.bfloat16)
    freq = b.chimera_rotary_frequencies(64).cuda()
    b.chimera_op_rotary(x, y, freq)
    want, tol = _turned(x, torch.arange(tokens, device="cuda").double()[:, None] * freq, 1.0, b.ROTARY_HALF, False)
    _within(y, want, tol + HALF[b.BF16] * want.abs(), "y")


# ----------------------------------------------------------------------- attention
class Packed:
    """Operands of attention over packed sequences as views of rows that hold more (NaN), rows of other owners before and behind the sequences (NaN)."""

    def __init__(self, dtype, lengths, heads, kv_heads, dim, causal=True, before=0, tail=0, gap=0, seed=0, gain=1.5, scale=None):
        torch = _torch()
        self.dtype, self.causal, self.heads, self.kv, self.dim, self.lengths = dtype, causal, heads, kv_heads, dim, lengths
        self.scale = dim ** -0.5 if scale is None else scale
        n = before + sum(lengths) + tail
        gen = _gen(seed)
        unit = 8
        self.rows = torch.full((n, (heads + 2 * kv_heads) * dim + unit * gap), float("nan"), device="cuda", dtype=_type(dtype))
        cut = lambda w, i, m: w[:, i * dim:(i + m) * dim].unflatten(1, (m, dim))  # noqa: E731
        self.q, self.k, self.v = cut(self.rows, 0, heads), cut(self.rows, heads, kv_heads), cut(self.rows, heads + kv_heads, kv_heads)
        self.dctx = torch.full((n, heads, dim), float("nan"), device="cuda", dtype=_type(dtype))
        live = slice(before, before + sum(lengths))
        self.q[live] = (gain * _randn(gen, sum(lengths), heads, dim)).to(_type(dtype))
        self.k[live] = _randn(gen, sum(lengths), kv_heads, dim).to(_type(dtype))
        self.v[live] = _randn(gen, sum(lengths), kv_heads, dim).to(_type(dtype))
        self.dctx[live] = _randn(gen, sum(lengths), heads, dim).to(_type(dtype))
        self.ends = [before]
        for m in lengths:
            self.ends.append(self.ends[-1] + m)
        self.offsets = torch.tensor(self.ends, dtype=torch.int32, device="cuda")
        self.live = live
        self.results()

    def results(self):
        torch = _torch()
        n, t = self.rows.shape[0], _type(self.dtype)
        self.ctx = torch.full((n, self.heads, self.dim), 7.0, device="cuda", dtype=t)
        self.lse = torch.full((self.heads, n), 7.0, device="cuda")
        self.drows = torch.full_like(self.rows, 7.0)
        cut = lambda i, m: self.drows[:, i * self.dim:(i + m) * self.dim].unflatten(1, (m, self.dim))  # noqa: E731
        self.dq, self.dk, self.dv = cut(0, self.heads), cut(self.heads, self.kv), cut(self.heads + self.kv, self.kv)

    def forward(self):
        b.chimera_op_attention_packed_fwd(self.q, self.k, self.v, self.offsets, self.ctx, self.lse, causal=self.causal, scale=self.scale)

    def backward(self, workspace=None):
        return b.chimera_op_attention_packed_bwd(self.q, self.k, self.v, self.offsets, self.ctx, self.lse, self.dctx, self.dq, self.dk, self.dv, causal=self.causal,
                                                 scale=self.scale, workspace=workspace)

    def untouched(self):
        """Rows without an owner, and what lies between a row's end and the next row, as they were."""
        for x in (self.ctx, self.drows):
            assert (x[:self.live.start] == 7.0).all() and (x[self.live.stop:] == 7.0).all()
        assert (self.lse[:, :self.live.start] == 7.0).all() and (self.lse[:, self.live.stop:] == 7.0).all()
        assert (self.drows[:, (self.heads + 2 * self.kv) * self.dim:] == 7.0).all()

    def _scores(self, lo, hi, h):
        """q, k, v of a head, its scores, and how far float scores may be off, per row."""
        torch = _torch()
        q, k, v = self.q[lo:hi, h].double(), self.k[lo:hi, h * self.kv // self.heads].double(), self.v[lo:hi, h * self.kv // self.heads].double()
        z = q @ k.t() * self.scale
        off = (q.abs() @ k.t().abs() * (self.scale * (self.dim + 3) * E24))
        if self.causal:
            hidden = torch.ones_like(z).triu(1).bool()
            z, off = z.masked_fill(hidden, -math.inf), off.masked_fill(hidden, 0.0)
        return q, k, v, z, off.amax(1, keepdim=True)

    def check_forward(self, some=None):
        torch = _torch()
        p_half = 0.0 if self.dtype == b.F32 else HALF[b.BF16]                 # probabilities are rounded to bf16 before their product with v
        for lo, hi in list(zip(self.ends, self.ends[1:]))[:some]:
            if lo == hi:
                continue
            for h in range(self.heads):
                q, k, v, z, off = self._scores(lo, hi, h)
                lse = torch.logsumexp(z, 1, keepdim=True)
                p = torch.exp(z - lse)
                want = p @ v
                # arguments of exp2 up to |z| + |max| (scaled by log2 e) are rounded; sums over hi - lo keys; rescaling once a tile of 32 or 64 keys at most
                span = (z.masked_fill(z == -math.inf, 0.0).abs().amax(1, keepdim=True) + lse.abs()) * 1.5
                rel = 2 * off + 2 * span * E23 + 4 * E22 + (hi - lo) * (1 / 32 + 1) * E24 * 2
                _within(self.ctx[lo:hi, h], want, (rel + p_half) * 1.01 * (p @ v.abs()) + HALF[self.dtype] * want.abs() + 1e-30, "ctx of head %d, rows %d to %d" % (h, lo, hi))
                _within(self.lse[h, lo:hi], lse[:, 0], (off + span * E23 + 4 * E22 + (hi - lo) * E24 * 2 + 4 * E24 * (1 + lse.abs()))[:, 0], "lse")

    def check_backward(self, some=None):
        """From ctx and lse as they are."""
        torch = _torch()
        half = 0.0 if self.dtype == b.F32 else HALF[b.BF16]
        t = lambda x: x.t().contiguous()  # noqa: E731
        for lo, hi in list(zip(self.ends, self.ends[1:]))[:some]:
            if lo == hi:
                continue
            n = hi - lo
            for g in range(self.kv):
                group = self.heads // self.kv
                dk, dv, dk_tol, dv_tol = (torch.zeros((n, self.dim), device="cuda", dtype=torch.float64) for _ in range(4))
                for h in range(g * group, (g + 1) * group):
                    q, k, v, z, off = self._scores(lo, hi, h)
                    lse, o, do = self.lse[h, lo:hi].double()[:, None], self.ctx[lo:hi, h].double(), self.dctx[lo:hi, h].double()
                    p = torch.exp(z - lse)
                    span = (z.masked_fill(z == -math.inf, 0.0).abs().amax(1, keepdim=True) + lse.abs()) * 1.5
                    p_off = p * (off + 2 * span * E23 + 4 * E22)
                    dp, delta = do @ t(v), (do * o).sum(1, keepdim=True)
                    d_off = (self.dim + 4) * E24 * (do.abs() @ t(v.abs()) + (do * o).abs().sum(1, keepdim=True))
                    ds = p * (dp - delta)
                    ds_off = p_off * (dp - delta).abs() + p * d_off + ds.abs() * (half + 2 * E24)
                    more = (n * group + 8) * E24
                    dq = self.scale * (ds @ k)
                    tol = self.scale * (1.01 * ds_off + more * ds.abs()) @ k.abs()
                    _within(self.dq[lo:hi, h], dq, tol + HALF[self.dtype] * dq.abs() + 1e-30, "dq of head %d, rows %d to %d" % (h, lo, hi))
                    dk += self.scale * (t(ds) @ q)
                    dk_tol += self.scale * (t(1.01 * ds_off + more * ds.abs()) @ q.abs())
                    dv += t(p) @ do
                    dv_tol += t(1.01 * p_off + p * (1.01 * half + more)) @ do.abs()
                _within(self.dk[lo:hi, g], dk, dk_tol + HALF[self.dtype] * dk.abs() + 1e-30, "dk of head %d, rows %d to %d" % (g, lo, hi))
                _within(self.dv[lo:hi, g], dv, dv_tol + HALF[self.dtype] * dv.abs() + 1e-30, "dv of head %d, rows %d to %d" % (g, lo, hi))


SHORT = [0, 5, 0, 1, 64, 65, 0, 33]
EDGES = [127, 128, 129, 32, 31]
MANY = [(i * 37) % 23 for i in range(150)]                       # more sequences than a wavefront has lanes, some empty
BF16_CASES = [([1], 1, 1, 8), ([1, 1, 1], 4, 4, 64), (SHORT, 6, 2, 64), (EDGES, 5, 1, 128), ([300], 8, 8, 40), (MANY, 3, 3, 64), ([0, 0, 0], 2, 1, 64), ([700, 3, 130], 16, 2, 72),
              ([257, 511], 25, 5, 64), ([200, 90], 8, 4, 120), ([1030], 2, 1, 128), ([1040], 3, 1, 64), ([1200, 1000], 9, 3, 64)]
F32_CASES = [([1], 1, 1, 4), (SHORT, 6, 2, 64), (EDGES, 5, 1, 128), ([300], 8, 8, 36), (MANY, 3, 3, 32), ([0, 0], 2, 1, 64), ([257, 40], 16, 2, 12), ([130, 90], 8, 4, 100)]


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "full"])
@pytest.mark.parametrize("dtype,lengths,heads,kv_heads,dim", [(b.BF16, *c) for c in BF16_CASES] + [(b.F32, *c) for c in F32_CASES],
                         ids=lambda v: "%d+%d" % (len(v), sum(v)) if isinstance(v, list) else str(v))
def test_attention_packed(dtype, lengths, heads, kv_heads, dim, causal):
    torch = _torch()
    a = Packed(dtype, lengths, heads, kv_heads, dim, causal, before=3, tail=5, gap=1, seed=sum(lengths) + dim)
    a.forward()
    torch.cuda.synchronize()
    a.check_forward()
    a.backward()
    torch.cuda.synchronize()
    a.check_backward()
    a.untouched()
    first = [x.clone() for x in (a.ctx, a.lse, a.drows)]
    a.results()
    a.forward()
    a.backward()
    for x, y in zip(first, (a.ctx, a.lse, a.drows)):
        assert torch.equal(x, y), "a second run differs"


# heads of a group in one, two and four parts of several: 16 x 38, 16 x 19 and 8 x 17 tiles of 128 keys
@pytest.mark.parametrize("heads,kv_heads,tiles", [(32, 16, 38), (64, 16, 19), (64, 8, 17)])
def test_attention_packed_groups_in_parts(heads, kv_heads, tiles):
    a = Packed(b.BF16, [60, 200, 128] * (tiles // 3) + [tiles * 128 - 388 * (tiles // 3)], heads, kv_heads, 8, seed=tiles)
    a.forward()
    a.backward()
    a.check_forward(some=2)
    a.check_backward(some=2)
    a.ends = a.ends[-2:]                         # the longest, and last
    a.check_forward()
    a.check_backward()
    a.untouched()


@pytest.mark.parametrize("dtype", [b.F32, b.BF16], ids=["f32", "bf16"])
def test_attention_packed_extreme_scores(dtype):
    """One key takes all of a row, scores of some hundreds, and a scale of the caller's."""
    a = Packed(dtype, [200, 70], 4, 2, 64, gain=60.0, seed=5, scale=0.3)
    a.forward()
    a.check_forward()
    a.backward()
    a.check_backward()


@pytest.mark.parametrize("dtype,lengths,kv_heads", [(b.F32, [200, 70], 2), (b.BF16, [200, 70], 2), (b.F32, [2100], 8)], ids=["f32", "bf16", "f32-large"])
def test_attention_packed_masks_hold_at_any_scale(dtype, lengths, kv_heads):
    """At the smallest scale every visible key has the same probability, and a masked one none."""
    torch = _torch()
    a = Packed(dtype, lengths, 8, kv_heads, 64, seed=6, scale=2.0 ** -100)
    a.forward()
    a.check_forward()
    n = torch.cat([torch.arange(1, m + 1) for m in lengths]).cuda().double()
    assert ((a.lse.double() - n.log()).abs() <= 4 * E22 + 2100 * E24).all()
    a.backward()
    a.check_backward()


@pytest.mark.parametrize("dtype", [b.F32, b.BF16], ids=["f32", "bf16"])
def test_attention_packed_queries_that_see_one_key(dtype):
    """Their probability is 1 whatever the score is: no gradient reaches q or k."""
    a = Packed(dtype, [1] * 40 + [0] + [1] * 60, 4, 2, 64, causal=False, seed=7)
    a.forward()
    a.backward()
    assert (a.dq == 0).all() and (a.dk == 0).all()
    a.check_backward()
    a = Packed(dtype, [30, 90], 4, 2, 64, seed=7)
    a.forward()
    a.backward()
    assert (a.dq[0] == 0).all() and (a.dq[30] == 0).all() and (a.dq[1] != 0).any()


@pytest.mark.parametrize("dtype", [b.F32, b.BF16], ids=["f32", "bf16"])
def test_attention_packed_thousands_of_sequences(dtype):
    a = Packed(dtype, [i % 3 for i in range(4000)], 2, 1, 32, causal=True, seed=10)
    a.forward()
    a.backward()
    a.ends = a.ends[:20] + a.ends[-20:]
    a.check_forward(some=19)
    a.check_backward(some=19)
    a.ends = a.ends[-20:]
    a.check_forward()
    a.check_backward()
    a.untouched()


@pytest.mark.parametrize("dtype", [b.F32, b.BF16], ids=["f32", "bf16"])
def test_attention_packed_sequences_do_not_see_each_other(dtype):
    torch = _torch()
    a = Packed(dtype, [100, 130, 77], 6, 3, 64, seed=8)
    a.forward()
    a.backward()
    want = [x.clone() for x in (a.ctx, a.lse, a.drows)]
    lo, hi = a.ends[1:3]
    for value in (float("nan"), float("inf")):
        a.rows[lo:hi], a.dctx[lo:hi] = value, value
        a.results()
        a.forward()
        a.backward()
        keep = torch.ones(a.rows.shape[0], dtype=torch.bool, device="cuda")
        keep[lo:hi] = False
        assert torch.equal(a.ctx[keep], want[0][keep]) and torch.equal(a.lse[:, keep], want[1][:, keep]) and torch.equal(a.drows[keep], want[2][keep])


def test_attention_packed_offsets_out_of_order_stay_in_bounds():
    """The result means nothing; rows outside the tensors are not touched (the host checks it on the tensors' neighbours) and the next call is right."""
    torch = _torch()
    a = Packed(b.BF16, [100, 130, 77], 4, 2, 64, tail=200, seed=9)
    a.rows.nan_to_num_(0.0)
    a.dctx.nan_to_num_(0.0)
    right = a.offsets.clone()
    for wrong in ([-5, 100, 50, 10 ** 9], [300, 200, 100, 0], [-2 ** 31, -1, 2 ** 31 - 1, 2 ** 31 - 1], [507, 600, 700, 800]):
        a.offsets.copy_(torch.tensor(wrong, dtype=torch.int64).to(torch.int32))
        a.forward()
        a.backward()
    torch.cuda.synchronize()
    a.offsets.copy_(right)
    a.results()
    a.forward()
    a.backward()
    a.check_forward()
    a.check_backward()


def test_attention_packed_with_equal_lengths_is_attention():
    """Beside the operator over equal sequences, on its layout: one head a group, rows of q, k and v side by side."""
    torch = _torch()
    for dtype in (b.F32, b.BF16):
        batch, seq, heads, dim = 3, 160, 4, 64
        a = Packed(dtype, [seq] * batch, heads, heads, dim, seed=11)
        a.forward()
        ctx, lse = torch.empty_like(a.ctx).view(batch * seq, -1), torch.empty((batch, heads, seq), device="cuda")
        b.chimera_op_attention_fwd(a.rows, ctx, lse, batch, seq, heads, dim, True)
        assert rel_err(a.ctx.view(batch * seq, -1).float().cpu(), ctx.float().cpu()) <= TOL[dtype]
        assert rel_err(a.lse.view(heads, batch, seq).transpose(0, 1).cpu(), lse.cpu()) <= 1e-5


@pytest.mark.parametrize("dtype", [b.F32, b.BF16], ids=["f32", "bf16"])
def test_attention_packed_keys_that_are_values(dtype):
    a = Packed(dtype, [150, 40], 4, 2, 64, seed=14)
    a.v = a.k
    a.forward()
    a.backward()
    a.check_forward()
    a.check_backward()


def test_two_calls_at_once():
    """On two streams, with workspaces of their own, beside each other and again."""
    torch = _torch()
    calls = [Packed(b.BF16, [500, 300], 8, 2, 64, seed=15), Packed(b.F32, [400, 111], 4, 1, 64, seed=16)]
    joins = [Join(b.BF16, b.F32, 900, 1024, L, R, 9, seed=17), Join(b.F32, b.F32, 1000, 520, R, L, 1, seed=18)]
    for a in calls + joins:
        a.forward()
        a.backward()
    want = [[x.clone() for x in (a.ctx, a.lse, a.drows)] for a in calls] + [[x.clone() for x in (a.y, a.h, a.dx, a.df, *a.grads.values())] for a in joins]
    for a in calls:
        a.results()
    for a in joins:
        a.reset()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for a, s in zip(calls + joins, streams * 2):
        with torch.cuda.stream(s):
            a.forward()
            a.backward()
    torch.cuda.synchronize()
    got = [[a.ctx, a.lse, a.drows] for a in calls] + [[a.y, a.h, a.dx, a.df, *a.grads.values()] for a in joins]
    for x, y in zip(want, got):
        for u, v in zip(x, y):
            assert torch.equal(u, v)


def test_attention_packed_rows_beyond_32_bits():
    """The last rows lie more than 2^31 elements behind the first."""
    torch = _torch()
    lengths, ld = [300] * 120 + [77], 65536
    n = sum(lengths)
    whole = torch.empty(n * ld, device="cuda", dtype=torch.bfloat16)
    a = Packed(b.BF16, lengths, 2, 1, 64, seed=12)
    cut = lambda i, m: whole.as_strided((n, m, 64), (ld, 64, 1), i * 64)  # noqa: E731
    for i, (name, m) in enumerate((("q", 2), ("k", 1), ("v", 1), ("ctx", 2), ("dctx", 2), ("dq", 2), ("dk", 1), ("dv", 1))):
        view = cut(4 * i, m)
        if name in ("q", "k", "v", "dctx"):
            view.copy_(getattr(a, name))
        setattr(a, name, view)
    a.forward()
    a.backward()
    a.ends = a.ends[-3:]
    a.check_forward()
    a.check_backward()


def test_attention_packed_of_more_than_2_to_the_28_rows_of_all_heads():
    """Sixteen threads for each row of a head would be more than a launch holds."""
    a = Packed(b.BF16, [300], 65, 13, 8, before=1 << 22, tail=2, seed=13)
    a.forward()
    a.backward()
    a.check_forward()
    a.check_backward()
    a.untouched()


def test_rotary_of_more_rows_than_a_launch_holds_workgroups():
    """Where a token is enough for a workgroup, two go to each."""
    torch = _torch()
    tokens, heads = (1 << 24) + 100, 400
    x = torch.zeros(tokens, heads, 2, device="cuda", dtype=torch.bfloat16)
    x[-200:] = _randn(_gen(14), 200, heads, 2).to(torch.bfloat16)
    last = x[-200:].clone()
    freq = torch.full((1,), 1e-7, dtype=torch.float64, device="cuda")
    b.chimera_op_rotary(x, x, freq)
    want, tol = _turned(last, torch.arange(tokens - 200, tokens, device="cuda").double()[:, None] * freq, 1.0, b.ROTARY_HALF, False)
    _within(x[-200:], want, tol + HALF[b.BF16] * want.abs(), "y")
    assert (x[:-200] == 0).all()


def _replayed(run, change, outputs):
    """Captures run(), replays it over inputs that change, and compares with the eager run each time."""
    torch = _torch()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        run()
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(4):
        change(i)
        start = [x.clone() for x in outputs()]
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in outputs()]
        for x, y in zip(outputs(), start):
            x.copy_(y)
        run()
        torch.cuda.synchronize()
        for x, y in zip(got, outputs()):
            assert torch.equal(x, y), "replay %d differs" % i


@pytest.mark.parametrize("dtype", [b.F32, b.BF16], ids=["f32", "bf16"])
def test_attention_packed_recorded_for_other_packings(dtype):
    torch = _torch()
    a = Packed(dtype, [100, 130, 77, 10], 4, 2, 64, seed=13)
    ws = torch.empty(b.lib().chimera_op_attention_packed_bwd_workspace_bytes(dtype, 4, 317, 4, 2, 64), dtype=torch.uint8, device="cuda")

    def run():
        a.forward()
        a.backward(ws)

    def change(i):
        a.offsets.copy_(torch.tensor([[0, 100, 230, 307, 317], [0, 317, 317, 317, 317], [5, 6, 7, 8, 300], [0, 0, 0, 0, 0]][i], dtype=torch.int32))
        a.rows.mul_(-1.0)
        for x in (a.ctx, a.lse, a.drows):
            x.fill_(7.0)

    _replayed(run, change, lambda: (a.ctx, a.lse, a.drows))


# ------------------------------------------------------------------- norms of a branch
class Off:
    """A number in 64 bits and how far floats may be from it; every operation adds its rounding."""

    def __init__(self, v, e=None):
        self.v, self.e = v, _torch().zeros_like(v) if e is None else e

    def _new(self, v, e):
        return Off(v, e + E24 * v.abs())

    def __add__(self, o):
        return self._new(self.v + o.v, self.e + o.e)

    def __sub__(self, o):
        return self._new(self.v - o.v, self.e + o.e)

    def __mul__(self, o):
        if not isinstance(o, Off):
            return self._new(self.v * o, self.e * abs(o))
        return self._new(self.v * o.v, self.e * o.v.abs() + o.e * self.v.abs() + self.e * o.e)

    def mean(self):
        """Over a row: a thread adds up to 32 numbers, a wavefront 6 times, wavefronts 8."""
        return self._new(self.v.mean(1, keepdim=True), self.e.mean(1, keepdim=True) + 48 * E24 * self.v.abs().mean(1, keepdim=True))

    def sum(self, rows, dim=0):
        """Over rows: up to one for each 256 in a workgroup's lane, 8 lanes, and sub-sums of an eighth of the workgroups, four at a time."""
        return self._new(self.v.sum(dim), self.e.sum(dim) + (rows / 256 + 120) * E24 * self.v.abs().sum(dim))

    def rsqrt(self):
        r = self.v.rsqrt()
        return self._new(r, self.e / (2 * self.v) * r * 1.01 + 4 * E24 * r)


def _norm(v, kind, gain, bias, eps):
    torch = _torch()
    mean = v.mean() if kind == b.NORM_LAYER else Off(torch.zeros_like(v.v[:, :1]))
    c = v - mean if kind == b.NORM_LAYER else v
    square = (c * c).mean()
    rstd = (square + Off(torch.full_like(square.v, eps))).rsqrt()
    h = c * rstd * gain
    return (h if bias is None else h + bias), mean, rstd


class Join:
    def __init__(self, dtype, stream, rows, cols, post, pre, gates, biases=True, x=True, alpha=0.9, beta=0.7, seed=0):
        torch = _torch()
        gen, t, ts = _gen(seed), _type(dtype), _type(stream)
        r = lambda *s: _randn(gen, *s)  # noqa: E731
        self.dtype, self.stream, self.rows, self.cols, self.post, self.pre, self.gates, self.alpha, self.beta = dtype, stream, rows, cols, post, pre, gates, alpha, beta
        self.f, self.x = (r(rows, cols) + 0.3).to(t), (2 * r(rows, cols)).to(ts) if x else None
        self.post_gain, self.pre_gain = [(1 + 0.2 * r(cols)).to(t) if k else None for k in (post, pre)]
        self.post_bias, self.pre_bias = [(0.2 * r(cols)).to(t) if k and biases else None for k in (post, pre)]
        self.gate = (0.5 + 0.3 * r(gates, cols)).to(t) if gates else None
        self.dy, self.dh = r(rows, cols).to(ts), r(rows, cols).to(t) if pre else None
        self.grads0 = {n: r(*v.shape) for n in ("post_gain", "post_bias", "pre_gain", "pre_bias", "gate") if (v := getattr(self, n)) is not None}
        self.reset()

    def reset(self):
        torch = _torch()
        nan = lambda t: torch.full((self.rows, self.cols), float("nan"), device="cuda", dtype=_type(t))  # noqa: E731
        self.y, self.h, self.dx, self.df = nan(self.stream), nan(self.dtype) if self.pre else None, nan(self.stream), nan(self.dtype)
        self.stats = torch.full((4, self.rows), 7.0, device="cuda")
        self.grads = {n: v.clone() for n, v in self.grads0.items()}

    def _params(self):
        return dict(post=self.post, post_gain=self.post_gain, post_bias=self.post_bias, pre=self.pre, pre_gain=self.pre_gain, gate=self.gate, alpha=self.alpha, beta=self.beta)

    def forward(self):
        b.chimera_op_branch_norm_fwd(self.f, self.x, self.y, self.h, self.stats, pre_bias=self.pre_bias, eps=1e-5, **self._params())

    def backward(self, overwrite=False, workspace=None, dy=True):
        return b.chimera_op_branch_norm_bwd(self.f, self.y if self.pre else None, self.stats, self.dy if dy else None, self.dh, self.dx, self.df, overwrite=overwrite,
                                            workspace=workspace, **self._params(), **{"d" + n: v for n, v in self.grads.items()})

    def _o(self, name):
        v = getattr(self, name)
        return None if v is None else Off(v.double())

    def _gate_rows(self):
        return None if self.gate is None else Off(self.gate.double().repeat_interleave(self.rows // self.gates, 0))

    def check_forward(self):
        u = self._o("f")
        if self.post:
            u, mean, rstd = _norm(u, self.post, self._o("post_gain"), self._o("post_bias"), 1e-5)
            self._check_stats(0, self.post, mean, rstd)
        if self.gate is not None:
            u = u * self._gate_rows()
        y = u * self.beta
        if self.x is not None:
            y = y + self._o("x") * self.alpha
        y = Off(y.v, y.e + 4 * E24 * (y.v.abs() + (u.v * self.beta).abs()))                        # (alpha, beta as floats)
        _within(self.y, y.v, y.e + HALF[self.stream] * y.v.abs(), "y")
        if self.pre:
            h, mean, rstd = _norm(y, self.pre, self._o("pre_gain"), self._o("pre_bias"), 1e-5)
            _within(self.h, h.v, h.e + HALF[self.dtype] * h.v.abs(), "h")
            self._check_stats(2, self.pre, mean, rstd)
        else:
            assert (self.stats[2:] == 7.0).all()

    def _check_stats(self, i, kind, mean, rstd):
        _within(self.stats[i], mean.v[:, 0], mean.e[:, 0], "mean")
        _within(self.stats[i + 1], rstd.v[:, 0], rstd.e[:, 0], "rstd")

    def _back(self, d, hat, kind, gain, rstd):
        d = d * gain
        out = d - hat * (d * hat).mean()
        return (out - d.mean() if kind == b.NORM_LAYER else out) * rstd

    def check_backward(self, overwrite=False, dy=True):
        """From y and the statistics as they are."""
        torch = _torch()
        s = [Off(self.stats[i].double()[:, None]) for i in range(4)]
        want = {}
        d = self._o("dy") if dy else Off(torch.zeros_like(self.f, dtype=torch.float64))
        if self.pre:
            hat, dh = (self._o("y") - s[2] if self.pre == b.NORM_LAYER else self._o("y")) * s[3], self._o("dh")
            want["pre_gain"], want["pre_bias"] = (dh * hat).sum(self.rows), dh.sum(self.rows)
            d = d + self._back(dh, hat, self.pre, self._o("pre_gain"), s[3])
        dx = d * self.alpha
        _within(self.dx, dx.v, dx.e + (HALF[self.stream] + 2 * E24) * dx.v.abs(), "dx")
        d = d * self.beta
        d.e += 2 * E24 * d.v.abs()
        u = self._o("f")
        if self.post:
            hat = (u - s[0] if self.post == b.NORM_LAYER else u) * s[1]
            u = hat * self._o("post_gain")
            u = u if self.post_bias is None else u + self._o("post_bias")
        if self.gate is not None:
            du = d * u
            n = self.rows // self.gates
            want["gate"] = Off(du.v.unflatten(0, (self.gates, n)), du.e.unflatten(0, (self.gates, n))).sum(self.rows, 1)
            d = d * self._gate_rows()
        if self.post:
            want["post_gain"], want["post_bias"] = (d * hat).sum(self.rows), d.sum(self.rows)
            d = self._back(d, hat, self.post, self._o("post_gain"), s[1])
        _within(self.df, d.v, d.e + HALF[self.dtype] * d.v.abs(), "df")
        for n, got in self.grads.items():
            w = want[n] if overwrite else want[n] + Off(self.grads0[n].double())
            _within(got, w.v, w.e, "d" + n)


N, L, R = b.NORM_NONE, b.NORM_LAYER, b.NORM_RMS
JOINS = [(1, 8, N, R, 0), (1, 64, R, R, 1), (60, 512, L, L, 0), (61, 520, R, N, 1), (300, 1024, L, R, 3), (37, 1600, N, L, 37), (129, 1032, R, L, 43), (515, 64, L, L, 103), (70, 2056, R, R, 7),
         (9, 4096, L, L, 3), (33, 4104, R, L, 1), (20, 8192, L, R, 20), (2600, 72, R, R, 2), (2050, 512, L, L, 1025), (700, 136, N, R, 350), (16, 256, N, N, 4)]


@pytest.mark.parametrize("dtype,stream", [(b.F32, b.F32), (b.BF16, b.BF16), (b.BF16, b.F32)], ids=["f32", "bf16", "bf16-float-stream"])
@pytest.mark.parametrize("rows,cols,post,pre,gates", JOINS)
def test_branch_norm(dtype, stream, rows, cols, post, pre, gates):
    torch = _torch()
    a = Join(dtype, stream, rows, cols, post, pre, gates, biases=(rows + cols) % 3 != 0, x=rows != 61, seed=rows + cols)
    a.forward()
    a.check_forward()
    a.backward()
    a.check_backward()
    first = [a.dx, a.df, *a.grads.values()]
    a.dx, a.df, a.grads = torch.zeros_like(a.dx), torch.zeros_like(a.df), {n: v.clone() for n, v in a.grads0.items()}
    a.backward()
    for x, y in zip(first, [a.dx, a.df, *a.grads.values()]):
        assert torch.equal(x, y), "a second run differs"
    a.grads = {n: torch.full_like(v, float("nan")) for n, v in a.grads0.items()}
    a.backward(overwrite=True)
    a.check_backward(overwrite=True)
    if pre:
        a.grads = {n: v.clone() for n, v in a.grads0.items()}
        a.backward(dy=False)
        a.check_backward(dy=False)


def test_branch_norm_in_place_and_gradients_not_wanted():
    torch = _torch()
    for dtype, stream in ((b.F32, b.F32), (b.BF16, b.F32), (b.BF16, b.BF16)):
        a = Join(dtype, stream, 130, 1600, R, L, 2, seed=4)
        a.forward()
        a.backward()
        want = [x.clone() for x in (a.y, a.h, a.dx, a.df)]
        x, f, keep = a.x.clone(), a.f.clone(), a.f
        b.chimera_op_branch_norm_fwd(f, x, x, f, a.stats, pre_bias=a.pre_bias, **a._params())
        assert torch.equal(x, want[0]) and torch.equal(f, want[1])
        dy, dh = a.dy.clone(), a.dh.clone()
        b.chimera_op_branch_norm_bwd(keep, a.y, a.stats, dy, dh, dy, dh, **a._params(), dpre_gain=a.grads["pre_gain"])
        assert torch.equal(dy, want[2]) and torch.equal(dh, want[3])
        df = torch.empty_like(want[3])
        b.chimera_op_branch_norm_bwd(keep, a.y, a.stats, a.dy, a.dh, None, df, **a._params())
        assert torch.equal(df, want[3])


def test_branch_norm_rows_that_are_not_finite_stay_alone():
    torch = _torch()
    a = Join(b.BF16, b.F32, 40, 512, L, R, 0, seed=6)
    a.forward()
    a.backward()
    want = [x.clone() for x in (a.y, a.h, a.dx, a.df)]
    a.f[7], a.x[20], a.dh[30] = float("nan"), float("inf"), float("nan")
    a.reset()
    a.forward()
    a.backward()
    keep = torch.ones(40, dtype=torch.bool, device="cuda")
    keep[[7, 20, 30]] = False
    for x, y in zip((a.y, a.h, a.dx, a.df), want):
        assert torch.equal(x[keep], y[keep])
    assert a.h[7].isnan().all() and a.df[30].isnan().all() and not a.h[30].isnan().any()


def test_branch_norm_more_than_2_31_values():
    torch = _torch()
    rows, cols = 270000, 8192
    gen = _gen(1)
    f = torch.empty((rows, cols), device="cuda", dtype=torch.bfloat16).normal_(generator=gen)
    y, h, stats = torch.empty_like(f), torch.empty_like(f), torch.empty((4, rows), device="cuda")
    g = torch.ones(cols, device="cuda", dtype=torch.bfloat16)
    b.chimera_op_branch_norm_fwd(f, f, y, h, stats, post=R, post_gain=g, pre=L, pre_gain=g)
    dx, df, dg = torch.empty_like(f), torch.empty_like(f), torch.zeros(cols, device="cuda")
    b.chimera_op_branch_norm_bwd(f, y, stats, y, h, dx, df, post=R, post_gain=g, pre=L, pre_gain=g, dpre_gain=dg)
    part = Join(b.BF16, b.BF16, 64, cols, R, L, 0, biases=False, alpha=1.0, beta=1.0)
    at = torch.cat((torch.arange(32), torch.arange(rows - 32, rows))).cuda()
    part.f, part.x, part.y, part.h, part.stats, part.dy, part.dh, part.dx, part.df = f[at], f[at], y[at], h[at], stats[:, at].contiguous(), y[at], h[at], dx[at], df[at]
    part.post_gain, part.pre_gain, part.grads = g, g, {}
    part.check_forward()
    part.check_backward()
    want = sum((h[i:i + 30000].double() * (y[i:i + 30000].double() - stats[2, i:i + 30000, None].double()) * stats[3, i:i + 30000, None].double()).sum(0) for i in range(0, rows, 30000))
    assert rel_err(dg.cpu(), want.cpu()) <= (rows / 256 + 130) * E24


def test_rotary_and_branch_norm_recorded():
    torch = _torch()
    a = Join(b.BF16, b.F32, 700, 1600, R, L, 7, seed=9)
    ws = torch.empty(b.lib().chimera_op_branch_norm_bwd_workspace_bytes(700, 1600, 7), dtype=torch.uint8, device="cuda")
    q = _randn(_gen(2), 700, 25, 64).bfloat16()
    turned, freq, positions = torch.empty_like(q), b.chimera_rotary_frequencies(64).cuda(), torch.arange(700, device="cuda", dtype=torch.int32)

    def run():
        a.forward()
        a.backward(workspace=ws)
        b.chimera_op_rotary(q, turned, freq, positions=positions)

    def change(i):
        a.f.mul_(-1.0)
        a.dy.mul_(0.5)
        positions.add_(1000 * i)

    _replayed(run, change, lambda: (a.y, a.h, a.dx, a.df, turned, *a.grads.values()))


# ------------------------------------------------------------------ against differences
def _slope(loss, at, direction, step=1e-4):
    """Along a direction, from four values: off by the fifth power of the step."""
    f = lambda s: float(loss([x + s * step * d for x, d in zip(at, direction)]))  # noqa: E731
    return (8 * (f(1) - f(-1)) - (f(2) - f(-2))) / (12 * step)


def test_gradients_against_differences():
    """The float operators' gradients along random directions against differences of the formulas in 64 bits."""
    torch = _torch()
    gen = _gen(21)
    rand = lambda x: torch.randn(x.shape, device="cuda", generator=gen, dtype=torch.float64)  # noqa: E731
    # attention, grouped heads, with the rotation of q and k in front of it
    a = Packed(b.F32, [40, 1, 23], 4, 2, 16, seed=22)
    freq = b.chimera_rotary_frequencies(12).cuda()
    turned, back = torch.empty((64, 6, 16), device="cuda"), torch.empty((64, 6, 16), device="cuda")
    x0 = a.rows.double().clone()
    b.chimera_op_rotary(a.rows.unflatten(1, (8, 16))[:, :6], turned, freq)
    a.q, a.k = turned[:, :4], turned[:, 4:]
    a.forward()
    a.backward()
    b.chimera_op_rotary(a.drows.unflatten(1, (8, 16))[:, :6], back, freq, transpose=True)
    grad = torch.cat((back.flatten(1), a.dv.flatten(1)), 1).double()

    def attention(rows):
        x = rows[0].unflatten(1, (8, 16))
        x = torch.cat((_turned(x[:, :6], torch.arange(64, device="cuda").double()[:, None] * freq, 1.0, b.ROTARY_HALF, False)[0], x[:, 6:]), 1)
        total = 0.0
        for lo, hi in zip(a.ends, a.ends[1:]):
            for h in range(4):
                z = (x[lo:hi, h] @ x[lo:hi, 4 + h // 2].t() * a.scale).masked_fill(torch.ones((hi - lo, hi - lo), device="cuda").triu(1).bool(), -math.inf)
                total = total + (torch.softmax(z, 1) @ x[lo:hi, 6 + h // 2] * a.dctx[lo:hi, h].double()).sum()
        return total

    for _ in range(4):
        d = rand(x0)
        want = _slope(attention, [x0], [d])
        # floats through two operators: 2^-24 for each of some 200 roundings of a term
        assert abs(float((grad * d).sum()) - want) <= 200 * E24 * float((grad * d).abs().sum())
    # norms, gate and residual
    j = Join(b.F32, b.F32, 24, 40, L, R, 6, seed=23)
    j.forward()
    j.backward(overwrite=True)
    names = ["f", "x", "post_gain", "post_bias", "pre_gain", "pre_bias", "gate"]
    start = [getattr(j, n).double() for n in names]
    grads = [j.df, j.dx] + [j.grads[n] for n in names[2:]]

    def norm(v, kind, gain, bias):
        c = v - v.mean(1, keepdim=True) if kind == L else v
        return c / (c.square().mean(1, keepdim=True) + 1e-5).sqrt() * gain + bias

    def join(v):
        f, x, g1, b1, g2, b2, gate = v
        y = j.alpha * x + j.beta * gate.repeat_interleave(4, 0) * norm(f, L, g1, b1)
        return (y * j.dy.double()).sum() + (norm(y, R, g2, b2) * j.dh.double()).sum()

    for k in range(len(names)):
        d = [rand(x) if i == k else torch.zeros_like(x) for i, x in enumerate(start)]
        want = _slope(join, start, d)
        assert abs(float((grads[k].double() * d[k]).sum()) - want) <= 200 * E24 * float((grads[k].double() * d[k]).abs().sum()), names[k]


# ------------------------------------------------------------------------ all together
@pytest.mark.parametrize("dtype", [b.F32, b.BF16], ids=["f32", "bf16"])
def test_attention_sublayer_of_these_operators(dtype):
    """Norm, projection, rotary positions, attention over packed sequences with grouped heads, projection, norm behind the branch, gate, residual, next norm:
    forward and backward through the framework's products, against autograd over the plain computation in 64 bits.  The bars are those of a stage."""
    torch = _torch()
    gen = _gen(31)
    t = _type(dtype)
    lengths, hidden, heads, kv, dim = [70, 33, 0, 25], 128, 4, 2, 32
    n, wide, total = sum(lengths), heads * dim, (heads + 2 * kv) * dim
    ends = [0]
    for m in lengths:
        ends.append(ends[-1] + m)
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    positions = torch.cat([torch.arange(m) for m in lengths]).to(torch.int32).cuda()
    freq = b.chimera_rotary_frequencies(dim, scaling=b.ROTARY_BLEND, factor=4.0, context=64).cuda()
    r = lambda *s: _randn(gen, *s)  # noqa: E731
    x, w_qkv, w_o = r(n, hidden).to(t), (r(hidden, total) * hidden ** -0.5).to(t), (r(wide, hidden) * wide ** -0.5).to(t)
    gains = [(1 + 0.1 * r(hidden)).to(t) for _ in range(3)]
    gate, dy, dh = (1 + 0.1 * r(1, hidden)).to(t), r(n, hidden).to(t), r(n, hidden).to(t)
    e = lambda *s, d=t: torch.empty(s, device="cuda", dtype=d)  # noqa: E731
    f = torch.float32

    # forward.  The first norm alone: a branch of zeros, whose stream is x
    zero, y0, h0, s0 = torch.zeros((n, hidden), device="cuda", dtype=t), e(n, hidden), e(n, hidden), e(4, n, d=f)
    b.chimera_op_branch_norm_fwd(zero, x, y0, h0, s0, pre=R, pre_gain=gains[0])
    assert torch.equal(y0, x)
    qkv, ctx, lse, o = e(n, total), e(n, heads, dim), e(heads, n, d=f), e(n, hidden)
    b.chimera_op_gemm(h0, w_qkv, qkv, n, total, hidden, 1, 0)
    rows = qkv.unflatten(1, (heads + 2 * kv, dim))
    b.chimera_op_rotary(rows[:, :heads + kv], rows[:, :heads + kv], freq, positions=positions)                                  # in place
    q, k, v = rows[:, :heads], rows[:, heads:heads + kv], rows[:, heads + kv:]
    b.chimera_op_attention_packed_fwd(q, k, v, offsets, ctx, lse)
    b.chimera_op_gemm(ctx, w_o, o, n, hidden, wide, 1, 0)
    y, h, s1 = e(n, hidden), e(n, hidden), e(4, n, d=f)
    b.chimera_op_branch_norm_fwd(o, x, y, h, s1, post=R, post_gain=gains[1], pre=R, pre_gain=gains[2], gate=gate, beta=0.5)
    # backward
    dgain = [torch.zeros(hidden, device="cuda") for _ in range(3)]
    dgate, dx, do = torch.zeros((1, hidden), device="cuda"), e(n, hidden), e(n, hidden)
    b.chimera_op_branch_norm_bwd(o, y, s1, dy, dh, dx, do, post=R, post_gain=gains[1], pre=R, pre_gain=gains[2], gate=gate, beta=0.5, dpost_gain=dgain[1], dpre_gain=dgain[2], dgate=dgate)
    dctx, dqkv, dh0, dw_o, dw_qkv = e(n, heads, dim), e(n, total), e(n, hidden), torch.zeros((wide, hidden), device="cuda"), torch.zeros((hidden, total), device="cuda")
    b.chimera_op_gemm(do, w_o, dctx, n, wide, hidden, 1, 1)
    b.chimera_op_gemm(ctx, do, dw_o, wide, hidden, n, 0, 0, epilogue=b.EPI_ACCUM_F32)
    drows = dqkv.unflatten(1, (heads + 2 * kv, dim))
    b.chimera_op_attention_packed_bwd(q, k, v, offsets, ctx, lse, dctx, drows[:, :heads], drows[:, heads:heads + kv], drows[:, heads + kv:])
    b.chimera_op_rotary(drows[:, :heads + kv], drows[:, :heads + kv], freq, positions=positions, transpose=True)
    b.chimera_op_gemm(dqkv, w_qkv, dh0, n, hidden, total, 1, 1)
    b.chimera_op_gemm(h0, dqkv, dw_qkv, hidden, total, n, 0, 0, epilogue=b.EPI_ACCUM_F32)
    dx_all = e(n, hidden)
    b.chimera_op_branch_norm_bwd(zero, x, s0, dx, dh0, dx_all, e(n, hidden), pre=R, pre_gain=gains[0], dpre_gain=dgain[0])

    leaves = [v.double().detach().requires_grad_() for v in (x, w_qkv, w_o, *gains, gate)]
    X, WQ, WO, G0, G1, G2, GATE = leaves
    rms = lambda u, g: u / (u.square().mean(1, keepdim=True) + 1e-5).sqrt() * g  # noqa: E731
    p = torch.matmul(rms(X, G0), WQ).unflatten(1, (heads + 2 * kv, dim))
    theta = positions.double()[:, None, None] * freq
    c, s = torch.cos(theta), torch.sin(theta)
    a0, a1 = p[:, :heads + kv, :dim // 2], p[:, :heads + kv, dim // 2:]
    turned = torch.cat((a0 * c - a1 * s, a0 * s + a1 * c), 2)
    parts = []
    for lo, hi in zip(ends, ends[1:]):
        hidden_keys = torch.ones((hi - lo, hi - lo), device="cuda").triu(1).bool()
        parts.append(torch.stack([torch.softmax((turned[lo:hi, i] @ turned[lo:hi, heads + i // 2].t() * dim ** -0.5).masked_fill(hidden_keys, -math.inf), 1)
                                  @ p[lo:hi, heads + kv + i // 2] for i in range(heads)], 1))
    Y = X + 0.5 * GATE * rms(torch.cat(parts).flatten(1) @ WO, G1)
    H = rms(Y, G2)
    ((Y * dy.double()).sum() + (H * dh.double()).sum()).backward()
    assert rel_err(y.float().cpu(), Y.detach().cpu()) <= TOL[dtype] and rel_err(h.float().cpu(), H.detach().cpu()) <= TOL[dtype]
    for got, leaf, what in zip((dx_all, dw_qkv, dw_o, *dgain, dgate), leaves, ("dx", "dw_qkv", "dw_o", "dgain0", "dgain1", "dgain2", "dgate")):
        assert rel_err(got.float().cpu(), leaf.grad.cpu()) <= TOL[dtype], what


def test_calls_on_another_stream_than_the_default():
    torch = _torch()
    a = Packed(b.BF16, [300, 45], 8, 2, 64, seed=41)
    a.forward()
    a.backward()
    want = [x.clone() for x in (a.ctx, a.lse, a.drows)]
    a.results()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a.forward()
        a.backward()
    side.synchronize()
    for x, y in zip(want, (a.ctx, a.lse, a.drows)):
        assert torch.equal(x, y)
