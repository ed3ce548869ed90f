"""What the loss without logits, the gradient norm and AdamW refuse, and the sizes they ask for: all decided on the host, before any launch."""
import ctypes as C

import pytest

from paper_2107_06925_amd import binding as b

P = 0x10000                                     # an aligned address that no call below follows
U64 = 1 << 62



def fwd(dtype=b.BF16, tokens=4, hidden=64, vocab=100, h=P, ldh=64, w=P, ldw=104, targets=P, rows=P, lse=P, loss=P, ws=P, size=U64):
    return b.lib().chimera_op_linear_xent_fwd(dtype, tokens, hidden, vocab, h, ldh, w, ldw, targets, 1.0, rows, lse, loss, ws, size, None)


def bwd(dtype=b.BF16, tokens=4, hidden=64, vocab=100, h=P, ldh=64, w=P, ldw=104, targets=P, lse=P, dloss=None, dh=P, lddh=64, dw=P, lddw=104,
        piece=0, ws=P, size=U64):
    return b.lib().chimera_op_linear_xent_bwd(dtype, tokens, hidden, vocab, h, ldh, w, ldw, targets, lse, 1.0, dloss, dh, lddh, dw, lddw, 0, piece, ws, size, None)


BAD_SIZES = [dict(dtype=2), dict(tokens=0), dict(tokens=-3), dict(tokens=(1 << 22) + 1), dict(hidden=0), dict(hidden=60), dict(hidden=(1 << 15) + 8, ldh=(1 << 15) + 8), dict(tokens=1 << 22, vocab=65537, ldw=65544),
             dict(vocab=0), dict(vocab=105), dict(vocab=(1 << 22) + 8, ldw=(1 << 22) + 8), dict(ldh=56), dict(ldh=68), dict(ldw=108), dict(ldw=1 << 23),
             dict(h=None), dict(w=None), dict(targets=None), dict(lse=None), dict(ws=None), dict(h=P + 8), dict(w=P + 2), dict(ws=P + 16)]


@pytest.mark.parametrize("bad", BAD_SIZES + [dict(rows=None)], ids=str)
def test_linear_xent_fwd_refuses(bad):
    assert fwd(**bad) == b.EINVAL, b.last_error()
    assert b.last_error()


@pytest.mark.parametrize("bad", BAD_SIZES + [dict(dh=None, dw=None), dict(piece=-1), dict(lddh=56), dict(lddh=68), dict(lddw=96), dict(lddw=106),
                                             dict(dh=P + 4), dict(dw=P + 4)], ids=str)
def test_linear_xent_bwd_refuses(bad):
    assert bwd(**bad) == b.EINVAL, b.last_error()
    assert b.last_error()


@pytest.mark.parametrize("dtype", [b.F32, b.BF16])
@pytest.mark.parametrize("tokens,hidden,vocab,piece", [(1, 8, 1, 0), (5, 64, 1001, 256), (4096, 1600, 50257, 0), (1 << 20, 2048, 65536, 0)])
def test_linear_xent_workspaces(dtype, tokens, hidden, vocab, piece):
    l = b.lib()
    f, g = l.chimera_op_linear_xent_fwd_workspace_bytes(dtype, tokens, hidden, vocab), l.chimera_op_linear_xent_bwd_workspace_bytes(dtype, tokens, hidden, vocab, piece)
    assert f > 0 and g > 0
    ld = (vocab + 7) // 8 * 8
    sizes = dict(dtype=dtype, tokens=tokens, hidden=hidden, vocab=vocab, ldh=hidden, ldw=ld)
    assert fwd(**sizes, size=f - 1) == b.ENOMEM
    assert bwd(**sizes, lddh=hidden, lddw=ld, piece=piece, size=g - 1) == b.ENOMEM
    if tokens >= 4096:                         # no logits: half of them at the very most, and the rows that the weight gradient takes
        e = 4 if dtype == b.F32 else 2
        assert f < tokens * vocab * e // 2
        assert l.chimera_head_pieces_workspace_bytes(dtype, tokens, hidden, vocab, 256) < tokens * vocab * e


def test_linear_xent_workspace_of_refused_sizes_is_zero():
    l = b.lib()
    for args in ((2, 4, 64, 100), (b.BF16, 0, 64, 100), (b.BF16, 4, 60, 100), (b.BF16, 4, 64, 0), (b.BF16, 4, 64, (1 << 22) + 1)):
        assert l.chimera_op_linear_xent_fwd_workspace_bytes(*args) == 0
        assert l.chimera_op_linear_xent_bwd_workspace_bytes(*args, 0) == 0
        assert l.chimera_head_pieces_workspace_bytes(*args, 0) == 0
    assert l.chimera_op_linear_xent_bwd_workspace_bytes(b.BF16, 4, 64, 100, -1) == 0


def test_head_loss_pieces_refuses():
    def call(**o):
        a = dict(dtype=b.BF16, tokens=4, hidden=64, vocab=100, y=P, t=P, g=P, be=P, w=P, ldw=104, dy=P, dg=P, db=P, dw=P, loss=P, piece=0, ws=P, size=U64)
        a.update(o)
        return b.lib().chimera_head_loss_pieces(a["dtype"], a["tokens"], a["hidden"], a["vocab"], a["y"], a["t"], a["g"], a["be"], a["w"], a["ldw"], 1.0, a["dy"],
                                                a["dg"], a["db"], a["dw"], a["loss"], a["piece"], a["ws"], a["size"], None)
    for bad in (dict(dtype=5), dict(tokens=0), dict(hidden=12), dict(ldw=100), dict(ldw=96), dict(y=None), dict(t=None), dict(loss=None), dict(dw=None),
                dict(piece=-1), dict(ws=P + 1), dict(dy=P + 8)):
        assert call(**bad) == b.EINVAL, bad
    need = b.lib().chimera_head_pieces_workspace_bytes(b.BF16, 4, 64, 100, 0)
    assert call(size=need - 1) == b.ENOMEM


def norm(n=(8, 0, 5), grads=(P, None, P), max_norm=1.0, out=P, ws=P, size=U64, count=None):
    c = len(n) if count is None else count
    return b.lib().chimera_op_grad_norm(c, (C.c_int64 * len(n))(*n), (C.c_void_p * len(grads))(*grads), max_norm, out, ws, size, None)


@pytest.mark.parametrize("bad", [dict(count=0), dict(count=-1), dict(n=(8, -1, 5)), dict(n=(8, 1 << 60, 5), grads=(P, P, P)), dict(grads=(P, None, None)),
                                 dict(grads=(P, None, P + 2)), dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(out=None),
                                 dict(ws=None), dict(ws=P + 4)], ids=str)
def test_grad_norm_refuses(bad):
    assert norm(**bad) == b.EINVAL
    assert b.last_error()


def test_grad_norm_workspace():
    need = b.lib().chimera_op_grad_norm_workspace_bytes(2)
    assert 0 < need < 10 ** 6
    assert norm(n=(10 ** 8, 3), grads=(P, P), size=need - 1) == b.ENOMEM
    assert b.lib().chimera_op_grad_norm_workspace_bytes(0) == 0 and b.lib().chimera_op_grad_norm_workspace_bytes(-1) == 0


def adamw(dtype=b.BF16, bits=32, n=(16, 0, 9), param=(P, None, 2 * P), master=(P, None, 2 * P), grad=(P, None, P), m=(P, None, 2 * P), v=(2 * P, None, P),
          scale=None, decay=None, hyper=(1e-3, 0.9, 0.95, 1e-8, 1, 0), device=None, count=None):
    arr = lambda x: None if x is None else (C.c_void_p * len(x))(*x)  # noqa: E731
    h = None if hyper is None else C.byref(b.AdamWHyper(*hyper))
    return b.lib().chimera_op_adamw(dtype, bits, len(n) if count is None else count, (C.c_int64 * len(n))(*n), arr(param), arr(master), arr(grad), arr(m), arr(v),
                                    arr(scale), None if decay is None else (C.c_float * len(decay))(*decay), h, device, None, None)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(bits=16), dict(bits=0), dict(count=0), dict(count=-5), dict(n=(16, 0, -9)), dict(n=(16, 0, (1 << 32) + 1)),
                                 dict(param=None), dict(master=None), dict(grad=None), dict(m=None), dict(v=None), dict(bits=8), dict(param=(P, None, None)),
                                 dict(master=(P, None, None)), dict(grad=(None, None, P)), dict(bits=8, scale=(P, None, None)), dict(param=(P, None, P)),
                                 dict(param=(P, None, P + 30)), dict(master=(P, None, P + 60)), dict(m=(2 * P, None, 2 * P + 32)), dict(v=(P + 32, None, P)), dict(param=(P + 1, None, 2 * P)), dict(grad=(P + 2, None, P)), dict(m=(P + 1, None, P)),
                                 dict(decay=(0.0, 0.0, -0.1)), dict(decay=(NAN, 0.0, 0.1)), dict(decay=(0.1, 0.0, INF)), dict(hyper=None), dict(device=P + 8),
                                 dict(hyper=(-1e-3, 0.9, 0.95, 1e-8, 1, 0)), dict(hyper=(NAN, 0.9, 0.95, 1e-8, 1, 0)), dict(hyper=(1e-3, 1.0, 0.95, 1e-8, 1, 0)),
                                 dict(hyper=(1e-3, 0.9, -0.1, 1e-8, 1, 0)), dict(hyper=(1e-3, 0.9, 0.95, 0.0, 1, 0)), dict(hyper=(1e-3, 0.9, 0.95, 1e-40, 1, 0)), dict(hyper=(1e-3, 0.9, 0.95, 2.0, 1, 0)), dict(hyper=(1e-3, 0.9, 0.95, 1e-8, 0, 0))],
                         ids=str)
def test_adamw_refuses(bad):
    assert adamw(**bad) == b.EINVAL
    assert b.last_error()


def test_stage_step_refuses_and_its_state_sizes():
    l = b.lib()
    for dtype, e in ((b.F32, 0), (b.BF16, 4)):
        st = l.chimera_stage_create(2, 64, 4, 16, 2, dtype)
        params = 2 * (12 * 64 * 64 + 13 * 64)
        assert l.chimera_stage_adamw_state_bytes(st, 32) >= params * (8 + e)
        assert params * (2 + e) <= l.chimera_stage_adamw_state_bytes(st, 8) < l.chimera_stage_adamw_state_bytes(st, 32)
        assert l.chimera_stage_adamw_state_bytes(st, 16) == 0 and l.chimera_stage_adamw_state_bytes(None, 32) == 0
        h = b.AdamWHyper(1e-3, 0.9, 0.95, 1e-8, 1, 0)
        assert l.chimera_stage_adamw_init(st, P, P, 32) == b.ESTATE                 # not bound
        assert l.chimera_stage_adamw_step(st, P, P, 32, 0.0, C.byref(h), None, None) == b.ESTATE
        assert l.chimera_stage_adamw_step(None, P, P, 32, 0.0, C.byref(h), None, None) == b.EINVAL
        l.chimera_stage_destroy(st)


def test_adamw_handle_checks_its_lists():
    torch = pytest.importorskip("torch")
    t = lambda n, d=torch.float32: torch.zeros(n, dtype=d)  # noqa: E731
    for bad in (dict(grads=[t(4)]), dict(grads=[t(4), t(4)]), dict(decay=[0.1]), dict(scales=[t(2)]), dict(scales=[t(2), t(1)]),
                dict(grads=[t(4), t((9, 2))[:, 0]]), dict(masters=[t(4), t(8)]),
                dict(params=[t(4), t(9, torch.float16)]), dict(grads=[t(4), t(9, torch.bfloat16)]), dict(ms=[t(4), t(9, torch.uint8)]),
                dict(scales=[t(2), t(2)]), dict(params=[])):
        args = dict(params=[t(4), t(9)], grads=[t(4), t(9)], ms=[t(4), t(9)], vs=[t(4), t(9)])
        args.update(bad)
        with pytest.raises(ValueError):
            b.AdamW(**args)


def test_binding_checks_matrices_and_vectors():
    torch = pytest.importorskip("torch")
    z = lambda *s, d=torch.float32: torch.zeros(s, dtype=d)  # noqa: E731
    i32 = torch.int32
    good = dict(h=z(3, 16), w=z(16, 24), targets=z(3, d=i32), scale=1.0, loss_rows=z(3), lse=z(3), loss=z(1), workspace=z(8, d=torch.uint8))
    for bad in (dict(h=z(16, 3).t()), dict(w=z(16, 24, d=torch.bfloat16)), dict(w=z(24, 16).t()), dict(targets=z(3, d=torch.int64)), dict(targets=z(4, d=i32)),
                dict(loss_rows=z(6)[::2]), dict(lse=z(3, d=torch.float64)), dict(loss=z(2))):
        with pytest.raises(ValueError):
            b.chimera_op_linear_xent_fwd(**dict(good, **bad))
    good = dict(h=z(3, 16), w=z(16, 24), targets=z(3, d=i32), lse=z(3), scale=1.0, dh=z(3, 16), dw=z(16, 24), workspace=z(8, d=torch.uint8))
    for bad in (dict(dh=z(3, 8)), dict(dw=z(16, 16)), dict(dw=z(16, 24, d=torch.bfloat16)), dict(dloss=z(2)), dict(dh=z(16, 3).t())):
        with pytest.raises(ValueError):
            b.chimera_op_linear_xent_bwd(**dict(good, **bad))
    for grads, out in (([z(4, d=torch.bfloat16)], z(2)), ([z(4, 2)[:, 0]], z(2)), ([z(4)], z(3))):
        with pytest.raises(ValueError):
            b.chimera_op_grad_norm(grads, 1.0, out, workspace=z(8, d=torch.uint8))


def test_binding_refuses_tensors_that_are_not_on_the_current_gpu():
    torch = pytest.importorskip("torch")
    z = lambda *s, d=torch.float32: torch.zeros(s, dtype=d)  # noqa: E731
    i32, ws = torch.int32, z(8, d=torch.uint8)
    t = dict(params=[z(4), z(9)], grads=[z(4), z(9)], ms=[z(4), z(9)], vs=[z(4), z(9)])
    for call in (lambda: b.chimera_op_linear_xent_fwd(z(3, 16), z(16, 24), z(3, d=i32), 1.0, z(3), z(3), workspace=ws),
                 lambda: b.chimera_op_linear_xent_bwd(z(3, 16), z(16, 24), z(3, d=i32), z(3), 1.0, dw=z(16, 24), workspace=ws),
                 lambda: b.chimera_head_loss_pieces(z(3, 16), z(3, d=i32), z(16), z(16), z(16, 24), 1.0, z(3, 16), z(16), z(16), z(16, 24), z(1), workspace=ws),
                 lambda: b.chimera_op_grad_norm([z(4)], 1.0, z(2), workspace=ws), lambda: b.AdamW(**t)):
        with pytest.raises(ValueError, match="current GPU"):
            call()


def test_head_in_pieces_checks_its_tensors():
    torch = pytest.importorskip("torch")
    z = lambda *s, d=torch.float32: torch.zeros(s, dtype=d)  # noqa: E731
    good = dict(y=z(3, 16), targets=z(3, d=torch.int32), lnf_g=z(16), lnf_b=z(16), w_head=z(16, 24), scale=1.0, dy=z(3, 16), dlnf_g=z(16), dlnf_b=z(16),
                dw_head=z(16, 24), loss=z(1), workspace=z(8, d=torch.uint8))
    for bad, what in ((dict(y=z(16, 3).t()), "contiguous"), (dict(dy=z(3, 32)[:, :16]), "contiguous"), (dict(dy=z(3, 8)), "one shape"), (dict(lnf_g=z(8)), "lnf_g"),
                      (dict(lnf_b=z(16, d=torch.bfloat16)), "lnf_b"), (dict(dlnf_g=z(32)[::2]), "dlnf_g"), (dict(dlnf_b=z(16, d=torch.float64)), "dlnf_b"),
                      (dict(loss=z(2)), "loss"), (dict(targets=z(3, d=torch.int64)), "targets"), (dict(dw_head=z(16, 32)), "w_head")):
        with pytest.raises(ValueError, match=what):
            b.chimera_head_loss_pieces(**dict(good, **bad))


def test_every_argument_has_a_type():
    """Arguments behind the declared ones travel as 32-bit numbers, pointers cut in half among them."""
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "chimera.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    declared = {name: 0 if args.strip() in ("", "void") else args.count(",") + 1 for name, args in re.findall(r"\b(chimera_\w+)\s*\(([^()]*)\)\s*;", text)}
    assert "chimera_op_adamw" in declared
    for name, (_, args) in b._SIGNATURES.items():
        assert declared.get(name) == len(args), name


def _handle(monkeypatch, sizes=(4, 9), **more):
    """A handle of CPU tensors whose steps reach no library: the arguments of each are kept in the list that comes with it."""
    torch = pytest.importorskip("torch")
    calls = []

    class Library:
        @staticmethod
        def chimera_op_adamw(*args):
            calls.append(args)
            return b.OK
    monkeypatch.setattr(b, "_stream_of", lambda *tensors: 0)
    monkeypatch.setattr(b, "lib", lambda: Library)
    lists = {k: [torch.zeros(n) for n in sizes] for k in ("params", "grads", "ms", "vs")}
    return b.AdamW(**lists, **more), lists, calls


def test_adamw_handle_keeps_what_its_addresses_name(monkeypatch):
    torch = pytest.importorskip("torch")
    handle, lists, _ = _handle(monkeypatch)
    arrays = (handle.param, handle.grad, handle.m, handle.v)
    named = [list(x) for x in arrays]
    assert named == [[t.data_ptr() for t in lists[k]] for k in ("params", "grads", "ms", "vs")]
    lists["grads"][0] = torch.ones(4)                       # a new gradient in the caller's list
    lists["params"][1].data = torch.ones(9)                 # a parameter whose memory is replaced
    lists["ms"].clear()
    for x in lists.values():
        x.clear()
    assert [[t.data_ptr() for t in x] for x in handle.tensors] == named and [list(x) for x in arrays] == named


def test_adamw_steps_share_no_hyperparameters(monkeypatch):
    """The library reads them while other threads run: a step beside another must not find the other's."""
    handle, _, calls = _handle(monkeypatch, beta1=0.8, beta2=0.9, eps=1e-6)
    handle.step(lr=1e-3, step=3, seed=5)
    handle.step(lr=2e-3, step=4, seed=6)
    seen = [next(a._obj for a in call if isinstance(getattr(a, "_obj", None), b.AdamWHyper)) for call in calls]
    assert [(h.lr, h.beta1, h.beta2, h.eps, h.step, h.seed) for h in seen] == [(1e-3, 0.8, 0.9, 1e-6, 3, 5), (2e-3, 0.8, 0.9, 1e-6, 4, 6)]


def _bad_device_hypers(torch):
    # the structure alone, without the bytes that the library uses behind it; one byte short; strided
    return [torch.zeros(C.sizeof(b.AdamWHyper), dtype=torch.uint8), torch.zeros(b.ADAMW_HYPER_BYTES - 1, dtype=torch.uint8), torch.zeros(15, dtype=torch.float64),
            torch.zeros(2 * b.ADAMW_HYPER_BYTES, dtype=torch.uint8)[::2]]


def test_adamw_checks_device_hyperparameters(monkeypatch):
    torch = pytest.importorskip("torch")
    handle, _, calls = _handle(monkeypatch)
    for bad in _bad_device_hypers(torch):
        with pytest.raises(ValueError, match="d_hyper"):
            handle.step(1e-3, 1, d_hyper=bad)
    assert not calls
    good = torch.zeros(b.ADAMW_HYPER_BYTES, dtype=torch.uint8)
    handle.step(1e-3, 1, d_hyper=good)
    assert good.data_ptr() in calls[0]


def test_stage_step_checks_its_tensors(monkeypatch):
    torch = pytest.importorskip("torch")
    from types import SimpleNamespace
    calls = []
    monkeypatch.setattr(b, "lib", lambda: SimpleNamespace(chimera_stage_adamw_step=lambda *a: calls.append(a) or b.OK))
    stage = SimpleNamespace(torch=torch, handle=1, weights=torch.zeros(8), adamw_state=torch.zeros(8), adamw_bits=32)
    for bad in _bad_device_hypers(torch):
        with pytest.raises(ValueError, match="d_hyper"):
            b.Stage.adamw_step(stage, 1e-3, 1, d_hyper=bad)
    for bad in (torch.zeros(1, dtype=torch.float64), torch.zeros(2), torch.zeros(0)):
        with pytest.raises(ValueError, match="grad_scale"):
            b.Stage.adamw_step(stage, 1e-3, 1, grad_scale=bad)
    elsewhere = SimpleNamespace(get_device=lambda: 3)
    for bad in (dict(grad_scale=elsewhere), dict(d_hyper=elsewhere)):
        with pytest.raises(ValueError, match="GPU"):
            b.Stage.adamw_step(stage, 1e-3, 1, **bad)
    assert not calls
    b.Stage.adamw_step(stage, 1e-3, 1, grad_scale=torch.ones(1), d_hyper=torch.zeros(b.ADAMW_HYPER_BYTES, dtype=torch.uint8))
    assert len(calls) == 1


def test_stage_state_is_initialised_behind_what_holds_its_memory(monkeypatch):
    """On a stage with a stream of its own: the state's memory comes from the current stream, whose work on it may not be done."""
    from types import SimpleNamespace
    did = []
    state = SimpleNamespace(record_stream=lambda s: did.append(("record", s)), data_ptr=lambda: 256)
    stream = SimpleNamespace(wait_stream=lambda s: did.append(("wait", s)))
    torch = SimpleNamespace(empty=lambda *a, **k: did.append("empty") or state, uint8=None, cuda=SimpleNamespace(current_stream=lambda d: "current"))
    monkeypatch.setattr(b, "lib", lambda: SimpleNamespace(chimera_stage_adamw_state_bytes=lambda *a: 64, chimera_stage_adamw_init=lambda *a: did.append("init") or b.OK))
    stage = SimpleNamespace(torch=torch, handle=1, weights=SimpleNamespace(data_ptr=lambda: 0), device="cuda:0", stream=stream)
    b.Stage.adamw_init(stage, 8)
    assert did.index("empty") < did.index(("wait", "current")) < did.index("init") and ("record", stream) in did


def test_adamw_refuses_overlaps_between_kinds():
    """What is written, tensor by tensor and kind by kind, shares no byte with anything else; 300 values a tensor, two blocks of 8-bit moments."""
    at = lambda k: P + 0x1000 * k  # noqa: E731
    good = dict(n=(300, 300), param=(at(0), at(1)), master=(at(2), at(3)), grad=(at(4), at(5)), m=(at(6), at(7)), v=(at(8), at(9)))
    scales = (at(10), at(11))
    for bits, bad in ((32, dict(v=(at(6), at(9)))), (32, dict(v=(at(8), at(6) + 1196))), (32, dict(m=(at(2) + 4, at(7)))), (32, dict(param=(at(0), at(9) + 1198))),
                      (32, dict(grad=(at(0), at(5)))), (32, dict(grad=(at(4), at(3) - 1196))), (32, dict(master=(at(2), at(5)))), (8, dict(m=(at(6), at(6) + 299))),
                      (8, dict(v=(at(6), at(9)))), (8, dict(scale=(at(10), at(10) + 12))), (8, dict(scale=(at(6) + 296, at(11)))), (8, dict(scale=(at(10), at(4) - 12)))):
        args = dict(good, bits=bits, scale=scales if bits == 8 else None)
        args.update(bad)
        assert adamw(**args) == b.EINVAL and "overlaps" in b.last_error(), (bits, bad, b.last_error())


def test_forward_only_stage_is_not_stepped():
    """It may be bound to the weights and gradients of another stage, and has none of its own."""
    l = b.lib()
    for bits in (32, 8):
        st = l.chimera_stage_create(2, 64, 4, 16, 2, b.BF16)
        for option in (b.OPT_KEEP, b.OPT_OVERLAP):
            b.check(l.chimera_stage_set_option(st, option, 0))
        b.check(l.chimera_stage_bind(st, P, P, P, 1, P, None))
        h = b.AdamWHyper(1e-3, 0.9, 0.95, 1e-8, 1, 0)
        for rc in (l.chimera_stage_adamw_init(st, 2 * P, 4 * P, bits), l.chimera_stage_adamw_step(st, 2 * P, 4 * P, bits, 0.0, C.byref(h), None, None)):
            assert rc == b.ESTATE and "forward-only" in b.last_error()
        l.chimera_stage_destroy(st)


def test_stage_step_refuses_overlapping_buffers():
    l = b.lib()
    params = 2 * (12 * 64 * 64 + 13 * 64)
    up = lambda n: (n + 255) // 256 * 256  # noqa: E731
    h = b.AdamWHyper(1e-3, 0.9, 0.95, 1e-8, 1, 0)
    for dtype, e in ((b.F32, 4), (b.BF16, 2)):
        for bits in (32, 8):
            st = l.chimera_stage_create(2, 64, 4, 16, 2, dtype)
            b.check(l.chimera_stage_set_option(st, b.OPT_OVERLAP, 0))
            far, state = 1 << 24, up(l.chimera_stage_adamw_state_bytes(st, bits))
            b.check(l.chimera_stage_bind(st, P, far, P, 1, P, None))
            for w, s in ((P, P), (P, P + up(params * e) - 256), (P + state - 256, P), (P, far), (P, far + up(params * 4) - 256), (P, far - state + 256), (far, P)):
                for rc in (l.chimera_stage_adamw_init(st, w, s, bits), l.chimera_stage_adamw_step(st, w, s, bits, 0.0, C.byref(h), None, None)):
                    assert rc == b.EINVAL and "overlap" in b.last_error(), (dtype, bits, w, s)
            l.chimera_stage_destroy(st)


FAR = 1 << 40                                   # places that are far apart, whatever lies at them


def test_linear_xent_refuses_overlaps():
    """4 tokens of 64, 100 words in rows of 104: every result over every operand and every other result, at its last bytes."""
    l = b.lib()
    for dtype, e in ((b.F32, 4), (b.BF16, 2)):
        at = {k: FAR * (i + 1) for i, k in enumerate(("h", "w", "targets", "rows", "lse", "loss", "ws"))}
        size = dict(h=4 * 64 * e, w=(63 * 104 + 100) * e, targets=16, rows=16, lse=16, loss=4, ws=l.chimera_op_linear_xent_fwd_workspace_bytes(dtype, 4, 64, 100))
        align = dict(h=16, w=16, targets=4, rows=4, lse=4, loss=4, ws=256)
        for out in ("rows", "lse", "loss", "ws"):
            for other in set(at) - {out}:
                first, second = (out, other) if align[out] > align[other] else (other, out)            # the second begins inside the first
                inside = at[first] + (size[first] - 1) // align[second] * align[second]
                assert fwd(dtype=dtype, **dict(at, **{second: inside})) == b.EINVAL and "overlap" in b.last_error(), (dtype, first, second)
        at = {k: FAR * (i + 1) for i, k in enumerate(("h", "w", "targets", "lse", "dloss", "dh", "dw", "ws"))}
        size = dict(h=4 * 64 * e, w=(63 * 104 + 100) * e, targets=16, lse=16, dloss=16, dh=4 * 64 * e, dw=(63 * 104 + 100) * 4,
                    ws=l.chimera_op_linear_xent_bwd_workspace_bytes(dtype, 4, 64, 100, 0))
        align = dict(h=16, w=16, targets=4, lse=4, dloss=4, dh=16, dw=16, ws=256)
        for out in ("dh", "dw", "ws"):
            for other in set(at) - {out}:
                if (out, other) == ("dh", "h"):
                    continue
                first, second = (out, other) if align[out] > align[other] else (other, out)
                inside = at[first] + (size[first] - 1) // align[second] * align[second]
                assert bwd(dtype=dtype, **dict(at, **{second: inside})) == b.EINVAL and "overlap" in b.last_error(), (dtype, first, second)
    # rows of dh between those of w, and on them: 64 rows of w, 512 bytes apart, hold 100 words; 4 rows of dh begin 256 bytes behind one of them
    at = dict(h=FAR, w=2 * FAR, targets=3 * FAR, lse=4 * FAR, dw=5 * FAR, ws=6 * FAR)
    assert bwd(dtype=b.BF16, ldw=256, dh=2 * FAR + 512 * 9 + 192, lddh=256, **at) == b.EINVAL and "overlap" in b.last_error()
    assert bwd(dtype=b.BF16, ldw=256, dh=2 * FAR + 512 * 62 + 192, lddh=512, **at) == b.EINVAL and "overlap" in b.last_error()


def test_head_loss_pieces_refuses_overlaps():
    l = b.lib()
    names = ("y", "t", "g", "be", "w", "dy", "dg", "db", "dw", "loss", "ws")
    for dtype, e in ((b.F32, 4), (b.BF16, 2)):
        size = dict(y=4 * 64 * e, t=16, g=64 * e, be=64 * e, w=(63 * 104 + 100) * e, dy=4 * 64 * e, dg=256, db=256, dw=(63 * 104 + 100) * 4, loss=4,
                    ws=l.chimera_head_pieces_workspace_bytes(dtype, 4, 64, 100, 0))
        align = {k: 256 if k == "ws" else 16 if k in ("y", "w", "dy", "dw") else 4 for k in names}
        for out in ("dy", "dg", "db", "dw", "loss", "ws"):
            for other in set(names) - {out}:
                at = {k: FAR * (i + 1) for i, k in enumerate(names)}
                first, second = (out, other) if align[out] > align[other] else (other, out)
                at[second] = at[first] + (size[first] - 1) // align[second] * align[second]
                rc = l.chimera_head_loss_pieces(dtype, 4, 64, 100, at["y"], at["t"], at["g"], at["be"], at["w"], 104, 1.0, at["dy"], at["dg"], at["db"], at["dw"],
                                                at["loss"], 0, at["ws"], U64, None)
                assert rc == b.EINVAL and "overlap" in b.last_error(), (dtype, first, second)


def test_grad_norm_refuses_overlaps():
    need = b.lib().chimera_op_grad_norm_workspace_bytes(3)
    for bad in (dict(out=FAR + 28), dict(out=3 * FAR + 16), dict(out=FAR - 4), dict(ws=FAR + 24), dict(ws=FAR - need + 8), dict(out=5 * FAR + need - 4), dict(ws=3 * FAR - need + 16)):
        args = dict(n=(8, 0, 5), grads=(FAR, None, 3 * FAR), out=4 * FAR, ws=5 * FAR)
        args.update(bad)
        assert norm(**args) == b.EINVAL and "overlaps" in b.last_error(), bad


def test_adamw_refuses_factors_and_device_hyperparameters_in_what_it_writes():
    at = lambda k: P + 0x1000 * k  # noqa: E731
    l, h = b.lib(), b.AdamWHyper(1e-3, 0.9, 0.95, 1e-8, 1, 0)
    two = lambda k: (C.c_void_p * 2)(at(k), at(k + 1))  # noqa: E731
    for device, factor in ((None, at(1) + 596), (None, at(3)), (None, at(6) + 1196), (at(8) + 1184, None), (at(2) - 112, None), (at(4) + 16, None),
                           (FAR, FAR + b.ADAMW_HYPER_BYTES - 4)):
        rc = l.chimera_op_adamw(b.BF16, 32, 2, (C.c_int64 * 2)(300, 300), two(0), two(2), two(4), two(6), two(8), None, None, C.byref(h), device, factor, None)
        assert rc == b.EINVAL and "overlaps" in b.last_error(), (device, factor, b.last_error())
    st = l.chimera_stage_create(2, 64, 4, 16, 2, b.BF16)
    b.check(l.chimera_stage_set_option(st, b.OPT_OVERLAP, 0))
    b.check(l.chimera_stage_bind(st, FAR, 2 * FAR, P, 1, P, None))
    for device, factor in ((FAR - 112, None), (None, FAR + 4), (None, 2 * FAR), (2 * FAR + 16, None), (None, 3 * FAR), (3 * FAR + 256, None), (4 * FAR, 4 * FAR + 48)):
        assert l.chimera_stage_adamw_step(st, FAR, 3 * FAR, 8, 0.0, C.byref(h), device, factor) == b.EINVAL and "overlap" in b.last_error(), (device, factor)
    l.chimera_stage_destroy(st)


def test_binding_refuses_matrices_whose_memory_ends_too_soon():
    """8 columns of bf16, 4 of float are read at a time, in the last row too, where no further row follows."""
    torch = pytest.importorskip("torch")
    for dtype, step in ((torch.float32, 4), (torch.bfloat16, 8)):
        for short in range(1, step):
            n = 24 - step + short                                             # columns; the last piece of 16 bytes holds `short` of them
            assert b._rows(torch.zeros(16 * 24, dtype=dtype).as_strided((16, n), (24, 1)), dtype, "w") == 24
            memory = torch.zeros(15 * 24 + n, dtype=dtype)
            with pytest.raises(ValueError, match="16 bytes"):
                b._rows(memory.as_strided((16, n), (24, 1)), dtype, "w")
            z = lambda *s, d=torch.float32: torch.zeros(s, dtype=d)  # noqa: E731
            with pytest.raises(ValueError, match="16 bytes"):
                b.chimera_op_linear_xent_fwd(z(3, 16, d=dtype), memory.as_strided((16, n), (24, 1)), z(3, d=torch.int32), 1.0, z(3), z(3), workspace=z(8, d=torch.uint8))
    # a part of a wider matrix that begins at a multiple of 16 bytes is whole
    assert b._rows(torch.zeros((16, 24))[:, 4:23], torch.float32, "w") == 24
    assert b._rows(torch.zeros((16, 24), dtype=torch.bfloat16)[:, 8:23], torch.bfloat16, "w") == 24


@pytest.mark.parametrize("tokens,vocab,wide", [(2048, 4096, 0), (2048, 4352, 4352), (2048, 12288, 8192), (2048, 12544, 12544), (2048, 32768, 32768), (2048, 50257, 49152),
                                               (128, 50257, 0), (129, 50257, 50432), (256, 32768, 0), (256, 33025, 33280)])
def test_linear_xent_forward_takes_large_tiles_from_half_a_round_on(tokens, vocab, wide):
    """Read off the workspace: 8 bytes for each token and tile column, 4 more a token."""
    need = b.lib().chimera_op_linear_xent_fwd_workspace_bytes(b.BF16, tokens, 64, vocab)
    columns = wide // 256 + max(0, -(-(vocab - wide) // 128))
    assert need == -(-8 * tokens * columns // 256) * 256 + -(-4 * tokens // 256) * 256


@pytest.mark.parametrize("tokens,hidden,vocab,piece", [(2048, 1600, 50257, 9216), (1024, 1600, 65536, 8192), (2048, 2304, 65536, 8192), (2048, 2560, 65536, 8192),
                                                       (8192, 2048, 65536, 8192), (4096, 1536, 50257, 10752), (8192, 1280, 65536, 7424), (2048, 1600, 37120, 7424),
                                                       (2048, 1536, 44032, 7424)])
def test_linear_xent_pieces_that_the_library_chooses(tokens, hidden, vocab, piece):
    """Without a piece the workspace is that of the piece of this size; and no other multiple of 256 near it has the same."""
    need = lambda p: b.lib().chimera_op_linear_xent_bwd_workspace_bytes(b.BF16, tokens, hidden, vocab, p)  # noqa: E731
    assert need(0) == need(piece) and need(0) not in (need(piece - 256), need(piece + 256))


@pytest.mark.parametrize("rows", [8, 24])
def test_binding_refuses_a_matrix_of_other_rows(rows):
    """The library reads (and writes) as many rows of w (and dw) as h has columns, whether the tensors hold them or not."""
    torch = pytest.importorskip("torch")
    z = lambda *s, d=torch.float32: torch.zeros(s, dtype=d)  # noqa: E731
    i32, ws = torch.int32, z(8, d=torch.uint8)
    for h, w in ((z(3, 16), z(rows, 24)), (z(3, 16), z(16, 24, 1)), (z(16), z(16, 24)), (z(1, 3, 16), z(16, 24))):
        for call in (lambda: b.chimera_op_linear_xent_fwd(h, w, z(3, d=i32), 1.0, z(3), z(3), workspace=ws),
                     lambda: b.chimera_op_linear_xent_bwd(h, w, z(3, d=i32), z(3), 1.0, dh=z(*h.shape), dw=z(*w.shape), workspace=ws),
                     lambda: b.chimera_head_loss_pieces(h, z(3, d=i32), z(16), z(16), w, 1.0, z(*h.shape), z(16), z(16), z(16, 24), z(1), workspace=ws)):
            with pytest.raises(ValueError, match="a row for each column"):
                call()


def test_grad_norm_refuses_results_that_lie_apart(monkeypatch):
    torch = pytest.importorskip("torch")
    calls = []
    monkeypatch.setattr(b, "_stream_of", lambda *tensors: 0)
    monkeypatch.setattr(b, "lib", lambda: type("Library", (), {"chimera_op_grad_norm": staticmethod(lambda *a: calls.append(a) or b.OK)}))
    with pytest.raises(ValueError, match="contiguous"):
        b.chimera_op_grad_norm([torch.zeros(4)], 1.0, torch.zeros(4)[::2], workspace=torch.zeros(8, dtype=torch.uint8))
    assert not calls


@pytest.mark.parametrize("dtype", ["float16", "float64", "int16", "uint8"])
def test_binding_refuses_other_types(dtype):
    """Two bytes that are not bfloat16 would be taken for it."""
    torch = pytest.importorskip("torch")
    d = getattr(torch, dtype)
    z = lambda *s, d=torch.float32: torch.zeros(s, dtype=d)  # noqa: E731
    i32, ws, h, w = torch.int32, z(8, d=torch.uint8), z(3, 16, d=d), z(16, 24, d=d)
    for call in (lambda: b.chimera_op_linear_xent_fwd(h, w, z(3, d=i32), 1.0, z(3), z(3), workspace=ws),
                 lambda: b.chimera_op_linear_xent_bwd(h, w, z(3, d=i32), z(3), 1.0, dh=z(3, 16, d=d), dw=z(16, 24), workspace=ws),
                 lambda: b.chimera_head_loss_pieces(h, z(3, d=i32), z(16, d=d), z(16, d=d), w, 1.0, z(3, 16, d=d), z(16), z(16), z(16, 24), z(1), workspace=ws)):
        with pytest.raises(ValueError, match="float32 or bfloat16"):
            call()


def test_stage_step_without_its_state_is_the_librarys_error(monkeypatch):
    """Refused like any other missing buffer, not by an attribute that is not there."""
    torch = pytest.importorskip("torch")
    stage = b.Stage.__new__(b.Stage)
    stage.torch, stage.weights = torch, torch.zeros(64)
    stage.handle = b.lib().chimera_stage_create(1, 64, 4, 16, 2, b.BF16)
    b.check(b.lib().chimera_stage_set_option(stage.handle, b.OPT_OVERLAP, 0))
    b.check(b.lib().chimera_stage_bind(stage.handle, P, P, P, 1, P, None))
    with pytest.raises(b.ChimeraError, match="NULL") as e:
        stage.adamw_step(1e-3, 1)
    assert e.value.code == b.EINVAL
    stage.close()
