"""The refusals of the recurrence's and the norms' entry points, which need no GPU:
bad arguments are turned down on the host before anything is enqueued (fake,
never-dereferenced device pointers), and by the binding."""

import ctypes
import os

import pytest
import torch

import paper_2609_32114_amd as P

pytestmark = pytest.mark.skipif(not os.path.exists(P.library_path()), reason="libhagdn.so not built")

OK, EINVAL, EUNSUP, EWS = 0, 1, 2, 3
F = 0x100000  # 16-byte aligned, never dereferenced
BIG = 1 << 40


def call(fn, defaults, **over):
    args = dict(defaults)
    assert set(over) <= set(args), set(over) - set(args)
    args.update(over)
    lib = P.load_library()
    rc = getattr(lib, fn)(*args.values())
    return rc, lib.hagdn_last_error().decode()


PREFILL = dict(x=F, xs=64, g=F, gs=64, s0=None, cu=F, N=2, T=10, D=64, dtype=1, gate=0, convex=0, pre=0, h=F, sf=None,
               ck=None, ws=F, wsb=64, stream=None)  # the workspace is too small: a valid call stops there
BACKWARD = dict(dh=F, dhs=64, x=F, xs=64, g=F, gs=64, ck=F, s0=None, df=None, cu=F, N=2, T=10, D=64, dtype=1, gate=0,
                convex=0, pre=0, dx=F, dg=F, ds0=None, ws=F, wsb=BIG, stream=None)
DECODE = dict(x=F, xs=64, g=F, gs=64, state=F, slots=None, pool=0, N=3, D=64, dtype=1, gate=0, convex=0, pre=0, h=F,
              stream=None)
ADD = dict(x=F, xs=64, res=F, rs=64, w=F, post=None, vec=None, scale=1.0, eps=1e-6, T=5, D=64, dtype=1, rt=0, y=F, out=F,
           stream=None)
ADD_BACK = dict(dy=F, dys=64, dres=F, drs=64, res=F, rs=64, x=F, xs=64, w=F, post=F, vec=F, scale=1.0, eps=1e-6, T=5,
                D=64, dtype=1, rt=0, dx=F, dro=F, dw=F, ds=F, dp=F, ws=F, wsb=64, stream=None)
GATE = dict(o=F, os=64, z=F, zs=64, w=F, eps=1e-6, T=5, H=1, d=64, dtype=1, act=0, y=F, stream=None)
GATE_BACK = dict(dy=F, dys=64, o=F, os=64, z=F, zs=64, w=F, eps=1e-6, T=5, H=1, d=64, dtype=1, act=0, do=F, dz=F, dw=F,
                 ws=F, wsb=64, stream=None)


def test_valid_calls_reach_the_workspace_check():
    for fn, d in (("glr_prefill", PREFILL), ("hagdn_add_norm_backward", ADD_BACK), ("hagdn_gate_norm_backward", GATE_BACK)):
        rc, msg = call(fn, d)
        assert rc == EWS and "workspace too small" in msg


@pytest.mark.parametrize("fn,d", [("glr_prefill", PREFILL), ("glr_backward", BACKWARD)], ids=["prefill", "backward"])
def test_glr_refusals(fn, d):
    for over in (dict(N=0), dict(T=-1), dict(D=0), dict(convex=2), dict(pre=1), dict(pre=4), dict(pre=8), dict(x=None),
                 dict(g=None), dict(ws=None), dict(ws=F + 8), dict(cu=None), dict(cu=F + 2), dict(xs=-1), dict(gs=1 << 31),
                 dict(x=F + 1), dict(g=F + 2), dict(N=1 << 20, D=1 << 12), dict(s0=F + 2)):
        assert call(fn, d, **{"wsb": BIG, **over})[0] == EINVAL, over
    for over in (dict(dtype=2), dict(gate=3), dict(dtype=0, gate=1), dict(N=1, D=(1 << 28) + 1)):
        assert call(fn, d, **{"wsb": BIG, **over})[0] == EUNSUP, over
    outs = dict(h=None) if fn == "glr_prefill" else dict(dx=None)
    assert call(fn, d, **{"wsb": BIG, **outs})[0] == EINVAL
    assert call(fn, d, wsb=0)[0] == EWS


def test_glr_aliases():
    assert call("glr_prefill", PREFILL, wsb=BIG, s0=F, sf=F + 64)[0] == EINVAL
    assert call("glr_backward", BACKWARD, df=F, ds0=F + 64)[0] == EINVAL
    assert call("glr_backward", BACKWARD, ck=None)[0] == EINVAL
    assert call("glr_backward", BACKWARD, dh=None)[0] == EINVAL
    assert call("glr_backward", BACKWARD, dhs=-5)[0] == EINVAL


def test_glr_workspace_size():
    lib = P.load_library()
    assert P.glr_workspace_size(0, 1) > 0
    assert P.glr_workspace_size(100000, 2048) >= P.glr_workspace_size(1000, 2048)
    assert lib.glr_workspace_size(-1, 64) == 0 and lib.glr_workspace_size(64, 0) == 0
    with pytest.raises(P.HagdnError):
        P.glr_workspace_size(5, 0)


def test_glr_decode_refusals():
    for over in (dict(N=-1), dict(D=0), dict(x=None), dict(g=None), dict(state=None), dict(h=None), dict(slots=F, pool=0),
                 dict(slots=F + 1, pool=4), dict(state=F + 2), dict(pre=1), dict(convex=-1), dict(xs=-1)):
        assert call("glr_decode", DECODE, **over)[0] == EINVAL, over
    assert call("glr_decode", DECODE, dtype=0, gate=1)[0] == EUNSUP
    assert call("glr_decode", DECODE, N=0, x=None)[0] == OK  # a no-op


def test_add_norm_refusals():
    for over in (dict(T=-1), dict(D=0), dict(x=None), dict(w=None), dict(y=None), dict(eps=-1.0), dict(eps=float("nan")),
                 dict(eps=float("inf")), dict(x=F + 1), dict(w=F + 2), dict(rs=-1), dict(res=F, out=F, rs=65)):
        assert call("hagdn_add_norm", ADD, **over)[0] == EINVAL, over
    for over in (dict(D=16385), dict(dtype=0, rt=1), dict(dtype=9), dict(rt=7)):
        assert call("hagdn_add_norm", ADD, **over)[0] == EUNSUP, over
    assert call("hagdn_add_norm", ADD, T=0, x=None, y=None)[0] == OK


def test_add_norm_backward_refusals():
    for over in (dict(dy=None), dict(res=None), dict(x=None), dict(dx=None), dict(dw=None), dict(ds=None), dict(dp=None),
                 dict(ws=None), dict(dres=F, dro=F, drs=99), dict(T=-1), dict(eps=-0.1)):
        assert call("hagdn_add_norm_backward", ADD_BACK, **{"wsb": BIG, **over})[0] == EINVAL, over
    assert call("hagdn_add_norm_backward", ADD_BACK, wsb=BIG, D=20000)[0] == EUNSUP
    lib = P.load_library()
    a, b = (lib.hagdn_add_norm_workspace_size(100, 64, v, v) for v in (0, 1))
    assert 0 < a < b and lib.hagdn_add_norm_workspace_size(1, 0, 0, 0) == 0


def test_gate_norm_refusals():
    for over in (dict(o=None), dict(z=None), dict(w=None), dict(y=None), dict(H=0), dict(H=-3), dict(d=0), dict(T=-1),
                 dict(act=2), dict(eps=-1.0), dict(T=1 << 20, H=1 << 12), dict(os=-1), dict(z=F + 1)):
        assert call("hagdn_gate_norm", GATE, **over)[0] == EINVAL, over
    assert call("hagdn_gate_norm", GATE, d=16385)[0] == EUNSUP and call("hagdn_gate_norm", GATE, dtype=4)[0] == EUNSUP
    for over in (dict(dy=None), dict(do=None), dict(dz=None), dict(dw=None), dict(ws=None), dict(dys=-1)):
        assert call("hagdn_gate_norm_backward", GATE_BACK, **{"wsb": BIG, **over})[0] == EINVAL, over
    assert P.load_library().hagdn_gate_norm_workspace_size(0, 1, 64) > 0


def test_binding_refusals():
    """Tensors of other devices, types and shapes are named before the library is called."""
    x = torch.zeros(4, 8)
    w = torch.ones(8)
    for fn in (lambda: P.glr_prefill(x, x), lambda: P.glr_backward(x, x, x, x), lambda: P.glr_decode(x, x, x),
               lambda: P.add_norm(x, w), lambda: P.add_norm_backward(x, x, w), lambda: P.gate_norm(x.view(4, 2, 4),
                                                                                                 x.view(4, 2, 4), w)):
        with pytest.raises(ValueError):
            fn()


def _cuda(call, error, match):
    with pytest.raises(error, match=match):
        call()


@pytest.mark.gpu
def test_binding_refusals_on_the_gpu():
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")
    x, w = z(4, 8), z(8)
    b = z(4, 8, dt=torch.bfloat16)
    _cuda(lambda: P.glr_prefill(z(4, 8, dt=torch.float16), x), TypeError, "x must be")
    _cuda(lambda: P.glr_prefill(x, b), TypeError, "g may be")
    _cuda(lambda: P.glr_prefill(x, z(4, 9)), ValueError, "g must have shape")
    _cuda(lambda: P.glr_prefill(z(8, 4).t(), x), ValueError, "contiguous rows")
    _cuda(lambda: P.glr_prefill(x, x.cpu()), ValueError, "g must be on")
    _cuda(lambda: P.glr_prefill(x, x, cu_seqlens=z(3)), TypeError, "cu_seqlens")
    _cuda(lambda: P.glr_prefill(x, x, initial_state=z(2, 8)), ValueError, "initial_state")
    _cuda(lambda: P.glr_prefill(x, x, out=b), TypeError, "out")
    _cuda(lambda: P.glr_prefill(x, x, workspace=z(4).to(torch.uint8)), P.HagdnError, "workspace too small")
    _cuda(lambda: P.glr_prefill(x, x, preprocess=P.PRE_ALL), P.HagdnError, "preprocessing")
    _cuda(lambda: P.glr_backward(b, x, x, z(1, 8)), TypeError, "dh must be")
    _cuda(lambda: P.glr_backward(x, x, x, z(2, 8)), ValueError, "checkpoints")
    _cuda(lambda: P.glr_decode(x, x, z(3, 8)), ValueError, "one state per sequence")
    _cuda(lambda: P.glr_decode(x, x, z(4, 8), slots=z(4)), TypeError, "slots")
    _cuda(lambda: P.add_norm(x, z(9)), ValueError, "weight")
    _cuda(lambda: P.add_norm(x, w, scale=z(7)), ValueError, "scale")
    _cuda(lambda: P.add_norm(x, w, residual=b), TypeError, "residual may be")
    _cuda(lambda: P.add_norm(x, w, eps=-1.0), P.HagdnError, "eps")
    _cuda(lambda: P.add_norm_backward(x, x, w, scale=w), ValueError, "x is needed")
    _cuda(lambda: P.add_norm_backward(x, x, w, dresidual=b), TypeError, "dresidual")
    _cuda(lambda: P.gate_norm(x.view(4, 2, 4), b.view(4, 2, 4), z(4)), TypeError, "z must be")
    _cuda(lambda: P.gate_norm(x.view(4, 2, 4), x.view(4, 2, 4), z(4), activation="relu"), ValueError, "activation")
    _cuda(lambda: P.gate_norm(x, x, w), ValueError, "o must be")


def test_glr_workspace_holds_what_a_call_uses():
    """A header; beyond 128 tokens a counter's memory line per 64 channels, and a word per
    channel of each tile, which has 128 tokens at least where a call has several."""
    for T in (0, 1, 64, 65, 128, 129, 256, 1000, 32768, 100000):
        for D in (1, 64, 65, 2048, 1 << 20):
            tiles = (T + 127) // 128
            want = 256 + ((D + 63) // 64 * 128 + tiles * D * 8 if tiles > 1 else 0)
            assert P.glr_workspace_size(T, D) == want, (T, D)
