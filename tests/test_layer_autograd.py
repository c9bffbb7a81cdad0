"""The differentiable forms and the example that runs the operators together, on the GPU."""

import os
import sys

import numpy as np
import pytest

import layer_ref as ref
from gpu_harness import say

pytestmark = pytest.mark.gpu


def _inputs(*shapes, seed=0):
    import torch
    gen = torch.Generator().manual_seed(seed)
    return [torch.randn(*s, generator=gen).cuda().requires_grad_() for s in shapes]


def _inside(got, want, label):
    off = ref.excess(got, want, "f32")
    say(f"[autograd] {label}: {off:.3f}")
    assert off <= 1.0, label


def test_glr_gradients():
    """Through a loss of h and the final state, from operands that are slices of one matrix."""
    import torch
    from paper_2609_32114_amd import autograd
    lens, D = (70, 0, 200), 96
    (wide, s0, dh, df) = _inputs((270, 2 * D), (3, D), (270, D), (3, D))
    cu = torch.tensor([0, 70, 70, 270], dtype=torch.int32, device="cuda")
    h, final = autograd.glr(wide[:, :D], wide[:, D:], s0, cu, convex=True, preprocess=2)
    ((h * dh.detach()).sum() + (final * df.detach()).sum()).backward()
    n = lambda t: t.detach().double().cpu().numpy()
    want = ref.glr(n(wide)[:, :D], n(wide)[:, D:], lens, n(s0), True, True, n(dh), n(df))
    _inside(wide.grad[:, :D], want["dx"], "dx")
    _inside(wide.grad[:, D:], want["dg"], "dg")
    _inside(s0.grad, want["ds0"], "ds0")


def test_glr_partial_gradients():
    """Only the final state reaches the loss, or only h, as an expanded gradient."""
    import torch
    from paper_2609_32114_amd import autograd
    x, g = _inputs((50, 64), (50, 64))
    n = lambda t: t.detach().double().cpu().numpy()
    _, final = autograd.glr(x, -g.abs())
    final.sum().backward()
    gd = n(-g.abs())
    want = ref.glr(n(x), gd, (50,), None, False, False, np.zeros((50, 64)), np.ones((1, 64)))
    _inside(x.grad, want["dx"], "dx of the final state")
    x.grad = None
    h, _ = autograd.glr(x, -g.abs())
    h.sum().backward()
    want = ref.glr(n(x), gd, (50,), None, False, False, np.ones((50, 64)), None)
    _inside(x.grad, want["dx"], "dx of h's sum")
    assert torch.isfinite(g.grad).all()


@pytest.mark.parametrize("post", [False, True])
def test_norm_gradients_join_the_stream(post):
    """Two blocks' add_norm on one stream: the gradient that reaches it comes from both."""
    import torch
    from paper_2609_32114_amd import autograd
    x1, x2, res, w, s, p = _inputs((20, 200), (20, 200), (20, 200), (200,), (200,), (200,))
    args = (x1, x2, res, w, s, p)
    y1, r1 = autograd.add_norm(x1, w, residual=res, scale=s, post_weight=p if post else None, eps=1e-3)
    y2, r2 = autograd.add_norm(x2, w, residual=r1, scale=0.5, eps=1e-3)
    (y1.sum() + (y2 * y2).sum() + r2.sin().sum()).backward()
    d = [a.detach().double().requires_grad_() for a in args]

    def plain(x, res, scale, pw):
        norm = lambda v: v * torch.rsqrt((v * v).mean(-1, keepdim=True) + 1e-3)
        r = res + scale * (norm(x) * pw if pw is not None else x)
        return norm(r) * d[3], r

    a1, b1 = plain(d[0], d[2], d[4], d[5] if post else None)
    a2, b2 = plain(d[1], b1, 0.5, None)
    (a1.sum() + (a2 * a2).sum() + b2.sin().sum()).backward()
    for i, (got, want) in enumerate(zip(args, d)):
        if want.grad is None:
            assert got.grad is None
            continue
        # two norms of 200 elements forward and back: some 100 roundings of the gradient's size
        assert (got.grad - want.grad).norm() <= 100 * ref.EPS * want.grad.norm(), i


def test_norm_of_an_unused_output():
    """Only the stream reaches the loss: the gradient passes the norm by, in x's type."""
    import torch
    from paper_2609_32114_amd import autograd
    x = torch.randn(9, 64, device="cuda").bfloat16().requires_grad_()
    res = torch.randn(9, 64, device="cuda", requires_grad=True)
    w = torch.ones(64, device="cuda", requires_grad=True)
    _, r = autograd.add_norm(x, w, residual=res, scale=0.5)
    r.sum().backward()
    assert x.grad.dtype == torch.bfloat16 and bool((x.grad == 0.5).all())
    assert bool((res.grad == 1).all()) and bool((w.grad == 0).all())


def test_gate_norm_gradients():
    import torch
    from paper_2609_32114_amd import autograd
    o, z, w = _inputs((30, 4, 64), (30, 4, 64), (64,))
    y = autograd.gate_norm(o, z, w, "sigmoid", 1e-3)
    y.pow(2).sum().backward()
    n = lambda t: t.detach().double().cpu().numpy()
    od, zd, dyd = n(o).reshape(-1, 64), n(z).reshape(-1, 64), 2 * n(y).reshape(-1, 64)
    want = ref.gate_norm(od, zd, n(w), False, 1e-3, dyd)
    _inside(o.grad, want["do"], "do")
    _inside(z.grad, want["dz"], "dz")
    _inside(w.grad, want["dw"], "dw")


def test_example_learns_and_serves():
    """The example's stack learns to copy (its loss starts at log 16 = 2.8 or above and
    falls below half of that), and tokens served one at a time agree with one prefill within
    a few bf16 roundings of the largest logit."""
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import recurrent_stack
    losses, stepped, whole = recurrent_stack.main(["--steps", "120"])
    say(f"[example] loss {losses[0]:.3f} -> {losses[-1]:.3f}")
    assert losses[0] > 2.5 and losses[-1] < 0.5 * np.log(16)
    assert float((stepped - whole).abs().max()) <= 16 * 2.0 ** -8 * float(whole.abs().max())


def test_norm_after_a_delta_rule_mixer():
    """gdn_prefill's output through gate_norm, its gate a slice of the projection: the layer's
    order of calls, against the same in 64 bits from the mixer's own output."""
    import torch
    import paper_2609_32114_amd as P
    gen = torch.Generator(device="cuda").manual_seed(3)
    T, H, d = 300, 4, 128
    q, k, v = (torch.randn(T, H, d, generator=gen, device="cuda") for _ in range(3))
    q, k = (torch.nn.functional.normalize(t, dim=-1).bfloat16() for t in (q, k))
    g = -torch.rand(T, H, generator=gen, device="cuda")
    beta = torch.rand(T, H, generator=gen, device="cuda")
    wide = torch.randn(T, 3 * H * d, generator=gen, device="cuda").bfloat16()
    z = wide[:, H * d:2 * H * d].unflatten(1, (H, d))
    w = torch.rand(d, generator=gen, device="cuda") + 0.5
    o, _ = P.gdn_prefill(q, k, v.bfloat16(), g, beta, scale=d ** -0.5)
    y = P.gate_norm(o, z, w)
    rows = lambda t: t.double().cpu().numpy().reshape(-1, d)
    want = ref.gate_norm(rows(o), rows(z), w.double().cpu().numpy(), True, 1e-6)
    assert ref.excess(y, want["y"], "bf16") <= 1.0


def test_glr_device_status():
    """Malformed offsets show in the status of the caller's workspace, after either direction."""
    import torch
    import paper_2609_32114_amd as P
    from paper_2609_32114_amd import autograd
    T, D = 700, 70
    x, g = _inputs((T, D), (T, D))
    ws = torch.full((P.glr_workspace_size(T, D),), 0xFF, dtype=torch.uint8, device="cuda")
    for last, code in ((T - 1, P.DEV_BAD_SEQLENS), (T, P.DEV_OK)):
        cu = torch.tensor([0, 300, last], dtype=torch.int32, device="cuda")
        h, final = autograd.glr(x, g, cu_seqlens=cu, workspace=ws)
        assert P.device_status(ws) == code
        ws.fill_(0xFF)
        final.sum().backward()
        assert P.device_status(ws) == code
