"""The differentiable forms have first derivatives only: a second one raises instead of
leaving its terms out.  On the CPU with plain stand-ins for the kernels, whose results carry
no graph as the kernels' do not; on the GPU with the kernels."""

import pytest
import torch

from paper_2609_32114_amd import autograd, layer


def _norm(x, eps):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)


def _gate(o, z, w, activation, eps):
    s = torch.sigmoid(z)
    return _norm(o, eps) * w * (z * s if activation == "silu" else s)


def _add(x, w, res, scale, post, eps):
    r = (0 if res is None else res) + scale * (x if post is None else _norm(x, eps) * post)
    return _norm(r, eps) * w, r


def _glr(x, g, s0):
    s, hs = torch.zeros_like(x[:1]) if s0 is None else s0, []
    for t in range(x.shape[0]):
        s = g[t].exp() * s + x[t]
        hs.append(s[0])
    return torch.stack(hs), s


def _grads(f, args, seeds):
    """f's gradients at the tensors among args, without a graph."""
    with torch.enable_grad():
        at = [a.detach().requires_grad_() if isinstance(a, torch.Tensor) else a for a in args]
        outs = f(*at)
        outs = outs if isinstance(outs, tuple) else (outs,)
        pairs = [(o, s) for o, s in zip(outs, seeds) if s is not None]
        return iter(torch.autograd.grad([o for o, _ in pairs], [a for a in at if isinstance(a, torch.Tensor)],
                                        [s.detach() for _, s in pairs], allow_unused=True))


@pytest.fixture
def stand_ins(monkeypatch):
    @torch.no_grad()
    def add_norm(x, w, residual, scale, post_weight, eps):
        return _add(x, w, residual, scale, post_weight, eps)

    def add_norm_backward(dy, res, w, dres, x, scale, post, eps):
        # from r' alone: enough for a scale without post weight
        dr, dw = _grads(lambda r, w: (_norm(r, eps) * w, r), (res, w), (dy, dres))
        ds = (dr * x).sum(0) if isinstance(scale, torch.Tensor) else None
        return (dr * scale).detach(), dr, dw, ds, None

    def gate_norm_backward(dy, o, z, w, activation, eps):
        return tuple(_grads(lambda *a: _gate(*a, activation, eps), (o, z, w), (dy,)))

    def glr_backward(dh, x, g, saved, s0, dfinal, cu, convex, preprocess, workspace):
        d = _grads(_glr, (x, g, s0), (dh, dfinal))
        return next(d), next(d), None if s0 is None else next(d)

    monkeypatch.setattr(layer, "gate_norm", torch.no_grad()(_gate))
    monkeypatch.setattr(layer, "gate_norm_backward", gate_norm_backward)
    monkeypatch.setattr(layer, "add_norm", add_norm)
    monkeypatch.setattr(layer, "add_norm_backward", add_norm_backward)
    monkeypatch.setattr(layer, "glr_prefill", torch.no_grad()(
        lambda x, g, s0, cu, convex, pre, output_checkpoints, workspace: _glr(x, g, s0) + (torch.zeros(1, x.shape[1]),)))
    monkeypatch.setattr(layer, "glr_backward", glr_backward)
    return "cpu"


def _cases(dev):
    gen = torch.Generator().manual_seed(1)
    leaf = lambda *s: torch.randn(*s, generator=gen).to(dev).requires_grad_()
    x, r, w, v = leaf(6, 8), leaf(6, 8), leaf(8), leaf(8)
    o, z, u = leaf(6, 2, 4), leaf(6, 2, 4), leaf(4)
    g, s0 = (-torch.rand(6, 8, generator=gen)).to(dev).requires_grad_(), leaf(1, 8)
    return {"glr": ((x, g, s0), lambda: autograd.glr(x, g, s0)[0]),
            "glr, final state": ((x, g), lambda: autograd.glr(x, g)[1]),
            "add_norm": ((x, r, w), lambda: autograd.add_norm(x, w, residual=r, scale=0.5)[0]),
            "add_norm, vector": ((x, r, w, v), lambda: autograd.add_norm(x, w, residual=r, scale=v)[0]),
            "gate_norm": ((o, z, u), lambda: autograd.gate_norm(o, z, u, "sigmoid"))}


NAMES = list(_cases("cpu"))


def _check(name, dev):
    leaves, f = _cases(dev)[name]
    for loss in (lambda y: y.sum(), lambda y: (y * y).sum()):  # the gradient that comes in: without a graph, with one
        plain = torch.autograd.grad(loss(f()), leaves)
        first = torch.autograd.grad(loss(f()), leaves, create_graph=True)
        assert all(torch.equal(a, b) for a, b in zip(plain, first))
        penalty = sum((d * d).sum() for d in first) + sum((p ** 3).sum() for p in leaves)
        with pytest.raises(RuntimeError, match="second derivative"):
            penalty.backward()


@pytest.mark.parametrize("name", NAMES)
def test_second_derivatives_are_refused(name, stand_ins):
    _check(name, stand_ins)


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_second_derivatives_of_the_kernels_are_refused(name):
    _check(name, "cuda")
