"""Binding of the operators around the delta-rule layers (``include/hagdn.h``):
the gated linear recurrence and the norms before and after a block.

    h, final = glr_prefill(x, g, initial_state=None, cu_seqlens=None, convex=False, preprocess=0)
    dx, dg, ds0 = glr_backward(dh, x, g, checkpoints, initial_state=None, dfinal=None, cu_seqlens=None)
    h = glr_decode(x1, g1, state_pool, slots=None)
    y, res = add_norm(x, weight, residual=None, scale=1.0, post_weight=None)
    y = gate_norm(o, z, weight, activation="silu")

Layouts: x, g, dh [T, D] (glr_decode: [N, D]); norms' rows [T, D]; o, z [T, H, d].
Inputs may be column slices of a wider matrix (rows of contiguous elements at any
row stride); outputs are contiguous.  bf16 or fp32, the gate and the residual
stream fp32 or the operands' type; states, weights and their gradients fp32.
"""

from __future__ import annotations

import torch

from . import (HAGDN_BF16, HAGDN_F32, HagdnError, _check_buffer, _err, _ptr, _raw_stream,
               load_library)

_F32 = torch.float32
_ACTIVATIONS = {"silu": 0, "sigmoid": 1}
_CODES = {torch.bfloat16: HAGDN_BF16, torch.float32: HAGDN_F32}


def _check(rc):
    if rc != 0:
        raise HagdnError(rc, _err(load_library()))


def _alike(t, shape, di):
    """Whether a tensor is contiguous, of this shape and on this GPU: the common case of
    every check below, told without building its message."""
    return t.get_device() == di and t.shape == shape and t.is_contiguous() and di >= 0


def _code(name, t, like=None):
    """The dtype code of a tensor; with ``like``, fp32 or that tensor's type."""
    code = _CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be torch.bfloat16 or torch.float32 (got {t.dtype})")
    if like is not None and code == HAGDN_BF16 and like.dtype != torch.bfloat16:
        raise TypeError(f"{name} may be torch.bfloat16 only beside bfloat16 operands")
    return code


def _rows(name, t, shape, di):
    """Row stride in elements of a tensor whose rows (all but the first dimension)
    are contiguous; checks its device and shape."""
    if _alike(t, shape, di):
        return t.stride(0)
    if t.get_device() != di or di < 0:
        raise ValueError(f"{name} must be on the GPU of the call's first tensor")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")
    inner = 1
    for size, stride in zip(reversed(shape[1:]), reversed(t.stride()[1:])):
        if size != 1 and stride != inner:
            raise ValueError(f"{name} must have contiguous rows (strides {t.stride()})")
        inner *= size
    return t.stride(0)


def _vector(name, t, size, device):
    if t is not None and not (t.dtype is _F32 and _alike(t, (size,), device.index)):
        _check_buffer(name, t, device, torch.float32, (size,))


def _workspace(workspace, size, device):
    if workspace is None:
        return torch.empty(size, dtype=torch.uint8, device=device)
    if workspace.device != device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {device}")
    return workspace


def _bytes(t):
    return t.numel() * t.element_size()


def _output(name, t, shape, dtype, device):
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _check_buffer(name, t, device, dtype, shape)
    return t


def _like(name, t, x):
    """A contiguous output of x's shape and type: t, or a new one."""
    if t is None:
        return torch.empty_like(x) if x.is_contiguous() else torch.empty(x.shape, dtype=x.dtype, device=x.device)
    _check_buffer(name, t, x.device, x.dtype, x.shape)
    return t


# ------------------------------------------------------- gated linear recurrence
def glr_workspace_size(T: int, D: int) -> int:
    """Bytes of workspace glr_prefill and glr_backward need for T tokens of D channels."""
    lib = load_library()
    n = lib.glr_workspace_size(T, D)
    if n == 0:
        raise HagdnError(1, _err(lib))
    return n


def _sequences(cu_seqlens, di):
    """(N, pointer) of the sequence offsets."""
    if cu_seqlens is None:
        return 1, None
    if cu_seqlens.dtype != torch.int32 or cu_seqlens.get_device() != di or not cu_seqlens.is_contiguous() \
            or cu_seqlens.dim() != 1:
        raise TypeError("cu_seqlens must be a contiguous 1-D int32 tensor on the operands' GPU")
    return cu_seqlens.shape[0] - 1, cu_seqlens.data_ptr()


def glr_prefill(x, g, initial_state=None, cu_seqlens=None, convex=False, preprocess=0, output_final_state=True,
                output_checkpoints=False, workspace=None, out=None, final_out=None):
    """Gated linear recurrence h_t = a_t h_{t-1} + w_t x_t over packed sequences, with
    a_t = exp(g_t) (PRE_GATE_SOFTPLUS: g holds raw values, a_t = 1 / (1 + e^g)) and
    w_t = 1, or 1 - a_t where ``convex``.  Returns (h, final state [N, D] fp32 or
    None); with ``output_checkpoints`` also the states that glr_backward takes."""
    lib = load_library()
    di, dev = x.get_device(), x.device
    if x.dim() != 2:
        raise ValueError(f"x must be [T, D] (got {tuple(x.shape)})")
    T, D = shape = x.shape
    xs, gs = _rows("x", x, shape, di), _rows("g", g, shape, di)
    dt, gt = _code("x", x), _code("g", g, x)
    N, cu = _sequences(cu_seqlens, di)
    if initial_state is not None:
        _check_buffer("initial_state", initial_state, dev, torch.float32, (N, D))
    h = _like("out", out, x)
    final = _output("final_out", final_out, (N, D), torch.float32, dev) if output_final_state else None
    saved = torch.empty(((T + 127) // 128, D), dtype=torch.float32, device=dev) if output_checkpoints else None
    ws = _workspace(workspace, glr_workspace_size(T, D) if workspace is None else 0, dev)
    _check(lib.glr_prefill(
        x.data_ptr(), xs, g.data_ptr(), gs, _ptr(initial_state), cu, N, T, D, dt, gt, int(convex), int(preprocess),
        h.data_ptr(), _ptr(final), _ptr(saved), ws.data_ptr(), _bytes(ws), _raw_stream(di)))
    return (h, final, saved) if output_checkpoints else (h, final)


def glr_backward(dh, x, g, checkpoints, initial_state=None, dfinal=None, cu_seqlens=None, convex=False, preprocess=0,
                 workspace=None):
    """Gradients of glr_prefill from that of h (``dh``) and of the final state
    (``dfinal``): (dx, dg, gradient of the initial state, or None without one).
    ``checkpoints`` is what the forward call returned."""
    lib = load_library()
    di, dev = x.get_device(), x.device
    if x.dim() != 2:
        raise ValueError(f"x must be [T, D] (got {tuple(x.shape)})")
    T, D = shape = x.shape
    xs, gs, dhs = _rows("x", x, shape, di), _rows("g", g, shape, di), _rows("dh", dh, shape, di)
    dt, gt = _code("x", x), _code("g", g, x)
    if dh.dtype != x.dtype:
        raise TypeError(f"dh must be {x.dtype} (got {dh.dtype})")
    N, cu = _sequences(cu_seqlens, di)
    _check_buffer("checkpoints", checkpoints, dev, torch.float32, ((T + 127) // 128, D))
    for name, t in (("initial_state", initial_state), ("dfinal", dfinal)):
        if t is not None:
            _check_buffer(name, t, dev, torch.float32, (N, D))
    dx, dg = _like("dx", None, x), _like("dg", None, g)
    ds0 = torch.empty((N, D), dtype=torch.float32, device=dev) if initial_state is not None else None
    ws = _workspace(workspace, glr_workspace_size(T, D) if workspace is None else 0, dev)
    _check(lib.glr_backward(
        dh.data_ptr(), dhs, x.data_ptr(), xs, g.data_ptr(), gs, checkpoints.data_ptr(), _ptr(initial_state),
        _ptr(dfinal), cu, N, T, D, dt, gt, int(convex), int(preprocess), dx.data_ptr(), dg.data_ptr(), _ptr(ds0),
        ws.data_ptr(), _bytes(ws), _raw_stream(di)))
    return dx, dg, ds0


def glr_decode(x, g, state, slots=None, convex=False, preprocess=0, out=None):
    """One token for each of N sequences, x and g [N, D]: updates the fp32 state pool
    [S, D] in place (sequence n in slot slots[n], or n; a slot outside the pool is
    padding and gives a row of zeros) and returns the new states h [N, D]."""
    lib = load_library()
    di, dev = x.get_device(), x.device
    if x.dim() != 2:
        raise ValueError(f"x must be [N, D] (got {tuple(x.shape)})")
    N, D = shape = x.shape
    xs, gs = _rows("x", x, shape, di), _rows("g", g, shape, di)
    dt, gt = _code("x", x), _code("g", g, x)
    if state.dim() != 2:
        raise ValueError(f"state must be [slots, {D}]")
    if not (state.dtype is _F32 and _alike(state, (state.shape[0], D), di)):
        _check_buffer("state", state, dev, _F32, (state.shape[0], D))
    if slots is None:
        if state.shape[0] < N:
            raise ValueError("without slots the state pool needs one state per sequence")
    else:
        _check_buffer("slots", slots, dev, torch.int32, (N,))
    h = _like("out", out, x)
    _check(lib.glr_decode(
        x.data_ptr(), xs, g.data_ptr(), gs, state.data_ptr(), _ptr(slots), state.shape[0], N, D, dt, gt, int(convex),
        int(preprocess), h.data_ptr(), _raw_stream(di)))
    return h


# --------------------------------------------------------------------- norms
def _scale(scale, D, device):
    """(number, vector or None) of a residual scale."""
    if isinstance(scale, torch.Tensor):
        _vector("scale", scale, D, device)
        return 1.0, scale
    return float(scale), None


def add_norm(x, weight, residual=None, scale=1.0, post_weight=None, eps=1e-6, out=None, residual_out=None):
    """A block's output x [T, D] joins the residual stream and the next block's input
    is normed: r = residual + scale * u with u = x, or norm(x) * post_weight;
    y = norm(r) * weight.  ``scale``: a number or fp32 [D].  Returns (y, r), r in the
    residual's type (x's without one); ``residual_out`` may be the residual itself."""
    lib = load_library()
    di, dev = x.get_device(), x.device
    if x.dim() != 2:
        raise ValueError(f"x must be [T, D] (got {tuple(x.shape)})")
    T, D = shape = x.shape
    xs, dt = _rows("x", x, shape, di), _code("x", x)
    rs, rt, rdtype = 0, dt, x.dtype
    if residual is not None:
        rs, rt, rdtype = _rows("residual", residual, shape, di), _code("residual", residual, x), residual.dtype
    elif residual_out is not None:
        rt, rdtype = _code("residual_out", residual_out, x), residual_out.dtype
    _vector("weight", weight, D, dev)
    _vector("post_weight", post_weight, D, dev)
    number, vector = _scale(scale, D, dev)
    y = _like("out", out, x)
    if residual_out is None and residual is not None:
        r = _like("residual_out", None, residual)
    else:
        r = _output("residual_out", residual_out, shape, rdtype, dev)
    _check(lib.hagdn_add_norm(
        x.data_ptr(), xs, _ptr(residual), rs, weight.data_ptr(), _ptr(post_weight), _ptr(vector), number, eps, T, D,
        dt, rt, y.data_ptr(), r.data_ptr(), _raw_stream(di)))
    return y, r


def add_norm_backward(dy, res, weight, dresidual=None, x=None, scale=1.0, post_weight=None, eps=1e-6, workspace=None):
    """Gradients of add_norm from those of y (``dy``) and of the stream it returned
    (``dresidual``, None: zero).  ``res`` is that stream; x is needed with a scale
    vector or post_weight.  Returns (dx, gradient of the residual, of weight, of
    the scale vector or None, of post_weight or None)."""
    lib = load_library()
    di, dev = dy.get_device(), dy.device
    if dy.dim() != 2:
        raise ValueError(f"dy must be [T, D] (got {tuple(dy.shape)})")
    T, D = shape = dy.shape
    number, vector = _scale(scale, D, dev)
    _vector("post_weight", post_weight, D, dev)
    _vector("weight", weight, D, dev)
    dys, rs, dt, rt = _rows("dy", dy, shape, di), _rows("res", res, shape, di), _code("dy", dy), _code("res", res, dy)
    drs = xs = 0
    if dresidual is not None:
        if dresidual.dtype != res.dtype:
            raise TypeError(f"dresidual must be {res.dtype} (got {dresidual.dtype})")
        drs = _rows("dresidual", dresidual, shape, di)
    reads_x = vector is not None or post_weight is not None
    if reads_x:
        if x is None:
            raise ValueError("x is needed with a scale vector or post_weight")
        if x.dtype != dy.dtype:
            raise TypeError(f"x must be {dy.dtype} (got {x.dtype})")
        xs = _rows("x", x, shape, di)
    dx, dres = _like("dx", None, dy), _like("dres", None, res)
    grads = torch.empty((1 + (vector is not None) + (post_weight is not None), D), dtype=torch.float32, device=dev)
    dw, dscale = grads[0], grads[1] if vector is not None else None
    dpost = grads[-1] if post_weight is not None else None
    ws = _workspace(workspace, lib.hagdn_add_norm_workspace_size(T, D, vector is not None, post_weight is not None)
                    if workspace is None else 0, dev)
    _check(lib.hagdn_add_norm_backward(
        dy.data_ptr(), dys, _ptr(dresidual), drs, res.data_ptr(), rs, x.data_ptr() if reads_x else None, xs,
        weight.data_ptr(), _ptr(post_weight), _ptr(vector), number, eps, T, D, dt, rt, dx.data_ptr(), dres.data_ptr(),
        dw.data_ptr(), _ptr(dscale), _ptr(dpost), ws.data_ptr(), _bytes(ws), _raw_stream(di)))
    return dx, dres, dw, dscale, dpost


def _activation(name):
    if name not in _ACTIVATIONS:
        raise ValueError(f"activation must be one of {sorted(_ACTIVATIONS)} (got {name!r})")
    return _ACTIVATIONS[name]


def gate_norm(o, z, weight, activation="silu", eps=1e-6, out=None):
    """The norm and gate between a mixer and its output projection, per token and
    head: norm(o) * weight * act(z), o and z [T, H, d], weight fp32 [d]."""
    lib = load_library()
    di, dev = o.get_device(), o.device
    if o.dim() != 3:
        raise ValueError(f"o must be [T, H, d] (got {tuple(o.shape)})")
    T, H, d = shape = o.shape
    os_, zs, dt = _rows("o", o, shape, di), _rows("z", z, shape, di), _code("o", o)
    if z.dtype != o.dtype:
        raise TypeError(f"z must be {o.dtype} (got {z.dtype})")
    _vector("weight", weight, d, dev)
    y = _like("out", out, o)
    _check(lib.hagdn_gate_norm(
        o.data_ptr(), os_, z.data_ptr(), zs, weight.data_ptr(), eps, T, H, d, dt, _activation(activation),
        y.data_ptr(), _raw_stream(di)))
    return y


def gate_norm_backward(dy, o, z, weight, activation="silu", eps=1e-6, workspace=None):
    """Gradients of gate_norm: (do, dz, gradient of weight)."""
    lib = load_library()
    di, dev = o.get_device(), o.device
    if o.dim() != 3:
        raise ValueError(f"o must be [T, H, d] (got {tuple(o.shape)})")
    T, H, d = shape = o.shape
    os_, zs, dys = _rows("o", o, shape, di), _rows("z", z, shape, di), _rows("dy", dy, shape, di)
    dt = _code("o", o)
    for name, t in (("z", z), ("dy", dy)):
        if t.dtype != o.dtype:
            raise TypeError(f"{name} must be {o.dtype} (got {t.dtype})")
    _vector("weight", weight, d, dev)
    act = _activation(activation)
    do, dz = _like("do", None, o), _like("dz", None, z)
    dw = torch.empty(d, dtype=torch.float32, device=dev)
    ws = _workspace(workspace, lib.hagdn_gate_norm_workspace_size(T, H, d) if workspace is None else 0, dev)
    _check(lib.hagdn_gate_norm_backward(
        dy.data_ptr(), dys, o.data_ptr(), os_, z.data_ptr(), zs, weight.data_ptr(), eps, T, H, d, dt, act,
        do.data_ptr(), dz.data_ptr(), dw.data_ptr(), ws.data_ptr(), _bytes(ws), _raw_stream(di)))
    return do, dz, dw
