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

_F32, _BF16 = torch.float32, torch.bfloat16
_ACTIVATIONS = {"silu": 0, "sigmoid": 1}
# the codes of the operands' type and of a second one, the gate's or the stream's
_TYPES = {(_BF16, _BF16): (HAGDN_BF16, HAGDN_BF16), (_BF16, _F32): (HAGDN_BF16, HAGDN_F32),
          (_F32, _F32): (HAGDN_F32, HAGDN_F32)}
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _raw_stream)  # of a device, as an int


def _check(rc):
    if rc != 0:
        raise HagdnError(rc, _err(load_library()))


def _types(name, t, other_name, other):
    """The dtype codes of the operands t and of a tensor that may also be fp32 beside bf16."""
    codes = _TYPES.get((t.dtype, other.dtype))
    if codes is None:
        if t.dtype not in (_BF16, _F32):
            raise TypeError(f"{name} must be torch.bfloat16 or torch.float32 (got {t.dtype})")
        if other.dtype is _BF16:
            raise TypeError(f"{other_name} may be torch.bfloat16 only beside bfloat16 operands")
        raise TypeError(f"{other_name} must be torch.bfloat16 or torch.float32 (got {other.dtype})")
    return codes


def _same_type(name, t, dtype):
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")


def _matrix(name, t, what):
    """The shape and device index of a call's first tensor."""
    shape = t.shape
    if len(shape) != 2:
        raise ValueError(f"{name} must be {what} (got {tuple(shape)})")
    return shape, t.get_device()


def _rows(name, t, shape, di):
    """Row stride in elements of a matrix [T, D] or heads [T, H, d] whose rows (all but the
    first dimension) are contiguous; checks its device and shape."""
    if t.get_device() != di or di < 0:
        raise ValueError(f"{name} must be on the GPU of the call's first tensor")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")
    s = t.stride()
    if s[-1] != 1 and shape[-1] != 1 or len(s) == 3 and s[1] != shape[2] and shape[1] != 1:
        if not t.is_contiguous():  # (a tensor without elements is)
            raise ValueError(f"{name} must have contiguous rows (strides {s})")
    return s[0]


def _fp32(name, t, shape, x):
    """Checks a contiguous fp32 tensor beside x."""
    if not (t.dtype is _F32 and t.shape == shape and t.get_device() == x.get_device() and t.is_contiguous()):
        _check_buffer(name, t, x.device, _F32, shape)


def _workspace(workspace, size, x):
    """(tensor, bytes) of a call's workspace: the caller's, or a new one of size() bytes."""
    if workspace is None:
        n = size()
        return x.new_empty(n, dtype=torch.uint8), n
    if workspace.get_device() != x.get_device() or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {x.device}")
    return workspace, workspace.numel() * workspace.element_size()


def _output(name, t, shape, dtype, x):
    if t is None:
        return x.new_empty(shape, dtype=dtype)
    _check_buffer(name, t, x.device, dtype, shape)
    return t


def _like(name, t, x):
    """A contiguous output of x's shape and type: t, or a new one."""
    if t is None:
        return torch.empty_like(x) if x.is_contiguous() else x.new_empty(x.shape)
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


def _groups(T):
    """Saved states of T tokens: one for every 128."""
    return (T + 127) // 128


def glr_prefill(x, g, initial_state=None, cu_seqlens=None, convex=False, preprocess=0, output_final_state=True,
                output_checkpoints=False, workspace=None, out=None, final_out=None):
    """Gated linear recurrence h_t = a_t h_{t-1} + w_t x_t over packed sequences, with
    a_t = exp(g_t) (PRE_GATE_SOFTPLUS: g holds raw values, a_t = 1 / (1 + e^g)) and
    w_t = 1, or 1 - a_t where ``convex``.  Returns (h, final state [N, D] fp32 or
    None); with ``output_checkpoints`` also the states that glr_backward takes.
    Malformed cu_seqlens are found on the device: h is then left as it was allocated,
    and device_status(workspace) of the caller's own workspace says so."""
    lib = load_library()
    shape, di = _matrix("x", x, "[T, D]")
    T, D = shape
    xs, gs = _rows("x", x, shape, di), _rows("g", g, shape, di)
    dt, gt = _types("x", x, "g", g)
    N, cu = _sequences(cu_seqlens, di)
    if initial_state is not None:
        _fp32("initial_state", initial_state, (N, D), x)
    h = _like("out", out, x)
    final = _output("final_out", final_out, (N, D), _F32, x) if output_final_state else None
    saved = x.new_empty((_groups(T), D), dtype=_F32) if output_checkpoints else None
    ws, ws_bytes = _workspace(workspace, lambda: glr_workspace_size(T, D), x)
    _check(lib.glr_prefill(
        x.data_ptr(), xs, g.data_ptr(), gs, _ptr(initial_state), cu, N, T, D, dt, gt, int(convex), int(preprocess),
        h.data_ptr(), _ptr(final), _ptr(saved), ws.data_ptr(), ws_bytes, _stream(di)))
    return (h, final, saved) if output_checkpoints else (h, final)


def glr_backward(dh, x, g, checkpoints, initial_state=None, dfinal=None, cu_seqlens=None, convex=False, preprocess=0,
                 workspace=None):
    """Gradients of glr_prefill from that of h (``dh``) and of the final state
    (``dfinal``): (dx, dg, gradient of the initial state, or None without one).
    ``checkpoints`` is what the forward call returned.  ``workspace``: as for
    glr_prefill."""
    lib = load_library()
    shape, di = _matrix("x", x, "[T, D]")
    T, D = shape
    xs, gs, dhs = _rows("x", x, shape, di), _rows("g", g, shape, di), _rows("dh", dh, shape, di)
    dt, gt = _types("x", x, "g", g)
    _same_type("dh", dh, x.dtype)
    N, cu = _sequences(cu_seqlens, di)
    _fp32("checkpoints", checkpoints, (_groups(T), D), x)
    ds0 = None
    if initial_state is not None:
        _fp32("initial_state", initial_state, (N, D), x)
        ds0 = torch.empty_like(initial_state)
    if dfinal is not None:
        _fp32("dfinal", dfinal, (N, D), x)
    dx, dg = _like("dx", None, x), _like("dg", None, g)
    ws, ws_bytes = _workspace(workspace, lambda: glr_workspace_size(T, D), x)
    _check(lib.glr_backward(
        dh.data_ptr(), dhs, x.data_ptr(), xs, g.data_ptr(), gs, checkpoints.data_ptr(), _ptr(initial_state),
        _ptr(dfinal), cu, N, T, D, dt, gt, int(convex), int(preprocess), dx.data_ptr(), dg.data_ptr(), _ptr(ds0),
        ws.data_ptr(), ws_bytes, _stream(di)))
    return dx, dg, ds0


def glr_decode(x, g, state, slots=None, convex=False, preprocess=0, out=None):
    """One token for each of N sequences, x and g [N, D]: updates the fp32 state pool
    [S, D] in place (sequence n in slot slots[n], or n; a slot outside the pool is
    padding and gives a row of zeros) and returns the new states h [N, D]."""
    lib = load_library()
    shape, di = _matrix("x", x, "[N, D]")
    N, D = shape
    xs, gs = _rows("x", x, shape, di), _rows("g", g, shape, di)
    dt, gt = _types("x", x, "g", g)
    S = state.shape[0] if state.dim() == 2 else 0
    _fp32("state", state, (S, D), x)
    if slots is None:
        if S < N:
            raise ValueError("without slots the state pool needs one state per sequence")
    else:
        _check_buffer("slots", slots, x.device, torch.int32, (N,))
    h = _like("out", out, x)
    _check(lib.glr_decode(
        x.data_ptr(), xs, g.data_ptr(), gs, state.data_ptr(), _ptr(slots), S, N, D, dt, gt, int(convex),
        int(preprocess), h.data_ptr(), _stream(di)))
    return h


# --------------------------------------------------------------------- norms
def _scale(scale, D, x):
    """(number, vector or None) of a residual scale."""
    if isinstance(scale, torch.Tensor):
        _fp32("scale", scale, (D,), x)
        return 1.0, scale
    return float(scale), None


def add_norm(x, weight, residual=None, scale=1.0, post_weight=None, eps=1e-6, out=None, residual_out=None):
    """A block's output x [T, D] joins the residual stream and the next block's input
    is normed: r = residual + scale * u with u = x, or norm(x) * post_weight;
    y = norm(r) * weight.  ``scale``: a number or fp32 [D].  Returns (y, r), r in the
    residual's type (x's without one); ``residual_out`` may be the residual itself."""
    lib = load_library()
    shape, di = _matrix("x", x, "[T, D]")
    T, D = shape
    xs, rs = _rows("x", x, shape, di), 0
    like = residual if residual is not None else residual_out if residual_out is not None else x
    if residual is not None:
        rs = _rows("residual", residual, shape, di)
    dt, rt = _types("x", x, "residual", like)
    _fp32("weight", weight, (D,), x)
    if post_weight is not None:
        _fp32("post_weight", post_weight, (D,), x)
    number, vector = _scale(scale, D, x)
    y = _like("out", out, x)
    r = _like("residual_out", None, like) if residual_out is None else \
        _output("residual_out", residual_out, shape, like.dtype, x)
    _check(lib.hagdn_add_norm(
        x.data_ptr(), xs, _ptr(residual), rs, weight.data_ptr(), _ptr(post_weight), _ptr(vector), number, eps, T, D,
        dt, rt, y.data_ptr(), r.data_ptr(), _stream(di)))
    return y, r


def add_norm_backward(dy, res, weight, dresidual=None, x=None, scale=1.0, post_weight=None, eps=1e-6, workspace=None):
    """Gradients of add_norm from those of y (``dy``) and of the stream it returned
    (``dresidual``, None: zero).  ``res`` is that stream; x is needed with a scale
    vector or post_weight.  Returns (dx, gradient of the residual, of weight, of
    the scale vector or None, of post_weight or None)."""
    lib = load_library()
    shape, di = _matrix("dy", dy, "[T, D]")
    T, D = shape
    dys, rs = _rows("dy", dy, shape, di), _rows("res", res, shape, di)
    dt, rt = _types("dy", dy, "res", res)
    number, vector = _scale(scale, D, dy)
    post = post_weight is not None
    _fp32("weight", weight, (D,), dy)
    if post:
        _fp32("post_weight", post_weight, (D,), dy)
    drs = xs = 0
    if dresidual is not None:
        _same_type("dresidual", dresidual, res.dtype)
        drs = _rows("dresidual", dresidual, shape, di)
    reads_x = vector is not None or post
    if reads_x:
        if x is None:
            raise ValueError("x is needed with a scale vector or post_weight")
        _same_type("x", x, dy.dtype)
        xs = _rows("x", x, shape, di)
    dx, dres = _like("dx", None, dy), _like("dres", None, res)
    dw = torch.empty_like(weight)
    dscale = torch.empty_like(vector) if vector is not None else None
    dpost = torch.empty_like(post_weight) if post else None
    ws, ws_bytes = _workspace(workspace, lambda: lib.hagdn_add_norm_workspace_size(T, D, vector is not None, post), dy)
    _check(lib.hagdn_add_norm_backward(
        dy.data_ptr(), dys, _ptr(dresidual), drs, res.data_ptr(), rs, x.data_ptr() if reads_x else None, xs,
        weight.data_ptr(), _ptr(post_weight), _ptr(vector), number, eps, T, D, dt, rt, dx.data_ptr(), dres.data_ptr(),
        dw.data_ptr(), _ptr(dscale), _ptr(dpost), ws.data_ptr(), ws_bytes, _stream(di)))
    return dx, dres, dw, dscale, dpost


def _activation(name):
    code = _ACTIVATIONS.get(name)
    if code is None:
        raise ValueError(f"activation must be one of {sorted(_ACTIVATIONS)} (got {name!r})")
    return code


def _heads(o):
    """The shape [T, H, d] and device index of gate_norm's first operand."""
    if o.dim() != 3:
        raise ValueError(f"o must be [T, H, d] (got {tuple(o.shape)})")
    return o.shape, o.get_device()


def gate_norm(o, z, weight, activation="silu", eps=1e-6, out=None):
    """The norm and gate between a mixer and its output projection, per token and
    head: norm(o) * weight * act(z), o and z [T, H, d], weight fp32 [d]."""
    lib = load_library()
    shape, di = _heads(o)
    T, H, d = shape
    os_, zs = _rows("o", o, shape, di), _rows("z", z, shape, di)
    _same_type("z", z, o.dtype)
    dt, _ = _types("o", o, "z", z)
    _fp32("weight", weight, (d,), o)
    y = _like("out", out, o)
    _check(lib.hagdn_gate_norm(
        o.data_ptr(), os_, z.data_ptr(), zs, weight.data_ptr(), eps, T, H, d, dt, _activation(activation),
        y.data_ptr(), _stream(di)))
    return y


def gate_norm_backward(dy, o, z, weight, activation="silu", eps=1e-6, workspace=None):
    """Gradients of gate_norm: (do, dz, gradient of weight)."""
    lib = load_library()
    shape, di = _heads(o)
    T, H, d = shape
    os_, zs, dys = _rows("o", o, shape, di), _rows("z", z, shape, di), _rows("dy", dy, shape, di)
    _same_type("z", z, o.dtype)
    dt, _ = _types("o", o, "z", z)
    _same_type("dy", dy, o.dtype)
    _fp32("weight", weight, (d,), o)
    act = _activation(activation)
    do, dz, dw = _like("do", None, o), _like("dz", None, z), torch.empty_like(weight)
    ws, ws_bytes = _workspace(workspace, lambda: lib.hagdn_gate_norm_workspace_size(T, H, d), o)
    _check(lib.hagdn_gate_norm_backward(
        dy.data_ptr(), dys, o.data_ptr(), os_, z.data_ptr(), zs, weight.data_ptr(), eps, T, H, d, dt, act,
        do.data_ptr(), dz.data_ptr(), dw.data_ptr(), ws.data_ptr(), ws_bytes, _stream(di)))
    return do, dz, dw
