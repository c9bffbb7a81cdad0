"""Binding of the short causal convolution and the selective state space scan
(``include/hagdn.h``).

    y, window = conv_prefill(x, weight, bias=None, initial_window=None, cu_seqlens=None, activation="silu")
    dx, dweight, dbias, dwindow = conv_backward(dy, x, weight, bias=None, initial_window=None, dfinal=None)
    y = conv_decode(x1, weight, window_pool, bias=None, slots=None)
    y, final = ssm_prefill(x, dt, A, B, C, skip=None, z=None, dt_bias=None, initial_state=None, cu_seqlens=None)
    dx, ddt, dA, dB, dC, dskip, dz, dbias, ds0 = ssm_backward(dy, x, dt, A, B, C, checkpoints, ..)
    y = ssm_decode(x1, dt1, A, B1, C1, state_pool, slots=None, ..)

Layouts: x, dt, z, dy [T, D] (decode: [N, D]); weight [D, W] and bias [D] fp32; windows
[N, W - 1, D] in x's type, the oldest input first; A [D, S], skip and dt_bias [D] fp32; B, C
[T, G, S], or [T, S] for one group; states [N, D, S] fp32.  Inputs may be column slices of
a wider matrix (rows of contiguous elements at any row stride); outputs are contiguous.  bf16
or fp32, dt fp32 or the operands' type.
"""

from __future__ import annotations

import torch

from . import HagdnError, _check_buffer, _err, _ptr, load_library
from .layer import (_F32, _check, _fp32, _like, _matrix, _output, _rows, _same_type, _sequences, _stream, _types,
                    _workspace)

_ACTIVATIONS = {"silu": 0, None: 2}
_CHECKED_IN_PLACE = 512  # sequences up to which hagdn_conv_prefill takes calls without a workspace


def _activation(name):
    code = _ACTIVATIONS.get(name)
    if code is None:
        raise ValueError(f"activation must be 'silu' or None (got {name!r})")
    return code


def _size(n):
    """A size from the library, which returns 0 for arguments that it turns down."""
    if n == 0:
        raise HagdnError(1, _err(load_library()))
    return n


def _call(di, fn, *args):
    """fn(*args) with the operands' GPU current, whose streams it launches on."""
    if torch._C._cuda_getDevice() == di:
        _check(fn(*args))
    else:
        with torch.cuda.device(di):
            _check(fn(*args))


def _slots(slots, S, N, x):
    if slots is None:
        if S < N:
            raise ValueError("without slots the state pool needs one state per sequence")
    else:
        _check_buffer("slots", slots, x.device, torch.int32, (N,))


# --------------------------------------------------------------- short convolution
def conv_workspace_size(T: int, D: int, W: int, backward: bool = False) -> int:
    """Bytes of workspace conv_prefill (or conv_backward) needs for T tokens of D channels."""
    return _size(load_library().hagdn_conv_workspace_size(T, D, W, int(backward)))


def _conv(x, weight, bias):
    """(shape, device index, row stride, dtype code, W, bias' pointer) of a call, its weights
    checked."""
    shape, di = _matrix("x", x, "[T, D]")
    xs = _rows("x", x, shape, di)
    dt, _ = _types("x", x, "x", x)
    if weight.dim() != 2:
        raise ValueError(f"weight must be [D, W] (got {tuple(weight.shape)})")
    D, W = shape[1], weight.shape[1]
    if weight.dtype is not _F32 or weight.get_device() != di or weight.shape[0] != D or weight.stride() != (W, 1):
        _fp32("weight", weight, (D, W), x)
    return shape, di, xs, dt, W, _vector("bias", bias, D, x, di)


def conv_prefill(x, weight, bias=None, initial_window=None, cu_seqlens=None, activation="silu",
                 output_final_window=True, workspace=None, out=None, final_out=None):
    """Causal convolution of W taps over packed sequences, y_t = act(bias + sum_j
    weight[:, j] x_{t-W+1+j}); ``activation`` "silu" or None.  Before a sequence stand the
    W - 1 inputs of its initial_window [N, W - 1, D] (None: zeros).  Returns (y, the window
    that continues each sequence or None).  Malformed cu_seqlens are found on the device: y is
    then left as it was allocated, and device_status(workspace) of the caller's own workspace
    says so."""
    lib = load_library()
    shape, di, xs, dt, W, pb = _conv(x, weight, bias)
    T, D = shape
    act = _activation(activation)
    N, cu = _sequences(cu_seqlens, di)
    windows = (N, W - 1, D)
    if initial_window is not None:
        _check_buffer("initial_window", initial_window, x.device, x.dtype, windows)
    ws, ws_bytes = None, 0  # only a caller's own tells of malformed offsets
    if workspace is not None or N > _CHECKED_IN_PLACE:
        ws, ws_bytes = _workspace(workspace, lambda: conv_workspace_size(T, D, W), x)
    y = _like("out", out, x)
    final = _output("final_out", final_out, windows, x.dtype, x) if output_final_window else None
    _call(di, lib.hagdn_conv_prefill, x.data_ptr(), xs, weight.data_ptr(), pb, _ptr(initial_window), cu, N, T, D, W,
          dt, act, y.data_ptr(), _ptr(final), _ptr(ws), ws_bytes, _stream(di))
    return y, final


def conv_backward(dy, x, weight, bias=None, initial_window=None, dfinal=None, cu_seqlens=None, activation="silu",
                  workspace=None):
    """Gradients of conv_prefill from that of y (``dy``) and of the window it returned
    (``dfinal``, None: zero): (dx, dweight, dbias or None, gradient of the initial window, or
    None without one)."""
    lib = load_library()
    shape, di, xs, dt, W, pb = _conv(x, weight, bias)
    T, D = shape
    act = _activation(activation)
    dys = _rows("dy", dy, shape, di)
    _same_type("dy", dy, x.dtype)
    N, cu = _sequences(cu_seqlens, di)
    windows, dw0 = (N, W - 1, D), None
    if initial_window is not None:
        _check_buffer("initial_window", initial_window, x.device, x.dtype, windows)
        dw0 = torch.empty_like(initial_window)
    if dfinal is not None:
        _check_buffer("dfinal", dfinal, x.device, x.dtype, windows)
    ws, ws_bytes = _workspace(workspace, lambda: conv_workspace_size(T, D, W, True), x)
    dx, dw = _like("dx", None, x), torch.empty_like(weight)
    db = torch.empty_like(bias) if bias is not None else None
    _call(di, lib.hagdn_conv_backward, dy.data_ptr(), dys, x.data_ptr(), xs, weight.data_ptr(), pb,
          _ptr(initial_window), _ptr(dfinal), cu, N, T, D, W, dt, act, dx.data_ptr(), dw.data_ptr(), _ptr(db),
          _ptr(dw0), ws.data_ptr(), ws_bytes, _stream(di))
    return dx, dw, db, dw0


def conv_decode(x, weight, state, bias=None, slots=None, activation="silu", out=None):
    """One token for each of N sequences, x [N, D]: moves the windows in the pool state
    [S, W - 1, D] (x's type) on in place (sequence n in slot slots[n], or n; a slot outside
    the pool is padding and gives a row of zeros) and returns y [N, D]."""
    lib = load_library()
    shape, di, xs, dt, W, pb = _conv(x, weight, bias)
    N, D = shape
    act = _activation(activation)
    S = state.shape[0] if state.dim() == 3 else 0
    _check_buffer("state", state, x.device, x.dtype, (S, W - 1, D))
    _slots(slots, S, N, x)
    y = _like("out", out, x)
    _call(di, lib.hagdn_conv_decode, x.data_ptr(), xs, weight.data_ptr(), pb, state.data_ptr(), _ptr(slots), S, N, D,
          W, dt, act, y.data_ptr(), _stream(di))
    return y


# ----------------------------------------------------------------- selective scan
def ssm_workspace_size(T: int, D: int, S: int, G: int = 1, backward: bool = False) -> int:
    """Bytes of workspace ssm_prefill (or ssm_backward) needs for T tokens of D channels with S
    states each, B and C in G groups."""
    return _size(load_library().ssm_workspace_size(T, D, S, G, int(backward)))


def ssm_checkpoints_size(T: int, D: int, S: int) -> int:
    """Elements of the checkpoints that ssm_prefill leaves for ssm_backward."""
    return load_library().ssm_checkpoints_size(T, D, S)


def _row(name, t, shape, di, inner=1):
    """The row stride of a matrix whose row's last elements, `inner` apart, follow each other;
    _rows has the other cases and the messages."""
    s = t.stride()
    if s[-1] == 1 and (len(s) == 2 or s[1] == inner) and t.get_device() == di and t.shape == shape:
        return s[0]
    return _rows(name, t, shape, di)


def _maps(B, C, T, S, x, di):
    """(groups, the token strides of B and C): [T, G, S], or [T, S] for one group."""
    shape = B.shape
    if len(shape) not in (2, 3) or shape[0] != T or shape[-1] != S:
        raise ValueError(f"B must be [{T}, G, {S}] or [{T}, {S}] (got {tuple(shape)})")
    Bs, Cs = _row("B", B, shape, di, S), _row("C", C, shape, di, S)
    if B.dtype is not x.dtype or C.dtype is not x.dtype:
        _same_type("B", B, x.dtype)
        _same_type("C", C, x.dtype)
    return (shape[1] if len(shape) == 3 else 1), Bs, Cs


def _vector(name, t, D, x, di):
    """The pointer of an fp32 vector beside x, or of none."""
    if t is None:
        return None
    if t.dtype is not _F32 or t.get_device() != di or t.shape != (D,) or t.stride() != (1,):
        _fp32(name, t, (D,), x)
    return t.data_ptr()


def _operands(x, dt, A, B, C, skip, z, dt_bias):
    """(shape of x, states, groups, device index, type codes, arguments) of what all the scan's
    calls share, checked."""
    shape, di = _matrix("x", x, "[T, D]")
    T, D = shape
    xs, dts = _rows("x", x, shape, di), _row("dt", dt, shape, di)
    types = _types("x", x, "dt", dt)
    if A.dim() != 2:
        raise ValueError(f"A must be [D, S] (got {tuple(A.shape)})")
    S = A.shape[1]
    if A.dtype is not _F32 or A.get_device() != di or A.shape[0] != D or A.stride() != (S, 1):
        _fp32("A", A, (D, S), x)
    G, Bs, Cs = _maps(B, C, T, S, x, di)
    zs = 0
    if z is not None:
        zs = _row("z", z, shape, di)
        if z.dtype is not x.dtype:
            _same_type("z", z, x.dtype)
    return shape, S, G, di, types, (
        x.data_ptr(), xs, dt.data_ptr(), dts, A.data_ptr(), B.data_ptr(), Bs, C.data_ptr(), Cs,
        _vector("skip", skip, D, x, di), None if z is None else z.data_ptr(), zs, _vector("dt_bias", dt_bias, D, x, di))


def ssm_prefill(x, dt, A, B, C, skip=None, z=None, dt_bias=None, initial_state=None, cu_seqlens=None, preprocess=0,
                output_final_state=True, output_checkpoints=False, workspace=None, out=None, final_out=None):
    """Selective state space scan over packed sequences, h_t = e^(dt_t A) h_{t-1} + dt_t x_t
    B_t and y_t = (C_t . h_t + skip x_t) silu(z_t).  PRE_GATE_SOFTPLUS: dt holds raw
    values, the step size is log(1 + e^(dt + dt_bias)).  Returns (y, final states [N, D, S]
    fp32 or None); with ``output_checkpoints`` also what ssm_backward takes.  Malformed
    cu_seqlens are found on the device: y is then left as it was allocated, and
    device_status(workspace) of the caller's own workspace says so."""
    lib = load_library()
    (T, D), S, G, di, types, args = _operands(x, dt, A, B, C, skip, z, dt_bias)
    N, cu = _sequences(cu_seqlens, di)
    if initial_state is not None:
        _fp32("initial_state", initial_state, (N, D, S), x)
    ws, ws_bytes = _workspace(workspace, lambda: ssm_workspace_size(T, D, S, G), x)
    y = _like("out", out, x)
    final = _output("final_out", final_out, (N, D, S), _F32, x) if output_final_state else None
    saved = x.new_empty(ssm_checkpoints_size(T, D, S), dtype=_F32) if output_checkpoints else None
    _call(di, lib.ssm_prefill, *args, _ptr(initial_state), cu, N, T, D, S, G, *types, int(preprocess), y.data_ptr(),
          _ptr(final), _ptr(saved), ws.data_ptr(), ws_bytes, _stream(di))
    return (y, final, saved) if output_checkpoints else (y, final)


def ssm_backward(dy, x, dt, A, B, C, checkpoints, skip=None, z=None, dt_bias=None, initial_state=None, dfinal=None,
                 cu_seqlens=None, preprocess=0, workspace=None):
    """Gradients of ssm_prefill from that of y (``dy``) and of the final states (``dfinal``,
    None: zero): (dx, ddt, dA, dB, dC, dskip, dz, gradient of dt_bias, of the initial state),
    None for what was not given.  ``checkpoints`` is what the forward call returned."""
    lib = load_library()
    shape, S, G, di, types, args = _operands(x, dt, A, B, C, skip, z, dt_bias)
    T, D = shape
    dys = _row("dy", dy, shape, di)
    _same_type("dy", dy, x.dtype)
    N, cu = _sequences(cu_seqlens, di)
    _fp32("checkpoints", checkpoints, (ssm_checkpoints_size(T, D, S),), x)
    ds0 = None
    if initial_state is not None:
        _fp32("initial_state", initial_state, (N, D, S), x)
        ds0 = torch.empty_like(initial_state)
    if dfinal is not None:
        _fp32("dfinal", dfinal, (N, D, S), x)
    ws, ws_bytes = _workspace(workspace, lambda: ssm_workspace_size(T, D, S, G, True), x)
    dx, ddt, dA, dB, dC = _like("dx", None, x), _like("ddt", None, dt), torch.empty_like(A), _like("dB", None, B), \
        _like("dC", None, C)
    dskip = torch.empty_like(skip) if skip is not None else None
    dz = _like("dz", None, z) if z is not None else None
    dbias = torch.empty_like(dt_bias) if dt_bias is not None else None
    _call(di, lib.ssm_backward, dy.data_ptr(), dys, *args, checkpoints.data_ptr(), _ptr(initial_state), _ptr(dfinal),
          cu, N, T, D, S, G, *types, int(preprocess), dx.data_ptr(), ddt.data_ptr(), dA.data_ptr(), dB.data_ptr(),
          dC.data_ptr(), _ptr(dskip), _ptr(dz), _ptr(dbias), _ptr(ds0), ws.data_ptr(), ws_bytes, _stream(di))
    return dx, ddt, dA, dB, dC, dskip, dz, dbias, ds0


def ssm_decode(x, dt, A, B, C, state, slots=None, skip=None, z=None, dt_bias=None, preprocess=0, out=None):
    """One token for each of N sequences, x, dt, z [N, D], B, C [N, G, S] or [N, S]: updates the
    fp32 state pool [slots, D, S] in place (sequence n in slot slots[n], or n; a slot outside
    the pool is padding and gives a row of zeros) and returns y [N, D]."""
    lib = load_library()
    (N, D), S, G, di, types, args = _operands(x, dt, A, B, C, skip, z, dt_bias)
    pool = state.shape[0] if state.dim() == 3 else 0
    _fp32("state", state, (pool, D, S), x)
    _slots(slots, pool, N, x)
    y = _like("out", out, x)
    _call(di, lib.ssm_decode, *args, state.data_ptr(), _ptr(slots), pool, N, D, S, G, *types, int(preprocess),
          y.data_ptr(), _stream(di))
    return y
