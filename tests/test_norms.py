"""The norms before and after a block against the 64-bit forms of layer_ref.py,
whose bounds are the tolerances."""

import numpy as np
import pytest

import layer_ref as ref
from gpu_harness import say

TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]
WIDTHS = [1, 2, 7, 8, 63, 64, 65, 127, 128, 256, 257, 511, 1000, 1001, 2048, 2049, 4096, 5000, 8192, 16383, 16384]


def rounded(v, t):
    import torch
    return torch.from_numpy(np.asarray(v, np.float32)).to(torch.bfloat16 if t == "bf16" else torch.float32)


def np64(t):
    return None if t is None else t.double().cpu().numpy()


def add_inputs(T, D, dtype, res, seed):
    r = np.random.default_rng(seed)
    n = lambda *s: r.standard_normal(s)
    return {"x": rounded(n(T, D), dtype), "res": rounded(2 * n(T, D), res), "dy": rounded(n(T, D), dtype),
            "dres": rounded(n(T, D), res), "w": rounded(1 + 0.1 * n(D), "f32"), "post": rounded(0.5 + 0.1 * n(D), "f32"),
            "vec": rounded(0.5 * (1 + 0.2 * n(D)), "f32")}


def check(got, want, kinds, label):
    off = {k: ref.excess(v, want[k], kinds[k]) for k, v in got.items() if v is not None}
    say(f"[norm] {label}: " + " ".join(f"{k}={v:.3f}" for k, v in off.items()))
    assert max(off.values()) <= 1.0, (label, off)


def add_case(d, dtype, res, post, vector, residual=True, dresidual=True, scale=0.5, eps=1e-6):
    """Forward and backward on the GPU against the oracle."""
    import paper_2609_32114_amd as P
    t = {k: v if v.is_cuda else v.cuda() for k, v in d.items()}
    s = t["vec"] if vector else scale
    how = dict(scale=s, post_weight=t["post"] if post else None, eps=eps)
    label = f"{tuple(d['x'].shape)} {dtype}/{res} post={post} vector={vector} residual={residual}/{dresidual}"
    y, r = P.add_norm(t["x"], t["w"], residual=t["res"] if residual else None, **how)
    s64, p64 = np64(d["vec"]) if vector else scale, np64(d["post"]) if post else None
    want = ref.add_norm(np64(d["x"]), np64(d["res"]) if residual else None, np64(d["w"]), s64, p64, eps)
    check({"y": y, "res": r}, want, {"y": dtype, "res": res if residual else dtype}, label)
    reads_x = post or vector
    dx, dres, dw, ds, dp = P.add_norm_backward(t["dy"], t["res"], t["w"], dresidual=t["dres"] if dresidual else None,
                                               x=t["x"] if reads_x else None, **how)
    assert (ds is None) == (not vector) and (dp is None) == (not post)
    want = ref.add_norm_back(np64(d["dy"]), np64(d["dres"]) if dresidual else None, np64(d["res"]),
                             np64(d["x"]) if reads_x else None, np64(d["w"]), s64, p64, eps)
    check({"dx": dx, "dres": dres, "dw": dw, "dscale": ds, "dpost": dp}, want,
          {"dx": dtype, "dres": res, "dw": "f32", "dscale": "f32", "dpost": "f32"}, "backward " + label)


def gate_inputs(T, H, d, dtype, seed):
    r = np.random.default_rng(seed)
    n = lambda *s: r.standard_normal(s)
    return {"o": rounded(0.3 * n(T, H, d), dtype), "z": rounded(2 * n(T, H, d), dtype), "dy": rounded(n(T, H, d), dtype),
            "w": rounded(1 + 0.1 * n(d), "f32")}


def gate_case(i, dtype, activation, place=lambda t: t.cuda(), eps=1e-6):
    import paper_2609_32114_amd as P
    o, z, dy, w = (place(i[k]) if k != "w" else i[k].cuda() for k in ("o", "z", "dy", "w"))
    T, H, d = i["o"].shape
    rows = lambda t: np64(t).reshape(T * H, d)
    label = f"{(T, H, d)} {dtype} {activation}"
    y = P.gate_norm(o, z, w, activation=activation, eps=eps)
    silu = activation == "silu"
    check({"y": y}, ref.gate_norm(rows(i["o"]), rows(i["z"]), np64(i["w"]), silu, eps), {"y": dtype}, label)
    do, dz, dw = P.gate_norm_backward(dy, o, z, w, activation=activation, eps=eps)
    check({"do": do, "dz": dz, "dw": dw},
          ref.gate_norm(rows(i["o"]), rows(i["z"]), np64(i["w"]), silu, eps, rows(i["dy"])),
          {"do": dtype, "dz": dtype, "dw": "f32"}, "backward " + label)


# ------------------------------------------------------------------ the oracle (CPU)
def _differences(loss, args, grads):
    """grads against central differences of loss(**args) in 64 bits (a step of 1e-6
    leaves 1e-12 of curvature and 1e-9 of rounding)."""
    for name, grad in grads.items():
        grad = np.asarray(grad)
        for i in np.ndindex(grad.shape):
            lo, hi = ({k: np.array(v, np.float64) for k, v in args.items()} for _ in range(2))
            lo[name][i] -= 1e-6
            hi[name][i] += 1e-6
            diff = (loss(**hi) - loss(**lo)) / 2e-6
            assert abs(diff - grad[i]) <= 1e-7 * (1 + abs(grad[i])), (name, i, diff, grad[i])


@pytest.mark.parametrize("post", [False, True])
def test_add_norm_oracle_gradient_is_that_of_its_values(post):
    d = {k: np64(v) for k, v in add_inputs(3, 5, "f32", "f32", 1).items()}

    def values(x, res, w, vec, post_w):
        return ref.add_norm(x, res, w, vec, post_w if post else None, 1e-3)

    def loss(**a):
        o = values(**a)
        return float((o["y"][0] * d["dy"]).sum() + (o["res"][0] * d["dres"]).sum())

    args = {"x": d["x"], "res": d["res"], "w": d["w"], "vec": d["vec"], "post_w": d["post"]}
    r = values(**args)["res"][0]
    b = ref.add_norm_back(d["dy"], d["dres"], r, d["x"], d["w"], d["vec"], d["post"] if post else None, 1e-3)
    grads = {"x": b["dx"][0], "res": b["dres"][0], "w": b["dw"][0], "vec": b["dscale"][0]}
    if post:
        grads["post_w"] = b["dpost"][0]
    _differences(loss, args, grads)


@pytest.mark.parametrize("silu", [False, True])
def test_gate_norm_oracle_gradient_is_that_of_its_values(silu):
    i = {k: np64(v) for k, v in gate_inputs(2, 2, 5, "f32", 1).items()}
    i = {k: v.reshape(-1, 5) if v.ndim > 1 else v for k, v in i.items()}
    loss = lambda o, z, w: float((ref.gate_norm(o, z, w, silu, 1e-3)["y"][0] * i["dy"]).sum())
    b = ref.gate_norm(i["o"], i["z"], i["w"], silu, 1e-3, i["dy"])
    _differences(loss, {"o": i["o"], "z": i["z"], "w": i["w"]}, {"o": b["do"][0], "z": b["dz"][0], "w": b["dw"][0]})


# -------------------------------------------------------------------------- GPU
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,res", TYPES, ids=lambda t: t)
@pytest.mark.parametrize("D", WIDTHS)
def test_add_norm_widths(D, dtype, res):
    T = 5 if D > 1000 else 9
    d = add_inputs(T, D, dtype, res, D)
    for post, vector in ((False, False), (True, True)):
        add_case(d, dtype, res, post, vector)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 3, 64, 1025, 2500])
def test_add_norm_rows(T):
    for (dtype, res), (post, vector) in zip(TYPES * 2, [(False, True), (True, False), (True, True), (False, False),
                                                        (True, True), (True, False)]):
        add_case(add_inputs(T, 200, dtype, res, T), dtype, res, post, vector)


@pytest.mark.gpu
@pytest.mark.parametrize("residual,dresidual", [(False, True), (True, False), (False, False)])
def test_add_norm_without_a_stream(residual, dresidual):
    for post in (False, True):
        add_case(add_inputs(33, 300, "bf16", "bf16", 3), "bf16", "bf16", post, False, residual, dresidual, scale=1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("offset", [0, 1, 2])
def test_add_norm_strided_rows(offset):
    import torch
    for dtype, res in TYPES:
        for D in (129, 2048):
            d = add_inputs(20, D, dtype, res, 4)
            for k in ("x", "res", "dy", "dres"):
                wide = torch.full((20, 2 * D + 7), float("nan"), dtype=d[k].dtype, device="cuda")
                wide[:, offset:offset + D] = d[k].cuda()
                d[k] = wide[:, offset:offset + D]
            add_case(d, dtype, res, True, True)


@pytest.mark.gpu
def test_add_norm_in_place():
    """The stream updated in place, forward and (as the gradient's buffer) backward."""
    import torch
    import paper_2609_32114_amd as P
    lib = P.load_library()
    for D in (100, 1001, 2048, 9000):
        d = {k: v.cuda() for k, v in add_inputs(40, D, "bf16", "f32", 5).items()}
        y, r = P.add_norm(d["x"], d["w"], residual=d["res"], scale=0.5)
        stream = d["res"].clone()
        y2, r2 = P.add_norm(d["x"], d["w"], residual=stream, scale=0.5, residual_out=stream)
        assert r2 is stream and torch.equal(r, stream) and torch.equal(y, y2)
        dx, dres, dw, _, _ = P.add_norm_backward(d["dy"], r, d["w"], dresidual=d["dres"], scale=0.5)
        grad, dx2, dw2 = d["dres"].clone(), torch.empty_like(dx), torch.empty_like(dw)
        ws = torch.empty(lib.hagdn_add_norm_workspace_size(40, D, 0, 0), dtype=torch.uint8, device="cuda")
        p = lambda t: t.data_ptr()
        rc = lib.hagdn_add_norm_backward(p(d["dy"]), D, p(grad), D, p(r), D, None, 0, p(d["w"]), None, None, 0.5, 1e-6, 40, D,
                                         1, 0, p(dx2), p(grad), p(dw2), None, None, p(ws), ws.numel(),
                                         torch.cuda.current_stream().cuda_stream)
        assert rc == 0 and torch.equal(grad, dres) and torch.equal(dx2, dx) and torch.equal(dw2, dw)


@pytest.mark.gpu
def test_add_norm_zero_and_wild_rows():
    """A row of zeros is zeros over sqrt(eps); a row's NaN or infinity stays in it."""
    import torch
    import paper_2609_32114_amd as P
    for D in (64, 1000, 6000):
        d = {k: v.cuda() for k, v in add_inputs(12, D, "f32", "f32", 6).items()}
        clean = P.add_norm(d["x"], d["w"], residual=d["res"])
        x, res = d["x"].clone(), d["res"].clone()
        x[2], res[2] = 0, 0
        x[5, 0], x[7, D - 1] = float("nan"), float("inf")
        y, r = P.add_norm(x, d["w"], residual=res)
        assert bool((y[2] == 0).all()) and bool((r[2] == 0).all())
        assert bool(y[5].isnan().all()) and bool(y[7, D - 1].isnan()) and bool((y[7, :D - 1] == 0).all())
        keep = [i for i in range(12) if i not in (2, 5, 7)]
        assert torch.equal(y[keep], clean[0][keep])
        g = P.add_norm_backward(d["dy"], r, d["w"], dresidual=d["dres"])
        ok = P.add_norm_backward(d["dy"], d["res"] + d["x"], d["w"], dresidual=d["dres"])
        assert torch.equal(g[0][keep], ok[0][keep]) and bool(g[0][2].isfinite().all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,d", [(1, 1), (3, 7), (4, 64), (5, 65), (16, 128), (2, 129), (7, 200), (1, 256), (2, 500),
                                 (3, 512), (1, 1000), (1, 2048), (2, 4097), (1, 16384)])
def test_gate_norm_widths(H, d, dtype):
    for activation in ("silu", "sigmoid"):
        gate_case(gate_inputs(9, H, d, dtype, d), dtype, activation)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 63, 1000, 3001])
def test_gate_norm_rows(T):
    for dtype in ("bf16", "f32"):
        gate_case(gate_inputs(T, 3, 128, dtype, T), dtype, "silu")
        gate_case(gate_inputs(T, 2, 90, dtype, T), dtype, "sigmoid")


@pytest.mark.gpu
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_gate_norm_strided_tokens(offset):
    import torch

    def place(t):
        T, H, d = t.shape
        wide = torch.full((T, 2 * H * d + 9), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, offset:offset + H * d] = t.reshape(T, -1).cuda()
        return wide[:, offset:offset + H * d].unflatten(1, (H, d))

    for dtype in ("bf16", "f32"):
        for H, d in ((4, 128), (3, 77)):
            gate_case(gate_inputs(50, H, d, dtype, 2), dtype, "silu", place)


@pytest.mark.gpu
def test_gate_norm_extreme_gates():
    """Gates far into both tails: the activations reach 0, 1 and z without overflow."""
    i = gate_inputs(6, 2, 128, "f32", 8)
    i["z"][0], i["z"][1], i["z"][2], i["z"][3] = 100.0, -100.0, 0.0, -85.0
    for activation in ("silu", "sigmoid"):
        gate_case(i, "f32", activation)


@pytest.mark.gpu
def test_gradients_against_differences():
    """The kernels' gradients along a direction against differences of their own fp32
    values.  A step of 2^-6 relative to unit inputs leaves a curvature term, under
    2^-10 of the norms' product, and rounding far below it."""
    import torch
    import paper_2609_32114_amd as P
    d = {k: v.cuda() for k, v in add_inputs(50, 300, "f32", "f32", 11).items()}
    at = {k: d[k] for k in ("x", "res", "w", "vec", "post")}

    def loss(x, res, w, vec, post):
        y, r = P.add_norm(x, w, residual=res, scale=vec, post_weight=post)
        return float((y.double() * d["dy"]).sum() + (r.double() * d["dres"]).sum())

    _, r = P.add_norm(d["x"], d["w"], residual=d["res"], scale=d["vec"], post_weight=d["post"])
    dx, dres, dw, ds, dp = P.add_norm_backward(d["dy"], r, d["w"], dresidual=d["dres"], x=d["x"], scale=d["vec"],
                                               post_weight=d["post"])
    i = {k: v.cuda() for k, v in gate_inputs(40, 3, 100, "f32", 12).items()}
    i["o"] *= 3
    gloss = lambda o, z, w: float((P.gate_norm(o, z, w).double() * i["dy"]).sum())
    do, dz, dgw = P.gate_norm_backward(i["dy"], i["o"], i["z"], i["w"])
    for f, point, grads in ((loss, at, {"x": dx, "res": dres, "w": dw, "vec": ds, "post": dp}),
                            (gloss, {k: i[k] for k in "ozw"}, {"o": do, "z": dz, "w": dgw})):
        for k, (name, grad) in enumerate(grads.items()):
            gen = torch.Generator(device="cuda").manual_seed(k)
            v = torch.randn(grad.shape, generator=gen, device="cuda") * 2 ** -6
            diff = f(**{**point, name: point[name] + v}) - f(**{**point, name: point[name] - v})
            want = 2 * float((grad.double() * v).sum())
            assert abs(diff - want) <= 2 ** -9 * float(grad.double().norm() * v.double().norm()), (name, diff, want)


@pytest.mark.gpu
def test_repeats_bit_for_bit():
    import torch
    import paper_2609_32114_amd as P
    d = {k: v.cuda() for k, v in add_inputs(5000, 512, "bf16", "bf16", 1).items()}
    i = {k: v.cuda() for k, v in gate_inputs(3000, 8, 128, "bf16", 1).items()}
    a = [P.add_norm_backward(d["dy"], d["res"], d["w"], d["dres"], d["x"], d["vec"], d["post"]) for _ in range(3)]
    b = [P.gate_norm_backward(i["dy"], i["o"], i["z"], i["w"]) for _ in range(3)]
    for runs in (a, b):
        for other in runs[1:]:
            assert all(torch.equal(p, q) for p, q in zip(runs[0], other))


@pytest.mark.gpu
def test_no_rows():
    import torch
    import paper_2609_32114_amd as P
    w = torch.ones(64, device="cuda")
    e = torch.empty(0, 64, device="cuda")
    y, r = P.add_norm(e, w, residual=e)
    assert y.shape == r.shape == (0, 64)
    dx, dres, dw, ds, dp = P.add_norm_backward(e, e, w, x=e, scale=w, post_weight=w)
    assert all(bool((g == 0).all()) for g in (dw, ds, dp))
    e = torch.empty(0, 4, 64, device="cuda")
    assert P.gate_norm(e, e, w).shape == (0, 4, 64)
    assert bool((P.gate_norm_backward(e, e, e, w)[2] == 0).all())


@pytest.mark.gpu
def test_beyond_two_gib():
    """Rows whose byte offsets pass 2^31 and 2^32, against the same rows alone."""
    import torch
    import paper_2609_32114_amd as P
    T, D = 1050000, 2048
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(T, D, generator=gen, device="cuda", dtype=torch.bfloat16)
    w = torch.rand(D, generator=gen, device="cuda")
    y, r = P.add_norm(x, w, scale=0.5)
    tail = x[-300:].contiguous()
    y1, r1 = P.add_norm(tail, w, scale=0.5)
    assert torch.equal(y[-300:], y1) and torch.equal(r[-300:], r1)
    dx, dres, dw, _, _ = P.add_norm_backward(x, r, w)
    dx1, dres1, _, _, _ = P.add_norm_backward(tail, r1, w)
    assert torch.equal(dx[-300:], dx1) and torch.equal(dres[-300:], dres1)
    del y, dx, dres
    o, wh = x.view(T, 16, 128), w[:128].contiguous()
    y = P.gate_norm(o, r.view(T, 16, 128), wh)
    assert torch.equal(y[-300:], P.gate_norm(o[-300:].contiguous(), r1.view(300, 16, 128), wh))
    do, dz, _ = P.gate_norm_backward(y, o, r.view(T, 16, 128), wh)
    do1, dz1, _ = P.gate_norm_backward(y[-300:].contiguous(), o[-300:].contiguous(), r1.view(300, 16, 128), wh)
    assert torch.equal(do[-300:], do1) and torch.equal(dz[-300:], dz1)


@pytest.mark.gpu
def test_writes_stay_inside():
    """Guard zones around every output and the workspace stay as they were."""
    import torch
    import paper_2609_32114_amd as P
    lib = P.load_library()
    st = torch.cuda.current_stream().cuda_stream
    for T, D in ((3, 1), (5, 7), (9, 130), (4, 1001), (300, 2048), (2, 9001), (2, 16384)):
        for dtype, res in TYPES:
            d = {k: v.cuda() for k, v in add_inputs(T, D, dtype, res, 1).items()}
            code, rcode, e, re = int(dtype == "bf16"), int(res == "bf16"), d["x"].element_size(), d["res"].element_size()
            raw = {}

            def guarded(name, nbytes):
                raw[name] = (torch.full((2048 + nbytes + 2048,), 0xA5, dtype=torch.uint8, device="cuda"), nbytes)
                return raw[name][0].data_ptr() + 2048

            p = lambda k: d[k].data_ptr()
            assert lib.hagdn_add_norm(p("x"), D, p("res"), D, p("w"), p("post"), p("vec"), 1.0, 1e-6, T, D, code, rcode,
                                      guarded("y", T * D * e), guarded("r", T * D * re), st) == 0
            n = lib.hagdn_add_norm_workspace_size(T, D, 1, 1)
            assert lib.hagdn_add_norm_backward(p("dy"), D, p("dres"), D, p("res"), D, p("x"), D, p("w"), p("post"), p("vec"),
                                               1.0, 1e-6, T, D, code, rcode, guarded("dx", T * D * e),
                                               guarded("dres", T * D * re), guarded("dw", 4 * D), guarded("ds", 4 * D),
                                               guarded("dp", 4 * D), guarded("ws", n), n, st) == 0
            assert lib.hagdn_gate_norm(p("x"), D, p("dy"), D, p("w"), 1e-6, T, 1, D, code, 0, guarded("gy", T * D * e), st) == 0
            n = lib.hagdn_gate_norm_workspace_size(T, 1, D)
            assert lib.hagdn_gate_norm_backward(p("dy"), D, p("x"), D, p("dy"), D, p("w"), 1e-6, T, 1, D, code, 0,
                                                guarded("do", T * D * e), guarded("dz", T * D * e), guarded("gw", 4 * D),
                                                guarded("gws", n), n, st) == 0
            torch.cuda.synchronize()
            for name, (buf, nbytes) in raw.items():
                v = buf.cpu().numpy()
                assert (v[:2048] == 0xA5).all() and (v[2048 + nbytes:] == 0xA5).all(), (name, T, D, dtype)


@pytest.mark.gpu
def test_graph_replays():
    import torch
    import paper_2609_32114_amd as P
    sets = [{k: v.cuda() for k, v in {**add_inputs(300, 256, "bf16", "bf16", s),
                                      **{"g" + k: v for k, v in gate_inputs(300, 4, 64, "bf16", s).items()}}.items()}
            for s in (1, 2, 3)]

    def call(d):
        y, r = P.add_norm(d["x"], d["w"], residual=d["res"], scale=d["vec"], post_weight=d["post"])
        return (y, r) + P.add_norm_backward(d["dy"], r, d["w"], d["dres"], d["x"], d["vec"], d["post"]) + \
            (P.gate_norm(d["go"], d["gz"], d["gw"]),) + P.gate_norm_backward(d["gdy"], d["go"], d["gz"], d["gw"])

    want = [[o.clone() for o in call(d)] for d in sets]
    fixed = {k: v.clone() for k, v in sets[0].items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(fixed)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(fixed)
    for i in (1, 2, 0, 1):
        for k, v in sets[i].items():
            fixed[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want[i]):
            assert torch.equal(a, b)
        call(sets[2])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,res", TYPES, ids=lambda t: t)
@pytest.mark.parametrize("D", [7, 64, 200, 2048, 5000, 9000])
def test_add_norm_row_scales(D, dtype, res):
    """Rows of root mean squares from 1e-14 to 1e14 without an eps: norms and their
    gradients are representable throughout, whatever a power of the reciprocal root is."""
    d = add_inputs(10, D, dtype, res, D + 1)
    rows = 10.0 ** np.array([-14, -7, 0, 7, 14, -14, 14, -3, 3, 13])[:, None]
    for k in ("x", "res"):
        d[k] = rounded(np64(d[k]) * rows, dtype if k == "x" else res)
    for post, vector in ((False, False), (True, True), (True, False), (False, True)):
        add_case(d, dtype, res, post, vector, dresidual=False, eps=0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [7, 128, 2048, 9000])
def test_gate_norm_row_scales(d, dtype):
    i = gate_inputs(10, 1, d, dtype, d)
    rows = 10.0 ** np.array([-14, -7, 0, 7, 14, -14, 14, -3, 3, 13])[:, None, None]
    i["o"] = rounded(np64(i["o"]) * rows, dtype)
    gate_case(i, dtype, "silu", eps=0.0)
