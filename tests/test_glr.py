"""The gated linear recurrence: forward, backward and single tokens against the
64-bit token-by-token form of layer_ref.py, whose bounds are the tolerances."""

import ctypes

import numpy as np
import pytest

import layer_ref as ref
from gpu_harness import say

# lengths of packed sequences: one token to several tiles, ends on and off every
# multiple of the kernels' 8, 16, 64 and 128 token pieces, empty sequences
LENS = [(1,), (7,), (64,), (65,), (129,), (1000,), (1, 1, 1), (0, 5, 0, 0, 130, 1, 0), (63, 65, 128, 256, 1),
        (200, 0, 57, 300, 3, 129)]
TYPES = [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")]


def make(lens, D, dtype, gate, raw, seed, s0=True, slow=False):
    """Seeded numpy inputs as the kernels will see them (rounded to their types)."""
    import torch
    r = np.random.default_rng(seed)
    T, N = sum(lens), len(lens)
    rate = np.exp(np.log(0.003) * (np.ones(D) if slow else r.random(D)))
    z = r.standard_normal((T, D))
    g = z + np.log(np.expm1(rate)) if raw else -rate * np.log1p(np.exp(z))
    rnd = lambda v, t: torch.from_numpy(np.asarray(v, np.float32)).to(torch.bfloat16 if t == "bf16" else torch.float32)
    return {"x": rnd(r.standard_normal((T, D)), dtype), "g": rnd(g, gate), "dh": rnd(r.standard_normal((T, D)), dtype),
            "s0": rnd(r.standard_normal((N, D)), "f32") if s0 else None,
            "dfinal": rnd(r.standard_normal((N, D)), "f32") if s0 else None}


def np64(t):
    return None if t is None else t.double().numpy()


def expected(d, lens, raw, convex, backward=True):
    return ref.glr(np64(d["x"]), np64(d["g"]), lens, np64(d["s0"]), raw, convex, np64(d["dh"]) if backward else None,
                   np64(d["dfinal"]) if backward else None)


def offsets(lens):
    import torch
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")


def run(d, lens, raw, convex, cu=None, place=lambda t: t.cuda()):
    """Forward and backward on the GPU; place moves a token matrix there."""
    import torch
    import paper_2609_32114_amd as P
    t = {k: None if v is None else (place(v) if k in ("x", "g", "dh") else v.cuda()) for k, v in d.items()}
    how = dict(cu_seqlens=offsets(lens) if cu is None else cu, convex=convex,
               preprocess=P.PRE_GATE_SOFTPLUS if raw else 0)
    h, final, saved = P.glr_prefill(t["x"], t["g"], initial_state=t["s0"], output_checkpoints=True, **how)
    dx, dg, ds0 = P.glr_backward(t["dh"], t["x"], t["g"], saved, initial_state=t["s0"], dfinal=t["dfinal"], **how)
    torch.cuda.synchronize()
    return {"h": h, "final": final, "dx": dx, "dg": dg, "ds0": ds0}


def check(got, want, dtype, gate, label):
    kinds = {"h": dtype, "dx": dtype, "dg": gate, "final": "f32", "ds0": "f32"}
    off = {k: ref.excess(v, want[k], kinds[k]) for k, v in got.items() if v is not None}
    say(f"[glr] {label}: " + " ".join(f"{k}={v:.3f}" for k, v in off.items()))
    assert max(off.values()) <= 1.0, (label, off)


# ------------------------------------------------------------------ the oracle (CPU)
@pytest.mark.parametrize("raw,convex", [(False, False), (False, True), (True, False), (True, True)])
def test_oracle_gradient_is_that_of_its_values(raw, convex):
    """The oracle's gradients against central differences of its own values, in 64 bits:
    a step of 1e-6 leaves 1e-12 of curvature and 1e-9 of rounding."""
    lens, D = (5, 0, 1, 9), 3
    d = {k: np64(v) for k, v in make(lens, D, "f32", "f32", raw, 3).items()}

    def loss(x, g, s0):
        o = ref.glr(x, g, lens, s0, raw, convex)
        return float((o["h"][0] * d["dh"]).sum() + (o["final"][0] * d["dfinal"]).sum())

    o = ref.glr(d["x"], d["g"], lens, d["s0"], raw, convex, d["dh"], d["dfinal"])
    for name, grad in (("x", o["dx"][0]), ("g", o["dg"][0]), ("s0", o["ds0"][0])):
        for i in np.ndindex(grad.shape):
            lo, hi = (dict(x=d["x"].copy(), g=d["g"].copy(), s0=d["s0"].copy()) for _ in range(2))
            lo[name][i] -= 1e-6
            hi[name][i] += 1e-6
            diff = (loss(**hi) - loss(**lo)) / 2e-6
            assert abs(diff - grad[i]) <= 1e-7 * (1 + abs(grad[i])), (name, i)


def test_oracle_closed_forms():
    """One token, a forgotten state, and a constant gate's geometric sum."""
    x, g = np.array([[2.0]]), np.array([[-np.inf]])
    o = ref.glr(x, g, (1,), np.array([[5.0]]))
    assert o["h"][0][0, 0] == 2.0
    T, a = 40, 0.75
    o = ref.glr(np.ones((T, 1)), np.full((T, 1), np.log(a)), (T,), None)
    assert np.allclose(o["h"][0][:, 0], (1 - a ** np.arange(1, T + 1)) / (1 - a), rtol=1e-13)
    o = ref.glr(np.ones((T, 1)), np.full((T, 1), np.log(a)), (T,), np.ones((1, 1)), convex=True)
    assert np.allclose(o["h"][0], 1.0, rtol=1e-13)  # a weighted mean of ones


# -------------------------------------------------------------------------- GPU
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,gate", TYPES, ids=lambda t: t)
@pytest.mark.parametrize("lens", LENS, ids=lambda n: "-".join(map(str, n)))
def test_against_oracle(lens, dtype, gate):
    for i, (raw, convex) in enumerate([(False, False), (False, True), (True, False), (True, True)]):
        D = (128, 200, 1, 67)[i]
        d = make(lens, D, dtype, gate, raw, 10 + i, s0=i != 2, slow=i == 3)
        check(run(d, lens, raw, convex), expected(d, lens, raw, convex), dtype, gate,
              f"{lens} D={D} {dtype}/{gate} raw={raw} convex={convex}")


@pytest.mark.gpu
@pytest.mark.parametrize("D", [1, 2, 3, 63, 64, 65, 127, 128, 129, 255, 513, 1280, 2048])
def test_widths(D):
    lens = (131, 70)
    for dtype, gate in TYPES:
        d = make(lens, D, dtype, gate, False, D)
        check(run(d, lens, False, True), expected(d, lens, False, True), dtype, gate, f"D={D} {dtype}/{gate}")


@pytest.mark.gpu
@pytest.mark.parametrize("lens,D", [((3000, 0, 2500, 1, 700), 704), ((255, 257, 256, 1, 5600), 1001), ((6000,), 768)])
def test_wide_calls(lens, D):
    """More tiles of 256 tokens than CUs: the largest tiles, several to a workgroup, with
    sequences that end on, before and after their boundaries."""
    for i, (dtype, gate) in enumerate(TYPES):
        raw, convex = i == 1, i != 0
        d = make(lens, D, dtype, gate, raw, 40 + i)
        check(run(d, lens, raw, convex), expected(d, lens, raw, convex), dtype, gate, f"{lens} D={D} {dtype}/{gate}")


@pytest.mark.gpu
@pytest.mark.parametrize("T", [5000, 20011])
def test_long_sequences(T):
    """Channels that remember thousands of tokens, over many tiles."""
    d = make((T,), 96, "bf16", "f32", False, T, slow=True)
    d["g"] *= 0.05
    check(run(d, (T,), False, False), expected(d, (T,), False, False), "bf16", "f32", f"T={T}")


@pytest.mark.gpu
def test_one_sequence_without_offsets():
    import torch
    import paper_2609_32114_amd as P
    d = make((300,), 130, "bf16", "bf16", True, 5)
    x, g, s0 = d["x"].cuda(), d["g"].cuda(), d["s0"].cuda()
    a = P.glr_prefill(x, g, initial_state=s0, preprocess=P.PRE_GATE_SOFTPLUS)
    b = P.glr_prefill(x, g, initial_state=s0, preprocess=P.PRE_GATE_SOFTPLUS, cu_seqlens=offsets((300,)))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.gpu
@pytest.mark.parametrize("N", [65, 300, 5000])
def test_many_short_sequences(N):
    """More sequences than lanes, some empty, tens of them inside one tile."""
    r = np.random.default_rng(N)
    lens = tuple(int(n) for n in r.integers(0, 4, N))
    d = make(lens, 66, "f32", "f32", True, N)
    check(run(d, lens, True, True), expected(d, lens, True, True), "f32", "f32", f"N={N} T={sum(lens)}")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,gate", TYPES, ids=lambda t: t)
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_strided_rows(dtype, gate, offset):
    """Operands as column slices of a wider matrix, at even and odd offsets."""
    import torch
    lens, D = (100, 33, 180), 130

    def place(t):
        wide = torch.full((t.shape[0], 3 * D + 5), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, offset:offset + D] = t.cuda()
        return wide[:, offset:offset + D]

    d = make(lens, D, dtype, gate, True, 21)
    check(run(d, lens, True, True, place=place), expected(d, lens, True, True), dtype, gate, f"offset {offset}")


@pytest.mark.gpu
def test_broadcast_rows():
    """A row stride of zero repeats one row (a constant gate)."""
    d = make((150,), 64, "f32", "f32", False, 8)
    d["g"] = d["g"][:1].expand(150, 64)
    got = run(d, (150,), False, False, place=lambda t: t[:1].cuda().expand(150, 64) if t.stride(0) == 0 else t.cuda())
    d["g"] = d["g"].contiguous()
    check(got, expected(d, (150,), False, False), "f32", "f32", "constant gate")


@pytest.mark.gpu
def test_extreme_gates():
    """Gates of -inf (forget all), 0 (keep all) and far tails; raw ones at +-inf."""
    lens, D = (90, 60, 140), 64
    for raw in (False, True):
        for convex in (False, True):
            d = make(lens, D, "f32", "f32", raw, 31)
            for row, v in ((3, -np.inf), (4, 0.0), (70, -1e-30), (95, -200.0), (150, -0.35), (151, -0.3500001), (289, 0.0)):
                d["g"][row] = -v if raw else v
            if raw:
                d["g"][100], d["g"][101], d["g"][102] = -np.inf, -100.0, 100.0
            check(run(d, lens, raw, convex), expected(d, lens, raw, convex), "f32", "f32", f"raw={raw} convex={convex}")


@pytest.mark.gpu
@pytest.mark.parametrize("lens,D", [((100, 77, 200, 1, 130), 70), ((20, 30, 40), 64), ((3000, 1500, 2000), 705),
                                    ((6000, 5000), 33)])
def test_no_value_reaches_another_sequence(lens, D):
    """NaN and infinities in one sequence's tokens, state and gradients leave the
    others' results as they were, bit for bit, wherever the tile boundaries fall."""
    import torch
    d = make(lens, D, "bf16", "f32", False, 17)
    clean = run(d, lens, False, True)
    starts = np.concatenate([[0], np.cumsum(lens)])
    for n in range(len(lens)):
        bad = {k: v.clone() for k, v in d.items()}
        lo, hi = starts[n], starts[n + 1]
        bad["x"][lo:hi] = float("nan")
        bad["dh"][hi - 1] = float("inf")
        bad["g"][lo] = float("nan")
        bad["s0"][n], bad["dfinal"][n] = float("inf"), float("nan")
        got = run(bad, lens, False, True)
        keep = torch.ones(sum(lens), dtype=torch.bool)
        keep[lo:hi] = False
        others = [i for i in range(len(lens)) if i != n]
        for k in ("h", "dx", "dg"):
            assert torch.equal(got[k].cpu()[keep], clean[k].cpu()[keep]), (n, k)
            assert got[k].cpu()[lo:hi].isnan().any()
        for k in ("final", "ds0"):
            assert torch.equal(got[k][others], clean[k][others]), (n, k)


@pytest.mark.gpu
def test_repeats_bit_for_bit():
    """However the tiles' order falls, results are the same bits."""
    import torch
    lens = (3000, 1500, 9000)
    d = make(lens, 512, "bf16", "f32", False, 2)
    first = run(d, lens, False, False)
    for _ in range(5):
        again = run(d, lens, False, False)
        for k, v in first.items():
            assert torch.equal(v, again[k]), k


@pytest.mark.gpu
def test_states_updated_in_place():
    """s_final written over s0, and ds0 over dfinal, in packed calls whose sequences span
    tiles, share them and are empty: the same bits as in buffers of their own."""
    import torch
    import paper_2609_32114_amd as P
    lib = P.load_library()
    for lens, D in (((300, 5, 0, 700, 2, 1, 129), 96), ((40, 3, 1, 20), 64), ((3000, 0, 2500, 1, 700), 705)):
        T, N = sum(lens), len(lens)
        d = {k: v.cuda() for k, v in make(lens, D, "bf16", "f32", False, 14).items()}
        cu, st = offsets(lens), torch.cuda.current_stream().cuda_stream
        h, final, saved = P.glr_prefill(d["x"], d["g"], initial_state=d["s0"], cu_seqlens=cu, output_checkpoints=True)
        state = d["s0"].clone()
        h2, _ = P.glr_prefill(d["x"], d["g"], initial_state=state, cu_seqlens=cu, final_out=state)
        assert torch.equal(h, h2) and torch.equal(final, state)
        want = P.glr_backward(d["dh"], d["x"], d["g"], saved, initial_state=d["s0"], dfinal=d["dfinal"], cu_seqlens=cu)
        grad, dx, dg = d["dfinal"].clone(), torch.empty_like(d["x"]), torch.empty_like(d["g"])
        ws = torch.empty(P.glr_workspace_size(T, D), dtype=torch.uint8, device="cuda")
        p = lambda t: t.data_ptr()
        rc = lib.glr_backward(p(d["dh"]), D, p(d["x"]), D, p(d["g"]), D, p(saved), p(d["s0"]), p(grad), p(cu), N, T, D, 1, 0,
                              0, 0, p(dx), p(dg), p(grad), p(ws), ws.numel(), st)
        assert rc == 0
        for a, b in zip((dx, dg, grad), want):
            assert torch.equal(a, b)


@pytest.mark.gpu
def test_continues_from_a_state():
    """Two calls joined by the state agree with one call, and a state updated in place
    is the same state."""
    import torch
    import paper_2609_32114_amd as P
    d = make((700,), 256, "f32", "f32", False, 4)
    x, g, s0 = d["x"].cuda(), d["g"].cuda(), d["s0"].cuda()
    h, s = P.glr_prefill(x, g, initial_state=s0)
    state = s0.clone()
    h1, _ = P.glr_prefill(x[:256], g[:256], initial_state=state, final_out=state)
    h2, _ = P.glr_prefill(x[256:], g[256:], initial_state=state, final_out=state)
    want = expected(d, (700,), False, False, backward=False)
    assert ref.excess(torch.cat([h1, h2]), want["h"], "f32") <= 1.0
    assert ref.excess(state, want["final"], "f32") <= 1.0
    assert ref.excess(h, want["h"], "f32") <= 1.0 and ref.excess(s, want["final"], "f32") <= 1.0


@pytest.mark.gpu
def test_no_tokens():
    import torch
    import paper_2609_32114_amd as P
    s0 = torch.randn(3, 100, device="cuda")
    x = torch.empty(0, 100, device="cuda")
    cu = torch.zeros(4, dtype=torch.int32, device="cuda")
    h, s, saved = P.glr_prefill(x, x, initial_state=s0, cu_seqlens=cu, output_checkpoints=True)
    assert h.shape == (0, 100) and torch.equal(s, s0)
    h, s = P.glr_prefill(x, x, cu_seqlens=cu)
    assert torch.equal(s, torch.zeros_like(s0))
    dx, dg, ds0 = P.glr_backward(x, x, x, saved, initial_state=s0, dfinal=2 * s0, cu_seqlens=cu)
    assert torch.equal(ds0, 2 * s0)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [100, 1000])
def test_malformed_offsets(T):
    """Bad sequence offsets: no token is touched, states pass through, the status says so."""
    import torch
    import paper_2609_32114_amd as P
    D, N = 70, 3
    x, g = torch.randn(T, D, device="cuda"), -torch.rand(T, D, device="cuda")
    s0 = torch.randn(N, D, device="cuda")
    ws = torch.empty(P.glr_workspace_size(T, D), dtype=torch.uint8, device="cuda")
    for bad in ([1, 10, 50, T], [0, 50, 10, T], [0, 10, 50, T - 1], [0, 10, 50, T + 1], [0, -5, 50, T],
                [0, 10, 2 ** 31 - 1, T]):
        cu = torch.tensor(bad, dtype=torch.int32, device="cuda")
        h = torch.full((T, D), 7.0, device="cuda")
        _, s = P.glr_prefill(x, g, initial_state=s0, cu_seqlens=cu, workspace=ws, out=h)
        assert P.device_status(ws) == P.DEV_BAD_SEQLENS
        assert torch.equal(s, s0) and bool((h == 7.0).all())
        saved = torch.zeros((T + 127) // 128, D, device="cuda")
        _, _, ds0 = P.glr_backward(x, x, g, saved, initial_state=s0, dfinal=3 * s0, cu_seqlens=cu, workspace=ws)
        assert P.device_status(ws) == P.DEV_BAD_SEQLENS and torch.equal(ds0, 3 * s0)
    _, s = P.glr_prefill(x, g, initial_state=s0, cu_seqlens=torch.tensor([0, 10, 50, T], dtype=torch.int32, device="cuda"),
                         workspace=ws)
    assert P.device_status(ws) == P.DEV_OK and not torch.equal(s, s0)


@pytest.mark.gpu
@pytest.mark.parametrize("N,D,pool", [(1, 2048, 0), (1, 1, 0), (5, 129, 9), (37, 200, 64), (256, 4096, 300)])
def test_decode(N, D, pool):
    import torch
    import paper_2609_32114_amd as P
    for dtype, gate in TYPES:
        for raw, convex in ((False, False), (True, True)):
            d = make((1,) * N, D, dtype, gate, raw, N + D)
            r = np.random.default_rng(N)
            state = torch.from_numpy(r.standard_normal((pool or N, D)).astype(np.float32))
            slots = None
            at = np.arange(N)
            if pool:
                at = r.permutation(pool)[:N]
                at[::4] = (-1, pool, -2 ** 31, 2 ** 31 - 1)[N % 4]  # padding entries
                slots = torch.tensor(at, dtype=torch.int32, device="cuda")
            live = (at >= 0) & (at < (pool or N))
            d["s0"] = torch.zeros(N, D)
            d["s0"][live] = state[at[live]]
            want = expected(d, (1,) * N, raw, convex, backward=False)
            dev = state.cuda()
            h = P.glr_decode(d["x"].cuda(), d["g"].cuda(), dev, slots=slots, convex=convex,
                             preprocess=P.PRE_GATE_SOFTPLUS if raw else 0).cpu()
            dev = dev.cpu()
            assert bool((h[~live] == 0).all())
            pick = lambda w: (w[0][live], w[1][live])
            assert ref.excess(h[live], pick(want["h"]), dtype) <= 1.0
            assert ref.excess(dev[at[live]], pick(want["h"]), "f32") <= 1.0
            rest = np.setdiff1d(np.arange(pool or N), at[live])
            assert torch.equal(dev[rest], state[rest])


@pytest.mark.gpu
def test_decode_continues_a_prefill():
    import torch
    import paper_2609_32114_amd as P
    d = make((40,), 192, "f32", "f32", False, 6)
    x, g = d["x"].cuda(), d["g"].cuda()
    _, state = P.glr_prefill(x[:30], g[:30], initial_state=d["s0"].cuda())
    hs = [P.glr_decode(x[t:t + 1], g[t:t + 1], state) for t in range(30, 40)]
    want = expected(d, (40,), False, False, backward=False)
    assert ref.excess(torch.cat(hs), (want["h"][0][30:], want["h"][1][30:]), "f32") <= 1.0


@pytest.mark.gpu
def test_beyond_two_gib():
    """Rows whose byte offsets pass 2^31 and 2^32: the last tokens of a long call against
    a short call over them from the state before."""
    import torch
    import paper_2609_32114_amd as P
    T, D, tail = 530000, 2048, 200
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(T, D, generator=gen, device="cuda", dtype=torch.bfloat16)
    g = -torch.rand(T, D, generator=gen, device="cuda", dtype=torch.bfloat16) - 0.05
    h, final, saved = P.glr_prefill(x, g, output_checkpoints=True)
    # a state of 2000 tokens before is forgotten (e^-100): start there from nothing
    lo = T - tail - 2000
    h1, final1 = P.glr_prefill(x[lo:].contiguous(), g[lo:].contiguous())
    assert torch.equal(h[-tail:], h1[-tail:]) or (h[-tail:].float() - h1[-tail:].float()).abs().max() <= 2 ** -7
    assert (final - final1).abs().max() <= 1e-5
    dh = torch.zeros_like(x)
    dh[-tail:] = 1
    dx, dg, _ = P.glr_backward(dh, x, g, saved)
    _, _, saved1 = P.glr_prefill(x[lo:].contiguous(), g[lo:].contiguous(), output_checkpoints=True)
    dx1, dg1, _ = P.glr_backward(dh[lo:].contiguous(), x[lo:].contiguous(), g[lo:].contiguous(), saved1)
    assert (dx[lo:].float() - dx1.float()).abs().max() <= 2 ** -8 * dx1.float().abs().max()
    assert (dg[lo:].float() - dg1.float()).abs().max() <= 2 ** -7 * dg1.float().abs().max()


@pytest.mark.gpu
def test_gradient_against_differences():
    """The kernels' gradient along a direction against differences of the fp32 kernel's
    own values.  A step of 2^-6 leaves a curvature term, under 2^-12 of the norms'
    product, and rounding of the values over the step, 2^-24 x 2^6 of them."""
    import torch
    import paper_2609_32114_amd as P
    lens, D = (150, 90), 64
    d = {k: v.cuda() for k, v in make(lens, D, "f32", "f32", True, 12).items()}
    cu, pre = offsets(lens), P.PRE_GATE_SOFTPLUS

    def loss(x, g, s0):
        h, s = P.glr_prefill(x, g, initial_state=s0, cu_seqlens=cu, convex=True, preprocess=pre)
        return float((h.double() * d["dh"].double()).sum() + (s.double() * d["dfinal"].double()).sum())

    _, _, saved = P.glr_prefill(d["x"], d["g"], initial_state=d["s0"], cu_seqlens=cu, convex=True, preprocess=pre,
                                output_checkpoints=True)
    grads = P.glr_backward(d["dh"], d["x"], d["g"], saved, initial_state=d["s0"], dfinal=d["dfinal"], cu_seqlens=cu,
                           convex=True, preprocess=pre)
    for i, name in enumerate(("x", "g", "s0")):
        gen = torch.Generator(device="cuda").manual_seed(i)
        v = torch.randn(d[name].shape, generator=gen, device="cuda") * 2 ** -6
        at = {k: d[k] for k in ("x", "g", "s0")}
        diff = loss(**{**at, name: d[name] + v}) - loss(**{**at, name: d[name] - v})
        want = 2 * float((grads[i].double() * v.double()).sum())
        bound = (2 ** -11) * 2 * float(grads[i].double().norm() * v.double().norm())
        assert abs(diff - want) <= bound, (name, diff, want, bound)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [90, 1500, 9001])
def test_graph_replays(T):
    """Captured calls replayed on new inputs, with eager work between, match eager calls."""
    import torch
    import paper_2609_32114_amd as P
    lens, D = (T // 3, T - T // 3), 130
    sets = [{k: v.cuda() for k, v in make(lens, D, "bf16", "f32", False, s).items()} for s in (1, 2, 3)]
    cu = offsets(lens)
    ws = torch.empty(P.glr_workspace_size(T, D), dtype=torch.uint8, device="cuda")

    def call(d, ws=None):
        h, s, saved = P.glr_prefill(d["x"], d["g"], initial_state=d["s0"], cu_seqlens=cu, output_checkpoints=True,
                                    workspace=ws)
        return (h, s) + P.glr_backward(d["dh"], d["x"], d["g"], saved, initial_state=d["s0"], dfinal=d["dfinal"],
                                       cu_seqlens=cu, workspace=ws)

    want = [[o.clone() for o in call(d)] for d in sets]
    fixed = {k: v.clone() for k, v in sets[0].items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(fixed, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(fixed, ws)
    for i in (1, 2, 0, 1):
        for k, v in sets[i].items():
            fixed[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want[i]):
            assert torch.equal(a, b)
        call(sets[2])


@pytest.mark.gpu
def test_writes_stay_inside():
    """Guard zones around every output and the workspace stay as they were."""
    import torch
    import paper_2609_32114_amd as P
    lib = P.load_library()
    for lens, D, dtype, gate in (((70,), 33, "bf16", "bf16"), ((300, 0, 77), 129, "bf16", "f32"), ((500,), 1, "f32", "f32"),
                                 ((129, 1), 256, "f32", "f32")):
        d = make(lens, D, dtype, gate, False, 9)
        T, N = sum(lens), len(lens)
        code = {"bf16": 1, "f32": 0}
        t = {k: v.cuda() for k, v in d.items()}
        raw = {}

        def guarded(name, nbytes):
            raw[name] = (torch.full((2048 + nbytes + 2048,), 0xA5, dtype=torch.uint8, device="cuda"), nbytes)
            return ctypes.c_void_p(raw[name][0].data_ptr() + 2048)

        esz = {"bf16": 2, "f32": 4}
        h, s = guarded("h", T * D * esz[dtype]), guarded("s", N * D * 4)
        ck = guarded("ck", (T + 127) // 128 * D * 4)
        n = P.glr_workspace_size(T, D)
        ws = guarded("ws", n)
        dx, dg, ds0 = guarded("dx", T * D * esz[dtype]), guarded("dg", T * D * esz[gate]), guarded("ds0", N * D * 4)
        cu, st = offsets(lens), torch.cuda.current_stream().cuda_stream
        p = lambda k: t[k].data_ptr()
        assert lib.glr_prefill(p("x"), D, p("g"), D, p("s0"), cu.data_ptr(), N, T, D, code[dtype], code[gate], 0, 0, h, s,
                               ck, ws, n, st) == 0
        assert lib.glr_backward(p("dh"), D, p("x"), D, p("g"), D, ck, p("s0"), p("dfinal"), cu.data_ptr(), N, T, D,
                                code[dtype], code[gate], 0, 0, dx, dg, ds0, ws, n, st) == 0
        torch.cuda.synchronize()
        for name, (buf, nbytes) in raw.items():
            v = buf.cpu().numpy()
            assert (v[:2048] == 0xA5).all() and (v[2048 + nbytes:] == 0xA5).all(), (name, lens, D)


# sequences that end on, before and after multiples of 256 and 512 tokens, and empty ones
LONG_LENS = (511, 1, 513, 0, 512, 2000, 4096, 3, 1500, 0, 900)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,gate", TYPES, ids=lambda t: t)
@pytest.mark.parametrize("D", [33, 67])
def test_long_packed_calls_of_few_channels(D, dtype, gate):
    """More than 8192 tokens in fewer tiles than CUs: the largest tiles, of 512 tokens
    forward and 256 backward, with sequences that begin and end inside them."""
    for i, (raw, convex) in enumerate([(False, False), (False, True), (True, False), (True, True)]):
        d = make(LONG_LENS, D, dtype, gate, raw, 60 + i, s0=i != 2, slow=i == 3)
        check(run(d, LONG_LENS, raw, convex), expected(d, LONG_LENS, raw, convex), dtype, gate,
              f"long, D={D} {dtype}/{gate} raw={raw} convex={convex}")


@pytest.mark.gpu
@pytest.mark.parametrize("lens,D", [(LONG_LENS, 33), (LONG_LENS, 130), ((3000, 0, 2500, 1, 700), 705), ((2000,), 300)])
def test_writes_of_long_calls_stay_inside(lens, D):
    """Guard zones around the outputs and a workspace of just the size asked for."""
    import torch
    import paper_2609_32114_amd as P
    lib = P.load_library()
    T, N = sum(lens), len(lens)
    t = {k: v.cuda() for k, v in make(lens, D, "bf16", "f32", False, 9).items()}
    n = P.glr_workspace_size(T, D)
    sizes = {"h": T * D * 2, "s": N * D * 4, "ck": (T + 127) // 128 * D * 4, "dx": T * D * 2, "dg": T * D * 4,
             "ds0": N * D * 4, "ws": n}
    raw = {k: torch.full((2048 + v + 2048,), 0xA5, dtype=torch.uint8, device="cuda") for k, v in sizes.items()}
    o = {k: v.data_ptr() + 2048 for k, v in raw.items()}
    cu, st = offsets(lens), torch.cuda.current_stream().cuda_stream
    p = lambda k: t[k].data_ptr()
    assert lib.glr_prefill(p("x"), D, p("g"), D, p("s0"), cu.data_ptr(), N, T, D, 1, 0, 0, 0, o["h"], o["s"], o["ck"],
                           o["ws"], n, st) == 0
    assert lib.glr_backward(p("dh"), D, p("x"), D, p("g"), D, o["ck"], p("s0"), p("dfinal"), cu.data_ptr(), N, T, D,
                            1, 0, 0, 0, o["dx"], o["dg"], o["ds0"], o["ws"], n, st) == 0
    torch.cuda.synchronize()
    for k, buf in raw.items():
        v = buf.cpu().numpy()
        assert (v[:2048] == 0xA5).all() and (v[2048 + sizes[k]:] == 0xA5).all(), k


@pytest.mark.gpu
@pytest.mark.parametrize("N,D", [(7000, 33), (6000, 512), (1023, 40), (1024, 40)])
def test_thousands_of_sequences_in_long_calls(N, D):
    """More than 8192 tokens: pieces of 32 tokens that hold tens of sequences' ends, whose
    offsets lie in LDS up to 1023 of them and in memory beyond."""
    r = np.random.default_rng(N)
    lens = tuple(int(n) for n in r.integers(0, 4 if N > 2000 else 20, N))
    d = make(lens, D, "bf16", "f32", False, N)
    check(run(d, lens, False, True), expected(d, lens, False, True), "bf16", "f32", f"N={N} D={D} T={sum(lens)}")


@pytest.mark.gpu
@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("D", [64, 67])
def test_decode_from_slices(D, offset):
    """Operands as column slices of a wider matrix at any offset, and one gate row for all."""
    import torch
    import paper_2609_32114_amd as P
    N = 9
    for dtype, gate in TYPES:
        d = make((1,) * N, D, dtype, gate, False, D)
        wide = {k: torch.full((N, 3 * D + 5), float("nan"), dtype=d[k].dtype, device="cuda") for k in "xg"}
        for k, w in wide.items():
            w[:, offset:offset + D] = d[k].cuda()
        state = d["s0"].cuda()
        h = P.glr_decode(*(wide[k][:, offset:offset + D] for k in "xg"), state)
        want = expected(d, (1,) * N, False, False, backward=False)
        assert ref.excess(h, want["h"], dtype) <= 1.0 and ref.excess(state, want["h"], "f32") <= 1.0
        d["g"] = d["g"][:1].expand(N, D)
        state = d["s0"].cuda()
        h = P.glr_decode(d["x"].cuda(), d["g"][:1].cuda().expand(N, D), state)
        want = expected(d, (1,) * N, False, False, backward=False)
        assert ref.excess(h, want["h"], dtype) <= 1.0 and ref.excess(state, want["h"], "f32") <= 1.0
