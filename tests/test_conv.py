"""The short causal convolution: forward, backward and single tokens against the 64-bit form of
mixer_ref.py, whose bounds are the tolerances."""

import numpy as np
import pytest

import mixer_ref as ref
from gpu_harness import say

# lengths of packed sequences: shorter than the window, ends on and off the kernels' runs of 8
# and 16 tokens, empty sequences
LENS = [(1,), (2,), (7,), (64,), (129,), (1000,), (1, 1, 1, 2, 3), (0, 5, 0, 0, 130, 1, 0), (15, 16, 17, 8, 1, 24),
        (200, 0, 57, 300, 3, 129)]


def make(lens, D, W, dtype, seed, s0=True, bias=True):
    """Seeded inputs as the kernels will see them (rounded to their types)."""
    import torch
    r = np.random.default_rng(seed)
    T, N = sum(lens), len(lens)
    rnd = lambda shape, t, s=1.0: torch.from_numpy(np.asarray(s * r.standard_normal(shape), np.float32)).to(
        torch.bfloat16 if t == "bf16" else torch.float32)
    return {"x": rnd((T, D), dtype), "dy": rnd((T, D), dtype), "w": rnd((D, W), "f32", 0.5),
            "b": rnd((D,), "f32", 0.3) if bias else None, "w0": rnd((N, W - 1, D), dtype) if s0 else None,
            "dfinal": rnd((N, W - 1, D), dtype) if s0 else None}


def np64(d):
    return {k: None if v is None else v.double().numpy() for k, v in d.items()}


def expected(d, lens, act):
    n = np64(d)
    return ref.conv(n["x"], n["w"], n["b"], lens, n["w0"], act is not None, n["dy"], n["dfinal"])


def offsets(lens):
    import torch
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")


def run(d, lens, act, cu=None, place=lambda t: t.cuda()):
    import torch
    import paper_2609_32114_amd as P
    t = {k: None if v is None else place(v) if k in ("x", "dy") else v.cuda() for k, v in d.items()}
    how = dict(bias=t["b"], initial_window=t["w0"], cu_seqlens=offsets(lens) if cu is None else cu, activation=act)
    y, final = P.conv_prefill(t["x"], t["w"], **how)
    dx, dw, db, dw0 = P.conv_backward(t["dy"], t["x"], t["w"], dfinal=t["dfinal"], **how)
    torch.cuda.synchronize()
    return {"y": y, "final": final, "dx": dx, "dw": dw, "db": db, "dw0": dw0}


def check(got, want, dtype, label):
    off = {k: ref.excess(v, want[k], "f32" if k in ("dw", "db") else dtype) for k, v in got.items() if v is not None}
    say(f"[conv] {label}: " + " ".join(f"{k}={v:.3f}" for k, v in off.items()))
    assert max(off.values()) <= 1.0, (label, off)


# ------------------------------------------------------------------ the oracle (CPU)
@pytest.mark.parametrize("act", ["silu", None])
@pytest.mark.parametrize("W", [2, 4])
def test_oracle_gradient_is_that_of_its_values(W, act):
    """Against central differences of the oracle's own values in 64 bits: a step of 1e-6 leaves
    1e-12 of curvature and 1e-9 of rounding."""
    lens, D = (1, 0, 6, 2), 2
    d = np64(make(lens, D, W, "f32", 5))

    def loss(x, w, b, w0):
        o = ref.conv(x, w, b, lens, w0, act is not None)
        return float((o["y"][0] * d["dy"]).sum() + (o["final"][0] * d["dfinal"]).sum())

    o = ref.conv(d["x"], d["w"], d["b"], lens, d["w0"], act is not None, d["dy"], d["dfinal"])
    for name, grad in (("x", "dx"), ("w", "dw"), ("b", "db"), ("w0", "dw0")):
        for i in np.ndindex(o[grad][0].shape):
            lo, hi = ({k: d[k].copy() for k in ("x", "w", "b", "w0")} for _ in range(2))
            lo[name][i] -= 1e-6
            hi[name][i] += 1e-6
            diff = (loss(**hi) - loss(**lo)) / 2e-6
            assert abs(diff - o[grad][0][i]) <= 1e-7 * (1 + abs(diff)), (name, i)


def test_oracle_closed_form():
    """A single tap picks an earlier input, from the window where the sequence has none."""
    x, w0 = np.arange(1.0, 6.0)[:, None], np.array([[[-3.0], [-2.0], [-1.0]]])
    for back in range(4):
        w = np.zeros((1, 4))
        w[0, 3 - back] = 1.0
        o = ref.conv(x, w, None, (5,), w0, act=False)
        assert np.array_equal(o["y"][0][:, 0], np.concatenate([w0[0, :, 0], x[:, 0]])[3 - back:8 - back])
        assert np.array_equal(o["final"][0][0, :, 0], [3.0, 4.0, 5.0])


# -------------------------------------------------------------------------- GPU
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", LENS, ids=lambda n: "-".join(map(str, n)))
def test_against_oracle(lens, dtype):
    for i, (W, act) in enumerate([(4, "silu"), (4, None), (2, "silu"), (8, "silu"), (3, None)]):
        D = (128, 256, 300, 67, 1)[i]
        d = make(lens, D, W, dtype, 10 + i, s0=i != 2, bias=i != 1)
        check(run(d, lens, act), expected(d, lens, act), dtype, f"{lens} D={D} W={W} {dtype} {act}")


@pytest.mark.gpu
@pytest.mark.parametrize("D", [1, 2, 3, 4, 5, 63, 64, 65, 255, 256, 257, 259, 511, 1027, 1280, 2048])
def test_widths(D):
    for dtype in ("bf16", "f32"):
        lens = (31, 0, 70)
        d = make(lens, D, 4, dtype, D)
        check(run(d, lens, "silu"), expected(d, lens, "silu"), dtype, f"D={D} {dtype}")


@pytest.mark.gpu
@pytest.mark.parametrize("W", range(2, 9))
def test_taps(W):
    for D in (40, 264):
        lens = (3, 1, 0, 9, 40)
        d = make(lens, D, W, "bf16", W)
        check(run(d, lens, "silu"), expected(d, lens, "silu"), "bf16", f"W={W} D={D}")


@pytest.mark.gpu
def test_long_and_many():
    """A call of several runs a wave, and more sequences than one workgroup checks alone."""
    for lens, D in (((5000, 1, 3300),), 768), ((tuple([1, 2, 0, 5] * 400),), 72):
        lens = lens[0]
        d = make(lens, D, 4, "bf16", 3)
        check(run(d, lens, "silu"), expected(d, lens, "silu"), "bf16", f"{len(lens)} sequences, {sum(lens)} x {D}")


@pytest.mark.gpu
@pytest.mark.parametrize("D", [66, 260])
def test_strides(D):
    """Column slices at odd places, and one row for all tokens."""
    import torch
    lens = (5, 40, 1)
    for dtype in ("bf16", "f32"):
        d = make(lens, D, 4, dtype, 7)

        def inside(t):
            wide = torch.full((t.shape[0], 2 * D + 3), float("nan"), dtype=t.dtype, device="cuda")
            wide[:, 1:1 + D] = t.cuda()
            return wide[:, 1:1 + D]

        check(run(d, lens, "silu", place=inside), expected(d, lens, "silu"), dtype, f"slices D={D} {dtype}")
        d["x"] = d["x"][:1].expand(sum(lens), D).clone()
        check(run(d, lens, "silu", place=lambda t: t.cuda() if t is not d["x"] else t[:1].cuda().expand(sum(lens), D)),
              expected(d, lens, "silu"), dtype, f"one row D={D} {dtype}")


@pytest.mark.gpu
def test_single_sequence_without_offsets():
    import torch
    import paper_2609_32114_amd as P
    d = make((77,), 130, 4, "bf16", 9)
    a = run(d, (77,), "silu")
    y, final = P.conv_prefill(d["x"].cuda(), d["w"].cuda(), bias=d["b"].cuda(), initial_window=d["w0"].cuda())
    dx, dw, db, dw0 = P.conv_backward(d["dy"].cuda(), d["x"].cuda(), d["w"].cuda(), bias=d["b"].cuda(),
                                      initial_window=d["w0"].cuda(), dfinal=d["dfinal"].cuda())
    for k, v in {"y": y, "final": final, "dx": dx, "dw": dw, "db": db, "dw0": dw0}.items():
        assert torch.equal(a[k], v), k


@pytest.mark.gpu
def test_no_tokens():
    import torch
    import paper_2609_32114_amd as P
    w, w0 = torch.randn(70, 4, device="cuda"), torch.randn(2, 3, 70, device="cuda")
    x, cu = torch.empty(0, 70, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    y, final = P.conv_prefill(x, w, initial_window=w0, cu_seqlens=cu)
    assert y.shape == (0, 70) and torch.equal(final, w0)
    dfinal = torch.randn_like(w0)
    _, dw, _, dw0 = P.conv_backward(x, x, w, initial_window=w0, dfinal=dfinal, cu_seqlens=cu)
    assert torch.equal(dw0, dfinal) and not dw.any()
    final = P.conv_prefill(x, w, cu_seqlens=cu)[1]
    assert not final.any()


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [[0, 5, 3, 20], [1, 5, 9, 20], [0, 5, 9, 19], [0, 30, 9, 20], [-4, 5, 9, 20]])
def test_malformed_offsets(bad):
    """No token is processed, windows pass through, the status says so."""
    import torch
    import paper_2609_32114_amd as P
    d = make((5, 4, 11), 68, 4, "bf16", 2)
    cu = torch.tensor(bad, dtype=torch.int32, device="cuda")
    ws = torch.zeros(P.conv_workspace_size(20, 68, 4, True), dtype=torch.uint8, device="cuda")
    out = torch.full((20, 68), 7.0, dtype=torch.bfloat16, device="cuda")
    y, final = P.conv_prefill(d["x"].cuda(), d["w"].cuda(), initial_window=d["w0"].cuda(), cu_seqlens=cu, workspace=ws, out=out)
    assert P.device_status(ws) == P.DEV_BAD_SEQLENS
    assert bool((y == 7).all()) and torch.equal(final, d["w0"].cuda())
    ws.zero_()
    _, dw, _, dw0 = P.conv_backward(d["dy"].cuda(), d["x"].cuda(), d["w"].cuda(), initial_window=d["w0"].cuda(),
                                    dfinal=d["dfinal"].cuda(), cu_seqlens=cu, workspace=ws)
    assert P.device_status(ws) == P.DEV_BAD_SEQLENS
    assert not dw.any() and torch.equal(dw0, d["dfinal"].cuda())


@pytest.mark.gpu
def test_no_value_of_another_sequence():
    """A sequence's results are the same beside neighbours of NaN and infinities."""
    import torch
    lens, D = (13, 3, 40), 260
    d = make(lens, D, 4, "f32", 4)
    clean = run(d, lens, "silu")
    for v in (float("nan"), float("inf")):
        bad = {k: None if t is None else t.clone() for k, t in d.items()}
        for k in ("x", "dy"):
            bad[k][:13] = v
            bad[k][16:] = v
        for k in ("w0", "dfinal"):
            bad[k][0] = v
            bad[k][2] = v
        got = run(bad, lens, "silu")
        for k in ("y", "dx"):
            assert torch.equal(got[k][13:16], clean[k][13:16]), (k, v)
        for k in ("final", "dw0"):
            assert torch.equal(got[k][1], clean[k][1]), (k, v)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,W", [(1, 1, 4), (1, 2048, 4), (5, 67, 3), (33, 260, 4), (256, 1284, 2), (7, 65, 8)])
def test_decode_continues_prefill(N, D, W, dtype):
    """Tokens fed one at a time through a shuffled pool give the same bits as one prefill (the same
    sums in the same order); padding and idle slots are left alone."""
    import torch
    import paper_2609_32114_amd as P
    steps, lens = 3, [1 + n % 5 for n in range(N)]
    d = make([n + steps for n in lens], D, W, dtype, N + D)
    cu = offsets([n + steps for n in lens])
    w, b = d["w"].cuda(), d["b"].cuda()
    whole, last = P.conv_prefill(d["x"].cuda(), w, bias=b, initial_window=d["w0"].cuda(), cu_seqlens=cu)
    parts = d["x"].cuda().split([n + steps for n in lens])
    _, window = P.conv_prefill(torch.cat([p[:n] for p, n in zip(parts, lens)]), w, bias=b,
                               initial_window=d["w0"].cuda(), cu_seqlens=offsets(lens))
    pool = torch.full((N + 3, W - 1, D), 5.0, dtype=whole.dtype, device="cuda")
    slots = torch.randperm(N + 3, device="cuda")[:N].to(torch.int32)
    pool[slots.long()] = window
    table = torch.cat([slots, torch.tensor([-1, N + 3], dtype=torch.int32, device="cuda")])
    for s in range(steps):
        x = torch.stack([p[n + s] for p, n in zip(parts, lens)] + [parts[0][0]] * 2)
        y = P.conv_decode(x, w, pool, bias=b, slots=table)
        want = torch.stack([p[n + s] for p, n in zip(whole.split([n + steps for n in lens]), lens)])
        assert torch.equal(y[:N], want) and not y[N:].any()
    assert torch.equal(pool[slots.long()], last)
    idle = torch.ones(N + 3, dtype=torch.bool, device="cuda")
    idle[slots.long()] = False
    assert bool((pool[idle] == 5).all())


@pytest.mark.gpu
def test_repeats_bit_for_bit():
    import torch
    d = make((700, 3, 900), 520, 4, "bf16", 6)
    a, b = run(d, (700, 3, 900), "silu"), run(d, (700, 3, 900), "silu")
    assert all(torch.equal(a[k], b[k]) for k in a)
