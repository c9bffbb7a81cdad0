"""The selective state space scan: forward, backward and single tokens against the 64-bit
form of mixer_ref.py, whose bounds are the tolerances."""

import numpy as np
import pytest

import mixer_ref as ref
from gpu_harness import say

# one token to several chunks of 32; ends on and off groups of 8, 16 and 32; empty sequences
LENS = [(1,), (7,), (32,), (33,), (129,), (500,), (1, 1, 1), (0, 5, 0, 0, 130, 1, 0), (31, 33, 64, 8, 1),
        (100, 0, 57, 96, 3, 32)]
GRADS = ("dx", "ddt", "dA", "dB", "dC", "dskip", "dz", "dbias", "ds0")


def make(lens, D, S, G=1, dtype="bf16", step="bf16", raw=True, z=True, skip=True, s0=True, seed=0, slow=False):
    """Seeded inputs as the kernels will see them (rounded to their types): channels that forget
    within a few tokens to ones that remember thousands."""
    import torch
    r = np.random.default_rng(seed)
    T, N = sum(lens), len(lens)
    rnd = lambda v, t: torch.from_numpy(np.asarray(v, np.float32)).to(torch.bfloat16 if t == "bf16" else torch.float32)
    base = np.exp(np.log(0.001) + (0.2 if slow else 1.0) * np.log(100) * r.random(D))
    bias = np.log(np.expm1(base))
    v = r.standard_normal((T, D))
    return {"x": rnd(r.standard_normal((T, D)), dtype), "dt": rnd(v if raw else np.log1p(np.exp(v + bias)), step),
            "A": rnd(-np.arange(1, S + 1) * (1 + 0.1 * r.random((D, S))), "f32"),
            "B": rnd(r.standard_normal((T, G, S)), dtype), "C": rnd(r.standard_normal((T, G, S)), dtype),
            "skip": rnd(1 + 0.1 * r.standard_normal(D), "f32") if skip else None,
            "z": rnd(r.standard_normal((T, D)), dtype) if z else None,
            "bias": rnd(bias, "f32") if raw else None, "s0": rnd(r.standard_normal((N, D, S)), "f32") if s0 else None,
            "dy": rnd(r.standard_normal((T, D)), dtype), "dfinal": rnd(r.standard_normal((N, D, S)), "f32") if s0 else None}


def np64(d):
    return {k: None if v is None else v.double().numpy() for k, v in d.items()}


def expected(d, lens, raw):
    n = np64(d)
    return ref.ssm(n["x"], n["dt"], n["A"], n["B"], n["C"], lens, n["skip"], n["z"], n["bias"], n["s0"], raw, n["dy"],
                   n["dfinal"])


def offsets(lens):
    import torch
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")


TOKENS = ("x", "dt", "B", "C", "z", "dy")


def run(d, lens, raw, cu=None, place=lambda t: t.cuda()):
    import torch
    import paper_2609_32114_amd as P
    t = {k: None if v is None else place(v) if k in TOKENS else v.cuda() for k, v in d.items()}
    how = dict(skip=t["skip"], z=t["z"], dt_bias=t["bias"], initial_state=t["s0"],
               cu_seqlens=offsets(lens) if cu is None else cu, preprocess=P.PRE_GATE_SOFTPLUS if raw else 0)
    args = (t["x"], t["dt"], t["A"], t["B"], t["C"])
    y, final = P.ssm_prefill(*args, **how)
    y2, final2, saved = P.ssm_prefill(*args, output_checkpoints=True, **how)
    assert torch.equal(y, y2) or bool(torch.isnan(y).any())
    grads = P.ssm_backward(t["dy"], *args, saved, dfinal=t["dfinal"], **how)
    torch.cuda.synchronize()
    return {"y": y, "final": final, **dict(zip(GRADS, grads))}


def kind(name, dtype, step):
    return step if name == "ddt" else "f32" if name in ("final", "dA", "dskip", "dbias", "ds0") else dtype


def check(got, want, dtype, step, label):
    off = {k: ref.excess(v, want[k], kind(k, dtype, step)) for k, v in got.items() if v is not None}
    say(f"[ssm] {label}: " + " ".join(f"{k}={v:.3f}" for k, v in off.items()))
    assert max(off.values()) <= 1.0, (label, off)


# ------------------------------------------------------------------ the oracle (CPU)
@pytest.mark.parametrize("raw", [False, True])
def test_oracle_gradient_is_that_of_its_values(raw):
    """Against central differences of the oracle's own values in 64 bits: a step of 1e-6 leaves
    1e-12 of curvature and 1e-9 of rounding."""
    lens, D, S, G = (4, 0, 1, 3), 4, 3, 2
    d = np64(make(lens, D, S, G, "f32", "f32", raw, seed=1))
    names = {"x": "dx", "dt": "ddt", "A": "dA", "B": "dB", "C": "dC", "skip": "dskip", "z": "dz", "s0": "ds0"}
    if raw:
        names["bias"] = "dbias"

    def loss(v):
        o = ref.ssm(v["x"], v["dt"], v["A"], v["B"], v["C"], lens, v["skip"], v["z"], v.get("bias"), v["s0"], raw)
        return float((o["y"][0] * d["dy"]).sum() + (o["final"][0] * d["dfinal"]).sum())

    o = ref.ssm(d["x"], d["dt"], d["A"], d["B"], d["C"], lens, d["skip"], d["z"], d["bias"], d["s0"], raw, d["dy"],
                d["dfinal"])
    for name, grad in names.items():
        for i in np.ndindex(o[grad][0].shape):
            lo, hi = ({k: d[k].copy() for k in names} for _ in range(2))
            lo[name][i] -= 1e-6
            hi[name][i] += 1e-6
            diff = (loss(hi) - loss(lo)) / 2e-6
            assert abs(diff - o[grad][0][i]) <= 1e-7 * (1 + abs(diff)), (name, i)


def test_oracle_closed_forms():
    """Constant inputs sum geometrically; a zero step keeps the state."""
    T, dt, A = 30, 0.25, -0.5
    one = np.ones((T, 1))
    o = ref.ssm(one, dt * one, np.array([[A]]), np.ones((T, 1, 1)), np.ones((T, 1, 1)), (T,))
    q = np.exp(dt * A)
    assert np.allclose(o["y"][0][:, 0], dt * (1 - q ** np.arange(1, T + 1)) / (1 - q), rtol=1e-13)
    o = ref.ssm(one, 0 * one, np.array([[A]]), np.ones((T, 1, 1)), np.ones((T, 1, 1)), (T,), s0=np.full((1, 1, 1), 3.0))
    assert np.array_equal(o["y"][0], 3 * one)


# -------------------------------------------------------------------------- GPU
TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,step", TYPES, ids=lambda t: t)
@pytest.mark.parametrize("lens", LENS, ids=lambda n: "-".join(map(str, n)))
def test_against_oracle(lens, dtype, step):
    for i, (raw, z, skip, s0) in enumerate([(True, True, True, True), (False, True, False, False), (True, False, True, False),
                                           (False, False, False, True)]):
        D = (128, 70, 1, 64)[i]
        d = make(lens, D, 16, 1, dtype, step, raw, z, skip, s0, seed=10 + i, slow=i == 3)
        check(run(d, lens, raw), expected(d, lens, raw), dtype, step, f"{lens} D={D} {dtype}/{step} form {i}")


@pytest.mark.gpu
@pytest.mark.parametrize("S", [1, 2, 3, 4, 8, 15, 16, 17, 31, 32, 33, 48, 63, 64])
def test_states(S):
    lens = (37, 0, 70, 1)
    d = make(lens, 67, S, 1, "bf16", "f32", seed=S)
    check(run(d, lens, True), expected(d, lens, True), "bf16", "f32", f"S={S}")


@pytest.mark.gpu
@pytest.mark.parametrize("D,G", [(1, 1), (2, 2), (6, 3), (63, 1), (65, 1), (128, 2), (130, 2), (192, 64), (255, 5), (257, 1),
                                 (520, 2), (1280, 1)])
def test_widths_and_groups(D, G):
    for S in (16, 5) if D < 500 else (16,):
        lens = (40, 33)
        d = make(lens, D, S, G, "bf16", "bf16", seed=D + S)
        check(run(d, lens, True), expected(d, lens, True), "bf16", "bf16", f"D={D} G={G} S={S}")


@pytest.mark.gpu
@pytest.mark.parametrize("D,G", [(256, 1), (300, 1), (520, 2)])
@pytest.mark.parametrize("S", [17, 32, 33, 64])
def test_many_states_in_wide_calls(S, D, G):
    """Workgroups of four waves with more than 16 states, some of whose columns are missing."""
    lens = (20, 0, 37, 1)
    d = make(lens, D, S, G, "bf16", "f32", seed=D + S)
    check(run(d, lens, True), expected(d, lens, True), "bf16", "f32", f"D={D} G={G} S={S}")


@pytest.mark.gpu
def test_many_sequences():
    """More sequences than a workgroup checks alone, of no, one, two and five tokens."""
    lens = tuple([1, 2, 0, 5] * 200)
    for dtype, S in (("bf16", 16), ("f32", 20)):
        d = make(lens, 40, S, 1, dtype, "f32", seed=S)
        check(run(d, lens, True), expected(d, lens, True), dtype, "f32", f"{len(lens)} sequences S={S}")


@pytest.mark.gpu
@pytest.mark.parametrize("S,G", [(16, 1), (40, 2)])
def test_long_sequences(S, G):
    """Many chunks to a run of the carry, channels that remember most of them."""
    lens = (2500, 1, 1111)
    d = make(lens, 32, S, G, "f32", "f32", False, seed=3, slow=True)
    check(run(d, lens, False), expected(d, lens, False), "f32", "f32", f"{lens} S={S}")


@pytest.mark.gpu
def test_chunks_of_all_lengths():
    """Calls wide enough for chunks of 64 tokens and more, on the plain form in 64 bits of a few
    channels (channels are independent but for dB and dC)."""
    import torch
    import paper_2609_32114_amd as P
    D, S, lens = 8192, 16, (1500, 700, 1, 400)
    T = sum(lens)
    pick = [0, 63, 64, 4097, 8191]
    d = make(lens, len(pick), S, 1, "bf16", "bf16", seed=8)
    wide = {}
    for k, v in d.items():
        if k in ("B", "C"):
            wide[k] = v
        else:
            axis = 1 if k in ("x", "dt", "z", "dy", "s0", "dfinal") else 0
            shape = list(v.shape)
            shape[axis] = D
            w = torch.zeros(shape, dtype=v.dtype)
            w.index_copy_(axis, torch.tensor(pick), v)
            wide[k] = w
    wide["A"][wide["A"] == 0] = -1.0
    got = run(wide, lens, True)
    assert P.ssm_workspace_size(T, D, S) < P.ssm_workspace_size(T, D, S, backward=True)
    want = expected(d, lens, True)
    narrow = {}
    for k, v in got.items():
        axis = {"y": 1, "dx": 1, "ddt": 1, "dz": 1, "final": 1, "ds0": 1, "dA": 0, "dskip": 0, "dbias": 0}.get(k)
        # x and dy are zero in the other channels: so are their parts of dB and dC
        narrow[k] = v if axis is None else v.index_select(axis, torch.tensor(pick, device="cuda"))
    check(narrow, want, "bf16", "bf16", "8192 channels")


@pytest.mark.gpu
@pytest.mark.parametrize("D", [66, 200])
def test_strides(D):
    """Column slices at odd places; B and C as slices of one projection; one row for all tokens."""
    import torch
    lens = (5, 40, 1)
    for dtype in ("bf16", "f32"):
        d = make(lens, D, 16, 2, dtype, dtype, seed=7)

        def inside(t):
            flat = t.reshape(t.shape[0], -1)
            wide = torch.full((flat.shape[0], 2 * flat.shape[1] + 3), float("nan"), dtype=t.dtype, device="cuda")
            wide[:, 1:1 + flat.shape[1]] = flat.cuda()
            part = wide[:, 1:1 + flat.shape[1]]
            return part.unflatten(1, t.shape[1:]) if t.dim() == 3 else part

        check(run(d, lens, True, place=inside), expected(d, lens, True), dtype, dtype, f"slices D={D} {dtype}")
        for k in TOKENS:
            d[k] = d[k][:1].expand(d[k].shape).clone()
        check(run(d, lens, True, place=lambda t: t[:1].cuda().expand(t.shape)), expected(d, lens, True), dtype, dtype,
              f"one row D={D} {dtype}")


@pytest.mark.gpu
def test_calls_of_one_group_and_sequence():
    """B and C without a group's dimension and no offsets: the same bits."""
    import torch
    import paper_2609_32114_amd as P
    d = make((300,), 130, 16, seed=9)
    a = run(d, (300,), True)
    t = {k: None if v is None else v.cuda() for k, v in d.items()}
    args = (t["x"], t["dt"], t["A"], t["B"][:, 0], t["C"][:, 0])
    how = dict(skip=t["skip"], z=t["z"], dt_bias=t["bias"], initial_state=t["s0"], preprocess=P.PRE_GATE_SOFTPLUS)
    y, final, saved = P.ssm_prefill(*args, output_checkpoints=True, **how)
    grads = P.ssm_backward(t["dy"], *args, saved, dfinal=t["dfinal"], **how)
    assert torch.equal(y, a["y"]) and torch.equal(final, a["final"])
    for k, v in zip(GRADS, grads):
        assert torch.equal(v.reshape(-1), a[k].reshape(-1)), k


@pytest.mark.gpu
def test_extreme_steps():
    """Raw steps far out on both sides: a step of zero keeps the state, a long one forgets it; and
    a state that decays by more than the least float within a token."""
    lens, D = (70,), 64
    d = make(lens, D, 16, 1, "f32", "f32", seed=2)
    d["dt"][::3] = -200.0
    d["dt"][1::7] = 30.0
    d["dt"][5] = float("-inf")
    check(run(d, lens, True), expected(d, lens, True), "f32", "f32", "far steps")


@pytest.mark.gpu
@pytest.mark.parametrize("S", [16, 40])
def test_no_tokens(S):
    import torch
    import paper_2609_32114_amd as P
    D = 70
    A, s0 = -torch.rand(D, S, device="cuda"), torch.randn(2, D, S, device="cuda")
    x, B, cu = torch.empty(0, D, device="cuda"), torch.empty(0, S, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    y, final, saved = P.ssm_prefill(x, x, A, B, B, initial_state=s0, cu_seqlens=cu, output_checkpoints=True)
    assert y.shape == (0, D) and torch.equal(final, s0)
    dfinal = torch.randn_like(s0)
    grads = dict(zip(GRADS, P.ssm_backward(x, x, x, A, B, B, saved, initial_state=s0, dfinal=dfinal, cu_seqlens=cu)))
    assert torch.equal(grads["ds0"], dfinal) and not grads["dA"].any()


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [[0, 5, 3, 200], [1, 5, 9, 200], [0, 5, 9, 199], [0, 300, 9, 200], [-4, 5, 9, 200]])
@pytest.mark.parametrize("S", [16, 40])
def test_malformed_offsets(bad, S):
    """No token is processed, states pass through, the status says so."""
    import torch
    import paper_2609_32114_amd as P
    d = make((5, 4, 191), 68, S, seed=2)
    t = {k: None if v is None else v.cuda() for k, v in d.items()}
    cu = torch.tensor(bad, dtype=torch.int32, device="cuda")
    ws = torch.zeros(P.ssm_workspace_size(200, 68, S, 1, True), dtype=torch.uint8, device="cuda")
    out = torch.full((200, 68), 7.0, dtype=torch.bfloat16, device="cuda")
    args = (t["x"], t["dt"], t["A"], t["B"], t["C"])
    how = dict(skip=t["skip"], z=t["z"], dt_bias=t["bias"], initial_state=t["s0"], cu_seqlens=cu, workspace=ws,
               preprocess=P.PRE_GATE_SOFTPLUS)
    y, final, saved = P.ssm_prefill(*args, out=out, output_checkpoints=True, **how)
    assert P.device_status(ws) == P.DEV_BAD_SEQLENS
    assert bool((y == 7).all()) and torch.equal(final, t["s0"])
    ws.zero_()
    grads = dict(zip(GRADS, P.ssm_backward(t["dy"], *args, torch.zeros_like(saved), dfinal=t["dfinal"], **how)))
    assert P.device_status(ws) == P.DEV_BAD_SEQLENS
    assert not grads["dA"].any() and not grads["dbias"].any() and torch.equal(grads["ds0"], t["dfinal"])


@pytest.mark.gpu
@pytest.mark.parametrize("S", [16, 40])
def test_no_value_of_another_sequence(S):
    """A sequence's results are the same beside neighbours of NaN and infinities, in its wave and
    in the chunks around it."""
    import torch
    lens = (45, 60, 70)
    d = make(lens, 66, S, 1, "f32", "f32", seed=4)
    clean = run(d, lens, True)
    mid = slice(45, 105)
    for v in (float("nan"), float("inf")):
        bad = {k: None if t is None else t.clone() for k, t in d.items()}
        for k in TOKENS:
            bad[k][:45] = v
            bad[k][105:] = v
        for k in ("s0", "dfinal"):
            bad[k][0] = v
            bad[k][2] = v
        got = run(bad, lens, True)
        for k in ("y", "dx", "ddt", "dz", "dB", "dC"):
            assert torch.equal(got[k][mid], clean[k][mid]), (k, v)
        for k in ("final", "ds0"):
            assert torch.equal(got[k][1], clean[k][1]), (k, v)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,step", TYPES, ids=lambda t: t)
@pytest.mark.parametrize("N,D,S,G", [(1, 1, 16, 1), (1, 2048, 16, 1), (5, 67, 16, 1), (33, 260, 8, 2), (7, 65, 5, 1),
                                     (3, 64, 64, 4), (2, 100, 32, 1), (64, 1280, 16, 1), (9, 130, 4, 1), (2, 5, 33, 1),
                                     (4, 70, 2, 1), (3, 66, 6, 2), (5, 65, 12, 1), (4, 130, 24, 2), (7, 97, 40, 1),
                                     (6, 260, 61, 4), (1, 3, 1, 1)])
def test_decode_against_oracle(N, D, S, G, dtype, step):
    """One token of each sequence from a shuffled pool; padding and idle slots are left alone."""
    import torch
    import paper_2609_32114_amd as P
    for raw, z, skip in ((True, True, True), (False, False, False)):
        lens = (1,) * N
        d = make(lens, D, S, G, dtype, step, raw, z, skip, seed=N + D)
        want = expected(d, lens, raw)
        pool = torch.full((N + 3, D, S), 5.0, device="cuda")
        slots = torch.randperm(N + 3, device="cuda")[:N].to(torch.int32)
        pool[slots.long()] = d["s0"].cuda()
        table = torch.cat([slots, torch.tensor([-1, N + 3], dtype=torch.int32, device="cuda")])
        t = {k: None if d[k] is None else torch.cat([d[k], d[k][:1], d[k][:1]]).cuda() for k in ("x", "dt", "B", "C", "z")}
        y = P.ssm_decode(t["x"], t["dt"], d["A"].cuda(), t["B"], t["C"], pool, slots=table,
                         skip=d["skip"].cuda() if skip else None, z=t["z"], dt_bias=d["bias"].cuda() if raw else None,
                         preprocess=P.PRE_GATE_SOFTPLUS if raw else 0)
        assert not y[N:].any()
        check({"y": y[:N], "final": pool[slots.long()]}, want, dtype, step, f"step N={N} D={D} S={S} G={G} {dtype}/{step}")
        idle = torch.ones(N + 3, dtype=torch.bool, device="cuda")
        idle[slots.long()] = False
        assert bool((pool[idle] == 5).all())


@pytest.mark.gpu
def test_decode_continues_prefill():
    """Tokens fed one at a time from the state a prefill left, against one prefill in 64 bits."""
    import torch
    import paper_2609_32114_amd as P
    lens, steps = [40, 1, 77], 4
    whole = [n + steps for n in lens]
    d = make(whole, 192, 16, 1, "f32", "f32", seed=12)
    want = expected(d, whole, True)
    t = {k: None if v is None else v.cuda() for k, v in d.items()}
    parts = {k: t[k].split(whole) for k in ("x", "dt", "B", "C", "z")}
    first = {k: torch.cat([p[:n] for p, n in zip(v, lens)]) for k, v in parts.items()}
    how = dict(skip=t["skip"], dt_bias=t["bias"], preprocess=P.PRE_GATE_SOFTPLUS)
    _, state = P.ssm_prefill(first["x"], first["dt"], t["A"], first["B"], first["C"], z=first["z"], initial_state=t["s0"],
                             cu_seqlens=offsets(lens), **how)
    rows = []
    for s in range(steps):
        at = {k: torch.stack([p[n + s] for p, n in zip(v, lens)]) for k, v in parts.items()}
        rows.append(P.ssm_decode(at["x"], at["dt"], t["A"], at["B"], at["C"], state, z=at["z"], **how))
    got = torch.stack(rows, 1).reshape(len(lens) * steps, -1)
    at = np.concatenate([np.arange(sum(whole[:i]) + n, sum(whole[:i + 1])) for i, n in enumerate(lens)])
    check({"y": got, "final": state}, {"y": tuple(v[at] for v in want["y"]), "final": want["final"]}, "f32", "f32",
          "decode after prefill")


@pytest.mark.gpu
@pytest.mark.parametrize("S", [16, 40])
def test_repeats_bit_for_bit(S):
    import torch
    lens = (700, 3, 900)
    d = make(lens, 520, S, seed=6)
    a, b = run(d, lens, True), run(d, lens, True)
    assert all(torch.equal(a[k], b[k]) for k in a)


@pytest.mark.gpu
@pytest.mark.parametrize("S", [2, 20])
def test_slow_growth_over_many_chunks(S):
    """Rates above zero, with less than e^60 in any 500 tokens but more than fp32 holds over a run of
    the carry's chunks: a state that is still zero, or small enough, stays what it is."""
    import torch
    D, T = 8, 16384
    for form in ("zero", "small"):
        d = make((T,), D, S, 1, "f32", "f32", False, False, False, form == "small", seed=S)
        d["A"][:, 0] = 0.6
        d["dt"] = torch.full((T, D), 0.2)
        if form == "zero":  # fed in the last 400 tokens only, read (in the backward pass) in the first 300
            d["A"][:, 1:] = -0.6
            d["x"][:T - 400] = 0.0
            d["dy"][300:] = 0.0
        else:  # e^120 in 1000 tokens, from 1e-20 on, and nothing after them
            d["dt"][:1024] = d["dt"][2024:] = 0.0
            d["s0"] *= 1e-20
            d["dfinal"] *= 1e-20
            d["x"][:] = d["dy"][:] = 0.0
        check(run(d, (T,), False), expected(d, (T,), False), "f32", "f32", f"growth from {form} S={S}")


@pytest.mark.gpu
@pytest.mark.parametrize("S", [16, 17, 20, 32, 33, 40, 64])
@pytest.mark.parametrize("D,G,pick", [(8192, 1, (0, 63, 64, 4097, 8191)), (4096, 64, (0, 63, 4032, 4095)),
                                      (4104, 2, (0, 2051, 2052, 4103))])
def test_chunks_of_many_groups(D, G, pick, S):
    """Backward chunks of several groups of 16 tokens for every padded number of states, in workgroups
    of one wave and of four, the last of whose lanes lie beyond a group of channels: a few channels
    against the plain form in 64 bits (in the others, x and dy are zero)."""
    import torch
    import paper_2609_32114_amd as P
    lens = (1500, 700, 1, 400)
    T, where = sum(lens), torch.tensor(pick)
    groups = sorted({c // (D // G) for c in pick})
    dtype = "f32" if S in (20, 40) else "bf16"
    d = make(lens, len(pick), S, len(groups), dtype, "f32", seed=D + S, slow=True)
    wide = {}
    for k, v in d.items():
        axis = 0 if k in ("A", "skip", "bias") else 1
        shape = list(v.shape)
        shape[axis] = G if k in ("B", "C") else D
        wide[k] = torch.zeros(shape, dtype=v.dtype)
        wide[k].index_copy_(axis, torch.tensor(groups) if k in ("B", "C") else where, v)
    wide["A"][wide["A"] == 0] = -1.0
    # tokens of a chunk, from the parts of the workspace that grow with the number of chunks
    padded = 16 if S <= 16 else 32 if S <= 32 else 64
    teams = -(-(D // G) // 64) if D // G < 193 else -(-(D // G) // 256)
    rest = P.ssm_workspace_size(T, D, S, G, True) - teams * T * G * 2 * padded * 4
    assert T / (rest / ((2 * padded + 3) * D * 4)) > 40
    got = run(wide, lens, True)
    narrow = {}
    for k, v in got.items():
        axis = 0 if k in ("dA", "dskip", "dbias") else 1
        narrow[k] = v.index_select(axis, torch.tensor(groups if k in ("dB", "dC") else pick, device="cuda"))
    check(narrow, expected(d, lens, True), dtype, "f32", f"{T} x {D} x {S}, {G} groups")
