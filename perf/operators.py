"""Cases of the operators around the delta-rule layers: a gated linear
recurrence (``glr_*``) and the norms before and after a block (``add_norm``,
``gate_norm``).

``run`` computes a case in plain torch operations, in 32 bits, or, where
``own`` is true, with the library's kernels; ``exact`` gives the same from the
definitions in 64 bits.  Cases are plain dicts; the key ``op`` names the
operator:

glr_decode   one token for each of N sequences over a pool of states (pool 0:
             one state per sequence, no slot table; pad entries are padding)
glr_prefill  packed sequences (lens), D channels
glr_train    the same, forward and backward
add_norm     T rows of D: residual add with its scale, then the norm
add_norm_back, gate_norm, gate_norm_back   likewise; gate_norm has H heads of d

dtype: "bf16" or "f32" inputs; gate / res: the type of the gate or of the
residual stream.  fused: the operands are column slices of one wider matrix, as
a fused projection leaves them.
"""

import math

import torch

own = False

EPS = 1e-6


def _glr(op, name, lens, D, dtype="bf16", gate="f32", raw=False, convex=False, s0=True, fused=False):
    return {"name": name, "op": op, "lens": ",".join(str(n) for n in lens), "D": D, "dtype": dtype, "gate": gate,
            "raw": raw, "convex": convex, "s0": s0, "fused": fused}


def _step(name, N, D, dtype="bf16", gate="f32", raw=False, convex=False, pool=0, pad=0):
    return {"name": name, "op": "glr_decode", "N": N, "D": D, "dtype": dtype, "gate": gate, "raw": raw,
            "convex": convex, "pool": pool, "pad": pad}


def _add(op, name, T, D, dtype="bf16", res="bf16", post=False, vector=False, scale=1.0):
    return {"name": name, "op": op, "T": T, "D": D, "dtype": dtype, "res": res, "post": post, "vector": vector,
            "scale": scale}


def _gate(op, name, T, H, d, dtype="bf16", act="silu", fused=False):
    return {"name": name, "op": op, "T": T, "H": H, "d": d, "dtype": dtype, "act": act, "fused": fused}


def listed():
    return [
        # one user's token through the recurrence: latency of the smallest call
        _step("glr_decode_n1", 1, 2048),
        # a full serving batch over a paged state pool, gates as projected
        _step("glr_decode_n256", 256, 4096, gate="bf16", raw=True, convex=True, pool=320, pad=5),
        # an ordinary short prompt, operands as the layer's fused projection leaves them
        _glr("glr_prefill", "glr_prefill_t777", [777], 1280, gate="bf16", raw=True, convex=True, s0=False, fused=True),
        # a long prompt continued from a state
        _glr("glr_prefill", "glr_prefill_t32768", [32768], 2048),
        # a reference-precision training step of a short sequence
        _glr("glr_train", "glr_train_t2048_f32", [2048], 2048, dtype="f32", convex=True),
        # a training step on a packed batch of mid-size and long documents (the largest)
        _glr("glr_train", "glr_train_varlen8", [4021, 7513, 611, 8130, 2048, 6899, 1277, 4301], 2048),
        # one user's token through the norm before a block
        _add("add_norm", "add_norm_t1", 1, 2048),
        # a prompt of 4096 tokens, the residual stream kept in 32 bits
        _add("add_norm", "add_norm_t4096", 4096, 2048, res="f32", scale=0.5),
        # an odd width in 32 bits with a norm after the block too
        _add("add_norm", "add_norm_t333_odd_f32", 333, 1001, dtype="f32", res="f32", post=True, vector=True),
        # the backward pass of norms after and before a block with a scale per channel
        _add("add_norm_back", "add_norm_back_t8192", 8192, 2048, post=True, vector=True),
        # the norm and gate after a delta-rule mixer, the gate a slice of the fused projection
        _gate("gate_norm", "gate_norm_t4096_h16", 4096, 16, 128, fused=True),
        # their backward pass over a packed batch of grouped-head layers
        _gate("gate_norm_back", "gate_norm_back_t8192_h32", 8192, 32, 128),
    ]


def draw(rng):
    def logint(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def types():
        dtype = rng.choice(["bf16", "bf16", "f32"])
        return dtype, "f32" if dtype == "f32" else rng.choice(["bf16", "f32"])

    def width(hi=8192):
        # heads x head size of the delta-rule layers, or any width
        D = rng.choice([64, 128, 512, 768, 1280, 2048, 4096, logint(33, hi), logint(33, hi)])
        return D if D != 3072 else 2048

    op = rng.choice(["glr_decode", "glr_prefill", "glr_prefill", "glr_train", "glr_train", "add_norm", "add_norm",
                     "add_norm_back", "gate_norm", "gate_norm_back"])
    dtype, other = types()
    if op == "glr_decode":
        N = logint(1, 512)
        pool = N + rng.randrange(0, 64) if rng.random() < 0.7 else 0
        c = _step("", N, width(4096), dtype, other, rng.random() < 0.5, rng.random() < 0.5, pool,
                  rng.randrange(0, max(1, N // 8)) if pool else 0)
    elif op in ("glr_prefill", "glr_train"):
        D = width(4096)
        # the largest listed case has 34800 tokens of 2048 channels, forward and backward, in bf16
        most = 32000 * 2048 // D // (2 if dtype == "f32" else 1)
        T = logint(16, min(100000, most))
        n = min(T, 1 if rng.random() < 0.5 else logint(2, 64))
        cuts = sorted(rng.sample(range(1, T), n - 1)) if n > 1 else []
        lens = [b - a for a, b in zip([0] + cuts, cuts + [T])]
        c = _glr(op, "", lens, D, dtype, other, rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.5,
                 dtype == other and rng.random() < 0.5)
    elif op in ("add_norm", "add_norm_back"):
        D = width()
        c = _add(op, "", logint(1, min(20000, (8192 if op == "add_norm_back" else 16384) * 2048 // D)), D, dtype, other,
                 rng.random() < 0.4, rng.random() < 0.4, rng.choice([1.0, 0.5, 0.125]))
    else:
        H, d = rng.choice([(4, 64), (12, 64), (16, 64), (8, 128), (10, 128), (16, 128), (32, 128), (1, logint(17, 2048)),
                           (rng.randrange(1, 9), logint(17, 500))])
        c = _gate(op, "", logint(1, min(30000, 8192 * 32 * 128 // (H * d) // (2 if dtype == "f32" else 1))), H, d, dtype,
                  rng.choice(["silu", "silu", "sigmoid"]), rng.random() < 0.5)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _lens(case):
    return [int(n) for n in case["lens"].split(",")]


def _gen(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return gen


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _slices(tensors, fused):
    """The tensors, or equal column slices of one matrix that hold their values."""
    if not fused:
        return tensors
    whole = torch.cat([t.reshape(t.shape[0], -1) for t in tensors], 1)
    width = whole.shape[1] // len(tensors)
    return [whole[:, i * width:(i + 1) * width].unflatten(1, t.shape[1:]) if t.dim() > 2 else
            whole[:, i * width:(i + 1) * width] for i, t in enumerate(tensors)]


def _gates(case, gen, *shape):
    """Log-gates of channels that forget within a few tokens to channels that
    remember hundreds, or the raw projections of such a layer."""
    rate = torch.exp(math.log(0.003) * torch.rand(shape[-1], generator=gen, device="cuda"))
    z = _normal(gen, *shape)
    g = z + torch.log(torch.expm1(rate)) if case["raw"] else -rate * torch.log1p(torch.exp(z))
    return g.to(_dt(case["gate"]))


def prepare(case, seed):
    gen, op, dt = _gen(seed), case["op"], _dt(case["dtype"])
    s = {"case": case}
    if op == "glr_decode":
        N, D = case["N"], case["D"]
        pool = case["pool"] or N
        s["x"], s["g"] = _normal(gen, N, D).to(dt), _gates(case, gen, N, D)
        s["state"] = _normal(gen, pool, D)
        s["slots"] = None
        if case["pool"]:
            slots = torch.randperm(pool, generator=gen, device="cuda")[:N].to(torch.int32)
            if case["pad"]:
                slots[torch.randperm(N, generator=gen, device="cuda")[:case["pad"]]] = -1
            s["slots"] = slots
    elif op in ("glr_prefill", "glr_train"):
        lens, D = _lens(case), case["D"]
        T, N = sum(lens), len(lens)
        s["x"], s["g"] = _slices([_normal(gen, T, D).to(dt), _gates(case, gen, T, D)], case["fused"])
        s["s0"] = _normal(gen, N, D) if case["s0"] else None
        cu = [0]
        for n in lens:
            cu.append(cu[-1] + n)
        s["cu"] = torch.tensor(cu, dtype=torch.int32, device="cuda") if N > 1 else None
        if op == "glr_train":
            s["dh"] = _normal(gen, T, D).to(dt)
            s["dfinal"] = _normal(gen, N, D) if case["s0"] else None
    elif op in ("add_norm", "add_norm_back"):
        T, D, rt = case["T"], case["D"], _dt(case["res"])
        s["x"], s["res"] = _normal(gen, T, D).to(dt), (2.0 * _normal(gen, T, D)).to(rt)
        s["w"] = 1.0 + 0.1 * _normal(gen, D)
        s["w_post"] = 0.5 + 0.1 * _normal(gen, D) if case["post"] else None
        s["scale"] = case["scale"] * (1.0 + 0.2 * _normal(gen, D)) if case["vector"] else case["scale"]
        if op == "add_norm_back":
            s["dy"], s["dres"] = _normal(gen, T, D).to(dt), _normal(gen, T, D).to(rt)
    else:
        T, H, d = case["T"], case["H"], case["d"]
        s["o"] = (0.3 * _normal(gen, T, H, d)).to(dt)
        # the gate beside another operand of the same width in the projection's output
        z, other = _normal(gen, T, H, d).to(dt), _normal(gen, T, H, d).to(dt) if case["fused"] else None
        s["z"] = _slices([other, z], True)[1] if case["fused"] else z
        s["w"] = 1.0 + 0.1 * _normal(gen, d)
        if op == "gate_norm_back":
            s["dy"] = _normal(gen, T, H, d).to(dt)
    return s


# ------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2609_32114_amd as hagdn
    c = s["case"]
    op = c["op"]
    if op.startswith("glr"):
        how = {"convex": c["convex"], "preprocess": hagdn.PRE_GATE_SOFTPLUS if c["raw"] else 0}
        if op == "glr_decode":
            h = hagdn.glr_decode(s["x"], s["g"], s["state"], slots=s["slots"], **how)
            return {"h": h, "state": s["state"]}
        if op == "glr_prefill":
            h, final = hagdn.glr_prefill(s["x"], s["g"], initial_state=s["s0"], cu_seqlens=s["cu"], **how)
            return {"h": h, "final": final}
        h, final, saved = hagdn.glr_prefill(s["x"], s["g"], initial_state=s["s0"], cu_seqlens=s["cu"],
                                            output_checkpoints=True, **how)
        dx, dg, ds0 = hagdn.glr_backward(s["dh"], s["x"], s["g"], saved, initial_state=s["s0"], dfinal=s["dfinal"],
                                         cu_seqlens=s["cu"], **how)
        return {"h": h, "final": final, "dx": dx, "dg": dg, "ds0": ds0}
    if op == "add_norm":
        y, res = hagdn.add_norm(s["x"], s["w"], residual=s["res"], scale=s["scale"], post_weight=s["w_post"], eps=EPS)
        return {"y": y, "res": res}
    if op == "add_norm_back":
        dx, dres, dw, dscale, dpost = hagdn.add_norm_backward(s["dy"], s["res"], s["w"], dresidual=s["dres"], x=s["x"],
                                                              scale=s["scale"], post_weight=s["w_post"], eps=EPS)
        return {"dx": dx, "dres": dres, "dw": dw, "dscale": dscale, "dpost": dpost}
    if op == "gate_norm":
        return {"y": hagdn.gate_norm(s["o"], s["z"], s["w"], activation=c["act"], eps=EPS)}
    do, dz, dw = hagdn.gate_norm_backward(s["dy"], s["o"], s["z"], s["w"], activation=c["act"], eps=EPS)
    return {"do": do, "dz": dz, "dw": dw}


# ------------------------------------------------------------- the plain forms
def _gate_plain(c, g):
    """(a, w): the decay and the input's weight, in 32 bits."""
    g = g.float()
    if c["raw"]:
        a, b = 1.0 / (1.0 + torch.exp(g)), 1.0 / (1.0 + torch.exp(-g))
    else:
        a, b = torch.exp(g), -torch.expm1(g)
    return a, b if c["convex"] else torch.ones_like(a)


def _scan_plain(a, b, longest):
    """All states of h_t = a_t h_{t-1} + b_t from zero along the first axis by
    doubling: after the step of width d every token holds the map of the 2 d
    tokens up to it.  A sequence starts where a is zero."""
    d = 1
    while d < longest:
        b = torch.cat([b[:d], b[d:] + a[d:] * b[:-d]])
        a = torch.cat([a[:d], a[d:] * a[:-d]])
        d *= 2
    return b


def _run_glr_plain(s):
    c = s["case"]
    lens, D = _lens(c), c["D"]
    first = [sum(lens[:n]) for n in range(len(lens))]
    last = [f + n - 1 for f, n in zip(first, lens)]
    x, dt = s["x"].float(), s["x"].dtype
    a, w = _gate_plain(c, s["g"])
    s0 = s["s0"] if s["s0"] is not None else x.new_zeros(len(lens), D)
    b = w * x
    b[first] += a[first] * s0
    inner = a.clone()
    inner[first] = 0.0
    h = _scan_plain(inner, b, max(lens))
    out = {"h": h.to(dt), "final": h[last]}
    if c["op"] == "glr_prefill":
        return out
    before = torch.cat([h[:1], h[:-1]])
    before[first] = s0
    # e_t = a_t (dh_t + e_{t+1}), from each sequence's last token back
    dh = s["dh"].float().clone()
    if s["dfinal"] is not None:
        dh[last] += s["dfinal"]
    inner = a.clone()
    inner[last] = 0.0
    e = _scan_plain(inner.flip(0), (a * dh).flip(0), max(lens)).flip(0)
    after = torch.cat([e[1:], e[:1]])
    after[last] = 0.0
    dg = e * (before - x) if c["convex"] else e * before
    if c["raw"]:
        dg = dg * -(1.0 / (1.0 + torch.exp(-s["g"].float())))
    return {**out, "dx": (w * (dh + after)).to(dt), "dg": dg.to(s["g"].dtype),
            "ds0": e[first] if s["s0"] is not None else None}


def _act_plain(name, z):
    """The activation and its derivative."""
    sig = 1.0 / (1.0 + torch.exp(-z))
    return (z * sig, sig * (1.0 + z * (1.0 - sig))) if name == "silu" else (sig, sig * (1.0 - sig))


def _rstd_plain(x):
    return torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)


def _run_plain(s):
    c = s["case"]
    op = c["op"]
    if op == "glr_decode":
        live = (torch.arange(c["N"], device="cuda"), torch.arange(c["N"], device="cuda"))
        if s["slots"] is not None:
            rows = (s["slots"] >= 0).nonzero().squeeze(-1)
            live = (rows, s["slots"].long()[rows])
        x = s["x"].float()
        a, w = _gate_plain(c, s["g"])
        new = a[live[0]] * s["state"][live[1]] + w[live[0]] * x[live[0]]
        h = torch.zeros_like(x)
        h[live[0]] = new
        s["state"][live[1]] = new
        return {"h": h.to(s["x"].dtype), "state": s["state"]}
    if op.startswith("glr"):
        return _run_glr_plain(s)
    w = s["w"]
    if op.startswith("add_norm"):
        x, res, scale, dt, rt = s["x"].float(), s["res"].float(), s["scale"], s["x"].dtype, s["res"].dtype
        rx = _rstd_plain(x) if c["post"] else None
        u = x * rx * s["w_post"] if c["post"] else x
        if op == "add_norm":
            new = res + scale * u
            return {"y": (new * _rstd_plain(new) * w).to(dt), "res": new.to(rt)}
        dy, r = s["dy"].float(), _rstd_plain(res)
        dw = (dy * res * r).sum(0)
        wdy = w * dy
        dres = s["dres"].float() + r * (wdy - res * (r * r * (res * wdy).mean(-1, keepdim=True)))
        du = scale * dres
        dx, dpost = du, None
        if c["post"]:
            dpost = (du * x * rx).sum(0)
            wdu = s["w_post"] * du
            dx = rx * (wdu - x * (rx * rx * (x * wdu).mean(-1, keepdim=True)))
        return {"dx": dx.to(dt), "dres": dres.to(rt), "dw": dw, "dscale": (dres * u).sum(0) if c["vector"] else None,
                "dpost": dpost}
    o, z, dt = s["o"].float(), s["z"].float(), s["o"].dtype
    r = _rstd_plain(o)
    act, slope = _act_plain(c["act"], z)
    n = o * r * w
    if op == "gate_norm":
        return {"y": (n * act).to(dt)}
    dy = s["dy"].float()
    dn = dy * act
    wdn = w * dn
    do = r * (wdn - o * (r * r * (o * wdn).mean(-1, keepdim=True)))
    return {"do": do.to(dt), "dz": (dy * n * slope).to(dt), "dw": (dn * o * r).sum((0, 1))}


# ------------------------------------------------------------- what it takes
def work(case):
    """Each input read once and each output written once; operations of the
    formulas, an exponential or root counted as one."""
    op, e = case["op"], 2 if case["dtype"] == "bf16" else 4
    if op.startswith("glr"):
        ge, D = 2 if case["gate"] == "bf16" else 4, case["D"]
        if op == "glr_decode":
            N, live = case["N"], case["N"] - case["pad"]
            return {"bytes": N * D * e + live * D * (e + ge + 8) + (4 * N if case["pool"] else 0), "flops": 6 * live * D}
        lens = _lens(case)
        T, N = sum(lens), len(lens)
        states = 4 * N * D * (2 if case["s0"] else 1)
        if op == "glr_prefill":
            return {"bytes": T * D * (2 * e + ge) + states, "flops": 6 * T * D}
        return {"bytes": T * D * (4 * e + 2 * ge) + states + (8 * N * D if case["s0"] else 0), "flops": 16 * T * D}
    if op.startswith("add_norm"):
        T, D, re = case["T"], case["D"], 2 if case["res"] == "bf16" else 4
        vectors = 4 * D * (1 + case["post"] + case["vector"])
        if op == "add_norm":
            return {"bytes": T * D * 2 * (e + re) + vectors, "flops": T * D * (11 if case["post"] else 7)}
        reads_x = case["post"] or case["vector"]
        return {"bytes": T * D * ((3 if reads_x else 2) * e + 3 * re) + 2 * vectors,
                "flops": T * D * (24 if case["post"] else 14)}
    n, d = case["T"] * case["H"] * case["d"], case["d"]
    if op == "gate_norm":
        return {"bytes": 3 * n * e + 4 * d, "flops": 9 * n}
    return {"bytes": 5 * n * e + 8 * d, "flops": 24 * n}


# ------------------------------------------------------- the result in 64 bits
def _exact_gate(case, g):
    """(a, 1 - a, d log a / d gate)."""
    g = g.double()
    if case["raw"]:
        return torch.sigmoid(-g), torch.sigmoid(g), -torch.sigmoid(g)
    return g.exp(), -torch.expm1(g), torch.ones_like(g)


def _exact_glr(case, s):
    """Token by token, all sequences at once: the longest first, so that the
    sequences still running are a leading part of the batch."""
    lens = _lens(case)
    order = sorted(range(len(lens)), key=lambda n: -lens[n])
    start = torch.tensor([sum(lens[:n]) for n in order], device="cuda")
    seq = torch.tensor(order, device="cuda")
    running = [sum(1 for n in lens if n > t) for t in range(max(lens))]
    x = s["x"].double()
    a, forget, slope = _exact_gate(case, s["g"])
    u = forget * x if case["convex"] else x
    S = s["s0"].double()[seq] if s["s0"] is not None else torch.zeros(len(lens), case["D"], dtype=torch.float64,
                                                                     device="cuda")
    h, before = torch.empty_like(x), torch.empty_like(x)
    for t, live in enumerate(running):
        at = start[:live] + t
        before[at] = S[:live]
        S[:live] = a[at] * S[:live] + u[at]
        h[at] = S[:live]
    final = torch.empty_like(S)
    final[seq] = S
    out = {"h": h, "final": final}
    if case["op"] == "glr_prefill":
        return out
    dh = s["dh"].double()
    G = s["dfinal"].double()[seq] if s["dfinal"] is not None else torch.zeros_like(S)  # gradient of the state
    d = torch.empty_like(x)
    for t in range(max(lens) - 1, -1, -1):
        live = running[t]
        at = start[:live] + t
        d[at] = dh[at] + G[:live]
        G[:live] = a[at] * d[at]
    dx = d * forget if case["convex"] else d
    dlog = a * d * (before - x if case["convex"] else before)
    ds0 = None
    if s["s0"] is not None:
        ds0 = torch.empty_like(G)
        ds0[seq] = G
    return {**out, "dx": dx, "dg": dlog * slope, "ds0": ds0}


def _exact_norm(x):
    """x over its root mean square, and the map of a gradient back through it."""
    rms = ((x ** 2).mean(-1, keepdim=True) + EPS).sqrt()
    n = x / rms
    return n, lambda dn: (dn - n * (dn * n).mean(-1, keepdim=True)) / rms


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "glr_decode":
        slots = s["slots"].long() if s["slots"] is not None else torch.arange(case["N"], device="cuda")
        state, x = s["state"].double(), s["x"].double()
        a, forget, _ = _exact_gate(case, s["g"])
        keep = slots >= 0
        new = a * state[slots.clamp_min(0)] + (forget * x if case["convex"] else x)
        h = torch.where(keep[:, None], new, torch.zeros_like(new))
        state[slots[keep]] = new[keep]
        return {"h": h, "state": state}
    if op.startswith("glr"):
        return _exact_glr(case, s)
    w = s["w"].double()
    if op.startswith("add_norm"):
        x, res = s["x"].double(), s["res"].double()
        scale = s["scale"].double() if case["vector"] else s["scale"]
        wp = s["w_post"].double() if case["post"] else None
        nx, back_x = _exact_norm(x) if case["post"] else (x, None)
        u = nx * wp if case["post"] else x
        if op == "add_norm":
            new = res + scale * u
            return {"y": _exact_norm(new)[0] * w, "res": new}
        n, back = _exact_norm(res)
        dy = s["dy"].double()
        total = s["dres"].double() + back(dy * w)
        du = total * scale
        return {"dx": back_x(du * wp) if case["post"] else du, "dres": total, "dw": (dy * n).sum(0),
                "dscale": (total * u).sum(0) if case["vector"] else None,
                "dpost": (du * nx).sum(0) if case["post"] else None}
    o, z = s["o"].double(), s["z"].double()
    n, back = _exact_norm(o)
    sig = torch.sigmoid(z)
    f, df = (z * sig, sig + z * sig * (1 - sig)) if case["act"] == "silu" else (sig, sig * (1 - sig))
    if op == "gate_norm":
        return {"y": n * w * f}
    dy = s["dy"].double()
    return {"do": back(dy * f * w), "dz": dy * n * w * df, "dw": (dy * f * n).sum((0, 1))}
