"""The differentiable convolution and scan: gradients through torch's graph equal the entry
points', alone and in a block as they are used together; streams, graphs and checks."""

import os

import pytest
import torch

import paper_2609_32114_amd as P

gpu = pytest.mark.gpu


def normal(gen, *shape, dtype=torch.float32, grad=True):
    return torch.randn(*shape, generator=gen, device="cuda").to(dtype).requires_grad_(grad)


def cu(lens):
    return torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int32, device="cuda")


def operands(lens, D, S, dtype, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T, N = sum(lens), len(lens)
    return {"x": normal(gen, T, D, dtype=dtype), "dt": normal(gen, T, D, dtype=dtype),
            "A": (-0.1 - torch.rand(D, S, generator=gen, device="cuda")).requires_grad_(),
            "B": normal(gen, T, 2, S, dtype=dtype), "C": normal(gen, T, 2, S, dtype=dtype), "skip": normal(gen, D),
            "z": normal(gen, T, D, dtype=dtype), "dt_bias": normal(gen, D), "initial_state": normal(gen, N, D, S)}


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_ssm_gradients(dtype):
    from paper_2609_32114_amd import autograd
    lens, D, S = (40, 1, 90), 70, 16
    o = operands(lens, D, S, dtype)
    how = dict(cu_seqlens=cu(lens), preprocess=P.PRE_GATE_SOFTPLUS)
    y, final = autograd.ssm(**o, **how)
    dy, dfinal = torch.randn_like(y), torch.randn_like(final)
    torch.autograd.backward([y, final], [dy, dfinal])
    plain = {k: v.detach() for k, v in o.items()}
    y2, final2, saved = P.ssm_prefill(**plain, output_checkpoints=True, **how)
    assert torch.equal(y, y2) and torch.equal(final, final2)
    grads = P.ssm_backward(dy, *[plain[k] for k in ("x", "dt", "A", "B", "C")], saved, skip=plain["skip"], z=plain["z"],
                           dt_bias=plain["dt_bias"], initial_state=plain["initial_state"], dfinal=dfinal, **how)
    for k, g in zip(("x", "dt", "A", "B", "C", "skip", "z", "dt_bias", "initial_state"), grads):
        assert torch.equal(o[k].grad, g), k
    # a gradient of only one of the results, and of one that is not contiguous
    for k in o:
        o[k].grad = None
    y, final = autograd.ssm(**o, **how)
    final.backward(dfinal)
    g = P.ssm_backward(torch.zeros_like(dy), *[plain[k] for k in ("x", "dt", "A", "B", "C")], saved, skip=plain["skip"],
                       z=plain["z"], dt_bias=plain["dt_bias"], initial_state=plain["initial_state"], dfinal=dfinal, **how)
    assert torch.equal(o["x"].grad, g[0])
    y, final = autograd.ssm(**o, **how)
    y.t().contiguous().t().sum().backward()


@gpu
def test_conv_gradients():
    from paper_2609_32114_amd import autograd
    gen = torch.Generator(device="cuda").manual_seed(1)
    lens, D = (40, 2, 0, 90), 300
    o = {"x": normal(gen, sum(lens), D, dtype=torch.bfloat16), "weight": normal(gen, D, 4), "bias": normal(gen, D),
         "initial_window": normal(gen, len(lens), 3, D, dtype=torch.bfloat16)}
    y, window = autograd.conv(**o, cu_seqlens=cu(lens))
    dy, dwin = torch.randn_like(y), torch.randn_like(window)
    torch.autograd.backward([y, window], [dy, dwin])
    plain = {k: v.detach() for k, v in o.items()}
    grads = P.conv_backward(dy, plain["x"], plain["weight"], plain["bias"], plain["initial_window"], dwin, cu(lens))
    for k, g in zip(o, grads):
        assert torch.equal(o[k].grad, g), k
    y, window = autograd.conv(o["x"], o["weight"], cu_seqlens=cu(lens), activation=None)
    o["x"].grad = None
    window.sum().backward()  # the last three inputs of each sequence
    assert float(o["x"].grad.sum()) == 3 * D + 2 * D + 3 * D


@gpu
def test_second_derivatives_raise():
    from paper_2609_32114_amd import autograd
    o = operands((20,), 10, 4, torch.float32)
    y, _ = autograd.ssm(**o, preprocess=P.PRE_GATE_SOFTPLUS)
    g, = torch.autograd.grad(y.sum(), o["x"], create_graph=True)
    with pytest.raises(RuntimeError, match="second derivative"):
        g.sum().backward()
    w = torch.randn(10, 4, device="cuda", requires_grad=True)
    y, _ = autograd.conv(o["x"], w)
    g, = torch.autograd.grad(y.sum(), w, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivative"):
        g.sum().backward()


class Block:
    """A block of this family: one projection gives the convolution's input and the gate, the
    convolution's output the step sizes, B and C, the scan mixes, a projection returns."""

    def __init__(self, width, inner, states, rank, gen):
        s = lambda *shape: (torch.randn(*shape, generator=gen, device="cuda") * shape[0] ** -0.5).requires_grad_()
        self.inner, self.states, self.rank = inner, states, rank
        self.p = {"norm": torch.ones(width, device="cuda", requires_grad=True), "in": s(width, 2 * inner),
                  "conv": (0.5 * torch.randn(inner, 4, generator=gen, device="cuda")).requires_grad_(),
                  "bias": torch.zeros(inner, device="cuda", requires_grad=True), "maps": s(inner, rank + 2 * states),
                  "step": s(rank, inner), "step_bias": torch.full((inner,), -3.0, device="cuda", requires_grad=True),
                  "A": (-torch.arange(1.0, states + 1, device="cuda")).repeat(inner, 1).requires_grad_(),
                  "skip": torch.ones(inner, device="cuda", requires_grad=True), "out": s(inner, width)}

    def __call__(self, x, res, mix):
        from paper_2609_32114_amd import autograd
        p, n, r = self.p, self.states, self.rank
        y, res = autograd.add_norm(x, p["norm"], residual=res)
        u, z = (y @ p["in"].to(y.dtype)).split(self.inner, 1)
        conv, scan = mix
        u = conv(u, p["conv"], p["bias"])
        m = u @ p["maps"].to(u.dtype)
        o = scan(u, m[:, :r] @ p["step"].to(u.dtype), p["A"], m[:, r:r + n], m[:, r + n:], skip=p["skip"], z=z,
                 dt_bias=p["step_bias"], preprocess=P.PRE_GATE_SOFTPLUS)
        return o @ p["out"].to(o.dtype), res


@gpu
def test_block_together():
    """Convolution and scan between this framework's norms, as a layer runs them: gradients of all
    parameters are finite and agree with differences, and tokens served one at a time from
    pools, over a fork and a compaction, continue a prefill."""
    from paper_2609_32114_amd import autograd
    gen = torch.Generator(device="cuda").manual_seed(0)
    lens = (50, 33, 1)
    block = Block(64, 128, 16, 8, gen)
    x = torch.randn(sum(lens), 64, generator=gen, device="cuda")
    probe = torch.randn(sum(lens), 64, generator=gen, device="cuda")
    off = cu(lens)
    mix = (lambda u, w, b: autograd.conv(u, w, b, cu_seqlens=off)[0],
           lambda *a, **k: autograd.ssm(*a, cu_seqlens=off, **k)[0])

    def loss():
        o, _ = block(x, None, mix)
        return (o * probe).sum()

    loss().backward()
    for k, v in block.p.items():
        assert v.grad is not None and bool(torch.isfinite(v.grad).all()), k
        # along a random direction: fp32 sums of some 5000 terms near 10 leave 1e-3 of rounding in the
        # loss, a step of 1e-2 as much of curvature
        d = torch.randn(v.shape, generator=gen, device="cuda")
        d /= d.norm()
        with torch.no_grad():
            v += 1e-2 * d
            hi = float(loss())
            v -= 2e-2 * d
            lo = float(loss())
            v += 1e-2 * d
        slope, want = (hi - lo) / 2e-2, float((v.grad * d).sum())
        assert abs(slope - want) <= 0.05 * float(v.grad.norm()) + 0.1, (k, slope, want)

    # serving: prefill, states into pools, a fork, tokens one at a time, compaction
    with torch.no_grad():
        finals = {}

        def conv(u, w, b):
            y, finals["window"] = P.conv_prefill(u, w, b, cu_seqlens=off)
            return y

        def scan(*a, **k):
            y, finals["state"] = P.ssm_prefill(*a, cu_seqlens=off, **k)
            return y

        block(x, None, (conv, scan))
        pools = [torch.zeros(9, 3, 128, device="cuda"), torch.zeros(9, 128, 16, device="cuda")]
        slots = torch.tensor([7, 2, 5], dtype=torch.int32, device="cuda")
        P.pool_copy(pools, dst=slots, sources=[finals["window"], finals["state"]])
        parents = torch.tensor([0, 2, 0, 1], dtype=torch.int32, device="cuda")
        slots = P.pool_fork(pools, slots, parents)
        slots = P.pool_compact(pools, slots)
        ahead = torch.randn(4, 5, 64, generator=gen, device="cuda")
        stepped = []
        for t in range(5):
            stepped.append(block(ahead[:, t], None, (
                lambda u, w, b: P.conv_decode(u, w, pools[0], b, slots=slots),
                lambda *a, **k: P.ssm_decode(*a[:5], pools[1], slots=slots, **k)))[0])
        docs = [torch.cat([x.split(lens)[p], ahead[i]]) for i, p in enumerate(parents.tolist())]
        off2 = cu([len(d) for d in docs])
        whole, _ = block(torch.cat(docs), None, (lambda u, w, b: P.conv_prefill(u, w, b, cu_seqlens=off2)[0],
                                                 lambda *a, **k: P.ssm_prefill(*a, cu_seqlens=off2, **k)[0]))
        want = torch.stack([d[-5:] for d in whole.split([len(d) for d in docs])], 1)
        got = torch.stack(stepped)
        # fp32 throughout; products of differently shaped matrices may sum in another order
        assert float((got - want).abs().max()) <= 1e-4 * float(want.abs().max())


@gpu
@pytest.mark.parametrize("S", [16, 40])
def test_graph_replays(S):
    """Prefill, backward, step and pools captured together, replayed on new inputs, with eager work
    and synchronisations between the replays."""
    lens, D = (70, 40), 130
    o = {k: v.detach() for k, v in operands(lens, D, S, torch.bfloat16).items()}
    off, w = cu(lens), torch.randn(D, 4, device="cuda")
    pools = [torch.zeros(6, 3, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(6, D, S, device="cuda")]
    slots = torch.tensor([3, 5], dtype=torch.int32, device="cuda")
    parents = torch.tensor([1, 1, 0], dtype=torch.int32, device="cuda")
    dy = torch.randn(sum(lens), D, device="cuda").bfloat16()

    def everything():
        for p in pools:
            p.zero_()
        how = dict(cu_seqlens=off, preprocess=P.PRE_GATE_SOFTPLUS)
        u, window = P.conv_prefill(o["x"], w, cu_seqlens=off)
        args = (u, o["dt"], o["A"], o["B"], o["C"])
        more = dict(skip=o["skip"], z=o["z"], dt_bias=o["dt_bias"], initial_state=o["initial_state"])
        y, final, saved = P.ssm_prefill(*args, output_checkpoints=True, **more, **how)
        grads = P.ssm_backward(dy, *args, saved, **more, **how)
        du = P.conv_backward(grads[0], o["x"], w, cu_seqlens=off)
        P.pool_copy(pools, dst=slots, sources=[window, final])
        new = P.pool_fork(pools, slots, parents)
        u1 = P.conv_decode(o["x"][:3], w, pools[0], slots=new)
        y1 = P.ssm_decode(u1, o["dt"][:3], o["A"], o["B"][:3], o["C"][:3], pools[1], slots=new)
        last = P.pool_compact(pools, new)
        return [y, final, *[g for g in grads if g is not None], *[g for g in du if g is not None], y1, last, *pools]

    eager = everything()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        everything()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = everything()
    for i in range(5):
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        want = [t.clone() for t in everything()]
        for j, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), (i, j)
        for k in ("x", "dt", "B", "C", "z"):
            o[k].copy_(torch.randn_like(o[k]))
        parents.copy_(torch.randint(0, 2, (3,), device="cuda"))
    assert len(eager) == len(outs)


@gpu
def test_two_streams_at_once():
    """Calls on two streams with workspaces of their own give what each gives alone."""
    lens, D, S = (300, 77), 520, 16
    a, b = ({k: v.detach() for k, v in operands(lens, D, S, torch.bfloat16, seed).items()} for seed in (1, 2))
    off = cu(lens)
    run = lambda o: P.ssm_prefill(**o, cu_seqlens=off, preprocess=P.PRE_GATE_SOFTPLUS)
    want = [run(a), run(b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(4):
        for i, o in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                got[i].append(run(o))
    torch.cuda.synchronize()
    for i in range(2):
        for y, final in got[i]:
            assert torch.equal(y, want[i][0]) and torch.equal(final, want[i][1])


@gpu
def test_nothing_behind_the_outputs_is_written():
    """Outputs lie between guards; a byte too many would show there."""
    lens, D, S = (70, 3), 66, 5
    o = {k: v.detach() for k, v in operands(lens, D, S, torch.bfloat16).items()}
    T = sum(lens)

    def guarded(shape, dtype):
        n = int(torch.tensor(shape).prod())
        whole = torch.full((n + 512,), 9.0, dtype=dtype, device="cuda")
        return whole, whole[256:256 + n].view(shape)

    pairs = {"y": guarded((T, D), torch.bfloat16), "final": guarded((2, D, S), torch.float32),
             "window": guarded((2, 3, D), torch.bfloat16), "conv": guarded((T, D), torch.bfloat16)}
    size = P.ssm_workspace_size(T, D, S, 2)
    ws, part = guarded((size,), torch.uint8)
    P.ssm_prefill(**o, cu_seqlens=cu(lens), preprocess=P.PRE_GATE_SOFTPLUS, out=pairs["y"][1], final_out=pairs["final"][1],
                  workspace=part)
    w = torch.randn(D, 4, device="cuda")
    P.conv_prefill(o["x"], w, cu_seqlens=cu(lens), out=pairs["conv"][1], final_out=pairs["window"][1])
    torch.cuda.synchronize()
    for name, (whole, _) in {**pairs, "workspace": (ws, part)}.items():
        assert bool((whole[:256] == 9).all()) and bool((whole[-256:] == 9).all()), name


# ----------------------------------------------------------- refusals of the binding (CPU)
@pytest.mark.skipif(not os.path.exists(P.library_path()), reason="libhagdn.so not built")
def test_binding_refuses_tensors_off_the_gpu():
    x, w = torch.zeros(4, 8), torch.zeros(8, 4)
    with pytest.raises(ValueError, match="GPU"):
        P.conv_prefill(x, w)
    with pytest.raises(ValueError, match="GPU"):
        P.ssm_prefill(x, x, torch.zeros(8, 2), torch.zeros(4, 2), torch.zeros(4, 2))
    with pytest.raises(ValueError, match="one GPU"):
        P.pool_copy([x], dst=torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError, match="empty"):
        P.pool_copy([])
    with pytest.raises(ValueError, match="activation"):
        from paper_2609_32114_amd import mixer
        mixer._activation("gelu")


@gpu
def test_binding_refusals():
    x, w = torch.zeros(4, 8, device="cuda"), torch.zeros(8, 4, device="cuda")
    A, B, s = torch.zeros(8, 2, device="cuda"), torch.zeros(4, 2, device="cuda"), torch.zeros(4, 8, 2, device="cuda")
    bad = [lambda: P.conv_prefill(x.half(), w), lambda: P.conv_prefill(x, w.double()), lambda: P.conv_prefill(x.t(), w),
           lambda: P.conv_prefill(x, torch.zeros(8, 9, device="cuda")), lambda: P.conv_prefill(x, w, activation="gelu"),
           lambda: P.conv_prefill(x, w, initial_window=torch.zeros(1, 4, 8, device="cuda")),
           lambda: P.conv_prefill(x, w, out=x), lambda: P.conv_decode(x, w, torch.zeros(3, 3, 8, device="cuda")),
           lambda: P.conv_decode(x, w, torch.zeros(4, 3, 8, device="cuda").bfloat16()),
           lambda: P.ssm_prefill(x, x.bfloat16(), A, B, B), lambda: P.ssm_prefill(x, x, A, B, B[:, :1]),
           lambda: P.ssm_prefill(x, x, A, torch.zeros(4, 3, 2, device="cuda"), torch.zeros(4, 3, 2, device="cuda")),
           lambda: P.ssm_prefill(x, x, torch.zeros(8, 65, device="cuda"), torch.zeros(4, 65, device="cuda"),
                                 torch.zeros(4, 65, device="cuda")),
           lambda: P.ssm_prefill(x, x, A, B, B, dt_bias=torch.zeros(8, device="cuda")),
           lambda: P.ssm_prefill(x, x, A, B, B, preprocess=1), lambda: P.ssm_prefill(x, x, A, B, B, z=x.bfloat16()),
           lambda: P.ssm_prefill(x, x, A, B, B, initial_state=s[:1], final_out=s[:1]),
           lambda: P.ssm_backward(x, x, x, A, B, B, torch.zeros(5, device="cuda")),
           lambda: P.ssm_decode(x, x, A, B, B, s[:3]),
           lambda: P.ssm_decode(x, x, A, B, B, s, slots=torch.zeros(4, dtype=torch.int64, device="cuda")),
           lambda: P.pool_copy([s, s]), lambda: P.pool_copy([s, x[:3]]), lambda: P.pool_copy(s, sources=s),
           lambda: P.pool_copy(s, dst=torch.zeros(1, dtype=torch.int64, device="cuda")),
           lambda: P.pool_copy(s, dst=torch.zeros(1, dtype=torch.int32, device="cuda"),
                               src=torch.zeros(2, dtype=torch.int32, device="cuda")),
           lambda: P.pool_copy(s, sources=torch.zeros(4, 8, 3, device="cuda")),
           lambda: P.pool_copy(s.transpose(1, 2)),
           lambda: P.pool_copy(torch.zeros(9000, 1, device="cuda"), src=torch.zeros(8193, dtype=torch.int32, device="cuda"))]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, TypeError, P.HagdnError)):
            call()
            print("not refused:", i)
