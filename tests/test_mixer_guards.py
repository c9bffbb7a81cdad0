"""Guard zones around everything that the convolution's, the scan's and the pools' entry points write:
outputs, workspaces and pools lie between bytes that must be the same afterwards."""

import pytest

import paper_2609_32114_amd as P
from test_mixer_abi import CONV_BACK, SSM, SSM_BACK, call

pytestmark = pytest.mark.gpu
ZONE = 1 << 16  # bytes on either side


class Guards:
    def __init__(self):
        self.all = {}

    def place(self, name, shape, dtype):
        """A tensor of bytes 9 between the zones."""
        import torch
        n = torch.Size(shape).numel() * torch.empty((), dtype=dtype).element_size()
        whole = torch.full((n + 2 * ZONE,), 9, dtype=torch.uint8, device="cuda")
        self.all[name] = whole
        return whole[ZONE:ZONE + n].view(dtype).view(shape)

    def check(self):
        import torch
        torch.cuda.synchronize()
        for name, whole in self.all.items():
            assert bool((whole[:ZONE] == 9).all()) and bool((whole[-ZONE:] == 9).all()), name


def inputs(T, N, D, S, G, W, dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(T + D + S)
    r = lambda *shape, t=torch.float32: torch.randn(*shape, generator=gen, device="cuda").to(t)
    return {"x": r(T, D, t=dtype), "dt": r(T, D), "z": r(T, D, t=dtype), "dy": r(T, D, t=dtype), "B": r(T, G, S, t=dtype),
            "C": r(T, G, S, t=dtype), "A": -r(D, S).abs(), "skip": r(D), "bias": r(D), "s0": r(N, D, S),
            "dfinal": r(N, D, S), "w": r(D, W), "w0": r(N, W - 1, D, t=dtype), "dwindow": r(N, W - 1, D, t=dtype)}


def lengths(T):
    """Offsets of three sequences over T tokens, the second one empty."""
    import torch
    return torch.tensor([0, T // 3, T // 3, T], dtype=torch.int32, device="cuda")


# one chunk and several, several groups of 16 tokens in a chunk (the last)
SIZES = [(1, 70, 1), (50, 66, 2), (300, 257, 1), (1200, 2049, 3)]


@pytest.mark.parametrize("T,D,G", SIZES)
@pytest.mark.parametrize("S", [5, 20, 40, 64])
def test_scan(T, D, G, S):
    import torch
    for dtype in (torch.bfloat16, torch.float32):
        i, cu, g = inputs(T, 3, D, S, G, 4, dtype), lengths(T), Guards()
        saved = g.place("checkpoints", (P.ssm_checkpoints_size(T, D, S),), torch.float32)
        outs = {"y": g.place("y", (T, D), dtype), "sf": g.place("final", (3, D, S), torch.float32), "ck": saved}
        size = P.ssm_workspace_size(T, D, S, G)
        shared = dict(x=i["x"], dt=i["dt"], A=i["A"], B=i["B"], C=i["C"], skip=i["skip"], z=i["z"], bias=i["bias"], s0=i["s0"],
                      cu=cu)
        sizes = dict(xs=D, dts=D, zs=D, Bs=G * S, Cs=G * S, N=3, T=T, D=D, S=S, G=G, dtype=int(dtype == torch.bfloat16), st=0, pre=2,
                     stream=torch.cuda.current_stream().cuda_stream)
        pointers = lambda d: {k: v.data_ptr() for k, v in d.items()}
        ws = g.place("workspace", (size,), torch.uint8)
        assert call("ssm_prefill", SSM, **pointers({**shared, **outs, "ws": ws}), **sizes, wsb=size)[0] == 0
        g.check()
        back = {"dx": g.place("dx", (T, D), dtype), "ddt": g.place("ddt", (T, D), torch.float32),
                "dA": g.place("dA", (D, S), torch.float32), "dB": g.place("dB", (T, G, S), dtype),
                "dC": g.place("dC", (T, G, S), dtype), "dskip": g.place("dskip", (D,), torch.float32),
                "dz": g.place("dz", (T, D), dtype), "dbias": g.place("dbias", (D,), torch.float32),
                "ds0": g.place("ds0", (3, D, S), torch.float32)}
        size = P.ssm_workspace_size(T, D, S, G, True)
        ws = g.place("backward workspace", (size,), torch.uint8)
        assert call("ssm_backward", SSM_BACK, **pointers({**shared, **back, "dy": i["dy"], "df": i["dfinal"], "ck": saved, "ws": ws}),
                    **sizes, dys=D, wsb=size)[0] == 0
        g.check()
        for name, t in {**outs, **back}.items():
            if name != "ck":  # (padded states have no values)
                assert bool(torch.isfinite(t).all()) and not bool((t.reshape(-1).view(torch.uint8) == 9).all()), name


@pytest.mark.parametrize("T,D,G", SIZES)
@pytest.mark.parametrize("W", [2, 4, 8])
def test_convolution(T, D, G, W):
    import torch
    for dtype in (torch.bfloat16, torch.float32):
        i, cu, g = inputs(T, 3, D, 1, 1, W, dtype), lengths(T), Guards()
        P.conv_prefill(i["x"], i["w"], i["bias"], i["w0"], cu, out=g.place("y", (T, D), dtype),
                       final_out=g.place("window", (3, W - 1, D), dtype),
                       workspace=g.place("workspace", (P.conv_workspace_size(T, D, W),), torch.uint8))
        size = P.conv_workspace_size(T, D, W, True)
        t = dict(dy=i["dy"], x=i["x"], w=i["w"], b=i["bias"], w0=i["w0"], df=i["dwindow"], cu=cu, dx=g.place("dx", (T, D), dtype),
                 dw=g.place("dw", (D, W), torch.float32), db=g.place("db", (D,), torch.float32),
                 dw0=g.place("dw0", (3, W - 1, D), dtype), ws=g.place("backward workspace", (size,), torch.uint8))
        assert call("hagdn_conv_backward", CONV_BACK, **{k: v.data_ptr() for k, v in t.items()}, dys=D, xs=D, N=3, T=T, D=D, W=W,
                    dtype=int(dtype == torch.bfloat16), wsb=size, stream=torch.cuda.current_stream().cuda_stream)[0] == 0
        g.check()


@pytest.mark.parametrize("N,D,S,G", [(1, 1, 1, 1), (5, 67, 5, 1), (3, 260, 16, 2), (17, 130, 61, 1)])
def test_single_tokens(N, D, S, G):
    import torch
    for dtype in (torch.bfloat16, torch.float32):
        i, g = inputs(N, 1, D, S, G, 4, dtype), Guards()
        slots = torch.randperm(N + 2, device="cuda")[:N].to(torch.int32)
        slots[0] = -1 if N > 1 else 0
        states, windows = g.place("states", (N + 2, D, S), torch.float32), g.place("windows", (N + 2, 3, D), dtype)
        states.zero_(), windows.zero_()
        P.conv_decode(i["x"], i["w"], windows, i["bias"], slots, out=g.place("conv", (N, D), dtype))
        P.ssm_decode(i["x"], i["dt"], i["A"], i["B"], i["C"], states, slots, i["skip"], i["z"], i["bias"], P.PRE_GATE_SOFTPLUS,
                     out=g.place("scan", (N, D), dtype))
        g.check()


@pytest.mark.parametrize("S", [9, 320, 4096, 4097, 6000])
def test_pools(S):
    """Copies, forks and compactions of pools at every alignment, with plans in LDS and in memory."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(S)
    g = Guards()
    pools = [g.place(f"pool {k}", (S, n), t) for k, (n, t) in enumerate(
        [(4, torch.float32), (3, torch.bfloat16), (5, torch.uint8), (70, torch.bfloat16)])]
    size, n = P.pool_workspace_size(S), max(1, S // 3)
    ws = g.place("workspace", (size,), torch.uint8)
    slots = torch.randperm(S, generator=gen, device="cuda")[:n].to(torch.int32)
    P.pool_copy(pools, dst=slots[:4000], src=slots.flip(0)[:4000].contiguous())
    for M in (n, S, 2 * S):  # the last: more children than slots
        parents = torch.randint(0, n, (M,), generator=gen, device="cuda").to(torch.int32)
        new = P.pool_fork(pools, slots, parents, workspace=ws, out=g.place(f"children {M}", (M,), torch.int32))
        assert int(new.max()) < S and P.device_status(ws) == (P.DEV_POOL_FULL if M > S else P.DEV_OK)
        P.pool_compact(pools, slots, workspace=ws, out=g.place(f"table {M}", (n,), torch.int32))
        g.check()
