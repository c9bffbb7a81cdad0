"""The refusals of the convolution's, the scan's and the pools' entry points, which need no GPU:
bad arguments are turned down on the host before anything is enqueued (fake,
never-dereferenced device pointers)."""

import ctypes
import os
import subprocess
import sys

import pytest

import paper_2609_32114_amd as P

pytestmark = pytest.mark.skipif(not os.path.exists(P.library_path()), reason="libhagdn.so not built")

EINVAL, EUNSUP, EWS = 1, 2, 3
BIG = 1 << 40
F = [(i + 1) << 32 for i in range(40)]  # 16-byte aligned, far apart, never dereferenced


def call(fn, defaults, **over):
    args = dict(defaults)
    assert set(over) <= set(args), set(over) - set(args)
    args.update(over)
    lib = P.load_library()
    return getattr(lib, fn)(*args.values()), lib.hagdn_last_error().decode()


CONV = dict(x=F[0], xs=64, w=F[1], b=F[2], w0=F[3], cu=F[4], N=2, T=10, D=64, W=4, dtype=1, act=0, y=F[5], wf=F[6], ws=F[7],
            wsb=64, stream=None)  # the workspace is too small: a valid call stops there
CONV_BACK = dict(dy=F[0], dys=64, x=F[1], xs=64, w=F[2], b=F[3], w0=F[4], df=F[5], cu=F[6], N=2, T=10, D=64, W=4, dtype=1, act=0,
                 dx=F[7], dw=F[8], db=F[9], dw0=F[10], ws=F[11], wsb=64, stream=None)
CONV_STEP = dict(x=F[0], xs=64, w=F[1], b=None, state=F[2], slots=None, pool=0, N=3, D=64, W=4, dtype=1, act=2, y=F[3],
                 stream=None)
SSM = dict(x=F[0], xs=64, dt=F[1], dts=64, A=F[2], B=F[3], Bs=16, C=F[4], Cs=16, skip=F[5], z=F[6], zs=64, bias=F[7], s0=F[8],
           cu=F[9], N=2, T=10, D=64, S=16, G=1, dtype=1, st=0, pre=2, y=F[10], sf=F[11], ck=F[12], ws=F[13], wsb=64, stream=None)
SSM_BACK = dict(dy=F[20], dys=64, x=F[0], xs=64, dt=F[1], dts=64, A=F[2], B=F[3], Bs=16, C=F[4], Cs=16, skip=F[5], z=F[6], zs=64,
                bias=F[7], ck=F[12], s0=F[8], df=F[21], cu=F[9], N=2, T=10, D=64, S=16, G=1, dtype=1, st=0, pre=2, dx=F[22],
                ddt=F[23], dA=F[24], dB=F[25], dC=F[26], dskip=F[27], dz=F[28], dbias=F[29], ds0=F[30], ws=F[13], wsb=64,
                stream=None)
SSM_STEP = dict(x=F[0], xs=64, dt=F[1], dts=64, A=F[2], B=F[3], Bs=16, C=F[4], Cs=16, skip=None, z=None, zs=0, bias=None,
                state=F[5], slots=None, pool=0, N=3, D=64, S=16, G=1, dtype=1, st=1, pre=0, y=F[6], stream=None)


def test_valid_calls_reach_the_workspace_check():
    for fn, d in (("hagdn_conv_prefill", CONV), ("hagdn_conv_backward", CONV_BACK), ("ssm_prefill", SSM),
                  ("ssm_backward", SSM_BACK)):
        rc, msg = call(fn, d)
        assert rc == EWS and "workspace too small" in msg, (fn, rc, msg)


@pytest.mark.parametrize("fn,d", [("hagdn_conv_prefill", CONV), ("hagdn_conv_backward", CONV_BACK)], ids=["prefill", "backward"])
def test_conv_refusals(fn, d):
    for over in (dict(N=0), dict(T=-1), dict(D=0), dict(act=1), dict(act=3), dict(x=None), dict(w=None), dict(ws=None, N=513),
                 dict(ws=F[7] + 8), dict(cu=None), dict(cu=F[4] + 2), dict(xs=-1), dict(xs=1 << 31), dict(x=F[0] + 1),
                 dict(w=F[1] + 2), dict(w0=F[3] + 1)):
        assert call(fn, d, **{"wsb": BIG, **over})[0] == EINVAL, over
    for over in (dict(dtype=2), dict(W=1), dict(W=9), dict(W=-3), dict(D=(1 << 28) + 1), dict(T=0x7fff0001)):
        assert call(fn, d, **{"wsb": BIG, **over})[0] == EUNSUP, over
    out = dict(y=None) if fn == "hagdn_conv_prefill" else dict(dx=None)
    assert call(fn, d, **{"wsb": BIG, **out})[0] == EINVAL


def test_conv_overlaps():
    for over in (dict(wf=F[3]), dict(wf=F[3] + 64), dict(y=F[0]), dict(y=F[0] + 128), dict(y=F[0] - 128), dict(wf=F[5] + 2),
                 dict(y=F[1] + 4), dict(wf=F[4])):
        rc, msg = call("hagdn_conv_prefill", CONV, wsb=BIG, **over)
        assert rc == EINVAL and "overlaps" in msg, over
    for over in (dict(dw0=F[5]), dict(dx=F[0]), dict(dw=F[2]), dict(dx=F[1] + 64), dict(db=F[3]), dict(db=F[8]), dict(db=None)):
        assert call("hagdn_conv_backward", CONV_BACK, wsb=BIG, **over)[0] == EINVAL, over


def test_conv_decode_refusals():
    for over in (dict(N=-1), dict(x=None), dict(state=None), dict(y=None), dict(slots=F[8], pool=0), dict(slots=F[8] + 2, pool=4),
                 dict(y=F[2]), dict(state=F[0]), dict(N=1 << 20, D=1 << 12), dict(xs=-2), dict(act=1)):
        assert call("hagdn_conv_decode", CONV_STEP, **over)[0] == EINVAL, over
    assert call("hagdn_conv_decode", CONV_STEP, dtype=5)[0] == EUNSUP
    assert call("hagdn_conv_decode", CONV_STEP, N=0, x=None, y=None, state=None)[0] == 0


@pytest.mark.parametrize("fn,d", [("ssm_prefill", SSM), ("ssm_backward", SSM_BACK)], ids=["prefill", "backward"])
def test_ssm_refusals(fn, d):
    for over in (dict(N=0), dict(T=-1), dict(D=0), dict(S=0), dict(G=0), dict(G=3), dict(G=-1), dict(pre=1), dict(pre=4),
                 dict(pre=0), dict(x=None), dict(dt=None), dict(A=None), dict(B=None), dict(C=None), dict(ws=None),
                 dict(ws=F[13] + 8), dict(cu=None), dict(xs=-1), dict(Bs=1 << 31), dict(zs=-4), dict(x=F[0] + 1),
                 dict(dt=F[1] + 2), dict(B=F[3] + 1), dict(N=1 << 20, D=1 << 12)):
        assert call(fn, d, **{"wsb": BIG, **over})[0] == EINVAL, over
    for over in (dict(dtype=2), dict(st=3), dict(dtype=0, st=1), dict(S=65), dict(N=1, D=(1 << 28) + 1, S=1),
                 dict(T=0x7fff0001)):
        assert call(fn, d, **{"wsb": BIG, **over})[0] == EUNSUP, over
    outs = ("y",) if fn == "ssm_prefill" else ("dx", "ddt", "dA", "dB", "dC", "dskip", "dz", "dbias", "ck")
    for name in outs:
        assert call(fn, d, **{"wsb": BIG, name: None})[0] == EINVAL, name


def test_ssm_overlaps():
    for over in (dict(sf=F[8]), dict(sf=F[8] + 16), dict(y=F[0]), dict(y=F[6] + 64), dict(ck=F[10]), dict(y=F[3])):
        assert call("ssm_prefill", SSM, wsb=BIG, **over)[0] == EINVAL, over
    for over in (dict(ds0=F[21]), dict(dx=F[20]), dict(ddt=F[1]), dict(dz=F[6]), dict(dB=F[25], dC=F[25]), dict(dA=F[2]),
                 dict(ds0=F[8])):
        assert call("ssm_backward", SSM_BACK, wsb=BIG, **over)[0] == EINVAL, over


def test_ssm_decode_refusals():
    for over in (dict(N=-1), dict(x=None), dict(state=None), dict(y=None), dict(slots=F[8], pool=0), dict(bias=F[9]),
                 dict(y=F[5]), dict(state=F[3]), dict(N=1 << 20, D=1 << 12), dict(Cs=-2), dict(G=5)):
        assert call("ssm_decode", SSM_STEP, **over)[0] == EINVAL, over
    for over in (dict(dtype=0), dict(S=65)):
        assert call("ssm_decode", SSM_STEP, **over)[0] == EUNSUP, over
    assert call("ssm_decode", SSM_STEP, N=0, x=None, y=None, state=None)[0] == 0


def test_workspace_sizes():
    lib = P.load_library()
    assert P.ssm_workspace_size(0, 1, 1) > 0 and P.conv_workspace_size(0, 1, 2) > 0
    assert P.ssm_workspace_size(100000, 2048, 16) > P.ssm_workspace_size(1000, 2048, 16)
    assert P.ssm_workspace_size(1000, 2048, 16, backward=True) > P.ssm_workspace_size(1000, 2048, 16)
    assert P.ssm_checkpoints_size(33, 10, 16) == 3 * 16 * 10 and P.ssm_checkpoints_size(0, 10, 16) == 0
    assert P.ssm_checkpoints_size(33, 10, 17) == 3 * 32 * 10 and P.ssm_checkpoints_size(33, 10, 64) == 3 * 64 * 10
    assert lib.ssm_workspace_size(-1, 64, 16, 1, 0) == 0 and lib.ssm_workspace_size(5, 64, 16, 3, 0) == 0
    assert lib.hagdn_conv_workspace_size(5, 64, 1, 0) == 0 and lib.hagdn_pool_workspace_size(0) == 0
    for bad in (lambda: P.ssm_workspace_size(5, 0, 16), lambda: P.conv_workspace_size(5, 64, 9),
                lambda: P.pool_workspace_size((1 << 20) + 1)):
        with pytest.raises(P.HagdnError):
            bad()


def test_conv_workspace_sizes_of_the_largest_calls():
    """Every size in the documented ranges gives a workspace's bytes or none, and the process goes on
    (in one of its own: a quotient by zero would end it)."""
    code = """
import paper_2609_32114_amd as P
lib = P.load_library()
MOST = 0x7fff0000
for T in (1 << 24, 1 << 30, 1 << 30 | 12345, MOST):
    for D in (1, 4096, 1 << 20, 1 << 28):
        for W in (2, 8):
            n = lib.hagdn_conv_workspace_size(T, D, W, 1)
            # a run's sums at least; at most one for every 16 tokens
            assert 256 + (W + 1) * D * 4 <= n <= 256 + ((T + 15) // 16) * (W + 1) * D * 4, (T, D, W, n)
print("sizes passed")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=120,
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0 and "sizes passed" in r.stdout, (r.returncode, r.stdout + r.stderr)


def test_ssm_workspace_sizes_of_the_largest_calls():
    """A size that does not fit is none, with its message, and a call of it is turned down, not taken
    for a smaller one."""
    lib = P.load_library()
    for T in (1, 1 << 24, 1 << 30, 0x7fff0000):
        for D in (1, 4096, 1 << 20, 1 << 28):
            for S, G in ((1, 1), (16, 1), (64, 1), (1, D), (64, D)):
                n = lib.ssm_workspace_size(T, D, S, G, 1)
                least = T * G * 2 * S * 4  # the sums of dB and dC alone
                assert n >= least if least < 1 << 58 else n == 0 if least >= 1 << 62 else True, (T, D, S, G, n)
                assert n or "too large" in lib.hagdn_last_error().decode(), (T, D, S, G)
    assert call("ssm_backward", SSM_BACK, wsb=BIG, N=1, T=1 << 30, D=1 << 24, S=64, G=1 << 24)[0] == EINVAL


# ------------------------------------------------------------------------- pools
def arrays(pools, sizes):
    n = len(pools)
    return (ctypes.c_void_p * n)(*pools), (ctypes.c_size_t * n)(*sizes)


def copy(pools, sizes, sources=None, dst=F[30], src=F[31], n=3, rows=8, src_rows=8, count=None):
    p, s = arrays(pools, sizes)
    f = arrays(sources, sizes)[0] if sources is not None else None
    lib = P.load_library()
    return lib.hagdn_pool_copy(p, f, s, len(pools) if count is None else count, dst, src, n, rows, src_rows, None)


def test_pool_copy_refusals():
    lib = P.load_library()
    assert copy([F[0]], [64], n=0) == 0 and copy([F[0]], [64], rows=0) == 0
    for args in (dict(n=-1), dict(rows=-1), dict(count=0), dict(count=1025), dict(dst=F[30] + 2), dict(src=F[31] + 1),
                 dict(dst=F[0] + 64)):
        assert copy([F[0]], [64], **args) == EINVAL, args
    assert copy([None], [64]) == EINVAL and copy([F[0]], [0]) == EINVAL and copy([F[0]], [1 << 41]) == EINVAL
    assert copy([F[0]], [64], n=8193, rows=10000) == EUNSUP
    assert copy([F[0]], [64], sources=[None]) == EINVAL and copy([F[0]], [64], sources=[F[1]], src_rows=-1) == EINVAL
    # pools over each other, in any order, and over sources
    assert copy([F[0], F[0]], [64, 64]) == EINVAL and copy([F[0], F[1], F[0] + 64 * 7], [64] * 3) == EINVAL
    assert copy([F[0]], [64], sources=[F[0]]) == EINVAL and copy([F[0]], [64], sources=[F[0] - 64]) == EINVAL
    assert copy([F[2], F[0]], [64, 64], sources=[F[1], F[2] + 64]) == EINVAL
    # neighbours are none
    assert copy([F[0], F[0] + 512, F[0] - 512], [64] * 3, n=0) == 0
    # sources may overlap each other
    assert copy([F[0], F[1]], [64, 64], sources=[F[2], F[2]], n=0) == 0
    assert lib.hagdn_pool_copy(None, None, None, 1, None, None, 1, 1, 1, None) == EINVAL


def test_pool_plan_refusals():
    lib = P.load_library()
    p, s = arrays([F[0]], [64])
    fork = lambda **o: lib.hagdn_pool_fork(*{**dict(p=p, s=s, n=1, slots=F[1], N=3, parents=F[2], M=4, S=8, out=F[3], ws=F[4],
                                                     wsb=BIG, stream=None), **o}.values())
    compact = lambda **o: lib.hagdn_pool_compact(*{**dict(p=p, s=s, n=1, slots=F[1], N=3, S=8, out=F[3], ws=F[4], wsb=BIG,
                                                           stream=None), **o}.values())
    for f in (fork, compact):
        for over in (dict(p=None), dict(s=None), dict(n=0), dict(slots=None), dict(slots=F[1] + 2), dict(out=None), dict(N=-1),
                     dict(S=0), dict(ws=None), dict(ws=F[4] + 8), dict(out=F[1] + 4)):
            assert f(**over) == EINVAL, over
        assert f(wsb=100) == EWS and f(S=(1 << 20) + 1) == EUNSUP
    for over in (dict(parents=None), dict(M=-1), dict(out=F[1]), dict(out=F[2])):
        assert fork(**over) == EINVAL, over
    assert fork(M=(1 << 20) + 1) == EUNSUP and compact(N=(1 << 20) + 1) == EUNSUP


def test_pools_of_more_bytes_than_there_are_addresses():
    """Rows whose bytes do not fit are turned down, and not taken for few."""
    lib = P.load_library()
    assert copy([F[0]], [1 << 39], rows=1 << 25, n=0) == EINVAL and "too large" in lib.hagdn_last_error().decode()
    assert copy([F[0], F[0] + 64], [1 << 39, 64], rows=1 << 25, n=0) == EINVAL
    assert copy([F[0]], [1 << 39], sources=[F[1]], rows=1, src_rows=1 << 25, n=0) == EINVAL
    p, s = arrays([F[0]], [(1 << 40) - 256])
    assert lib.hagdn_pool_compact(p, s, 1, F[1], 3, 1 << 20, F[3], F[4], 100, None) == EWS  # 2^60 bytes do


def test_plans_overlaps():
    """A plan's tables and workspace lie apart from the pools that it moves rows of and from each other:
    the copies would write over them while they are read."""
    lib = P.load_library()
    p, s = arrays([F[5], F[0]], [64, 64])
    size = lib.hagdn_pool_workspace_size(8)
    fork = lambda **o: lib.hagdn_pool_fork(*{**dict(p=p, s=s, n=2, slots=F[1], N=3, parents=F[2], M=4, S=8, out=F[3], ws=F[4],
                                                     wsb=BIG, stream=None), **o}.values())
    compact = lambda **o: lib.hagdn_pool_compact(*{**dict(p=p, s=s, n=2, slots=F[1], N=3, S=8, out=F[3], ws=F[4], wsb=BIG,
                                                           stream=None), **o}.values())
    inside = F[0] + 64 * 7 + 48  # the last pool's last row
    for f in (fork, compact):
        for over in (dict(slots=inside), dict(out=inside), dict(ws=inside), dict(ws=F[0] - 16), dict(slots=F[5] - 4),
                     dict(ws=F[1]), dict(ws=F[3]), dict(slots=F[4] + 16), dict(out=F[4] + size - 4), dict(slots=F[4] - 4)):
            assert f(**over) == EINVAL and "overlaps" in lib.hagdn_last_error().decode(), over
    for over in (dict(parents=inside), dict(ws=F[2]), dict(parents=F[4] + 64)):
        assert fork(**over) == EINVAL and "overlaps" in lib.hagdn_last_error().decode(), over
    # neighbours do not overlap: these stop at the workspace that is too small
    for f in (fork, compact):
        assert f(wsb=size - 4, slots=F[0] + 512, ws=F[0] - 16 * (size // 16 + 1), out=F[5] - 16) == EWS


@pytest.mark.parametrize("fn,d", [("hagdn_conv_prefill", CONV), ("hagdn_conv_backward", CONV_BACK), ("ssm_prefill", SSM),
                                  ("ssm_backward", SSM_BACK)], ids=["conv", "conv backward", "scan", "scan backward"])
def test_workspace_overlaps(fn, d):
    """A workspace lies apart from everything else that the call reads or writes."""
    for name, place in d.items():
        if isinstance(place, int) and place >= F[0] and name != "ws":
            rc, msg = call(fn, d, wsb=BIG, ws=place)
            assert rc == EINVAL and "overlaps" in msg, (name, rc, msg)
            rc, msg = call(fn, d, wsb=BIG, ws=place - 16)
            assert rc == EINVAL and "overlaps" in msg, (name, rc, msg)
