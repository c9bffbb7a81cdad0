"""Copies, forks and compaction of state pools: every bit, against the rules carried out one
row at a time on the host."""

import numpy as np
import pytest

from gpu_harness import say

# rows of every alignment: (type, shape of a row)
ROWS = [("float32", (16, 33)), ("bfloat16", (3, 70)), ("float32", (7,)), ("bfloat16", (1,)), ("uint8", (5,)),
        ("float32", (2, 64, 64)), ("int64", (3,)), ("uint8", (4099,))]


def make(slots, rows=ROWS, seed=0):
    """Pools whose bytes are all different sequences."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for name, shape in rows:
        dtype = getattr(torch, name)
        size = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
        raw = torch.randint(0, 256, (slots, size), generator=gen, device="cuda", dtype=torch.uint8)
        out.append(raw.view(dtype).view(slots, *shape))
    return out


def raw(t):
    import torch
    return t.contiguous().view(t.shape[0], -1).view(torch.uint8).cpu().numpy() if t.shape[0] else None


def same(pools, want):
    for i, (p, w) in enumerate(zip(pools, want)):
        assert np.array_equal(raw(p), w), f"pool {i}"


def table(values):
    import torch
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def copied(before, dst, src, sources=None):
    """The rule of pool_copy."""
    after = [b.copy() for b in before]
    from_ = before if sources is None else sources
    for d, s in zip(dst, src):
        for a, f in zip(after, from_):
            if 0 <= d < len(a):
                a[d] = f[s] if 0 <= s < len(f) else 0
    return after


def forked(slots, parents, S):
    """The rule of pool_fork: (new slots, moves, children without a slot)."""
    at = [slots[p] if 0 <= p < len(slots) and 0 <= slots[p] < S else -1 for p in parents]
    kept = set(at)
    free = [s for s in range(S) if s not in kept]
    seen, new, moves, missing = set(), [], [], 0
    for s in at:
        if s < 0 or s not in seen:
            new.append(s)
            seen.add(s)
        elif free:
            moves.append((free.pop(0), s))
            new.append(moves[-1][0])
        else:
            new.append(-1)
            missing += 1
    return new, moves, missing


def compacted(slots, S):
    """The rule of pool_compact: (new table, moves)."""
    live = sorted({s for s in slots if 0 <= s < S})
    holes = [h for h in range(len(live)) if h not in live]
    to = dict(zip([s for s in live if s >= len(live)], holes))
    return [to.get(s, s) for s in slots], [(d, s) for s, d in to.items()]


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 2, 5, 37, 64])
def test_copy_within_pools(n):
    """Any mapping, as if all rows were read before any is written: permutations, one source for
    many, padding and new sequences."""
    import paper_2609_32114_amd as P
    r = np.random.default_rng(n)
    for i in range(4):
        pools = make(64, seed=i)
        before = [raw(p) for p in pools]
        dst = r.permutation(64)[:n]
        src = (r.permutation(64)[:n], r.integers(0, 64, n), r.permutation(dst), r.integers(-2, 70, n))[i]
        if i == 3:
            dst = np.where(r.random(n) < 0.3, r.choice([-1, 64, 2 ** 31 - 1, -2 ** 31], n), dst)
        P.pool_copy(pools, dst=table(dst.tolist()), src=table(src.tolist()))
        same(pools, copied(before, dst.tolist(), src.tolist()))


@pytest.mark.gpu
@pytest.mark.parametrize("n", [2000, 2049, 5000, 8192])
def test_copy_of_many_rows(n):
    """A permutation of more rows than 256 threads hold."""
    import paper_2609_32114_amd as P
    rows = [("float32", (12,)), ("uint8", (3,)), ("bfloat16", (100,))]
    pools = make(n, rows)
    before = [raw(p) for p in pools]
    src = np.random.default_rng(1).permutation(n)
    P.pool_copy(pools, src=table(src.tolist()))
    same(pools, copied(before, range(n), src.tolist()))


@pytest.mark.gpu
def test_copy_between_tensors():
    """A prefill's states into their slots, a snapshot out of them, all rows, and zeros."""
    import torch
    import paper_2609_32114_amd as P
    pools, finals = make(20), make(6, seed=1)
    before, other = [raw(p) for p in pools], [raw(f) for f in finals]
    slots = [7, -1, 19, 0, 20, 3]
    P.pool_copy(pools, dst=table(slots), sources=finals)
    want = copied(before, slots, range(6), other)
    same(pools, want)
    same(finals, other)
    P.pool_copy(finals, src=table([0, 1, -1, 19, 20, 3]), sources=pools)
    same(finals, copied(other, range(6), [0, 1, -1, 19, 20, 3], want))
    copy = [torch.empty_like(p) for p in pools]
    P.pool_copy(copy, sources=pools)
    same(copy, want)
    P.pool_copy(pools, dst=table([2, 4]), src=table([-1, -1]))
    same(pools, copied(want, [2, 4], [-1, -1]))


@pytest.mark.gpu
def test_rows_at_odd_addresses():
    """Pools whose first bytes are aligned to less than their rows, and one tensor alone."""
    import torch
    import paper_2609_32114_amd as P
    flat = torch.randint(0, 256, (4096 * 9 + 16,), device="cuda", dtype=torch.uint8)
    for off in (0, 1, 2, 4, 8, 12):
        pool = flat[off:off + 4096 * 9].view(9, 4096)
        before = [raw(pool)]
        P.pool_copy(pool, dst=table([8, 0]), src=table([0, 5]))
        same([pool], copied(before, [8, 0], [0, 5]))


@pytest.mark.gpu
def test_more_pools_than_a_launch_takes():
    import paper_2609_32114_amd as P
    rows = [("float32", (4,)), ("bfloat16", (3,))] * 80
    pools, finals = make(5, rows), make(2, rows, seed=1)
    before = [raw(p) for p in pools]
    P.pool_copy(pools, dst=table([4, 1]), sources=finals)
    same(pools, copied(before, [4, 1], [0, 1], [raw(f) for f in finals]))


@pytest.mark.gpu
@pytest.mark.parametrize("N,M,S", [(1, 1, 1), (1, 8, 8), (8, 8, 8), (8, 8, 20), (64, 64, 70), (5, 40, 41), (300, 256, 320),
                                   (3, 0, 9), (1500, 2100, 4000)])
def test_fork(N, M, S):
    import paper_2609_32114_amd as P
    r = np.random.default_rng(N + M)
    rows = ROWS if S < 100 else [("float32", (9,)), ("bfloat16", (70,))]
    for i in range(3):
        pools = make(S, rows, seed=i)
        before = [raw(p) for p in pools]
        slots = r.permutation(max(S, N))[:N].tolist()  # some beyond the pools where N > S
        parents = r.integers(0, N, M).tolist() if i else [0] * M
        if i == 2:
            parents = [p if r.random() > 0.2 else int(r.choice([-1, N])) for p in parents]
            slots = [s if r.random() > 0.2 else -1 for s in slots]
        new, moves, missing = forked(slots, parents, S)
        ws = make(1, [("uint8", (P.pool_workspace_size(S),))])[0].view(-1)
        got = P.pool_fork(pools, table(slots), table(parents), workspace=ws)
        assert got.tolist() == new
        assert P.device_status(ws) == (P.DEV_POOL_FULL if missing else P.DEV_OK)
        same(pools, copied(before, [d for d, _ in moves], [s for _, s in moves]))


@pytest.mark.gpu
def test_fork_without_enough_slots():
    import paper_2609_32114_amd as P
    pools = make(5)
    before = [raw(p) for p in pools]
    ws = make(1, [("uint8", (P.pool_workspace_size(5),))])[0].view(-1)
    got = P.pool_fork(pools, table([3, 1]), table([0, 0, 1, 0, 1, 0, 0]), workspace=ws)
    assert got.tolist() == [3, 0, 1, 2, 4, -1, -1] and P.device_status(ws) == P.DEV_POOL_FULL
    same(pools, copied(before, [0, 2, 4], [3, 3, 1]))


@pytest.mark.gpu
@pytest.mark.parametrize("N,S", [(1, 1), (1, 9), (8, 8), (8, 20), (64, 200), (512, 512), (2500, 5000), (0, 3)])
def test_compact(N, S):
    import paper_2609_32114_amd as P
    r = np.random.default_rng(N + S)
    rows = ROWS if S < 300 else [("float32", (9,)), ("bfloat16", (70,))]
    for i in range(3):
        pools = make(S, rows, seed=i)
        before = [raw(p) for p in pools]
        slots = r.permutation(S)[:N].tolist()
        slots += [-1] * (N - len(slots))
        if i:
            slots = [s if r.random() > 0.6 else int(r.choice([-1, S, -7])) for s in slots]
        if i == 2 and N > 4:
            slots[3] = slots[1]  # two entries of one state
        new, moves = compacted(slots, S)
        given = table(slots)
        got = P.pool_compact(pools, given)
        assert got.tolist() == new and given.tolist() == slots
        want = copied(before, [d for d, _ in moves], [s for _, s in moves])
        same(pools, want)
        assert P.pool_compact(pools, given, out=given) is given  # in place (rows beyond the live ones were kept)
        assert given.tolist() == new
        same(pools, want)


@pytest.mark.gpu
def test_rows_beyond_4_gib():
    """Offsets past 32 bits: the last rows of a pool of 6 GiB."""
    import torch
    import paper_2609_32114_amd as P
    pool = torch.zeros(6, 1 << 28, dtype=torch.float32, device="cuda")
    pool[5, -5:] = torch.arange(1.0, 6.0, device="cuda")
    pool[5, :5] = 7.0
    P.pool_copy(pool, dst=table([4]), src=table([5]))
    assert torch.equal(pool[4, -5:], torch.arange(1.0, 6.0, device="cuda")) and bool((pool[4, :5] == 7).all())
    P.pool_copy(pool, dst=table([0, 5]), src=table([5, -1]))
    assert torch.equal(pool[0], pool[4]) and not pool[5].any()
    assert P.pool_compact(pool, table([4, -1])).tolist() == [0, -1]
    assert torch.equal(pool[0], pool[4])


@pytest.mark.gpu
def test_beam_search_over_states():
    """Beams of the scan behind its convolution: forked states go on exactly as their parents' would."""
    import torch
    import paper_2609_32114_amd as P
    gen = torch.Generator(device="cuda").manual_seed(3)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    D, S, slots = 96, 16, table([4, 9])
    windows, states = normal(12, 3, D).bfloat16(), normal(12, D, S)
    w, A = normal(D, 4), -torch.rand(D, S, generator=gen, device="cuda")

    def step(x, dt, B, C, where, windows, states):
        u = P.conv_decode(x, w, windows, slots=where)
        return P.ssm_decode(u, dt, A, B, C, states, slots=where, preprocess=P.PRE_GATE_SOFTPLUS)

    parents = [1, 0, 1, 1]
    old = (windows[slots.long()].clone(), states[slots.long()].clone())
    new = P.pool_fork([windows, states], slots, table(parents))
    assert new.tolist() == [9, 4, 0, 1]
    x, dt, B, C = normal(4, D).bfloat16(), normal(4, D).bfloat16(), normal(4, S).bfloat16(), normal(4, S).bfloat16()
    y = step(x, dt, B, C, new, windows, states)
    apart = (old[0][parents].clone(), old[1][parents].clone())
    want = step(x, dt, B, C, None, *apart)
    assert torch.equal(y, want)
    assert torch.equal(windows[new.long()], apart[0]) and torch.equal(states[new.long()], apart[1])
    table_after = P.pool_compact([windows, states], new)
    assert sorted(table_after.tolist()) == [0, 1, 2, 3]
    assert torch.equal(states[table_after.long()], apart[1])


@pytest.mark.gpu
@pytest.mark.parametrize("N,M,S", [(40, 4096, 4096), (3, 4097, 4096), (3000, 4096, 4097), (3000, 4500, 6000), (1, 5000, 100),
                                   (100, 5000, 100), (200, 4097, 1), (2000, 9000, 5000)])
def test_fork_of_thousands(N, M, S):
    """Plans in LDS and in memory, with enough free slots and with far fewer than children; nothing
    around the workspace and the new table is written."""
    import torch
    import paper_2609_32114_amd as P
    r = np.random.default_rng(M + S)
    rows = [("float32", (2,)), ("uint8", (5,))]
    size = P.pool_workspace_size(S)
    for i in range(3):
        pools = make(S, rows, seed=i)
        before = [raw(p) for p in pools]
        slots = r.permutation(max(S, N))[:N].tolist()
        parents = r.integers(0, N, M).tolist() if i else [0] * M
        if i == 2:
            parents = [p if r.random() > 0.2 else int(r.choice([-1, N])) for p in parents]
            slots = [s if r.random() > 0.2 else -1 for s in slots]
        new, moves, missing = forked(slots, parents, S)
        around = torch.full((size + 131072,), 9, dtype=torch.uint8, device="cuda")
        tables = torch.full((M + 4096,), 9, dtype=torch.int32, device="cuda")
        ws, out = around[65536:65536 + size], tables[2048:2048 + M]
        say(f"fork of {N} sequences into {M} children, {S} slots, form {i}")
        got = P.pool_fork(pools, table(slots), table(parents), workspace=ws, out=out)
        assert got.tolist() == new
        assert P.device_status(ws) == (P.DEV_POOL_FULL if missing else P.DEV_OK)
        same(pools, copied(before, [d for d, _ in moves], [s for _, s in moves]))
        for guard in (around[:65536], around[65536 + size:], tables[:2048], tables[2048 + M:]):
            assert bool((guard == 9).all())


def test_rules_on_the_host():
    """The rules themselves, on cases worked out by hand."""
    assert forked([3, 1], [0, 0, 1, 0], 5) == ([3, 0, 1, 2], [(0, 3), (2, 3)], 0)
    assert forked([3, -1], [1, 0, 5, 0], 4) == ([-1, 3, -1, 0], [(0, 3)], 0)
    assert forked([0], [0, 0], 1) == ([0, -1], [], 1)
    assert compacted([4, -1, 0, 7], 8) == ([1, -1, 0, 2], [(1, 4), (2, 7)])
    assert compacted([2, 0, 1], 3) == ([2, 0, 1], [])
