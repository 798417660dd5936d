"""kv_fork_blk, kv_copy_blk, kv_free_blk and kv_compact_blk against their definitions: whole numbers and copied bytes, equal."""
import random

import pytest
import torch

from pages_common import E4M3, ints
from oracle import pages
from paper_2411_18077_amd import api

pytestmark = pytest.mark.gpu


def pool_shape(R, block, N, width, Hkv=1):
    return api.make_blk_shape(R, Hkv, Hkv, 128, block, N, width, torch.float16)


def some_tables(rng, R, block, N, width, share=0.3, absent=0.0):
    """Lengths and rows (of `width` entries) over a pool of N blocks, some of them shared; entries behind the length are anything."""
    order, at = rng.sample(range(N), N), 0
    q_len, table = [], []
    for r in range(R):
        n = rng.choice([0, 1, block - 1, block, block + 1, rng.randint(0, width * block), rng.randint(0, width * block)])
        n = min(n, width * block, (N - at) * block)
        row = []
        for i in range(-(-n // block)):
            if r and rng.random() < share and i < len(table[0]) and i < -(-q_len[0] // block) and (i + 1) * block <= n:
                row.append(table[0][i])
            elif rng.random() < absent:
                row.append(rng.choice([-1, N, 2 ** 31 - 1, -2 ** 31]))
            else:
                row.append(order[at])
                at += 1
        q_len.append(n)
        table.append(row + [rng.choice([-1, 0, N - 1, -9, 2 ** 31 - 1]) for _ in range(width - len(row))])
    return q_len, table, order[at:]


def cut(table, rows):
    return [t[:len(r)] for t, r in zip(table.tolist(), rows)]


def behind(table, rows):
    return [t[len(r):] for t, r in zip(table.tolist(), rows)]


def run_fork(q_len, parent, n_keep, table, free, block, N, head=0, stream=None):
    R, width = len(q_len), len(table[0])
    ring = [-5] * N
    for i, b in enumerate(free):
        ring[(head + i) % N] = b
    want = pages.fork(q_len, parent, n_keep, table, ring, (head, len(free)), block)
    up = lambda v: ints(v).cuda()  # noqa: E731
    outs = [torch.full((R,), 77, dtype=torch.int32, device="cuda"), torch.full((R, width), 77, dtype=torch.int32, device="cuda"),
            torch.full((2,), 77, dtype=torch.int32, device="cuda")] + [torch.full((R,), 77, dtype=torch.int32, device="cuda") for _ in range(2)]
    shape = pool_shape(R, block, N, width)
    api.kv_fork_blk(shape, up(q_len), up(parent), up(n_keep), up(table), up(ring), up([head, len(free)]), *outs)
    torch.cuda.synchronize()
    assert outs[0].tolist() == want["q_len"]
    assert cut(outs[1], want["table"]) == want["table"]
    assert all(set(rest) <= {77} for rest in behind(outs[1], want["table"]))
    assert outs[2].tolist() == want["state"] and outs[3].tolist() == want["src"] and outs[4].tolist() == want["dst"]
    return want


@pytest.mark.parametrize("R", [1, 2, 7, 64, 65, 300, 1023, 1025, 2100])
@pytest.mark.parametrize("block", [16, 64])
def test_forks(R, block):
    rng = random.Random(R * block)
    width = 5
    N = R * 6 + 3
    q_len, table, free = some_tables(rng, R, block, N, width, absent=0.05)
    parent = [rng.choice([r, rng.randrange(R), rng.randrange(R), -1, rng.randrange(min(R, 3))]) for r in range(R)]
    n_keep = [rng.choice([10 ** 9, 2 ** 31 - 1, rng.randint(0, width * block), 0, -3, block]) for _ in range(R)]
    head = rng.randrange(N)
    for some in (len(free), len(free) // 8, 1, 0):     # (the ring wraps, and runs out)
        run_fork(q_len, parent, n_keep, table, free[:some], block, N, head)


def test_fork_everybody_from_one():
    q_len, table = [100, 0, 0, 0], [[3, 1, 4, 5, 9, 2, 6], [-1] * 7, [-1] * 7, [-1] * 7]
    got = run_fork(q_len, [0, 0, 0, 0], [100, 100, 96, 70], table, [0, 7, 8], 16, 10)
    assert got["src"] == [-1, 6, -1, 9] and got["dst"] == [-1, 0, -1, 7]          # 0 keeps its own, 2 ends with a whole block
    got = run_fork(q_len, [-1, 0, 0, 0], [0, 100, 100, 100], table, [0, 7, 8], 16, 10)
    assert got["src"] == [-1, -1, 6, 6]                # the lowest heir
    got = run_fork(q_len, [0, -1, -1, -1], [70, 0, 0, 0], table, [], 16, 10)
    assert got["q_len"][0] == 64                       # cut inside a block that others may hold: a copy, and there is none


@pytest.mark.parametrize("parent", [[7, 2 ** 31 - 1, -2 ** 31, 4, 0]])
def test_fork_parents_out_of_range(parent):
    got = run_fork([20, 20, 20, 20, 20], parent, [20] * 5, [[2 * r, 2 * r + 1] for r in range(5)], [10, 11, 12], 16, 13)
    assert got["q_len"] == [0, 0, 0, 20, 20]


def test_fork_lengths_out_of_range():
    run_fork([2 ** 31 - 1, -7, 33, -2 ** 31], [0, 1, 0, 3], [2 ** 31 - 1, 5, 40, 9], [[0, 1, 2], [3, 4, 5], [6, 7, 8], [9, 10, 11]], [12, 13], 16, 14)


def test_fork_long_rows():
    """Rows of more than one segment, and of many."""
    rng = random.Random(4)
    width, N = 5000, 12000
    order = rng.sample(range(N), N)
    table = [order[:width], order[width:2 * width], [0] * width]
    run_fork([5000 * 16 - 3, 1024 * 16, 1], [1, 0, 0], [10 ** 9, 10 ** 9, 3000 * 16 + 5], table, order[2 * width:], 16, N, head=N - 1)


@pytest.mark.parametrize("R", [4096, 8191, 8192])
def test_forks_of_the_most_requests(R):
    rng = random.Random(R)
    N = R * 3
    q_len, table, free = some_tables(rng, R, 16, N, 3)
    parent = [rng.choice([r, rng.randrange(R), R - 1, rng.randrange(3)]) for r in range(R)]
    n_keep = [rng.choice([10 ** 9, rng.randint(0, 48)]) for _ in range(R)]
    for some in (len(free), len(free) // 2):
        run_fork(q_len, parent, n_keep, table, free[:some], 16, N, N - 2)


def test_fork_captured():
    up = lambda v: ints(v).cuda()  # noqa: E731
    shape = pool_shape(3, 16, 12, 3)
    args = [up([20, 33, 0]), up([0, 0, 1]), up([20, 20, 33]), up([[0, 1, -1], [2, 3, 4], [-1, -1, -1]]), up([5, 6, 7, 8, 9, 10, 11, 0, 0, 0, 0, 0]), up([0, 7])]
    outs = [torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, 3, dtype=torch.int32, device="cuda"),
            torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")]
    api.kv_fork_blk(shape, *args, *outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.kv_fork_blk(shape, *args, *outs)
    for parent in ([0, 0, 1], [1, 1, 1], [-1, 0, 0], [2, 1, 0]):
        args[1].copy_(ints(parent))
        for t in outs:
            t.fill_(5)
        graph.replay()
        got = [t.tolist() for t in outs]
        for t in outs:
            t.fill_(5)
        api.kv_fork_blk(shape, *args, *outs)
        assert got == [t.tolist() for t in outs]


# ---------------------------------------------------------------------------------------------------------

def layers_of(n, N, Hkv, block, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    byte = lambda: torch.randint(0, 256, (N, Hkv, block, 128), generator=g, dtype=torch.uint8, device="cuda")  # noqa: E731
    scale = lambda: torch.randn(N, Hkv, generator=g, device="cuda")  # noqa: E731
    return [dict(K=byte().view(E4M3), V=byte().view(E4M3), Ks=scale(), Vs=scale()) for _ in range(n)]


def check_copy(N, Hkv, block, n_layers, pairs, seed=0):
    shape = pool_shape(1, block, N, 1, Hkv)
    layers = layers_of(n_layers, N, Hkv, block, seed)
    want = []
    for x in layers:
        y = {k: t.view(torch.uint8).clone() if t.dtype is E4M3 else t.clone() for k, t in x.items()}
        for t in y.values():
            old = t.clone()
            for a, b in pairs:
                if 0 <= a < N and 0 <= b < N:
                    t[b] = old[a]
        want.append(y)
    src, dst = ints([p[0] for p in pairs]).cuda(), ints([p[1] for p in pairs]).cuda()
    api.kv_copy_blk(shape, api.BlkCaches(shape, layers), src, dst)
    for x, y in zip(layers, want):
        for k in x:
            got = x[k].view(torch.uint8) if x[k].dtype is E4M3 else x[k]
            assert torch.equal(got, y[k]), k


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("Hkv", [1, 3, 8])
@pytest.mark.parametrize("n_layers", [1, 5])
def test_copies(block, Hkv, n_layers):
    rng = random.Random(block + Hkv)
    N = 60
    ends = rng.sample(range(N), N)
    pairs = [(ends[i], ends[i + 20]) for i in range(20)]
    for i in range(0, 30, 3):                          # holes, and pairs that are none
        pairs.insert(i, rng.choice([(-1, -1), (N, 3), (3, N), (-1, ends[50]), (2 ** 31 - 1, ends[51]), (ends[52], -2 ** 31)]))
    check_copy(N, Hkv, block, n_layers, pairs)


def test_one_source_for_many():
    check_copy(50, 4, 16, 2, [(7, b) for b in range(8, 40)] + [(6, 6)])


@pytest.mark.parametrize("n_pairs", [0, 1, 255, 2048, 2049, 5000])
def test_many_pairs_with_few_that_count(n_pairs):
    rng = random.Random(n_pairs)
    pairs = [(-1, -1)] * n_pairs
    ends = rng.sample(range(64), 64)
    for i, p in enumerate(rng.sample(range(n_pairs), min(n_pairs, 30))):
        pairs[p] = (ends[i], ends[i + 32])
    check_copy(64, 2, 16, 3, pairs)


def test_many_caches():
    """More caches than one launch takes."""
    check_copy(6, 1, 16, 70, [(0, 5), (-1, -1), (2, 3)])


def test_large_blocks():
    """Blocks of 2 MB: more than 64 chunks of 16 KB."""
    check_copy(5, 128, 128, 2, [(0, 4), (2, 1)])


def test_copies_beyond_2_to_32():
    Hkv, block, N = 8, 64, 70000
    shape = pool_shape(1, block, N, 1, Hkv)
    K = torch.zeros(N, Hkv, block, 128, dtype=torch.uint8, device="cuda")
    V = torch.zeros_like(K)
    Ks, Vs = torch.zeros(N, Hkv, device="cuda"), torch.zeros(N, Hkv, device="cuda")
    K[3], V[3], Ks[3], Vs[3] = 17, 18, 2.0, 3.0
    caches = api.BlkCaches(shape, [dict(K=K.view(E4M3), V=V.view(E4M3), Ks=Ks, Vs=Vs)])
    api.kv_copy_blk(shape, caches, ints([3]).cuda(), ints([N - 1]).cuda())
    api.kv_copy_blk(shape, caches, ints([N - 1]).cuda(), ints([66000]).cuda())
    for b in (N - 1, 66000):
        assert (K[b] == 17).all() and (V[b] == 18).all() and (Ks[b] == 2).all() and (Vs[b] == 3).all()
    assert int(K[66001:N - 1].max()) == 0 and int(K[4:66000].max()) == 0


# ---------------------------------------------------------------------------------------------------------

def check_pool(q_len, table, N, block, n_pairs, ws=None):
    R, width = len(q_len), len(table[0])
    up = lambda v: ints(v).cuda()  # noqa: E731
    shape = pool_shape(R, block, N, width)
    if ws is None:
        ws = torch.zeros(api.kv_free_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    full = lambda n: torch.full((n,), 77, dtype=torch.int32, device="cuda")  # noqa: E731
    want, ring, state = pages.free(q_len, table, N, block), full(N), full(2)
    api.kv_free_blk(shape, up(q_len), up(table), ring, state, ws)
    assert state.tolist() == [0, len(want)] and ring.tolist() == want + [77] * (N - len(want))
    moves, rows, want = pages.compact(q_len, table, N, block, n_pairs)
    ring, state, src, dst, new = full(N), full(2), full(n_pairs), full(n_pairs), full(R * width).view(R, width)
    api.kv_compact_blk(shape, up(q_len), up(table), new, ring, state, src, dst, ws)
    assert state.tolist() == [0, len(want)] and ring.tolist() == want + [77] * (N - len(want))
    rest = [-1] * (n_pairs - len(moves))
    assert src.tolist() == [m[0] for m in moves] + rest and dst.tolist() == [m[1] for m in moves] + rest
    assert cut(new, rows) == rows and all(set(x) <= {77} for x in behind(new, rows))
    words = ws[128:128 + -(-N // 1024) * 384].view(torch.int32).view(-1, 96)
    assert int(ws[:4].sum()) == 0 and not words[:, :32].any()          # ready for the next call
    return ws


@pytest.mark.parametrize("R", [1, 3, 64, 400])
@pytest.mark.parametrize("block", [16, 128])
def test_pools(R, block):
    rng = random.Random(R + block)
    for N in (R * 4, R * 4 + 31, R * 7 + 1, 4096, 4097, 9000):
        q_len, table, _ = some_tables(rng, R, block, N, 4, absent=0.05)
        for n_pairs in (N // 2 + 1, 5, 0):
            check_pool(q_len, table, N, block, n_pairs)


@pytest.mark.parametrize("R,N,width", [(400, 17000, 30), (3, 16385, 40), (4200, 16384, 4), (64, 40003, 300), (2000, 65536, 9)])
def test_pools_beyond_one_workgroup(R, N, width):
    """More than 16384 blocks or entries."""
    rng = random.Random(R + N)
    q_len, table, _ = some_tables(rng, R, 16, N, width, absent=0.02)
    ws = check_pool(q_len, table, N, 16, N // 2 + 1)
    check_pool(q_len[::-1], table, N, 16, 7, ws)
    check_pool([0] * R, table, N, 16, 0, ws)


@pytest.mark.parametrize("R,N,width", [(1, 16384, 16384), (8192, 16384, 2), (4096, 500, 4)])
def test_pools_at_the_border_of_one_workgroup(R, N, width):
    rng = random.Random(R)
    q_len, table, _ = some_tables(rng, R, 16, N, width, absent=0.02)
    check_pool(q_len, table, N, 16, N // 2)
    check_pool(q_len, table, N, 16, 3)


def test_pools_of_one_and_of_none():
    check_pool([0], [[0]], 1, 16, 1)
    check_pool([16], [[0]], 1, 16, 1)
    check_pool([1], [[32]], 33, 16, 4)
    check_pool([0, 0], [[1, 2], [3, 4]], 40, 16, 7)
    check_pool([32, 32], [[1, 0], [2, 3]], 4, 16, 7)


def test_pool_lengths_out_of_range():
    check_pool([2 ** 31 - 1, -2 ** 31, 17], [[9, 8], [7, 6], [5, 4]], 12, 16, 4)


def test_large_pool_and_long_rows():
    rng = random.Random(1)
    N, width = 150001, 9000
    order = rng.sample(range(N), N)
    table = [order[i * width:(i + 1) * width] for i in range(8)]
    ws = check_pool([width * 16, 5, 4000 * 16, 8000 * 16 - 7, 0, 16 * 1024, 16 * 1025, 3], table, N, 16, N // 2)
    check_pool([width * 16] * 8, table, N, 16, 1000, ws)


def test_one_workspace_for_many_calls():
    rng = random.Random(2)
    ws = None
    for _ in range(12):
        q_len, table, _ = some_tables(rng, 20, 16, 333, 6)
        ws = check_pool(q_len, table, 333, 16, 40, ws)


def test_one_workspace_for_pools_of_any_size():
    rng = random.Random(5)
    ws = torch.zeros(api.kv_free_workspace_bytes(pool_shape(1, 16, 70000, 1)), dtype=torch.uint8, device="cuda")
    for N in (70000, 333, 20001, 16400, 40, 69999, 17000, 70000):
        q_len, table, _ = some_tables(rng, 60, 16, N, 300)
        check_pool(q_len, table, N, 16, N // 3, ws)


def test_pool_captured():
    """A captured free and compaction, replayed with other lengths, the program's own work between."""
    rng = random.Random(3)
    R, N, block, width = 16, 500, 16, 8
    shape = pool_shape(R, block, N, width)
    ws = torch.zeros(api.kv_free_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    q_len, table = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((R,), (R, width)))
    ring, state, src, dst, new, ring2, state2 = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((N,), (2,), (30,), (30,), (R, width), (N,), (2,)))
    call = lambda: (api.kv_free_blk(shape, q_len, table, ring, state, ws),  # noqa: E731
                    api.kv_compact_blk(shape, q_len, table, new, ring2, state2, src, dst, ws))
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        ql, tb, _ = some_tables(rng, R, block, N, width)
        q_len.copy_(ints(ql)), table.copy_(ints(tb))
        graph.replay()
        torch.cuda.synchronize()
        moves, rows, after = pages.compact(ql, tb, N, block, 30)
        want = pages.free(ql, tb, N, block)
        assert state.tolist() == [0, len(want)] and ring.tolist()[:len(want)] == want
        assert cut(new, rows) == rows and ring2.tolist()[:len(after)] == after and src.tolist()[:len(moves)] == [m[0] for m in moves]
