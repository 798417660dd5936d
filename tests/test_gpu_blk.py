"""The paged 8-bit cache on the GPU against the plain definitions: block assignment (whole numbers, equal), filing (codes and
scales, equal), attention (within a tolerance derived from its roundings)."""
import random

import numpy as np
import pytest
import torch

from blk_common import HALF, SM, attn_tolerance, rand_cache, tables
from oracle import blk

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available()
    from paper_2411_18077_amd import api as _api
    return _api


# ---------------------------------------------------------------------------------------------------------
# kv_assign_blk

def assign_state(R, block, width, hi, seed, new, free=None, over=0.1, n_extra=5):
    """A consistent state of R requests; new(rng, held) gives each one's n_new."""
    rng = random.Random(seed)
    held = [rng.choice([0, rng.randint(0, hi), rng.randint(0, hi) // block * block]) for _ in range(R)]
    n_new = [-1 if rng.random() < over else new(rng, h) for h in held]
    need = [-(-h // block) for h in held]
    want = sum(max(-(-(h + max(n, 0)) // block) - k, 0) for h, n, k in zip(held, n_new, need))
    free = want + n_extra if free is None else int(want * free)
    N = max(sum(need) + free + rng.randint(0, 3), 1)
    ids = list(range(N))
    rng.shuffle(ids)
    table = [[-1] * width for _ in range(R)]
    for r in range(R):
        for b in range(need[r]):
            table[r][b] = ids.pop()
    head = rng.randrange(N)
    ring = [-5] * N
    for i in range(free):
        ring[(head + i) % N] = ids[i]
    return held, n_new, table, ring, [head, free]


def run_assign(api, held, n_new, table, ring, state, block, n_slots, R=None):
    R, width, N = len(held), len(table[0]), len(ring)
    i = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    shape = api.make_blk_shape(R, 1, 1, 128, block, N, width, F16)
    q, n, t, g, s = i(held), i(n_new), i(table), i(ring), i(state)
    q2, s2, cu, slots = torch.full_like(q, -9), torch.full_like(s, -9), i([-9] * (R + 1)), i([-9] * n_slots)
    api.kv_assign_blk(shape, q, n, t, g, s, q2, s2, cu, slots)
    assert q.tolist() == held and s.tolist() == state and n.tolist() == n_new
    return dict(table=t.tolist(), ring=g.tolist(), q_len=q2.tolist(), state=s2.tolist(), cu=cu.tolist(), slots=slots.tolist())


@pytest.mark.parametrize("R,block,width,hi,new,n_slots,free", [
    (1, 16, 4, 40, 1, 1, None), (1, 64, 9, 0, 500, 500, None), (3, 32, 8, 90, 100, 301, None), (64, 16, 20, 250, 1, 64, None),
    (256, 128, 40, 4000, 1, 300, 0.5), (257, 16, 64, 600, 333, 20000, 0.6), (1000, 32, 30, 800, 7, 2500, None),
    (8192, 16, 4, 60, 1, 8192, None), (300, 64, 10, 500, 120, 20000, 0.0), (5, 16, 700, 0, 11000, 60000, None),
])
def test_assignment_equals_the_definition(api, R, block, width, hi, new, n_slots, free):
    for seed in range(2):
        st = assign_state(R, block, width, hi, seed, lambda rng, h: rng.choice([0, new, rng.randint(0, new)]), free)
        want = blk.assign(*st, block, n_slots)
        got = run_assign(api, *st, block, n_slots)
        for k in want:
            assert got[k] == want[k], k


@pytest.mark.parametrize("new", [8, 9])
def test_assignment_of_few_rows_each_and_of_one_more(api, new):
    """Up to eight new rows a request are written by the request's own thread, more by a search: the same numbers."""
    for R, n_slots in ((1, 9), (70, 700), (1500, 20000), (3000, 900)):
        st = assign_state(R, 16, 20, 200, new, lambda rng, h: rng.choice([0, 1, new]), free=0.9)
        assert run_assign(api, *st, 16, n_slots) == blk.assign(*st, 16, n_slots)


def test_assignment_refuses_by_table_slots_and_pool(api):
    st = ([15, 32, 0, 0, 10], [2, 1, 3, 40, 30], [[0, -1], [1, 2], [-1, -1], [-1, -1], [3, -1]], [7, 8, 9, 4, 5, 6], [4, 3])
    for n_slots in (0, 5, 6, 46, 76, 200):
        got, want = run_assign(api, *st, 16, n_slots), blk.assign(*st, 16, n_slots)
        assert got == want, n_slots


def test_values_out_of_range_stay_inside_the_buffers(api):
    """Lengths, counts and ring states that no program means: clamped or refused, nothing outside the buffers is touched."""
    st = ([-5, 1 << 30, 20, 3], [1, 5, 2 ** 31 - 1, -(2 ** 31)], [[0, 1], [2, 3], [4, 5], [6, 7]], [8, 9, 10, 11, 12, 13, 14, 15], [99, 1000])
    got = run_assign(api, *st, 16, 8)
    assert got["q_len"] == [1, 32, 20, 0]                                            # clamped; too many; too many; over
    assert got["cu"] == [0, 1, 6, 2 ** 31 - 1, 2 ** 31 - 1] and got["slots"] == [got["table"][0][0] * 16] + [-1] * 7
    got = run_assign(api, *st[:4], [-3, -1], 16, 8)
    assert got["state"] == [0, 1] and got["q_len"][0] == 0


def test_the_largest_slot_map(api):
    """2^31 - 1 slots: the loop over them steps beyond what 32 bits hold."""
    R, block, n = 3, 16, 2 ** 31 - 1
    shape = api.make_blk_shape(R, 1, 1, 128, block, 40, 8, F16)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    table, ring = torch.zeros(R, 8, dtype=torch.int32, device="cuda"), torch.arange(40, dtype=torch.int32, device="cuda")
    nxt, state, cu, slots = ints(0, 0, 0), ints(0, 0), ints(0, 0, 0, 0), torch.zeros(n, dtype=torch.int32, device="cuda")
    api.kv_assign_blk(shape, ints(0, 0, 0), ints(20, 0, 30), table, ring, ints(0, 40), nxt, state, cu, slots)
    assert nxt.tolist() == [20, 0, 30] and state.tolist() == [4, 36] and cu.tolist() == [0, 20, 20, 50]
    assert slots[:50].tolist() == list(range(20)) + list(range(32, 62))
    assert int(slots[50:].max()) == -1 and int(slots[50:].min()) == -1


def test_assignment_captured_and_replayed_over_steps(api):
    """A decoding loop whose bookkeeping is one captured launch per parity: blocks go out, come back, and are handed out again."""
    R, block, width, N = 12, 16, 6, 40
    i = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    shape = api.make_blk_shape(R, 1, 1, 128, block, N, width, F16)
    rng = random.Random(5)
    want = dict(q_len=[0] * R, table=[[-1] * width for _ in range(R)], ring=list(range(N)), state=[0, N])
    q, s = [i(want["q_len"]), i(want["q_len"])], [i(want["state"]), i(want["state"])]
    t, ring, n, cu, slots = i(want["table"]), i(want["ring"]), i([0] * R), i([0] * (R + 1)), i([0] * 50)
    graphs = []
    for k in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            api.kv_assign_blk(shape, q[k], n, t, ring, s[k], q[1 - k], s[1 - k], cu, slots)
        graphs.append(g)
    for step in range(60):
        n_new = [-1 if want["q_len"][r] > 40 and rng.random() < 0.3 else rng.choice([0, 1, 1, 5, 17]) for r in range(R)]
        n.copy_(i(n_new))
        graphs[step % 2].replay()
        want = blk.assign(want["q_len"], n_new, want["table"], want["ring"], want["state"], block, 50)
        assert q[1 - step % 2].tolist() == want["q_len"] and slots.tolist() == want["slots"] and cu.tolist() == want["cu"], step
        assert t.tolist() == want["table"] and ring.tolist() == want["ring"] and s[1 - step % 2].tolist() == want["state"], step


# ---------------------------------------------------------------------------------------------------------
# kv_quantize_blk

def filed(api, shape, K, V, slots, cache):
    """Runs the call on device copies; codes and scales back on the host."""
    Kc, Ks, Vc, Vs = (x.cuda() for x in cache)
    e4m3 = torch.float8_e4m3fn
    c = api.BlkCache(shape, K=Kc.view(e4m3), V=Vc.view(e4m3), Ks=Ks, Vs=Vs)
    api.kv_quantize_blk(shape, K, V, slots.cuda(), c)
    return [x.cpu() for x in (Kc, Ks, Vc, Vs)]


def check_filed(api, Hkv, block, N, slots, dtype, seed, spread=3, gain=1.0, stride=None):
    g = torch.Generator().manual_seed(seed)
    T = len(slots)
    wide = torch.randn(T, stride or 3 * Hkv, 128, generator=g) * gain * 2.0 ** torch.randint(-spread, spread + 1, (T, 1, 1), generator=g)
    wide = wide.to(dtype).cuda()
    K, V = wide[:, :Hkv], wide[:, -Hkv:]                                             # slices of a fused projection
    Kc, Ks = rand_cache(N, Hkv, block, seed + 1, spread)
    Vc, Vs = rand_cache(N, Hkv, block, seed + 2, spread)
    shape = api.make_blk_shape(1, Hkv, Hkv, 128, block, N, 1, dtype)
    got = filed(api, shape, K, V, torch.tensor(slots, dtype=torch.int32), (Kc, Ks, Vc, Vs))
    for x, c, s, gc, gs in ((K, Kc, Ks, got[0], got[1]), (V, Vc, Vs, got[2], got[3])):
        wc, ws = blk.file_rows(x.cpu(), c, s, torch.tensor(slots))
        assert torch.equal(gs.double(), ws)
        assert torch.equal(blk.decode_codes(gc).nan_to_num(nan=1e9), blk.decode_codes(wc).nan_to_num(nan=1e9))      # (+0 and -0 alike)


def prompt_slots(lens, block, N, seed, held=None):
    """Slots of `lens` new tokens of requests that hold `held` ones, over shuffled blocks."""
    t = tables([(h + n) for n, h in zip(lens, held or [0] * len(lens))], block, 64, N, seed)
    return [int(t[r, (h + i) // block]) * block + (h + i) % block for r, (n, h) in enumerate(zip(lens, held or [0] * len(lens))) for i in range(n)]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("Hkv,lens,held", [
    (1, [1], [0]), (2, [1], [5]), (8, [1] * 9, [0, 1, 15, 16, 31, 32, 63, 64, 127]), (3, [130, 1, 63], None), (2, [7, 40], [9, 100]),
    (4, [256], None),
])
def test_filing_equals_the_definition(api, dtype, block, Hkv, lens, held):
    check_filed(api, Hkv, block, 40, prompt_slots(lens, block, 40, 3, held), dtype, seed=len(lens) + block)


def test_filing_nothing(api):
    shape = api.make_blk_shape(1, 2, 2, 128, 16, 3, 1, F16)
    cache = api.BlkCache(shape)
    x = torch.zeros(0, 2, 128, dtype=F16, device="cuda")
    api.kv_quantize_blk(shape, x, x, torch.zeros(0, dtype=torch.int32, device="cuda"), cache)
    x = torch.ones(5, 2, 128, dtype=F16, device="cuda")
    api.kv_quantize_blk(shape, x, x, torch.full((5,), -1, dtype=torch.int32, device="cuda"), cache)          # padding alone
    assert not bool(cache.K.view(torch.uint8).any()) and not bool(cache.Ks.any()) and not bool(cache.Vs.any())


def test_filing_more_rows_than_waves_fit_a_launch(api):
    """8192 requests' tokens of 4104 heads, K and V: 2^26 rows and more.  The last sixteen have a block."""
    n, Hkv, block = 8192, 4104, 16
    x = torch.zeros(n, Hkv, 128, dtype=F16, device="cuda")
    x[-block:] = torch.randn(block, Hkv, 128, generator=torch.Generator().manual_seed(1)).half().cuda()
    slots = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    slots[-block:] = torch.arange(block, 2 * block, dtype=torch.int32, device="cuda")
    many, few = api.make_blk_shape(8192, Hkv, Hkv, 128, block, 2, 1, F16), api.make_blk_shape(1, Hkv, Hkv, 128, block, 2, 1, F16)
    one, two = api.BlkCache(many), api.BlkCache(few)
    api.kv_quantize_blk(many, x, x, slots, one)
    api.kv_quantize_blk(few, x[-block:], x[-block:], slots[-block:], two)
    assert bool((one.Ks[1] > 0).all()) and not bool(one.Ks[0].any())
    for a, b in ((one.K, two.K), (one.V, two.V), (one.Ks, two.Ks), (one.Vs, two.Vs)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_filing_many_tokens_a_wave(api):
    """More tokens than the form of a wave per token takes: waves that begin several runs, runs across waves, padding."""
    slots = prompt_slots([700, 333, 16, 1, 1, 1, 50, 900], 16, 140, 7)
    check_filed(api, 8, 16, 140, slots + [-1] * 100, F16, seed=11)
    slots = prompt_slots([1] * 60 + [900], 64, 90, 8, [i for i in range(60)] + [37])
    cut = 60 + (64 - 37) + 64 * 6                      # (a block's first row: rows of one block stand together)
    check_filed(api, 8, 64, 90, [-1] * 3 + slots[:cut] + [-1] + slots[cut:] + [90 * 64, 2 ** 31 - 1, -(2 ** 31)], BF16, seed=12)
    check_filed(api, 9, 128, 12, prompt_slots([1000], 128, 12, 9), BF16, seed=13)


@pytest.mark.parametrize("dtype,gain", [(F16, 2.0 ** -20), (F16, 4000.0), (BF16, 2.0 ** -120), (BF16, 2.0 ** -128), (BF16, 2.0 ** 118), (F16, 0.0)])
def test_filing_at_the_ends_of_the_range(api, dtype, gain):
    check_filed(api, 2, 32, 9, prompt_slots([40, 3], 32, 9, 4, [10, 32]), dtype, seed=21, spread=0, gain=gain)


def test_rows_that_stand_in_the_pool_keep_their_values_when_the_scale_grows(api):
    """Appending ever larger rows: each step doubles the scale, codes shift without loss until they are subnormal."""
    block, N = 64, 2
    shape = api.make_blk_shape(1, 1, 1, 128, block, N, 1, F16)
    cache = [torch.full((N, 1, block, 128), 0x7f, dtype=torch.uint8), torch.full((N, 1), 7.0)] * 2           # what a last use left
    want = None
    for i in range(12):
        x = (torch.randn(1, 1, 128, generator=torch.Generator().manual_seed(i)) * 2.0 ** i).half()
        cache = filed(api, shape, x.cuda(), -x.cuda(), torch.tensor([block + i], dtype=torch.int32), cache)
        want = blk.file_rows(x, *(want or (torch.full((N, 1, block, 128), 0x7f, dtype=torch.uint8), torch.full((N, 1), 7.0))), torch.tensor([block + i]))
        got_v, want_v = blk.decode_codes(cache[0]), blk.decode_codes(want[0])
        assert torch.equal(cache[1].double(), want[1]) and torch.equal(got_v.nan_to_num(nan=1e9), want_v.nan_to_num(nan=1e9))
        assert torch.equal(got_v[1, 0, :i + 1], -blk.decode_codes(cache[2])[1, 0, :i + 1])
        assert torch.equal(cache[0][0], torch.full((1, block, 128), 0x7f, dtype=torch.uint8))                # the other block


# ---------------------------------------------------------------------------------------------------------
# minikv_decode_attn_blk

def attend(api, lens, Hq, Hkv, block, dtype, seed=1, width=None, spread=2, spoil=True, table=None, extra=2, gain=1.0, sm=SM, scale=None):
    """Runs the call on a cache whose unused rows hold NaN codes; compares with the definition; returns the output."""
    n_blocks = sum(-(-n // block) for n in lens) + extra
    width = width or max(max(-(-n // block) for n in lens), 1)
    t = tables(lens, block, width, n_blocks, seed) if table is None else table
    Kc, Ks = rand_cache(n_blocks, Hkv, block, seed + 1, spread)
    Vc, Vs = rand_cache(n_blocks, Hkv, block, seed + 2, spread)
    if scale is not None:
        Ks, Vs = Ks * scale, Vs * scale
    if spoil:
        used = torch.zeros(n_blocks, block, dtype=torch.bool)
        for r, n in enumerate(lens):
            for b in range(-(-n // block)):
                if 0 <= t[r, b] < n_blocks:
                    used[t[r, b], :min(n - b * block, block)] = True
        for c, s in ((Kc, Ks), (Vc, Vs)):
            c.view(n_blocks, Hkv, block, 128).transpose(1, 2)[~used] = 0x7f
            s[~used.any(dim=1)] = float("nan")
    g = torch.Generator().manual_seed(seed + 3)
    q = (torch.randn(len(lens), Hq + 2, 128, generator=g) * gain).to(dtype).cuda()[:, 1:Hq + 1]       # a slice
    shape = api.make_blk_shape(len(lens), Hq, Hkv, 128, block, n_blocks, width, dtype)
    e4m3 = torch.float8_e4m3fn
    cache = api.BlkCache(shape, K=Kc.cuda().view(e4m3), V=Vc.cuda().view(e4m3), Ks=Ks.cuda(), Vs=Vs.cuda())
    out = torch.full((len(lens), Hq, 128), float("nan"), dtype=dtype, device="cuda")
    q_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    args = (shape, q, cache, t.cuda(), q_len, sm, out)
    api.minikv_decode_attn_blk(*args)
    want, mean, score = blk.decode_attn(q.cpu(), Kc, Ks, Vc, Vs, t, lens, sm)
    real = blk.decode_codes(Vc).nan_to_num(0.0).abs() * Vs.nan_to_num(0.0).double()[:, :, None, None]
    tol = attn_tolerance(want, mean, score, max(max(lens), 1), float(real.max()), 2.0 ** -11, dtype)
    err = (out.cpu().double() - want).abs()
    assert bool((err <= tol).all()), (float(err.max()), float((err / tol).max()))
    first = out.clone()
    out.fill_(float("nan"))
    api.minikv_decode_attn_blk(*args)                                                # the workspace is as it was
    assert torch.equal(first, out)
    assert not bool(cache.workspace[:5120].any())
    return out


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("Hq,Hkv,lens", [
    (1, 1, [1]), (8, 8, [64]), (8, 1, [65, 63]), (6, 2, [0, 1, 17, 0, 400]), (32, 4, [257, 16, 15]), (4, 4, [1000, 3]),
    (16, 2, [2500]), (5, 1, [128] * 7),
])
def test_attention_over_the_paged_cache(api, dtype, block, Hq, Hkv, lens):
    attend(api, lens, Hq, Hkv, block, dtype)


def test_long_and_many_requests(api):
    attend(api, [20000], 4, 1, 16, F16)                # one unit over many workgroups, table fetched in batches
    attend(api, [9000, 33], 8, 2, 128, BF16)
    attend(api, [i % 90 for i in range(700)], 2, 1, 16, F16)          # several units a workgroup, empty ones between
    attend(api, [3000] * 9 + [1] * 9, 8, 4, 32, BF16)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("Hq,Hkv,block", [(1, 1, 16), (3, 1, 64), (8, 1, 128), (16, 8, 32)])
def test_the_line_of_work(api, dtype, Hq, Hkv, block):
    """More units than workgroups: waves with several units, units over many waves and workgroups, merged by the last one."""
    few = max(300 // Hkv, 40)
    attend(api, [9000, 5000 // Hkv] + [10, 0, 70] * (few // 3) + [3000 // Hkv], Hq, Hkv, block, dtype)
    attend(api, [64] * few + [12000 // Hkv, 1], Hq, Hkv, block, dtype, seed=4)
    attend(api, [70, 0] + [0] * 2000 + [65, 1, 0, 0, 128], Hq, Hkv, block, dtype, seed=5)         # a padded batch


@pytest.mark.parametrize("Hq,Hkv,lens,block", [
    (8, 8, [512], 16), (8, 8, [513], 16), (4, 1, [700, 30], 32), (5, 1, [1100, 1000, 900], 64), (8, 1, [4097], 128), (2, 2, [9000, 100], 16),
    (7, 1, [16000], 64), (32, 32, [300] * 8, 16),
])
def test_workgroups_shared_out_to_units(api, Hq, Hkv, lens, block):
    """Few units: one workgroup each up to eight tiles, several beyond, whose results meet by ticket."""
    attend(api, lens, Hq, Hkv, block, F16)
    attend(api, lens, Hq, Hkv, block, BF16, seed=9)


def test_requests_without_tokens_and_wide_tables(api):
    out = attend(api, [0, 0, 0], 8, 2, 32, F16)
    assert not bool(out.any())
    attend(api, [40, 0, 7], 8, 2, 16, F16, width=50)


def test_table_entries_out_of_range_are_absent(api):
    lens, block = [100, 64, 40], 16
    t = tables(lens, block, 8, 20, 3)
    t[0, 2], t[0, 6], t[2, 0], t[2, 1], t[2, 2] = -1, 20, 2 ** 31 - 1, -(2 ** 31), -1
    out = attend(api, lens, 4, 2, block, BF16, table=t, width=8, extra=6)
    assert not bool(out[2].any())
    for block, width in ((64, 3), (128, 2), (32, 5)):
        t = tables([150, 100], block, width, 9, 3)
        t[0, 1] = -1
        attend(api, [150, 100], 4, 2, block, F16, table=t, width=width, extra=9 - sum(-(-n // block) for n in [150, 100]))


def test_shared_blocks_and_lengths_beyond_the_table(api):
    t = torch.tensor([[3, 1], [3, 2], [3, 1]], dtype=torch.int32)                    # a prefix in three tables
    attend(api, [20, 32, 20], 4, 1, 16, F16, table=t, width=2, extra=2, spoil=False)
    attend(api, [32, 32, 20], 4, 1, 16, F16, table=t, width=2, extra=2, spoil=False)
    # a length past the table is clamped to it
    n_blocks = 5
    Kc, Ks = rand_cache(n_blocks, 1, 16, 1)
    shape = api.make_blk_shape(1, 2, 1, 128, 16, n_blocks, 2, F16)
    e4m3 = torch.float8_e4m3fn
    cache = api.BlkCache(shape, K=Kc.cuda().view(e4m3), V=Kc.cuda().view(e4m3), Ks=Ks.cuda(), Vs=Ks.cuda())
    q, out = torch.randn(1, 2, 128).half().cuda(), [torch.zeros(1, 2, 128, dtype=F16, device="cuda") for _ in range(2)]
    for o, n in zip(out, (32, 2 ** 31 - 1)):
        api.minikv_decode_attn_blk(shape, q, cache, t[:1].cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"), SM, o)
    assert torch.equal(out[0], out[1])


@pytest.mark.parametrize("scale", [2.0 ** -60, 2.0 ** 20, 0.37, 0.0])
def test_scales_of_any_size(api, scale):
    """Power-of-two or not, tiny, large, zero: the weights of the second product stay below 1."""
    attend(api, [333, 64], 4, 2, 32, BF16, scale=scale, sm=SM / (scale or 1.0), spread=6)


def test_peaked_rows_and_negative_scale_factor(api):
    attend(api, [700, 90], 8, 2, 64, F16, gain=12.0)
    attend(api, [200], 8, 2, 64, F16, sm=-SM)
    attend(api, [200], 8, 2, 64, F16, sm=0.0)


def test_shapes_take_turns_on_one_workspace(api):
    """Calls of different shapes on one workspace, and two captured graphs of them, replayed in turn with eager calls between."""
    made = []
    e4m3 = torch.float8_e4m3fn
    for lens, Hq, Hkv, block in (([5000, 77], 8, 1, 16), ([300] * 40, 8, 4, 64), ([12000], 4, 2, 128)):
        N = sum(-(-n // block) for n in lens)
        Kc, Ks = rand_cache(N, Hkv, block, 5)
        shape = api.make_blk_shape(len(lens), Hq, Hkv, 128, block, N, max(-(-n // block) for n in lens), F16)
        cache = api.BlkCache(shape, K=Kc.cuda().view(e4m3), V=Kc.cuda().view(e4m3), Ks=Ks.cuda(), Vs=Ks.cuda())
        t = tables(lens, block, shape.max_blocks, N, 5).cuda()
        q = torch.randn(len(lens), Hq, 128, generator=torch.Generator().manual_seed(1)).half().cuda()
        made.append((shape, q, cache, t, torch.tensor(lens, dtype=torch.int32, device="cuda"), SM, torch.zeros_like(q)))
    own = []
    for m in made:
        api.minikv_decode_attn_blk(*m)
        own.append(m[-1].clone())
    ws = made[0][2].workspace
    graphs = []
    for m in made:
        m[-1].zero_()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            api.minikv_decode_attn_blk(*m, workspace=ws)
        graphs.append(g)
    for _ in range(4):
        for m, g, o in zip(made, graphs, own):
            m[-1].zero_()
            g.replay()
            assert torch.equal(m[-1], o)
            m[-1].zero_()
            api.minikv_decode_attn_blk(*m, workspace=ws)
            assert torch.equal(m[-1], o)


def test_offsets_beyond_32_bits(api):
    """A pool of more than 4 GB of codes: the last blocks are filed and attended to."""
    Hkv, block, N = 8, 128, 40000                      # 128 KB of codes per block: 5.2 GB
    shape = api.make_blk_shape(1, 8, Hkv, 128, block, N, 3, F16)
    cache = api.BlkCache(shape)
    ids = [39999, 33000, 20]
    slots = [b * block + i for b in ids for i in range(block)]
    g = torch.Generator().manual_seed(9)
    K, V = torch.randn(len(slots), Hkv, 128, generator=g).half(), torch.randn(len(slots), Hkv, 128, generator=g).half()
    api.kv_quantize_blk(shape, K.cuda(), V.cuda(), torch.tensor(slots, dtype=torch.int32, device="cuda"), cache)
    z = torch.zeros(3, Hkv, block, 128, dtype=torch.uint8)
    local = torch.tensor([i * block + j for i in range(3) for j in range(block)])
    small = [blk.file_rows(x, z, torch.zeros(3, Hkv), local) for x in (K, V)]
    for c, s, (wc, ws) in ((cache.K, cache.Ks, small[0]), (cache.V, cache.Vs, small[1])):
        got = c.view(torch.uint8)[torch.tensor(ids, device="cuda")].cpu()
        assert torch.equal(blk.decode_codes(got), blk.decode_codes(wc)) and torch.equal(s[torch.tensor(ids, device="cuda")].cpu().double(), ws)
    q, out = torch.randn(1, 8, 128, generator=g).half(), torch.zeros(1, 8, 128, dtype=F16, device="cuda")
    api.minikv_decode_attn_blk(shape, q.cuda(), cache, torch.tensor([ids], dtype=torch.int32, device="cuda"),
                               torch.tensor([380], dtype=torch.int32, device="cuda"), SM, out)
    want, mean, score = blk.decode_attn(q, small[0][0], small[0][1].float(), small[1][0], small[1][1].float(), torch.tensor([[0, 1, 2]]), [380], SM)
    assert bool(((out.cpu().double() - want).abs() <= attn_tolerance(want, mean, score, 380, 6.0, 2.0 ** -11, F16)).all())


def test_filing_captured_and_replayed(api):
    """Each replay files other rows at other slots; a program's own calls stand between the replays."""
    shape = api.make_blk_shape(2, 2, 2, 128, 16, 12, 6, F16)
    one, two = api.BlkCache(shape), api.BlkCache(shape)
    gen = torch.Generator().manual_seed(4)
    rows = [torch.randn(20, 2, 128, generator=gen).half().cuda() * 3 ** k for k in range(4)]
    slots = [torch.tensor([(5 * k + i) % 192 for i in range(20)], dtype=torch.int32, device="cuda") for k in range(4)]
    x, s = rows[0].clone(), slots[0].clone()
    api.kv_quantize_blk(shape, x, x, s, two)
    two.K.view(torch.uint8).zero_(), two.V.view(torch.uint8).zero_(), two.Ks.zero_(), two.Vs.zero_()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        api.kv_quantize_blk(shape, x, x, s, two)
    for r, n in zip(rows, slots):
        x.copy_(r), s.copy_(n)
        g.replay()
        api.kv_quantize_blk(shape, r, r, n, one)
        for a, b in ((one.K, two.K), (one.V, two.V), (one.Ks, two.Ks), (one.Vs, two.Vs)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert bool((one.Ks > 0).any())


def test_two_calls_at_once(api):
    """Attention on two streams with workspaces of their own: the results of one after the other."""
    lens, block, Hkv, N = [4000, 300, 900], 64, 2, 90
    shape = api.make_blk_shape(3, 8, Hkv, 128, block, N, 64, BF16)
    gen = torch.Generator().manual_seed(6)
    cache = api.BlkCache(shape)
    t = tables(lens, block, 64, N, 2).cuda()
    slots = torch.tensor([int(t[r, i // block]) * block + i % block for r, n in enumerate(lens) for i in range(n)], dtype=torch.int32, device="cuda")
    x = torch.randn(sum(lens), Hkv, 128, generator=gen).bfloat16().cuda()
    api.kv_quantize_blk(shape, x, x, slots, cache)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    q = [torch.randn(3, 8, 128, generator=gen).bfloat16().cuda() for _ in range(2)]
    want = [torch.zeros_like(v) for v in q]
    for v, o in zip(q, want):
        api.minikv_decode_attn_blk(shape, v, cache, t, n, SM, o)
    out = [[torch.zeros_like(v) for _ in range(20)] for v in q]
    ws = [torch.zeros_like(cache.workspace) for _ in q]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for k in range(20):
        for v, o, w, st in zip(q, out, ws, streams):
            api.minikv_decode_attn_blk(shape, v, cache, t, n, SM, o[k], workspace=w, stream=st)
    torch.cuda.synchronize()
    for o, w in zip(out, want):
        assert all(torch.equal(v, w) for v in o)


def test_calls_on_a_side_stream(api):
    """The calls go to the stream that is current, or to the one given."""
    lens, block, Hkv = [70, 200], 32, 2
    N = 12
    shape = api.make_blk_shape(2, 4, Hkv, 128, block, N, 7, F16)
    t = tables(lens, block, 7, N, 1).cuda()
    slots = torch.tensor([int(t[r, i // block]) * block + i % block for r, n in enumerate(lens) for i in range(n)], dtype=torch.int32, device="cuda")
    x = torch.randn(270, Hkv, 128, generator=torch.Generator().manual_seed(3)).half().cuda()
    q, n = torch.randn(2, 4, 128).half().cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    outs = []
    for stream in (None, torch.cuda.Stream(), "given"):
        cache, out = api.BlkCache(shape), torch.zeros(2, 4, 128, dtype=F16, device="cuda")
        torch.cuda.synchronize()
        if stream == "given":
            s = torch.cuda.Stream()
            api.kv_quantize_blk(shape, x, x, slots, cache, stream=s)
            api.minikv_decode_attn_blk(shape, q, cache, t, n, SM, out, stream=s)
        else:
            with torch.cuda.stream(stream or torch.cuda.current_stream()):
                api.kv_quantize_blk(shape, x, x, slots, cache)
                api.minikv_decode_attn_blk(shape, q, cache, t, n, SM, out)
        torch.cuda.synchronize()
        outs.append(out.clone())
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
