"""Every token counted once: attention over the paged cache with equal weights and values that name their tokens, so that a tile left out or taken
twice shows whatever the lengths; and results of calls that other tests look at from one side only."""
import pytest
import torch

from blk_common import HALF, SM, attn_tolerance, rand_cache, tables
from oracle import blk
from test_gpu_packed import fused, run

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available()
    from paper_2411_18077_amd import api as _api
    return _api


def count(api, lens, Hq, Hkv, block, dtype, absent=()):
    """Queries of zeros; token i's value is 1 in channel i / 16 % 128 and 0 elsewhere, under scales of 1, 2 and 4.  An output is the share of
    the request's tokens in its channel: weights, their products with the scales and sums of up to 2^24 of them are exact, the quotient
    passes two roundings in fp32 and one to its type."""
    need = [-(-n // block) for n in lens]
    N, width = sum(need) + 1, max(max(need), 1)
    t = tables(lens, block, width, N, 3)
    Kc, Ks = rand_cache(N, Hkv, block, 4, 2) if N * Hkv * block < 40000 else (torch.zeros(N, Hkv, block, 128, dtype=torch.uint8), torch.ones(N, Hkv))
    power = torch.arange(N) % 3
    one = blk.encode(2.0 ** -power.double())           # of each block
    Vc = torch.zeros(N, block, 128, dtype=torch.uint8)
    want = torch.zeros(len(lens), 128, dtype=torch.float64)
    for r, n in enumerate(lens):
        token = torch.arange(n)
        b, at = t[r, token // block].long(), token // 16 % 128
        Vc[b, token % block, at] = one[b]
        there = torch.tensor([(r, i) not in absent for i in range(need[r])])[token // block] if n else token > 0
        want[r] = torch.bincount(at[there], minlength=128).double() / max(int(there.sum()), 1)
    for r, i in absent:
        t[r, i] = -1
    shape = api.make_blk_shape(len(lens), Hq, Hkv, 128, block, N, width, dtype)
    Vc, Vs = Vc[:, None].expand(N, Hkv, block, 128).contiguous().cuda(), (2.0 ** power).float()[:, None].expand(N, Hkv).contiguous().cuda()
    cache = api.BlkCache(shape, K=Kc.cuda().view(E4M3), V=Vc.view(E4M3), Ks=Ks.cuda(), Vs=Vs)
    q = torch.zeros(len(lens), Hq, 128, dtype=dtype, device="cuda")
    out = torch.full_like(q, float("nan"))
    api.minikv_decode_attn_blk(shape, q, cache, t.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), SM, out)
    want = want[:, None].expand(len(lens), Hq, 128)
    err = (out.cpu().double() - want).abs()
    assert bool((err <= want * (HALF[dtype] + 4 * 2.0 ** -24) + 2.0 ** -25).all()), float((err / (want + 1e-9)).max())


@pytest.mark.parametrize("Hq,Hkv,lens,block", [
    (4, 1, [20000], 16), (8, 2, [9000, 33], 128), (2, 1, [i % 90 for i in range(700)], 16), (8, 4, [3000] * 9 + [1] * 9, 32),        # long and many
    (8, 8, [512], 16), (8, 8, [513], 16), (4, 1, [700, 30], 32), (5, 1, [1100, 1000, 900], 64), (8, 1, [4097], 128),                 # workgroups shared
    (2, 2, [9000, 100], 16), (7, 1, [16000], 64), (32, 32, [300] * 8, 16), (1, 1, [131072 + 5], 128),                               # out to units
])
def test_every_token_counts_once(api, Hq, Hkv, lens, block):
    count(api, lens, Hq, Hkv, block, F16)
    count(api, lens, Hq, Hkv, block, BF16)


@pytest.mark.parametrize("Hq,Hkv,block", [(1, 1, 16), (3, 1, 64), (8, 1, 128), (16, 8, 32)])
def test_every_token_counts_once_on_the_line(api, Hq, Hkv, block):
    few = max(300 // Hkv, 40)
    count(api, [9000, 5000 // Hkv] + [10, 0, 70] * (few // 3) + [3000 // Hkv], Hq, Hkv, block, F16)
    count(api, [64] * few + [12000 // Hkv, 1], Hq, Hkv, block, BF16)
    count(api, [70, 0] + [0] * 2000 + [65, 1, 0, 0, 128], Hq, Hkv, block, F16)
    count(api, [40000] + [129] * (2 * few) + [2500], Hq, Hkv, block, BF16)


@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_every_present_token_counts_once(api, block):
    """Blocks that are absent: first, last, in the middle, next to each other, and all of a request."""
    n = 20 * block + 5
    count(api, [n, 3 * block, 40, n], 4, 2, block, F16, absent={(0, 0), (0, 7), (0, 8), (0, 20), (1, 1), (2, 0), (2, 1), (2, 2)} if block == 16 else
          {(0, 0), (0, 7), (0, 8), (0, 20), (1, 1), (2, 0)})


def test_lengths_beyond_the_table_give_the_whole_table(api):
    """A length past the table's end against the definition (which clamps it as the header says)."""
    for block, width in ((16, 2), (64, 3)):
        Kc, Ks = rand_cache(5, 1, block, 1)
        Vc, Vs = rand_cache(5, 1, block, 2)
        shape = api.make_blk_shape(2, 2, 1, 128, block, 5, width, F16)
        cache = api.BlkCache(shape, K=Kc.cuda().view(E4M3), V=Vc.cuda().view(E4M3), Ks=Ks.cuda(), Vs=Vs.cuda())
        t = torch.tensor([[3, 1, 4][:width], [0, 2, 1][:width]], dtype=torch.int32)
        q = torch.randn(2, 2, 128, generator=torch.Generator().manual_seed(4)).half()
        for lens in ([2 ** 31 - 1, width * block + 1], [width * block, -(2 ** 31)]):
            out = torch.full((2, 2, 128), float("nan"), dtype=F16, device="cuda")
            api.minikv_decode_attn_blk(shape, q.cuda(), cache, t.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), SM, out)
            want, mean, score = blk.decode_attn(q, Kc, Ks, Vc, Vs, t, lens, SM)
            real = float((blk.decode_codes(Vc).abs() * Vs.double()[:, :, None, None]).max())
            tol = attn_tolerance(want, mean, score, width * block, real, 2.0 ** -11, F16)
            assert bool(((out.cpu().double() - want).abs() <= tol).all())


@pytest.mark.parametrize("cu,good", [([-5, 40, 300], 1), ([0, 300, 200], 0), ([0, 100, 310], 0), ([-5, 0, 300], 1), ([0, 100, 301, 300], 0)])
def test_the_prompts_beside_one_that_does_not_fit(api, cu, good):
    """Of a batch with a prompt outside the rows or backwards the other prompt's numbers are its own, and no other row is written."""
    Q, K, V = fused(300, 2, 1, F16, 5)
    got = run(api, Q, K, V, cu, True, max_len=300, fill=7.0)
    a, e = cu[good], cu[good + 1]
    want = blk.prompt_attn(Q[a:e], K[a:e], V[a:e], [0, e - a], SM)
    tol = attn_tolerance(want[0], want[3], want[4], e - a, float(V.abs().max()), HALF[F16], F16)
    assert bool(((got[0][a:e].double() - want[0]).abs() <= tol).all())
    # as in the tests of packed prompts: scores' errors, four half steps of the logarithm's sum; weights: both of these and a half step per addition
    rel = 137 * 2.0 ** -24 * want[4] * 1.01
    ltol = rel + 4 * 2.0 ** -24 * (want[1].abs() + want[4] + 1)
    assert bool(((got[1][2 * a:2 * e].double() - want[1]).abs() <= ltol).all())
    assert bool(((got[2][2 * a:2 * e].double() - want[2]).abs() <= want[2] * (rel + float(ltol.max()) + 80 * 2.0 ** -24) + 1e-30).all())
    for x, f in ((got[0], 1), (got[1], 2), (got[2], 2)):
        assert bool((x[:a * f] == 7.0).all()) and bool((x[e * f:] == 7.0).all())


def test_the_largest_batches(api):
    """8192 requests, most of local memory taken by their lengths; 8192 prompts, whose counts take a tile of the second pass."""
    count(api, [(i * 7) % 50 if i % 3 else 0 for i in range(8191)] + [5000], 2, 1, 16, F16)
    count(api, [0] * 8192, 1, 1, 128, BF16)
    count(api, [0] * 8191 + [1], 8, 8, 64, BF16)
    for lens in ([i % 2 for i in range(8192)], [0] * 8000 + [300] + [0] * 190 + [170]):
        cu = [0] + torch.tensor(lens).cumsum(0).tolist()
        Q, K, V = fused(cu[-1], 2, 1, BF16, 3)
        for scores in (True, False):
            X, lse, A = run(api, Q, K, V, cu, scores)
            want = blk.prompt_attn(Q, K, V, [c for i, c in enumerate(cu) if i == 0 or c > cu[i - 1]], SM)
            tol = attn_tolerance(want[0], want[3], want[4], max(lens), float(V.abs().max()), HALF[BF16], BF16)
            assert bool(((X.double() - want[0]).abs() <= tol).all())
            rel = 137 * 2.0 ** -24 * want[4] * 1.01
            ltol = rel + 4 * 2.0 ** -24 * (want[1].abs() + want[4] + 1)
            assert bool(((lse.double() - want[1]).abs() <= ltol).all())
            if scores:
                assert bool(((A.double() - want[2]).abs() <= want[2] * (rel + float(ltol.max()) + 80 * 2.0 ** -24) + 1e-30).all())


@pytest.mark.parametrize("Hq,Hkv", [(32, 1), (24, 2), (10, 1)])
def test_more_than_eight_query_heads_of_a_kv_head(api, Hq, Hkv):
    """The packed prompts have no bound of their own on the heads that share keys."""
    for lens in ([100, 28], [333, 1, 90], [1200]):
        cu = [0] + torch.tensor(lens).cumsum(0).tolist()
        Q, K, V = fused(cu[-1], Hq, Hkv, F16, 4)
        X, lse, A = run(api, Q, K, V, cu, True)
        want = blk.prompt_attn(Q, K, V, cu, SM)
        tol = attn_tolerance(want[0], want[3], want[4], max(lens), float(V.abs().max()), HALF[F16], F16)
        assert bool(((X.double() - want[0]).abs() <= tol).all())
        rel = 137 * 2.0 ** -24 * want[4] * 1.01
        ltol = rel + 4 * 2.0 ** -24 * (want[1].abs() + want[4] + 1)
        assert bool(((lse.double() - want[1]).abs() <= ltol).all())
        assert bool(((A.double() - want[2]).abs() <= want[2] * (rel + float(ltol.max()) + (max(lens) / 64 + 80) * 2.0 ** -24) + 1e-30).all())


def test_attention_captured_and_replayed_with_other_lengths(api):
    """One captured call whose requests grow, shrink and end between replays: a workgroup per unit, several, the line of work, nothing."""
    R, Hq, Hkv, block, width = 40, 16, 8, 32, 300
    N = R * width
    gen = torch.Generator().manual_seed(8)
    shape = api.make_blk_shape(R, Hq, Hkv, 128, block, N, width, BF16)
    codes = [torch.randint(0, 120, (N, Hkv, block, 128), generator=gen, dtype=torch.uint8).cuda() for _ in range(2)]
    ones = torch.full((N, Hkv), 2.0 ** -8, device="cuda")
    cache = api.BlkCache(shape, K=codes[0].view(E4M3), V=codes[1].view(E4M3), Ks=ones, Vs=ones.clone())
    table = torch.arange(N, dtype=torch.int32).view(R, width).cuda()
    q = torch.randn(R, Hq, 128, generator=gen).bfloat16().cuda()
    n, out, want = torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros_like(q), torch.zeros_like(q)
    own = torch.zeros_like(cache.workspace)
    api.minikv_decode_attn_blk(shape, q, cache, table, n, SM, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        api.minikv_decode_attn_blk(shape, q, cache, table, n, SM, out)
    for lens in ([0] * R, [40] * R, [9600] * 3 + [1] * 37, [0] * 39 + [9000], [i * 200 for i in range(R)], [9600] * R, [0] * R, [5] + [0] * 39):
        n.copy_(torch.tensor(lens, dtype=torch.int32))
        out.fill_(float("nan"))
        g.replay()
        api.minikv_decode_attn_blk(shape, q, cache, table, n, SM, want, workspace=own)
        assert torch.equal(out, want)
        for r in (0, R - 1):                           # (against the definition: two requests of each)
            k = (lens[r] + block - 1) // block
            some = [c[r * width:r * width + max(k, 1)].cpu() for c in codes]
            s = torch.full((max(k, 1), Hkv), 2.0 ** -8)
            exact, mean, score = blk.decode_attn(q[r:r + 1].cpu(), some[0], s, some[1], s, torch.arange(max(k, 1)).view(1, -1), [lens[r]], SM)
            tol = attn_tolerance(exact, mean, score, max(lens[r], 1), 448 * 2.0 ** -8, 2.0 ** -11, BF16)
            assert bool(((out[r:r + 1].cpu().double() - exact).abs() <= tol).all())


def test_keys_and_values_of_different_strides(api):
    """Keys as a slice of a projection, values standing alone, and the other way round."""
    g = torch.Generator().manual_seed(5)
    shape = api.make_blk_shape(3, 2, 2, 128, 32, 6, 2, F16)
    wide, alone = torch.randn(70, 7, 128, generator=g).half().cuda(), torch.randn(70, 2, 128, generator=g).half().cuda()
    slots = torch.arange(96, 166, dtype=torch.int32, device="cuda")
    for K, V in ((wide[:, 3:5], alone), (alone, wide[:, 5:])):
        cache = api.BlkCache(shape)
        api.kv_quantize_blk(shape, K, V, slots, cache)
        for x, c, s in ((K, cache.K, cache.Ks), (V, cache.V, cache.Vs)):
            wc, ws = blk.file_rows(x.cpu(), torch.zeros(6, 2, 32, 128, dtype=torch.uint8), torch.zeros(6, 2), slots.cpu())
            assert torch.equal(s.cpu().double(), ws) and torch.equal(blk.decode_codes(c.view(torch.uint8).cpu()), blk.decode_codes(wc))


def test_a_step_of_prompts_and_decoding_requests(api):
    """One step in which requests begin, go on and end, on what kv_assign_blk left on the device: the packed call takes its cu as it is (requests
    that go on are prompts of one token there), the cache gets all rows, and the decoding requests attend with the lengths after the step."""
    R, Hq, Hkv, block, width, N, T = 6, 8, 2, 32, 8, 40, 300
    shape = api.make_blk_shape(R, Hq, Hkv, 128, block, N, width, F16)
    cache = api.BlkCache(shape)
    i = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    table, ring, cu, slots = i([-1] * (R * width)), i(list(range(N))), i([0] * (R + 1)), i([0] * T)
    now, nxt, state, s_nxt = i([0] * R), i([0] * R), i([0, N]), i([0, 0])
    for k, plan in enumerate(([70, 0, 33, 1, 0, 20], [1, 90, 1, 1, 0, -1], [1, 1, 64, -1, 5, 130])):        # (request 2 gets 64 more: filed only)
        api.kv_assign_blk(shape, now, i(plan), table, ring, state, nxt, s_nxt, cu, slots)
        now, nxt, state, s_nxt = nxt, now, s_nxt, state
        Q, K, V = fused(T, Hq, Hkv, F16, 20 + k)       # (rows of no request behind the step's)
        X, lse = torch.full((T, Hq, 128), 7.0, dtype=F16, device="cuda"), torch.full((T * Hq,), 7.0, device="cuda")
        api.selective_flash_attn_packed(R, Hq, Hkv, T, max(plan), Q, K, V, cu, SM, X, lse, None)
        api.kv_quantize_blk(shape, K, V, slots, cache)
        at = [sum(max(n, 0) for n in plan[:r]) for r in range(R + 1)]
        assert cu.tolist() == at
        rows = [a for j, a in enumerate(at) if j == 0 or a > at[j - 1]]
        want = blk.prompt_attn(Q[:at[-1]], K[:at[-1]], V[:at[-1]], rows, SM)
        tol = attn_tolerance(want[0], want[3], want[4], max(plan), float(V.abs().max()), HALF[F16], F16)
        assert bool(((X[:at[-1]].double() - want[0]).abs() <= tol).all()) and bool((X[at[-1]:] == 7.0).all())
        assert bool((lse[at[-1] * Hq:] == 7.0).all())
        for r, n in enumerate(plan):                   # a single token's own value
            if n == 1:
                assert torch.equal(X[at[r]], V[at[r]].repeat_interleave(Hq // Hkv, 0))
        q = torch.randn(R, Hq, 128, generator=torch.Generator().manual_seed(k)).half()
        out = torch.full((R, Hq, 128), float("nan"), dtype=F16, device="cuda")
        api.minikv_decode_attn_blk(shape, q.cuda(), cache, table, now, SM, out)
        codes = [c.view(torch.uint8).cpu() for c in (cache.K, cache.V)]
        exact, mean, score = blk.decode_attn(q, codes[0], cache.Ks.cpu(), codes[1], cache.Vs.cpu(), table.view(R, width).cpu(), now.tolist(), SM)
        tol = attn_tolerance(exact, mean, score, 300, 6.0, 2.0 ** -11, F16)
        assert bool(((out.cpu().double() - exact).abs() <= tol).all())
    assert now.tolist() == [72, 91, 98, 0, 5, 130]
