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
    N, width = sum(need) + 1, max(need)
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
