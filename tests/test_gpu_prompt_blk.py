"""minikv_prompt_attn_blk against its definition in 64 bits."""
import math

import pytest
import torch

from pages_common import E4M3, HALF, SM, check_prompt, ints, lse_tolerance, make_cache, prompt_tolerance, rand_cache, tables
from oracle import pages
from paper_2411_18077_amd import api

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


class Case:
    def __init__(self, held, new, Hq, Hkv, block, dtype, seed=0, spread=0, extra_rows=2, gain=1.0, fused=True, width=None):
        total = [h + n for h, n in zip(held, new)]
        R = len(held)
        self.width = width or max(-(-max(total) // block), 1)
        self.N = sum(-(-t // block) for t in total) + 2
        self.Kc, self.Ks = rand_cache(self.N, Hkv, block, seed, spread)
        self.Vc, self.Vs = rand_cache(self.N, Hkv, block, seed + 1, spread)
        self.table = tables(total, block, self.width, self.N, seed)
        for r, t in enumerate(total):                  # NaN codes behind the last token
            if t % block:
                b = int(self.table[r, t // block])
                self.Kc[b, :, t % block:], self.Vc[b, :, t % block:] = 0x7f, 0xff
        self.q_len, self.cu = ints(total), ints([sum(new[:i]) for i in range(R + 1)])
        self.T = sum(new) + extra_rows
        g = torch.Generator().manual_seed(seed + 2)
        x = (torch.randn(self.T, Hq + (3 if fused else 0), 128, generator=g) * gain).to(dtype)
        self.q = x[:, :Hq]
        self.q_dev = x.cuda()[:, :Hq]
        self.shape = api.make_blk_shape(R, Hq, Hkv, 128, block, self.N, self.width, dtype)
        self.dtype, self.Hq = dtype, Hq

    def run(self, lse=True, ws=None, T=None):
        T = self.T if T is None else T
        self.cache = make_cache(self.shape, self.Kc, self.Ks, self.Vc, self.Vs)
        self.out = torch.full((self.T, self.Hq, 128), 7.0, dtype=self.dtype, device="cuda")
        self.lse = torch.full((self.T, self.Hq), 7.0, device="cuda")
        if ws is None:
            ws = torch.zeros(api.minikv_prompt_blk_workspace_bytes(self.shape, T), dtype=torch.uint8, device="cuda")
        self.ws = ws
        self.args = (self.shape, T, self.q_dev, self.cache, self.table.cuda(), self.q_len.cuda(), self.cu.cuda(), SM, self.out,
                     self.lse if lse else None, ws)
        api.minikv_prompt_attn_blk(*self.args)
        return self

    def check(self, spread=64):
        check_prompt(self.shape, self.q, (self.Kc, self.Ks, self.Vc, self.Vs), self.table, self.q_len, self.cu, self.out, self.lse, spread=spread)
        return self


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (8, 2), (6, 2), (8, 1), (5, 1), (14, 2)])
def test_blocks_and_heads(Hq, Hkv, block, dtype):
    Case([70, 0, 33], [20, 9, 40], Hq, Hkv, block, dtype, seed=Hq + block).run().check()


@pytest.mark.parametrize("held,new", [
    ([0], [1]), ([1], [1]), ([0], [2]), ([63], [1]), ([64], [1]), ([62], [1]), ([0], [64]), ([0], [65]), ([1], [63]), ([127], [2]), ([500], [1]),
    ([0], [33]), ([31], [32]), ([3], [129]), ([130], [257]), ([1000], [3]), ([5, 0, 0, 7], [0, 0, 3, 0]), ([0, 0], [0, 1]), ([9] * 70, [1] * 70),
    ([3, 100, 0] * 30, [1, 2, 3] * 30), ([2000, 3], [1, 150]),
])
def test_lengths(held, new):
    Case(held, new, 4, 2, 16, F16, seed=len(held) + sum(new)).run().check()


@pytest.mark.parametrize("held,new,Hq,Hkv", [([6000], [1], 2, 2), ([9000], [5], 8, 2), ([4000, 100], [40, 3], 4, 1), ([3000], [200], 3, 1), ([20000], [2], 1, 1)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_walks_in_parts(held, new, Hq, Hkv, dtype):
    Case(held, new, Hq, Hkv, 64, dtype, seed=3).run().check()


# Blocks of 32 rows up to 512 of them in all, of 128 beyond: many heads make many.
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("held,new,Hq,Hkv", [([0], [150], 128, 128), ([70], [130], 128, 128), ([5, 200], [100, 64], 128, 128), ([333, 0], [40, 90], 256, 128),
                                             ([64], [200], 192, 64)])
def test_wide_blocks(held, new, Hq, Hkv, block, dtype):
    Case(held, new, Hq, Hkv, block, dtype, seed=Hq + block + sum(new)).run().check()


@pytest.mark.parametrize("held,new", [([0], [2016]), ([0], [2048]), ([0], [2049]), ([1], [2080])])
def test_blocks_next_to_the_border_of_512(held, new):
    """63 and 64 blocks of 32 rows for each of 8 heads, 65 (513 and more: of 128 rows)."""
    Case(held, new, 8, 8, 64, BF16, seed=30).run().check()


@pytest.mark.parametrize("block,dtype", [(16, F16), (64, BF16), (32, BF16)])
def test_wide_walks_in_parts(block, dtype):
    """One long walk among many short ones."""
    Case([6000] + [10] * 12, [130] + [64] * 12, 32, 32, block, dtype, seed=31).run().check()
    Case([10] * 12 + [3000], [64] * 12 + [100], 64, 32, block, dtype, seed=32).run().check()


def test_wide_blocks_in_the_corners():
    """What the other tests look at, with blocks of 128 rows: more new rows than tokens, absent blocks, scales far apart, zero, of no power of two."""
    c = Case([64, 40, 100], [100, 100, 100], 64, 64, 16, F16, seed=33, spread=6, gain=2.0 ** -6)
    c.q_len[0], c.q_len[1] = 70, 3
    c.Kc, c.Ks = rand_cache(c.N, 64, 16, 81)
    c.Vs[c.table[0].long()[:3]] = 0.0
    c.Vs[c.table[2, 4].long()] *= 0.77
    c.Ks[c.table[2, 5].long()] *= 1.37
    c.Ks[c.table[2, 6].long()] = 0.0
    c.table[2, 1], c.table[2, 9] = -1, c.N
    c.run().check(spread=80)


@pytest.mark.parametrize("block,dtype", [(64, BF16), (32, F16), (16, F16)])
def test_calls_that_read_more_than_caches_hold(block, dtype):
    """64 requests behind one prefix of 2048 tokens, 8 KV heads: 16896 tiles of 64 tokens."""
    R, Hkv, prefix = 64, 8, 2048 // block
    new = [1 + r % 4 for r in range(R)]
    c = Case([0], [4], 16, Hkv, block, dtype, seed=34)  # (its own tokens are replaced)
    c.N, c.width = prefix + R, prefix + 1
    (c.Kc, c.Ks), (c.Vc, c.Vs) = rand_cache(c.N, Hkv, block, 35), rand_cache(c.N, Hkv, block, 36)
    c.table = torch.cat([torch.arange(prefix).expand(R, prefix), prefix + torch.arange(R)[:, None]], dim=1).int().contiguous()
    c.q_len, c.cu, c.T = ints([2048 + n for n in new]), ints([sum(new[:r]) for r in range(R + 1)]), sum(new) + 1
    c.q = torch.randn(c.T, 16, 128, generator=torch.Generator().manual_seed(37)).to(dtype)
    c.q_dev = c.q.cuda()
    c.shape = api.make_blk_shape(R, 16, Hkv, 128, block, c.N, c.width, dtype)
    c.run().check()


@pytest.mark.parametrize("R", [256, 257, 700])
def test_many_requests(R):
    held, new = [(r * 37) % 90 for r in range(R)], [(r * 11) % 4 for r in range(R)]
    Case(held, new, 2, 1, 16, F16, seed=R).run().check()
    new[R // 2] = 150
    Case(held, new, 2, 2, 32, BF16, seed=R).run().check()


@pytest.mark.parametrize("R", [63, 64, 65, 128])
def test_requests_of_all_lengths(R):
    """Walks in parts, long and short ones in one, more of them than run at once."""
    held, new = [(3000, 700, 90, 5, 0)[r % 5] + r for r in range(R)], [(40, 1, 130, 70, 9, 0, 260)[r % 7] for r in range(R)]
    Case(held, new, 8, 4, 16, F16, seed=R).run().check()


@pytest.mark.parametrize("R,n", [(4097, 1), (8192, 1), (8191, 2)])
def test_the_most_requests(R, n):
    held, new = [(r * 7) % 30 for r in range(R)], [(r % 5 == 0) * n for r in range(R)]
    new[R - 1], held[R - 1] = 40, 3000                 # (in parts)
    Case(held, new, 2, 1, 64, BF16, seed=R).run().check()


def test_rows_before_the_first_token():
    """More new rows than tokens: those in front see nothing."""
    c = Case([0, 40], [30, 20], 4, 2, 16, F16, seed=4)
    c.q_len[0] = 12
    c.q_len[1] = 0
    c.run().check()


def test_lengths_out_of_range():
    c = Case([54, 20, 30], [10, 10, 10], 4, 2, 16, BF16, seed=5)      # (request 0 fills its blocks: the third, clamped to them, counts no NaN code)
    c.q_len = ints([64, -5, 10 ** 9])
    c.table[2, :] = c.table[0, :]
    c.run().check()


@pytest.mark.parametrize("cu", [[0, 40, 30, 45], [-3, 4, 20, 30], [0, 10, 20, 1000], [5, 5, 5, 5], [2 ** 31 - 1, -2 ** 31, 0, 3], [30, 30, 10, 20]])
def test_rows_out_of_range(cu):
    """Requests whose rows do not lie inside are left alone."""
    c = Case([50, 20, 30], [10, 10, 10], 4, 2, 16, F16, seed=6)
    c.cu = ints(cu)
    c.run().check()


def test_rows_that_many_requests_claim():
    """cu that falls and rises: more parts than the launch has workgroups.  What is written is nobody's business, but the workspace stays good."""
    c = Case([3000] + [0] * 199, [1] + [0] * 199, 4, 2, 64, F16, seed=26)
    c.run().check()
    c.table[:] = c.table[0]
    c.q_len[:], c.cu = 3001, ints([r % 2 for r in range(201)])
    c.run(ws=c.ws)
    again = Case([3000, 2000], [1, 3], 4, 2, 64, F16, seed=27)
    ws = torch.zeros(max(c.ws.numel(), api.minikv_prompt_blk_workspace_bytes(again.shape, again.T)), dtype=torch.uint8, device="cuda")
    c.run(ws=ws)
    assert not ws[:3 * 1024 * 4].any()                 # (the tickets)
    again.run(ws=ws).check()


@pytest.mark.parametrize("block", [16, 32, 64])
def test_absent_blocks(block):
    c = Case([200, 100, 40], [30, 5, 8], 4, 2, block, F16, seed=7)
    c.table[0, 1], c.table[0, 0], c.table[1, 0] = -1, c.N, 2 ** 31 - 1
    c.table[2, :] = -4                                 # nothing left of this one
    c.run().check()


@pytest.mark.parametrize("dtype,spread", [(F16, 12), (BF16, 12), (BF16, 28)])
@pytest.mark.parametrize("block", [16, 64])
def test_scales_far_apart(dtype, spread, block):
    """V scales 2^(2 spread) apart, keys alike: no weight loses bits to a large scale."""
    c = Case([300, 150], [40, 3], 4, 2, block, dtype, seed=8, spread=spread, gain=2.0 ** -spread)
    c.Kc, c.Ks = rand_cache(c.N, 2, block, 80)
    c.run().check(spread=64 + 2 * spread)


def test_small_scales_that_carry_all_weight():
    """The block with the largest V scale has hardly any weight: outputs are the small ones' to full precision."""
    c = Case([64], [3], 4, 4, 16, F16, seed=9)
    b = c.table[0].long()
    c.Kc[:], c.Ks[:] = 0x38, 1.0                       # keys of ones
    c.Ks[b[0]] = 2.0 ** -3                             # block 0: smaller scores
    c.Vs[b[0]] *= 2.0 ** 20
    x = torch.full_like(c.q, 4.0)
    c.q, c.q_dev = x, x.cuda()
    c.run().check()
    want = pages.prompt_attn(c.q, c.Kc, c.Ks, c.Vc, c.Vs, c.table, c.q_len, c.cu, SM)[0]
    assert float(want.abs().max()) < 100.0             # (the test's own premise)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_scales_of_zero_and_of_no_power_of_two(dtype):
    c = Case([100, 33], [20, 4], 4, 2, 16, dtype, seed=10)
    b = c.table[0].long()
    c.Ks[b[1]], c.Vs[b[2]], c.Vs[b[0]] = 0.0, 0.0, 0.0
    c.Ks[b[3]] *= 1.37
    c.Vs[b[3]] *= 0.77
    c.Vs[c.table[1].long()[:3]] = 0.0                  # request 1: no value at all
    c.run().check()
    assert (c.out[20:24] == 0).all() and (c.lse[20:24].abs() < 100).all()


@pytest.mark.parametrize("sm", [1e-45, 1e-30, 1e-6])
@pytest.mark.parametrize("held,new", [([90, 40], [20, 33]), ([200, 0], [150, 170])])
def test_small_factors_of_scores(held, new, sm):
    """Scores of next to nothing, so that a row is the mean of what it sees: what it does not see stays out."""
    c = Case(held, new, 16, 4, 16, BF16, seed=28)
    b = c.table[0].long()
    c.Ks[b[0]], c.Ks[b[5]], c.Ks[b[6]] = 0.0, 0.0, 2.0 ** -126
    c.run()
    c.out.fill_(7.0), c.lse.fill_(7.0)
    api.minikv_prompt_attn_blk(*c.args[:7], sm, *c.args[8:])
    check_prompt(c.shape, c.q, (c.Kc, c.Ks, c.Vc, c.Vs), c.table, c.q_len, c.cu, c.out, c.lse, sm=sm)


def test_bf16_scales_at_the_ends_of_the_range():
    """V scales 2^200 apart: what lies 2^60 below may count as 0, weights do not change by it."""
    c = Case([64], [4], 2, 2, 16, BF16, seed=11)
    b = c.table[0].long()
    c.Vs[b[0]], c.Vs[b[1]], c.Vs[b[2]] = 2.0 ** -110, 2.0 ** 90, 2.0 ** -20
    c.run()
    want, wlse, live, mean, score = pages.prompt_attn(c.q, c.Kc, c.Ks, c.Vc, c.Vs, c.table, c.q_len, c.cu, SM)
    got = c.out.cpu().double()
    assert ((got - want)[live].abs() <= prompt_tolerance(want, mean, score, 68, 0.0, 400, BF16)[live] + 448 * 2.0 ** 30).all()
    assert ((c.lse.cpu().double() - wlse)[live].abs() <= lse_tolerance(wlse[live], score)).all()


def test_one_token_is_decode_attention():
    """A step of one new token each: the same as minikv_decode_attn_blk within both tolerances."""
    c = Case([700, 3, 0, 64], [1, 1, 1, 1], 8, 2, 32, BF16, seed=12, extra_rows=0).run().check()
    out = torch.zeros(4, 8, 128, dtype=BF16, device="cuda")
    api.minikv_decode_attn_blk(c.shape, c.q_dev, c.cache, c.table.cuda(), c.q_len.cuda(), SM, out)
    assert ((out.float() - c.out.float()).abs() <= 4 * HALF[BF16] * out.float().abs() + 2.0 ** -7).all()


def test_without_lse_and_contiguous():
    c = Case([70, 5], [20, 9], 8, 2, 16, F16, seed=13, fused=False).run()
    first = c.out.clone()
    c.run(lse=False)
    assert torch.equal(c.out, first) and (c.lse == 7.0).all()


def test_fewer_rows_than_q_has():
    c = Case([70, 5], [20, 9], 8, 2, 16, F16, seed=14)
    c.run(T=25)                                        # the second request's rows end behind
    want = Case([70, 5], [20, 9], 8, 2, 16, F16, seed=14).run()
    assert torch.equal(c.out[:20], want.out[:20]) and (c.out[20:] == 7.0).all()


@pytest.mark.parametrize("block", [16, 64])
def test_twice_the_same(block):
    c = Case([3000, 20, 64], [3, 40, 1], 8, 2, block, F16, seed=15).run()
    first, l1 = c.out.clone(), c.lse.clone()
    for _ in range(3):
        api.minikv_prompt_attn_blk(*c.args)
        assert torch.equal(c.out, first) and torch.equal(c.lse, l1)


def test_workspace_taken_by_other_shapes_between():
    big = Case([5000], [60], 8, 1, 16, F16, seed=16)
    ws = torch.zeros(max(api.minikv_prompt_blk_workspace_bytes(big.shape, 4096), 1 << 20), dtype=torch.uint8, device="cuda")
    small = Case([2500, 9], [2, 3], 4, 4, 64, BF16, seed=17)
    for _ in range(2):
        big.run(ws=ws).check()
        small.run(ws=ws).check()


def test_captured_with_lengths_that_change():
    c = Case([900, 40, 0], [3, 30, 7], 8, 2, 16, F16, seed=18).run()
    q_len, cu = c.args[5], c.args[6]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.minikv_prompt_attn_blk(*c.args)
    for lens, rows in (([903, 70, 7], [0, 3, 33, 40]), ([17, 70, 7], [0, 1, 2, 2]), ([903, 5, 3], [0, 0, 5, 8]), ([0, 0, 0], [0, 0, 0, 0])):
        q_len.copy_(ints(lens)), cu.copy_(ints(rows))
        c.out.fill_(7.0), c.lse.fill_(7.0)
        graph.replay()
        got, gl = c.out.clone(), c.lse.clone()
        c.out.fill_(7.0), c.lse.fill_(7.0)
        api.minikv_prompt_attn_blk(*c.args)
        assert torch.equal(got, c.out) and torch.equal(gl, c.lse)
        c.q_len, c.cu = ints(lens), ints(rows)
        c.check()


def test_two_streams():
    a, b = Case([3000, 20], [9, 30], 8, 2, 16, F16, seed=19).run(), Case([100, 2600], [50, 2], 4, 4, 64, BF16, seed=20).run()
    want = a.out.clone(), b.out.clone()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for c in (a, b):
        c.out.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip((a, b), streams):
            api.minikv_prompt_attn_blk(*c.args, stream=s)
    torch.cuda.synchronize()
    live = [int(c.cu[-1]) for c in (a, b)]
    assert torch.equal(a.out[:live[0]], want[0][:live[0]]) and torch.equal(b.out[:live[1]], want[1][:live[1]])


def test_shared_blocks():
    """Requests whose tables name the same blocks."""
    c = Case([64, 64, 64], [5, 6, 7], 4, 2, 16, F16, seed=21)
    c.table[1, :4] = c.table[0, :4]
    c.table[2, :4] = c.table[0, :4]
    c.run().check()


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_one_key_decides(dtype):
    """Scores far apart: the weights are 1 and 0, the output is that value to a rounding."""
    c = Case([200], [30], 4, 2, 32, dtype, seed=22, gain=40.0).run().check()
    assert math.isfinite(float(c.lse[:30].max()))


def test_blocks_far_into_a_large_pool():
    """Blocks whose codes lie beyond 2^32 bytes."""
    Hkv, block, N = 8, 64, 70000                       # 4.6 GB of keys
    K = torch.zeros(N, Hkv, block, 128, dtype=torch.uint8, device="cuda")
    V = torch.zeros_like(K)
    Ks, Vs = torch.zeros(N, Hkv, device="cuda"), torch.zeros(N, Hkv, device="cuda")
    small = rand_cache(3, Hkv, block, 23), rand_cache(3, Hkv, block, 24)
    at = torch.tensor([N - 1, 66001, 5])
    for (big, sc), (c, s) in zip(((K, Ks), (V, Vs)), small):
        big[at], sc[at] = c.cuda(), s.cuda()
    shape = api.make_blk_shape(1, 16, Hkv, 128, block, N, 3, F16)
    cache = api.BlkCache(shape, K=K.view(E4M3), V=V.view(E4M3), Ks=Ks, Vs=Vs)
    q = torch.randn(10, 16, 128, generator=torch.Generator().manual_seed(25)).half()
    out, lse = torch.full((10, 16, 128), 7.0, dtype=F16, device="cuda"), torch.full((10, 16), 7.0, device="cuda")
    ws = torch.zeros(api.minikv_prompt_blk_workspace_bytes(shape, 10), dtype=torch.uint8, device="cuda")
    api.minikv_prompt_attn_blk(shape, 10, q.cuda(), cache, at[None].int().cuda(), ints([180]).cuda(), ints([0, 10]).cuda(), SM, out, lse, ws)
    (Kc, ks), (Vc, vs) = small
    check_prompt(shape, q, (Kc, ks, Vc, vs), torch.arange(3)[None].int(), ints([180]), ints([0, 10]), out, lse)


def test_outputs_between_the_rows_of_queries():
    """Rows of q far apart, out and lse in the room between them: no overlap, no refusal."""
    c = Case([40], [2], 4, 2, 16, F16, seed=38, extra_rows=0).run()
    want, lse = c.out.clone(), c.lse.clone()
    buf = torch.zeros(2, 8 * 1024, dtype=F16, device="cuda")
    q = buf.as_strided((2, 4, 128), (8 * 1024, 128, 1))
    q.copy_(c.q_dev)
    out, sums = buf[0, 512:1536].view(2, 4, 128), buf[0, 1536:1552].view(torch.float32).view(2, 4)
    api.minikv_prompt_attn_blk(*c.args[:2], q, *c.args[3:8], out, sums, c.ws)
    assert torch.equal(out, want) and torch.equal(sums, lse) and torch.equal(q, c.q_dev)


def test_outputs_over_queries_are_refused():
    c = Case([40], [2], 4, 2, 16, F16, seed=39, extra_rows=0).run()
    flat = torch.zeros(4096, dtype=F16, device="cuda")
    q = flat[1024:2048].view(2, 4, 128)
    for out, lse in ((q, c.lse), (flat[:1032][8:].view(2, 4, 128), c.lse), (flat[2040:3064].view(2, 4, 128), c.lse),
                     (c.out, flat[2040:2056].view(torch.float32).view(2, 4)), (c.out, c.out.view(-1)[1008:].view(torch.float32).view(2, 4))):
        before = flat.clone(), c.out.clone()
        with pytest.raises(api.MinikvError):
            api.minikv_prompt_attn_blk(*c.args[:2], q, *c.args[3:8], out, lse, c.ws)
        torch.cuda.synchronize()
        assert torch.equal(flat, before[0]) and torch.equal(c.out, before[1])
