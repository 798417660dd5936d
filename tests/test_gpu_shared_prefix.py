"""The operators together, as a program uses them: prompts, forks behind a shared prefix, a step of several new tokens, the end of requests that
share blocks, the pool compacted, decoding on.  At every step what the cache holds for a request is compared with the same tokens filed
alone, and attention with its definition."""
import pytest
import torch

from blk_common import SM, rand_cache  # noqa: F401
from pages_common import check_prompt, ints
from oracle import blk, pages
from paper_2411_18077_amd import api

pytestmark = pytest.mark.gpu


class Program:
    """Two layers, R places in the batch, all state on the device."""

    def __init__(self, R, Hq, Hkv, block, N, width, dtype):
        self.shape = api.make_blk_shape(R, Hq, Hkv, 128, block, N, width, dtype)
        self.layers = [api.BlkCache(self.shape) for _ in range(2)]
        self.caches = api.BlkCaches(self.shape, self.layers)
        z = lambda *n: torch.zeros(*n, dtype=torch.int32, device="cuda")  # noqa: E731
        self.q_len, self.q_len_next, self.table, self.table_next = z(R), z(R), z(R, width), z(R, width)
        self.ring, self.state, self.state_next = torch.arange(N, dtype=torch.int32, device="cuda"), ints([0, N]).cuda(), z(2)
        self.cu, self.src, self.dst, self.z = z(R + 1), z(R), z(R), z
        self.ws = torch.zeros(api.kv_free_workspace_bytes(self.shape), dtype=torch.uint8, device="cuda")
        g = torch.Generator().manual_seed(1)
        self.w = [(1 + 0.2 * torch.randn(128, generator=g)).to(dtype).cuda() for _ in range(2)]
        self.inv = (10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)).float().cuda()
        self.dtype, self.R, self.Hq, self.Hkv, self.block, self.N = dtype, R, Hq, Hkv, block, N
        self.said = [[] for _ in range(R)]             # the tokens of every request: numbers that stand for their rows

    def rows(self, tokens, layer):
        """Rows of the fused projection of tokens (a token's are the same wherever it stands)."""
        g = torch.Generator().manual_seed(7 + layer)
        bank = torch.randn(400, self.Hq + 2 * self.Hkv, 128, generator=g)
        return bank[torch.tensor(tokens, dtype=torch.long) % 400].to(self.dtype)

    def step(self, new):
        """New tokens (a list each) filed, and attended from: both layers."""
        T = sum(len(n) for n in new) + 2
        slots, n_new = self.z(T), ints([len(n) for n in new]).cuda()
        api.kv_assign_blk(self.shape, self.q_len, n_new, self.table, self.ring, self.state, self.q_len_next, self.state_next, self.cu, slots)
        t = torch.arange(T, device="cuda")             # positions, from what lies on the device
        r = torch.searchsorted(self.cu[1:].contiguous(), t.int(), right=True)
        at = r.clamp(max=self.R - 1)
        pos = torch.where(r < self.R, self.q_len[at] + t - self.cu[at], -1).int()
        tokens = [x for n in new for x in n] + [0, 0]
        for layer, cache in enumerate(self.layers):
            qkv = self.rows(tokens, layer).cuda()
            q, k, v = qkv[:, :self.Hq], qkv[:, self.Hq:self.Hq + self.Hkv], qkv[:, self.Hq + self.Hkv:]
            api.minikv_norm_rope(self.Hq, self.Hkv, T, q, k, self.w[0], self.w[1], 1e-6, self.inv, 128, False, pos, q, k)
            api.kv_quantize_blk(self.shape, k, v, slots, cache)
            out, lse = torch.full((T, self.Hq, 128), 7.0, dtype=self.dtype, device="cuda"), torch.full((T, self.Hq), 7.0, device="cuda")
            ws = torch.zeros(api.minikv_prompt_blk_workspace_bytes(self.shape, T), dtype=torch.uint8, device="cuda")
            api.minikv_prompt_attn_blk(self.shape, T, q, cache, self.table, self.q_len_next, self.cu, SM, out, lse, ws)
            raw = [x.view(torch.uint8).cpu() if x.element_size() == 1 else x.cpu() for x in (cache.K, cache.Ks, cache.V, cache.Vs)]
            check_prompt(self.shape, q, raw, self.table.cpu(), self.q_len_next.cpu(), self.cu.cpu(), out, lse)
        self.q_len, self.q_len_next, self.state, self.state_next = self.q_len_next, self.q_len, self.state_next, self.state
        for said, n in zip(self.said, new):
            said += n

    def fork(self, parent, keep):
        api.kv_fork_blk(self.shape, self.q_len, ints(parent).cuda(), ints(keep).cuda(), self.table, self.ring, self.state, self.q_len_next,
                        self.table_next, self.state_next, self.src, self.dst)
        api.kv_copy_blk(self.shape, self.caches, self.src, self.dst)
        self.q_len, self.q_len_next, self.state, self.state_next = self.q_len_next, self.q_len, self.state_next, self.state
        self.table, self.table_next = self.table_next, self.table
        self.said = [list(self.said[p][:k]) if p >= 0 else [] for p, k in zip(parent, keep)]

    def free(self):
        api.kv_free_blk(self.shape, self.q_len, self.table, self.ring, self.state, self.ws)

    def compact(self):
        src, dst = self.z(self.N // 2), self.z(self.N // 2)
        api.kv_compact_blk(self.shape, self.q_len, self.table, self.table_next, self.ring, self.state, src, dst, self.ws)
        api.kv_copy_blk(self.shape, self.caches, src, dst)
        self.table, self.table_next = self.table_next, self.table
        return src

    def check(self):
        """Each request's filed rows stand for its tokens' (turned at their places) to the codes' rounding, no block lost and none held twice."""
        q_len, table = self.q_len.tolist(), self.table.tolist()
        assert q_len == [len(s) for s in self.said]
        head, n = self.state.tolist()
        free = [self.ring.tolist()[(head + i) % self.N] for i in range(n)]
        used = pages.named(q_len, table, self.N, self.block)
        assert len(set(free)) == n and not used & set(free)
        writable = [row[m // self.block] for m, row in zip(q_len, table) if m % self.block]
        assert all(sum(b in row[:-(-m // self.block)] for m, row in zip(q_len, table)) == 1 for b in writable)
        for layer, cache in enumerate(self.layers):
            K, V = (blk.decode_codes(c.view(torch.uint8).cpu()) * s.cpu().double()[..., None, None] for c, s in ((cache.K, cache.Ks), (cache.V, cache.Vs)))
            for said, row in zip(self.said, table):
                if not said:
                    continue
                x = self.rows(said, layer)
                k, _ = pages.norm_rope(x[:, self.Hq:self.Hq + self.Hkv], self.w[1].cpu(), 1e-6, self.inv.cpu(), 128, False, torch.arange(len(said)))
                v = x[:, self.Hq + self.Hkv:].double()
                b, o = torch.tensor(row)[torch.arange(len(said)) // self.block], torch.arange(len(said)) % self.block
                for got, want in ((K[b, :, o], k), (V[b, :, o], v)):   # e4m3: 2^-4 of the value, or a subnormal's half step under a scale of at most amax / 224
                    assert ((got - want).abs() <= want.abs() * (2.0 ** -4 + 2.0 ** -7) + 2.0 ** -10 * 16.0 / 224 + 2.0 ** -9).all()
        return used, free


@pytest.mark.parametrize("dtype,block", [(torch.float16, 16), (torch.bfloat16, 32)])
def test_a_program(dtype, block):
    p = Program(6, 6, 2, block, 60, 12, dtype)
    tokens = iter(range(10 ** 6))
    some = lambda n: [next(tokens) for _ in range(n)]  # noqa: E731
    p.step([some(100), some(37), [], [], [], []])
    p.check()
    p.fork([0, 1, 0, 0, 1, -1], [100, 37, 100, 64, 37, 0])             # two answers to prompt 0, a third behind its first 64 tokens, one more to prompt 1
    p.check()
    p.step([some(1), some(1), some(30), some(5), some(2), some(50)])   # decoding, parts of prompts, drafted tokens and a new prompt in one step
    p.check()
    p.fork([0, 1, 2, 3, 4, 5], [101, 36, 130, 66, 38, 50])             # drafted tokens taken back (all but 3's third, 4's second)
    p.check()
    p.step([some(1)] * 0 + [some(1), some(2), [], some(1), some(1), some(3)])
    p.check()
    p.fork([-1, 1, 2, 3, -1, 5], [0, 38, 130, 67, 0, 53])              # two requests over; their blocks are the others' too
    before, _ = p.check()
    p.free()
    used, free = p.check()
    assert len(used) + len(free) == p.N and used == before
    moved = p.compact()
    used, free = p.check()
    assert used == set(range(len(used))) and int((moved >= 0).sum()) > 0
    p.step([some(40), some(1), some(1), some(1), some(20), some(1)])
    p.check()
