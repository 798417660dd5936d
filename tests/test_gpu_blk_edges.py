"""The paged 8-bit cache at the ends of what its entry points accept: the longest lines of work, scales far apart, every tile counted once,
slot maps and tables with values out of range, shared prefixes."""
import pytest
import torch

from blk_common import HALF, SM
from oracle import blk

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available()
    from paper_2411_18077_amd import api as _api
    return _api


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------------------------------------
# minikv_decode_attn_blk

def test_the_longest_line_of_work(api):
    """As many tiles as a shape may have, fewer than 2048 below 2^31: rounding them up to the waves' share passes 2^31.  All tables name one
    block, keys are zeros, values one power of two per head: weights are equal, sums are whole numbers below 2^29 times a power of
    two (a rounding of 2^-24 for each merge of parts), and one rounding of the output follows."""
    R, Hkv, block = 2, 130, 128
    units = R * Hkv
    tiles = ((1 << 31) - 1) // units - 2               # 64 tokens each; the bound counts two more
    width = tiles // 2
    assert units > 256 and units * (2 * width + 2) < 1 << 31 <= units * (2 * width + 1) + 2047
    shape = api.make_blk_shape(R, Hkv, Hkv, 128, block, 1, width, F16)
    cache = api.BlkCache(shape)
    value = 2.0 ** (torch.arange(Hkv) % 9 - 4)
    cache.V.view(torch.uint8)[0] = blk.encode(value.double()).cuda()[:, None, None]
    cache.Ks.fill_(1.0), cache.Vs.fill_(1.0)
    table, n = torch.zeros(R, width, dtype=torch.int32, device="cuda"), ints(*[width * block] * R)
    out = torch.full((R, Hkv, 128), float("nan"), dtype=F16, device="cuda")
    api.minikv_decode_attn_blk(shape, torch.zeros_like(out), cache, table, n, SM, out)
    want = value[None, :, None].expand(R, Hkv, 128)
    assert bool(((out.cpu() - want).abs() <= want * (HALF[F16] + 64 * 2.0 ** -24)).all())
    assert not bool(cache.workspace[:5120].any())


def coded(x):
    """Codes and power-of-two scales of rows x [blocks][Hkv][block][128] in 64 bits."""
    s = torch.tensor([[blk.scale_for(float(a)) for a in row] for row in x.abs().amax(dim=(2, 3))], dtype=torch.float64)
    return blk.encode(x / torch.where(s > 0, s, 1.0)[:, :, None, None]), s.float()


def largest_product(q, Kc, Ks, Vs, table, lens, sm):
    """Per request and head the largest softmax weight times V scale."""
    R, Hq, _ = q.shape
    Hkv, block = Kc.shape[1:3]
    rep, top = Hq // Hkv, torch.zeros(R, Hq, 1, dtype=torch.float64)
    for r, n in enumerate(lens):
        at = [(int(table[r, i // block]), i % block) for i in range(n)]
        if at:
            b, o = torch.tensor([p[0] for p in at]), torch.tensor([p[1] for p in at])
        for h in range(Hkv if at else 0):
            k = blk.decode_codes(Kc[b, h, o]) * Ks[b, h].double()[:, None]
            p = torch.softmax(q[r, h * rep:(h + 1) * rep].double() @ k.t() * sm, dim=1)
            top[r, h * rep:(h + 1) * rep, 0] = (p * Vs[b, h].double()).amax(dim=1)
    return top


SPREADS = {
    # (V scale, score) of block i of n, r octaves apart
    "large blocks without weight": lambda i, n, r: (r, -300.0) if i % 3 == 1 else (0, 0.0),
    "large blocks of little weight": lambda i, n, r: (r, -r * 0.6931) if i % 3 == 1 else (0, 0.0),
    "large and small blocks of the same weight": lambda i, n, r: (0, 0.0) if i % 3 == 1 else (-r, 0.0),
    "zeros with the weight": lambda i, n, r: (None, min(r, 40) * 0.6931) if i % 4 == 0 else (0, 0.0),
    "ever larger": lambda i, n, r: (r * (i + 1) / n, -r * (i + 1) / n * 0.6931),
    "ever smaller": lambda i, n, r: (r * (n - i) / n, -r * (n - i) / n * 0.6931),
}


@pytest.mark.parametrize("kind", SPREADS)
@pytest.mark.parametrize("r", [13, 18, 30, 90])
@pytest.mark.parametrize("Hq,Hkv,block,lens,dtype", [
    (4, 1, 16, [330], F16), (8, 2, 32, [0, 70, 1000], BF16), (3, 1, 64, [5000, 200], F16), (4, 4, 128, [700, 129, 64], BF16),
    (2, 1, 16, [60 + i % 40 for i in range(280)] + [4000], BF16), (1, 1, 64, [450] * 258, F16),
])
def test_scales_far_apart(api, kind, r, Hq, Hkv, block, lens, dtype):
    """The V scales of a request's blocks are r octaves apart, with or without weight to go with them.  Per output: each weight's product
    with its scale is rounded to fp16's 11 bits (half a step 2^-11), or where it is below fp16's normal numbers by at most 2^-28 of the largest
    such product of the row (see the kernel), times a code of at most 448; scores, sums and the output's own rounding as
    in attn_tolerance, here with every token's addition counted."""
    g = torch.Generator().manual_seed(r + block)
    need = [-(-n // block) for n in lens]
    N, width = sum(need) + 1, max(need)
    K, V = (torch.randn(N, Hkv, block, 128, generator=g, dtype=torch.float64) for _ in range(2))
    q = torch.randn(len(lens), Hq, 128, generator=g)
    q[:, :, 0] = 16.0
    q = q.to(dtype)
    K[..., 0] = 0.0
    order, table, at = torch.randperm(N, generator=g), torch.full((len(lens), width), -7, dtype=torch.int32), 0
    for row, n in zip(table, need):
        for i in range(n):
            b = int(order[at])
            row[i], at = b, at + 1
            octaves, score = SPREADS[kind](i, n, r)
            V[b] *= 0.0 if octaves is None else 2.0 ** octaves
            K[b, :, :, 0] = score / (16.0 * SM)
    (Kc, Ks), (Vc, Vs) = coded(K), coded(V)
    shape = api.make_blk_shape(len(lens), Hq, Hkv, 128, block, N, width, dtype)
    cache = api.BlkCache(shape, K=Kc.cuda().view(E4M3), V=Vc.cuda().view(E4M3), Ks=Ks.cuda(), Vs=Vs.cuda())
    out = torch.full((len(lens), Hq, 128), float("nan"), dtype=dtype, device="cuda")
    api.minikv_decode_attn_blk(shape, q.cuda(), cache, table.cuda(), ints(*lens), SM, out)
    want, mean, score = blk.decode_attn(q, Kc, Ks, Vc, Vs, table, lens, SM)
    n = torch.tensor(lens)[:, None, None]
    rel = 2.0 ** -11 + 2 * (136 * 2.0 ** -24 * score * 1.01) + (64 + n) * 2.0 ** -24
    tol = mean * rel + n * 2.0 ** -28 * 448 * largest_product(q, Kc, Ks, Vs, table, lens, SM) + want.abs() * HALF[dtype] * 1.001 + \
        (2.0 ** -25 if dtype is F16 else 2.0 ** -130)
    got = out.cpu().double()
    # (fp16 rounds what is 65520 or more to infinity: the keys' codes miss the intended scores by up to 2^-4 of them, and 200 tokens of
    # 90 octaves then give outputs of 1.9e7, 3.1e8)
    err = (got - want).abs().where((got.abs() != float("inf")) | (want * got.sign() + tol < 65520.0), 0.0)
    assert bool((err <= tol).all()), (float(err.max()), float((err / tol).max()))


# ---------------------------------------------------------------------------------------------------------
# kv_assign_blk

@pytest.mark.parametrize("n_new,ok", [((2 ** 31 - 1, 1), (False, False)), ((2 ** 31 - 1, 0, 1), (False, False, False)), ((2 ** 31 - 2, 1), (False, True)),
                                      ((2 ** 31 - 1, 2 ** 31 - 1, 20), (False, False, False))])
def test_rows_behind_the_largest_slot_map(api, n_new, ok):
    """2^31 - 1 slots: a request whose rows begin behind them is refused, although what cu holds of the sum ends at 2^31 - 1."""
    R, n = len(n_new), 2 ** 31 - 1
    shape = api.make_blk_shape(R, 1, 1, 128, 16, 40, 8, F16)
    table, ring = torch.full((R, 8), -1, dtype=torch.int32, device="cuda"), torch.arange(40, dtype=torch.int32, device="cuda")
    nxt, state, cu, slots = ints(*[-9] * R), ints(-9, -9), ints(*[-9] * (R + 1)), torch.zeros(n, dtype=torch.int32, device="cuda")
    api.kv_assign_blk(shape, ints(*[0] * R), ints(*n_new), table, ring, ints(0, 40), nxt, state, cu, slots)
    at = [sum(n_new[:i]) for i in range(R + 1)]
    want = [k if o else 0 for k, o in zip(n_new, ok)]
    assert cu.tolist() == [min(a, n) for a in at] and nxt.tolist() == want
    assert state.tolist() == [sum(ok), 40 - sum(ok)]
    for r, o in enumerate(ok):
        assert table[r].tolist() == [0 if o else -1] + [-1] * 7
        if o:
            assert slots[at[r]:at[r] + n_new[r]].tolist() == list(range(n_new[r]))
            slots[at[r]:at[r] + n_new[r]] = -1
    assert int(slots.max()) == -1 and int(slots.min()) == -1


@pytest.mark.parametrize("new", [3, 9])
def test_blocks_outside_the_pool_have_no_slots_in_it(api, new):
    """A table or a ring that names a block outside the pool: its rows' slots lie outside it too, whatever the product with the block's size
    wraps to, in the form for few rows each and in the other one."""
    block = 16
    bad = [1 << 28, -(1 << 28), -1, 5, 2 ** 31 - 1]
    q_len, n_new = [block - 2] * 5 + [0, 0, 0], [new] * 5 + [2, 2, 2]
    table = [[b, -1] for b in bad] + [[-1, -1]] * 3
    ring = [0, 1 << 28, 1, -7, 2, 3, 4, 1 << 30, 5, 6]                # (ids outside the pool among the free ones)
    got = dict(table=ints(*sum(table, [])), ring=ints(*ring), q_len=ints(*[0] * 8), state=ints(0, 0), cu=ints(*[0] * 9), slots=ints(*[7] * 60))
    shape = api.make_blk_shape(8, 1, 1, 128, block, 10, 2, F16)
    api.kv_assign_blk(shape, ints(*q_len), ints(*n_new), got["table"], got["ring"], ints(0, 10), got["q_len"], got["state"], got["cu"], got["slots"])
    want = blk.assign(q_len, n_new, table, ring, [0, 10], block, 60)
    assert got["table"].view(8, 2).tolist() == want["table"] and got["slots"].tolist() == want["slots"]
    assert all(got[k].tolist() == want[k] for k in ("ring", "q_len", "state", "cu"))
    assert got["slots"][:2].tolist() == [-1, -1] and got["slots"][3 * new:3 * new + 2].tolist() == [94, 95]
    free = [b for b in ring if 0 <= b < 10] + [5]
    assert all(s < 0 or s >= 160 or s // 16 in free for s in got["slots"].tolist())


def test_a_shared_prefix_through_the_end_of_its_requests(api):
    """Two requests name the same first two blocks.  Each is ended by the program (length 0, own blocks behind the last free one), the shared
    blocks with the second: the other's attention does not change while new requests take what is free, and no block is lost or doubled."""
    R, block, width, N, Hkv = 3, 16, 6, 12, 2
    shape = api.make_blk_shape(R, 4, Hkv, 128, block, N, width, F16)
    cache = api.BlkCache(shape)
    table, ring, cu, slots = ints(*[-1] * (R * width)).view(R, width), ints(*range(N)), ints(*[0] * (R + 1)), ints(*[0] * 80)
    s = dict(q=ints(0, 0, 0), q2=ints(0, 0, 0), state=ints(0, N), state2=ints(0, 0))
    gen = torch.Generator().manual_seed(3)

    def step(*n_new):
        api.kv_assign_blk(shape, s["q"], ints(*n_new), table, ring, s["state"], s["q2"], s["state2"], cu, slots)
        s.update(q=s["q2"], q2=s["q"], state=s["state2"], state2=s["state"])
        x = torch.randn(sum(max(n, 0) for n in n_new), Hkv, 128, generator=gen).half().cuda()
        api.kv_quantize_blk(shape, x, -x, slots[:len(x)], cache)

    def attend():
        out = torch.zeros(R, 4, 128, dtype=F16, device="cuda")
        api.minikv_decode_attn_blk(shape, q, cache, table, s["q"], SM, out)
        return out

    def end(r, blocks):                                # what the header tells a program to do
        for b in blocks:
            head, n_free = s["state"].tolist()
            ring[(head + n_free) % N] = b
            s["state"][1] += 1
        s["q"][r] = 0

    q = torch.randn(R, 4, 128, generator=gen).half().cuda()
    step(40, 0, 0)                                     # blocks 0, 1, 2
    table[1, :2], s["q"][1] = table[0, :2], 32         # the second one begins with the first one's 32 tokens
    step(1, 20, 0)
    assert table[0, :3].tolist() == [0, 1, 2] and table[1, :4].tolist() == [0, 1, 3, 4] and s["q"].tolist() == [41, 52, 0]
    before = attend()
    end(0, [2])
    for n in (60, 1):
        step(n, 0, 0)
        assert torch.equal(attend()[1], before[1])
    assert not {0, 1, 3, 4} & set(table[0, :4].tolist())
    step(0, 0, 30)
    assert torch.equal(attend()[1], before[1]) and not {0, 1, 3, 4} & set(table[2, :2].tolist())
    end(1, [0, 1, 3, 4])
    assert not bool(attend()[1].any())
    step(-1, 0, -1)
    head, n_free = s["state"].tolist()
    assert n_free == N and sorted(ring.tolist()) == list(range(N)) and s["q"].tolist() == [0, 0, 0]


def test_a_new_token_sees_itself(api):
    """The order of a step: assignment, filing, attention with the lengths after the step.  A request's first token gets its own value, the
    second one, whose score is far larger, as good as its own again."""
    shape = api.make_blk_shape(2, 2, 1, 128, 16, 4, 2, BF16)
    cache = api.BlkCache(shape)
    cache.K.view(torch.uint8).fill_(0x7f), cache.V.view(torch.uint8).fill_(0x7f)      # what a last use left: NaN
    table, ring, cu, slots = ints(-1, -1, -1, -1), ints(0, 1, 2, 3), ints(0, 0, 0), ints(0, 0)
    q_len, nxt, state, s_nxt = ints(0, 0), ints(0, 0), ints(0, 4), ints(0, 0)
    q, out = torch.ones(2, 2, 128, dtype=BF16, device="cuda"), torch.zeros(2, 2, 128, dtype=BF16, device="cuda")
    for k in range(3):
        api.kv_assign_blk(shape, q_len, ints(1, 1), table, ring, state, nxt, s_nxt, cu, slots)
        K = torch.full((2, 1, 128), 8.0 * k, dtype=BF16, device="cuda")
        V = torch.full((2, 1, 128), 3.0 + k, dtype=BF16, device="cuda")              # (codes hold it exactly)
        api.kv_quantize_blk(shape, K, V, slots, cache)
        api.minikv_decode_attn_blk(shape, q, cache, table, nxt, SM, out)
        assert bool((out == 3.0 + k).all())                                          # (the others weigh e^-90)
        q_len, nxt, state, s_nxt = nxt, q_len, s_nxt, state


# ---------------------------------------------------------------------------------------------------------
# kv_quantize_blk

def file_both(api, x, codes, scales, slots, dtype):
    """Files x as K and -x as V into copies of one pool; checks both against the definition."""
    N, Hkv, block, _ = codes.shape
    shape = api.make_blk_shape(1, Hkv, Hkv, 128, block, N, 1, dtype)
    t = [codes.clone().cuda(), scales.clone().cuda(), codes.clone().cuda(), scales.clone().cuda()]
    cache = api.BlkCache(shape, K=t[0].view(E4M3), V=t[2].view(E4M3), Ks=t[1], Vs=t[3])
    api.kv_quantize_blk(shape, x.cuda(), -x.cuda(), ints(*slots), cache)
    for y, c, s in ((x, t[0], t[1]), (-x, t[2], t[3])):
        wc, ws = blk.file_rows(y, codes, scales, torch.tensor(slots))
        assert torch.equal(s.cpu().double(), ws)
        assert torch.equal(blk.decode_codes(c.cpu()), blk.decode_codes(wc))


# halfway between neighbouring codes, ordinary and subnormal ones
TIES = [(17 + 2 * i) / 16 for i in range(8)] + [2.0 ** -10 * k for k in (1, 3, 5, 13)]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("block", [16, 128])
def test_filing_behind_a_scale_that_is_no_power_of_two(api, dtype, block):
    """A block's scale from elsewhere: rows next to it are x / s rounded once.  The scales are those nearest to x / tie, so that the
    quotient in 32 bits lies on the tie where the real one does not."""
    g = torch.Generator().manual_seed(block)
    for i, t in enumerate(TIES):
        x = (1 + torch.rand(1, 8, 128, generator=g)).to(dtype)
        s = (x[0, :, 0].double() / t).float()          # one x of each head decides; the others are multiples of it
        x = (x[:, :, :1].float() * 2.0 ** -(torch.arange(128) % 9)).to(dtype).repeat(5, 1, 1)
        scales = torch.stack([s, s * 2.0 ** -100 if dtype is BF16 else s * 0.37]) + 0.0
        if dtype is BF16:
            x[3:] = (x[3:].float() * 2.0 ** -100).to(dtype)
        codes = torch.randint(0, 127, (2, 8, block, 128), generator=g).to(torch.uint8)
        file_both(api, x, codes, scales, [5, 6, 7, block + 3, block + 4], dtype)


def test_scales_far_below_one_are_divided_by_exactly(api):
    """bf16 rows of 2^-118 behind scales as small: the remainder of such a quotient is below binary32's numbers."""
    g = torch.Generator().manual_seed(2)
    x = ((1 + torch.rand(3, 4, 128, generator=g)) * 2.0 ** -118).to(BF16)
    for t in TIES[:8]:
        scales = (x[0, :, 0].double() / t).float()[None]
        file_both(api, x, torch.zeros(1, 4, 16, 128, dtype=torch.uint8), scales, [3, 4, 5], BF16)


@pytest.mark.parametrize("block", [32, 128])
def test_a_scale_that_is_no_power_of_two_grows(api, block):
    """A larger row: the block's other rows are code * old / s, rounded once.  The old scales are those nearest to tie / code."""
    codes = torch.arange(block * 128).reshape(1, 1, block, 128).remainder(127).to(torch.uint8)
    for code in (9.0, 11.0, 13.0, 15.0):
        old = torch.tensor([[t / code * 2.0 ** 3 for t in TIES[:8]]], dtype=torch.float64).float()
        x = torch.full((1, 8, 128), 448.0 * 16).to(F16)
        file_both(api, x, codes.expand(1, 8, block, 128).contiguous(), old, [1], F16)


@pytest.mark.parametrize("R", [1, 5, 1024, 1025, 2048, 2049, 3500, 8192])
@pytest.mark.parametrize("new", [0, 1, 2, 3, 4])
def test_assignment_on_both_sides_of_its_rule(api, R, new):
    """Threads with one to eight requests, of no more rows each than they write themselves and of one more: the definition's numbers."""
    block, width, N = 16, 3, 2 * R + 7
    q_len = [(7 * r) % 33 for r in range(R)]
    n_new = [-1 if r % 11 == 3 else new if r % 5 else min(new, 1) for r in range(R)]
    ids = iter(torch.randperm(N, generator=torch.Generator().manual_seed(R)).tolist())
    table = [[next(ids) if 16 * b < n else -1 for b in range(width)] for n in q_len]
    ring = list(ids)
    n_free = min(len(ring), R // 3 + 1)
    ring += [-1] * (N - len(ring))
    n_slots = sum(max(n, 0) for n in n_new) + 3
    want = blk.assign(q_len, n_new, table, ring, [0, n_free], block, n_slots)
    t, g, q, s = ints(*sum(table, [])), ints(*ring), ints(*[-9] * R), ints(-9, -9)
    cu, slots = ints(*[-9] * (R + 1)), ints(*[-9] * n_slots)
    shape = api.make_blk_shape(R, 1, 1, 128, block, N, width, F16)
    api.kv_assign_blk(shape, ints(*q_len), ints(*n_new), t, g, ints(0, n_free), q, s, cu, slots)
    got = dict(table=t.view(R, width).tolist(), ring=g.tolist(), q_len=q.tolist(), state=s.tolist(), cu=cu.tolist(), slots=slots.tolist())
    for k in want:
        assert got[k] == want[k], k
