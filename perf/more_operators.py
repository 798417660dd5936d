"""The operators of requests that share a prefix in the paged 8-bit cache, as they are timed and compared.

A program that lets requests share what they have in common does, beside a step's filing and attention: give new requests the
blocks of an old one (`kv_fork_blk`, and `kv_copy_blk` for the block that is only partly filled), prepare the new tokens' queries and
keys (`minikv_norm_rope`), attend from several new tokens of a request over its filed ones (`minikv_prompt_attn_blk`), take the blocks
back that no request names any more (`kv_free_blk`), and now and then move the used blocks to the front of the pool
(`kv_compact_blk`, and `kv_copy_blk` again).

Every kind has its plain form here: elementary torch operations in 32 bits (angles in 64), vectorised over requests and heads.
Requests are padded to the longest one where the plain form needs a rectangle.
"""
import math
import random

import torch

own = False

D = 128
DEV = "cuda"
SM = 1.0 / math.sqrt(D)
EPS = 1e-6
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn


def listed():
    return [
        # the queries and keys of a decoding step of 64 requests, whole heads rotated by halves: all latency
        dict(name="norm_step_64", kind="norm", T=64, Hq=32, Hkv=8, rot=128, adjacent=False, weights=True, far=8192, dtype="bf16", mix=1),
        # an odd number of prompt tokens, multi-head, half of each head rotated by adjacent pairs, no norm
        dict(name="norm_odd_777", kind="norm", T=777, Hq=8, Hkv=8, rot=64, adjacent=True, weights=False, far=1000, dtype="f16", mix=2),
        # prompt tokens at far positions, the largest call of this kind
        dict(name="norm_prompts_32k", kind="norm", T=32768, Hq=32, Hkv=8, rot=128, adjacent=False, weights=True, far=1000000, dtype="bf16", mix=3),
        # four drafted tokens of one short conversation: the smallest attention call, all latency
        dict(name="attend_draft_1k", kind="attend", R=1, Hq=8, Hkv=8, block=32, lo=1000, hi=1000, new_lo=4, new_hi=4, one=0, dtype="f16", mix=4),
        # a step of decoding requests and parts of prompts together, lengths very different, three heads to a KV head
        dict(name="attend_mixed_24", kind="attend", R=24, Hq=24, Hkv=8, block=16, lo=0, hi=6000, new_lo=20, new_hi=256, one=18, dtype="f16", mix=5),
        # eight drafted tokens each of 16 requests of a long context: bound by reading the cache
        dict(name="attend_draft_16x16k", kind="attend", R=16, Hq=32, Hkv=8, block=64, lo=16384, hi=16384, new_lo=8, new_hi=8, one=0, dtype="bf16", mix=6),
        # the next turn of a long conversation: the largest call
        dict(name="attend_turn_32k", kind="attend", R=1, Hq=32, Hkv=8, block=64, lo=32768, hi=32768, new_lo=2048, new_hi=2048, one=0, dtype="bf16", mix=7),
        # a step of a beam search, eight beams to a request: most beams take another's blocks, one cache
        dict(name="fork_beams_64", kind="fork", R=64, group=8, Hkv=8, block=16, lo=10, hi=2000, layers=1, mix=8),
        # one long prefix shared by 256 requests, the partly filled block copied in every layer
        dict(name="fork_prefix_256", kind="fork", R=256, group=256, Hkv=8, block=64, lo=8000, hi=8191, layers=12, mix=9),
        # blocks of 256 requests after a third of them ended, prefixes shared, a pool of 60000 blocks
        dict(name="free_60k", kind="free", R=256, block=16, lo=1, hi=6000, pool=60000, shared=0.3, mix=10),
        # a small pool of few requests
        dict(name="free_300", kind="free", R=7, block=32, lo=0, hi=1500, pool=301, shared=0.5, mix=11),
        # the used blocks of a half-empty pool moved to its front, in every layer's cache
        dict(name="compact_8k", kind="compact", R=48, Hkv=8, block=16, lo=1, hi=4000, pool=8192, shared=0.2, layers=6, mix=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm", "attend", "attend", "attend", "attend", "fork", "fork", "free", "compact", "compact"])
    mix = rng.randrange(1 << 30)
    block = rng.choice([16, 32, 64, 64, 128])
    dtype = rng.choice(["f16", "bf16"])
    Hq, Hkv = rng.choice([(8, 8), (32, 32), (32, 8), (32, 8), (16, 8), (32, 4), (12, 2), (24, 8), (10, 2)])
    if kind == "norm":
        return dict(kind=kind, T=min(_log_int(rng, 1, 32768), 1300000 // (Hq + Hkv)), Hq=Hq, Hkv=Hkv, rot=rng.choice([128, 128, 64, 32, 96, 16]),
                    adjacent=rng.random() < 0.4, weights=rng.random() < 0.7, far=_log_int(rng, 100, 2000000), dtype=dtype, mix=mix)
    if kind == "attend":
        R = _log_int(rng, 1, 64)
        new_hi = _log_int(rng, 2, min(2048, 65536 // R))
        hi = max(min(_log_int(rng, 16, 32768), 1_500_000_000 // (R * Hq * new_hi) - new_hi, 3_000_000 // (R * Hkv)), 1)
        return dict(kind=kind, R=R, Hq=Hq, Hkv=Hkv, block=block, lo=rng.choice([0, 1, hi]), hi=hi, new_lo=rng.choice([1, new_hi]), new_hi=new_hi,
                    one=rng.randrange(R) if rng.random() < 0.5 else 0, dtype=dtype, mix=mix)
    if kind == "fork":
        R = _log_int(rng, 2, 256)
        Hkv = rng.choice([2, 4, 8])
        hi = _log_int(rng, 16, 8191)
        return dict(kind=kind, R=R, group=rng.choice([2, 4, 8, R]), Hkv=Hkv, block=block, lo=rng.choice([1, hi]), hi=hi,
                    layers=max(min(_log_int(rng, 1, 12), 4_000_000 // (R * Hkv * max(block, hi // 8))), 1), mix=mix)
    R = _log_int(rng, 1, 256)
    hi = _log_int(rng, 16, 8000)
    pool = R * (hi // block + 1) + _log_int(rng, 1, 4000)
    if kind == "free":
        return dict(kind=kind, R=R, block=block, lo=0, hi=hi, pool=pool, shared=rng.choice([0.0, 0.3, 0.7]), mix=mix)
    R = min(R, 64)
    hi = min(hi, 400_000 // R)
    pool = R * (hi // block + 1) + _log_int(rng, 1, 4_000_000 // (8 * block))
    Hkv = rng.choice([2, 4, 8])
    return dict(kind=kind, R=R, Hkv=Hkv, block=block, lo=1, hi=hi, pool=pool, shared=rng.choice([0.0, 0.3]),
                layers=max(min(_log_int(rng, 1, 8), 6_000_000 // (pool * Hkv * block)), 1), mix=mix)


# ---------------------------------------------------------------------------------------------------------
# lengths: they belong to the case (work() needs them), the contents to the seed

def _spread(rng, n, lo, hi):
    """n lengths between lo and hi, spread over their logarithm."""
    return [min(max(int(math.exp(rng.uniform(math.log(lo + 1), math.log(hi + 2)))) - 1, lo), hi) for _ in range(n)]


def _plan(case):
    """attend: tokens held before, new tokens.  fork: tokens held, parent, tokens kept.  free, compact: tokens held, tokens shared with request 0."""
    rng = random.Random(case["mix"])
    R = case["R"]
    held = [case["hi"]] * R if case["lo"] == case["hi"] else _spread(rng, R, case["lo"], case["hi"])
    if case["kind"] == "attend":
        new = [case["new_hi"]] * R if case["new_lo"] == case["new_hi"] else _spread(rng, R, case["new_lo"], case["new_hi"])
        for r in rng.sample(range(R), case["one"]):        # decoding requests among them
            new[r] = 1
        if R > 6:                                          # and a place of the batch without a request
            held[rng.randrange(R)] = 0
            new[rng.randrange(R)] = 0
        return held, new
    if case["kind"] == "fork":
        group = case["group"]
        parent, keep = [], []
        for r in range(R):
            first = r // group * group
            if group == R:                                 # everybody behind request 0
                p = 0
            else:
                p = min(first + rng.choice([0, 0, 1, rng.randrange(group)]), R - 1)
            p = -1 if rng.random() < 0.03 and R > 8 and r else p
            parent.append(p)
            keep.append(held[p] if rng.random() < 0.8 else rng.randint(0, held[p]))
        return held, parent, keep
    block = case["block"]
    held = [0 if rng.random() < 0.33 and R > 2 and r else h for r, h in enumerate(held)]
    common = held[0] // block * block
    shared = [min(h // block * block, common) if r and rng.random() < case["shared"] else 0 for r, h in enumerate(held)]
    return held, shared


def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1009 + salt)
    return g


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _tables(held, shared, block, width, pool, gen):
    """Block tables of requests that hold `held` tokens, the first `shared` of them in request 0's blocks, and the order of the pool's blocks they
    were taken from, with how many of it were."""
    need = [-(-h // block) - s // block for h, s in zip(held, shared)]
    total = sum(need)
    pool = max(pool, total + 1)
    order = torch.randperm(pool, generator=gen, device=DEV).to(torch.int32)
    count, common = _ints(need).long(), _ints([s // block for s in shared]).long()
    first = count.cumsum(0) - count
    cols = torch.arange(width, device=DEV)
    mine = order[(first[:, None] + cols - common[:, None]).clamp(0, pool - 1)]
    table = torch.where(cols < common[:, None], order[cols.clamp(max=pool - 1)], mine)
    return torch.where(cols < (common + count)[:, None], table, -1).to(torch.int32).contiguous(), order, total


def _pow2_scale(amax):
    """The smallest power of two s with amax <= 448 s (e4m3's largest value); 0 for amax 0."""
    m, e = torch.frexp(amax)                       # amax = m 2^e, 0.5 <= m < 1; 448 = 0.875 * 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-126)
    return torch.where(amax > 0, ((e + 127) << 23).view(torch.float32), torch.zeros_like(amax))


def _cache(n_blocks, Hkv, block, gen, far):
    """Codes and scales of a pool of filed rows, N(0,1) values; `far`: a few key channels eight times the others."""
    codes = torch.empty(n_blocks, Hkv, block, D, dtype=E4M3, device=DEV)
    scales = torch.empty(n_blocks, Hkv, device=DEV)
    mult = torch.ones(Hkv, 1, D, device=DEV)
    if far:
        mult[:, :, ::43] = 8.0
    step = max(1, (1 << 25) // (Hkv * block * D))
    for i in range(0, n_blocks, step):
        x = torch.randn(min(step, n_blocks - i), Hkv, block, D, generator=gen, device=DEV) * mult
        s = _pow2_scale(x.abs().amax(dim=(2, 3)))
        scales[i:i + step] = s
        codes[i:i + step] = (x / s[:, :, None, None]).to(E4M3)
    return codes, scales


def _prepare_norm(case, gen):
    T, Hq, Hkv, rot = case["T"], case["Hq"], case["Hkv"], case["rot"]
    dtype = TYPES[case["dtype"]]
    x = torch.randn(T, Hq + 2 * Hkv, D, generator=gen, device=DEV).to(dtype)          # one fused projection
    s = dict(Q=x[:, :Hq], K=x[:, Hq:Hq + Hkv])
    s["w_q"] = s["w_k"] = None
    if case["weights"]:
        s["w_q"], s["w_k"] = ((1.0 + 0.3 * torch.randn(D, generator=gen, device=DEV)).to(dtype) for _ in range(2))
    s["inv_freq"] = 10000.0 ** (-torch.arange(rot // 2, device=DEV) / (rot // 2))
    s["pos"] = torch.randint(0, case["far"], (T,), generator=gen, device=DEV, dtype=torch.int32)
    if T > 8:
        s["pos"][torch.randint(0, T, (T // 16 + 1,), generator=gen, device=DEV)] = -1       # padding of the batch
    s["q_out"] = torch.zeros(T, Hq, D, dtype=dtype, device=DEV)
    s["k_out"] = torch.zeros(T, Hkv, D, dtype=dtype, device=DEV)
    return s


def _prepare_attend(case, gen):
    held, new = _plan(case)
    block, R, Hq, Hkv = case["block"], case["R"], case["Hq"], case["Hkv"]
    total = [h + n for h, n in zip(held, new)]
    width = max(-(-max(total) // block), 1)
    s = {}
    s["table"], order, _ = _tables(total, [0] * R, block, width, sum(-(-t // block) for t in total) + 3, gen)
    s["Kc"], s["Ks"] = _cache(len(order), Hkv, block, gen, True)
    s["Vc"], s["Vs"] = _cache(len(order), Hkv, block, gen, False)
    s["len"] = _ints(total)
    s["cu"] = _ints([sum(new[:i]) for i in range(R + 1)])
    T = sum(new) + (3 if R > 1 else 0)                     # a few rows behind the last request
    s["q"] = torch.randn(T, Hq + 2 * Hkv, D, generator=gen, device=DEV).to(TYPES[case["dtype"]])[:, :Hq]
    s["T"], s["max_new"] = T, max(max(new), 1)
    # behind a request's last token a block holds whatever its last use left there, NaN codes among it
    last = torch.tensor([(r, t) for r, t in enumerate(total) if t % block] or [(0, 0)], device=DEV)
    at = s["table"][last[:, 0], (last[:, 1] // block).clamp(max=width - 1)].clamp(min=0).long()
    tail = (torch.arange(block, device=DEV) >= (last[:, 1] % block)[:, None]) & (last[:, 1] % block > 0)[:, None]
    for c in (s["Kc"], s["Vc"]):
        raw = c.view(torch.uint8)
        raw[at] = torch.where(tail[:, None, :, None], 0x7f, raw[at])
    s["out"] = torch.zeros(T, Hq, D, dtype=s["q"].dtype, device=DEV)
    s["lse"] = torch.zeros(T, Hq, device=DEV)
    return s


def _layers(case, pool, gen):
    """One cache for each layer: K and V codes, K and V scales."""
    return [[*_cache(pool, case["Hkv"], case["block"], gen, True), *_cache(pool, case["Hkv"], case["block"], gen, False)]
            for _ in range(case["layers"])]


def _prepare_fork(case, gen):
    held, parent, keep = _plan(case)
    block, R = case["block"], case["R"]
    if case["group"] == R:                                 # one prefix: the other places of the batch are empty
        held = [h if r == 0 else 0 for r, h in enumerate(held)]
    width = max(held) // block + 2
    extra = max(R - R // 16, 1)                            # (a tight pool: the last ones may find no block)
    s = {}
    used = sum(-(-h // block) for h in held)
    s["table"], order, _ = _tables(held, [0] * R, block, width, used + extra, gen)
    N = len(order)
    head = int(torch.randint(0, N, (1,), generator=gen, device=DEV))
    s["ring"] = torch.zeros(N, dtype=torch.int32, device=DEV)
    s["ring"][(torch.arange(N - used, device=DEV) + head) % N] = order[used:]
    s["state"] = _ints([head, N - used])
    s["len"], s["parent"], s["keep"] = _ints(held), _ints(parent), _ints(keep)
    s["len_next"], s["state_next"] = torch.zeros_like(s["len"]), torch.zeros_like(s["state"])
    s["table_next"] = torch.zeros_like(s["table"])
    s["src"], s["dst"] = torch.zeros_like(s["len"]), torch.zeros_like(s["len"])
    s["layers"] = _layers(case, N, gen)
    return s


def _prepare_pool(case, gen):
    held, shared = _plan(case)
    block = case["block"]
    width = max(held) // block + 1
    s = {}
    s["table"], order, _ = _tables(held, shared, block, width, case["pool"], gen)
    N = len(order)
    s["len"] = _ints(held)
    s["ring"] = torch.zeros(N, dtype=torch.int32, device=DEV)
    s["state"] = torch.zeros(2, dtype=torch.int32, device=DEV)
    if case["kind"] == "compact":
        s["table_next"] = torch.zeros_like(s["table"])
        s["src"], s["dst"] = (torch.zeros(N // 2 + 1, dtype=torch.int32, device=DEV) for _ in range(2))
        s["layers"] = _layers(case, N, gen)
    return s


def prepare(case, seed):
    kind = case["kind"]
    make = {"norm": _prepare_norm, "attend": _prepare_attend, "fork": _prepare_fork, "free": _prepare_pool, "compact": _prepare_pool}[kind]
    return dict(make(case, _gen(seed, len(kind))), kind=kind, case=case)


# ---------------------------------------------------------------------------------------------------------
# plain forms

def _turned(x, w, cos, sin, adjacent):
    """Rows x [T][H][128]: normed (w given), the first channels rotated; in the type of cos."""
    x = x.to(cos.dtype)
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(dim=2, keepdim=True) + EPS) * w.to(cos.dtype)
    half = cos.shape[1]
    c, s = cos[:, None], sin[:, None]
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if adjacent else (x[..., :half], x[..., half:2 * half])
    u, v = a * c - b * s, b * c + a * s
    turned = torch.stack([u, v], dim=3).flatten(2) if adjacent else torch.cat([u, v], dim=2)
    return torch.cat([turned, x[..., 2 * half:]], dim=2)


def _plain_norm(s):
    angle = s["pos"].double()[:, None] * s["inv_freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    live = (s["pos"] >= 0)[:, None, None]
    for x, w, out in ((s["Q"], s["w_q"], s["q_out"]), (s["K"], s["w_k"], s["k_out"])):
        y = _turned(x, w, cos, sin, s["case"]["adjacent"])
        out.copy_(torch.where(live, y.to(out.dtype), out))
    return dict(q=s["q_out"], k=s["k_out"])


def _plain_attend(s):
    q, table, ln, cu, n = s["q"], s["table"].long().clamp(min=0), s["len"].long(), s["cu"].long(), s["max_new"]
    T, Hq, _ = q.shape
    R = len(ln)
    N, Hkv, block, _ = s["Kc"].shape
    new = cu[1:] - cu[:-1]
    i, tok = torch.arange(n, device=DEV), torch.arange(table.shape[1] * block, device=DEV)
    row = (cu[:-1, None] + i).clamp(max=T - 1)                         # [R][n]
    past = tok >= ln[:, None]

    def rows(codes, scales):                                           # [R][Hkv][tokens][128], nothing behind the last token
        x = codes[table].float() * scales[table][..., None, None]      # [R][blocks][Hkv][block][128]
        return x.transpose(1, 2).reshape(R, Hkv, -1, D).masked_fill_(past[:, None, :, None], 0.0)

    qs = q[row].float().transpose(1, 2).reshape(R, Hkv, -1, D)         # [R][Hkv][rep * n][128]
    x = torch.matmul(qs, rows(s["Kc"], s["Ks"]).transpose(2, 3).contiguous()).mul_(SM)
    dead = tok[None, None] > (ln - new)[:, None, None] + i[None, :, None]              # [R][n][tokens]
    x.view(R, Hq, n, -1).masked_fill_(dead[:, None], float("-inf"))
    m = x.amax(dim=-1, keepdim=True).clamp(min=-3e38)
    w = x.sub_(m).exp_()
    total = w.sum(dim=-1, keepdim=True)
    o = (torch.matmul(w, rows(s["Vc"], s["Vs"])) / total.clamp(min=1e-38)).reshape(R, Hq, n, D)
    lse = (m + torch.log(total)).reshape(R, Hq, n)
    t = torch.arange(T, device=DEV)
    r = torch.searchsorted(cu, t, right=True) - 1
    live = (r < R)[:, None]
    r = r.clamp(max=R - 1)
    s["out"].copy_(torch.where(live[..., None], o[r, :, (t - cu[r]).clamp(max=n - 1)].to(q.dtype), s["out"]))
    s["lse"].copy_(torch.where(live, lse[r, :, (t - cu[r]).clamp(max=n - 1)], s["lse"]))
    return dict(out=s["out"], lse=s["lse"])


def _plain_copy(layers, src, dst):
    """Blocks dst of every layer become what blocks src are; pairs outside the pool are none."""
    N = len(layers[0][0])
    live = (src >= 0) & (src < N) & (dst >= 0) & (dst < N)
    take = torch.arange(N + 1, device=DEV).index_put_((torch.where(live, dst.long(), N),), src.long())[:N]     # who each block becomes
    to = torch.where(live, dst.long(), 0)
    for layer in layers:
        for t in layer:
            raw = t.view(torch.uint8) if t.dtype is E4M3 else t
            raw[to] = raw[take[to]]


def _plain_fork(s):
    block, ring, table = s["case"]["block"], s["ring"].long(), s["table"]
    ln, parent = s["len"].long(), s["parent"].long()
    R, N = len(ln), len(ring)
    head, n_free = s["state"].long()[0], s["state"].long()[1]
    width = table.shape[1]
    me = torch.arange(R, device=DEV)
    live = parent >= 0
    p = parent.clamp(min=0)
    keep = torch.where(live, torch.minimum(s["keep"].long(), ln[p]).clamp(min=0), 0)
    part = keep % block > 0
    whole = live & part & (keep == ln[p])
    first = torch.where(whole & (p == me), -1, me)                     # the parent itself comes first
    heir = torch.full((R + 1,), R, device=DEV).scatter_reduce_(0, torch.where(whole, p, R), first, "amin")[:R]
    need = part & ~(whole & (heir[p] == first))
    rank = need.long().cumsum(0)
    ok = need & (rank <= n_free)
    len_next = torch.where(need & ~ok, keep // block * block, keep)
    fresh = ring[(head + rank - 1) % N]
    cols = torch.arange(width, device=DEV)
    entry = torch.where(ok[:, None] & (cols == (keep // block)[:, None]), fresh[:, None], table[p].long())
    count = (len_next + block - 1) // block
    table_next = torch.where(cols < count[:, None], entry, s["table_next"].long())
    tail = table[p, (keep // block).clamp(max=width - 1)].long()
    i32 = lambda x: x.to(torch.int32)  # noqa: E731
    src, dst = i32(torch.where(ok, tail, -1)), i32(torch.where(ok, fresh, -1))
    _plain_copy(s["layers"], src, dst)
    given = ok.long().sum()
    return dict(len=i32(len_next), table=i32(table_next), state=i32(torch.stack([(head + given) % N, n_free - given])), src=src, dst=dst,
                layers=s["layers"])


def _used(s):
    """Which blocks a table names, and which entries of the tables count."""
    table, block = s["table"].long(), s["case"]["block"]
    N = len(s["ring"])
    cols = torch.arange(table.shape[1], device=DEV)
    named = cols < ((s["len"].long() + block - 1) // block)[:, None]
    used = torch.zeros(N + 1, dtype=torch.bool, device=DEV)
    used.index_fill_(0, torch.where(named, table, N).flatten(), True)
    return used[:N], named


def _ring_of(free, ring):
    """The free blocks ascending, in front of what the ring held."""
    N = len(free)
    out = torch.cat([ring, ring[:1]])
    out.index_put_((torch.where(free, free.long().cumsum(0) - 1, N),), torch.arange(N, device=DEV, dtype=torch.int32))
    return out[:N]


def _plain_free(s):
    used, _ = _used(s)
    n_free = (~used).sum()
    return dict(ring=_ring_of(~used, s["ring"]), state=torch.stack([torch.zeros_like(n_free), n_free]).to(torch.int32))


def _plain_compact(s):
    used, named = _used(s)
    N, n = len(used), s["src"].numel()
    at = torch.arange(N, device=DEV)
    moves = (used & (at >= used.sum())).sum().clamp(max=n)
    from_top = used.long().flip(0).cumsum(0).flip(0) - 1               # of a used block: how many lie above
    from_low = (~used).long().cumsum(0) - 1                            # of a free block: how many lie below
    gone, taken = used & (from_top < moves), ~used & (from_low < moves)
    src, dst = (torch.full((n + 1,), -1, device=DEV) for _ in range(2))
    src = src.index_put_((torch.where(gone, from_top, n),), at)[:n]
    dst = dst.index_put_((torch.where(taken, from_low, n),), at)[:n]
    k = torch.arange(n, device=DEV)
    src, dst = torch.where(k < moves, src, -1), torch.where(k < moves, dst, -1)
    to = torch.where(gone, dst[from_top.clamp(0, n - 1)], at)
    table_next = torch.where(named, to[s["table"].long().clamp(min=0)], s["table_next"].long())
    free = (~used & ~taken) | gone
    _plain_copy(s["layers"], src, dst)
    n_free = free.sum()
    i32 = lambda x: x.to(torch.int32)  # noqa: E731
    return dict(table=i32(table_next), ring=_ring_of(free, s["ring"]), state=i32(torch.stack([torch.zeros_like(n_free), n_free])), src=i32(src),
                dst=i32(dst), layers=s["layers"])


PLAIN = {"norm": _plain_norm, "attend": _plain_attend, "fork": _plain_fork, "free": _plain_free, "compact": _plain_compact}


# ---------------------------------------------------------------------------------------------------------
# the framework's calls

def _handle(s):
    """The shape, the cache handles and the workspace that a program makes once."""
    if "handle" not in s:
        from paper_2411_18077_amd import api
        c = s["case"]
        N = len(s["Kc"]) if c["kind"] == "attend" else len(s["ring"])
        shape = api.make_blk_shape(c["R"], c.get("Hq", c.get("Hkv", 1)), c.get("Hkv", 1), D, c["block"], N, s["table"].shape[1],
                                   TYPES[c.get("dtype", "f16")])
        if c["kind"] == "attend":
            caches = api.BlkCache(shape, K=s["Kc"], V=s["Vc"], Ks=s["Ks"], Vs=s["Vs"])
            ws = torch.zeros(api.minikv_prompt_blk_workspace_bytes(shape, s["T"]), dtype=torch.uint8, device=DEV)
        else:
            caches = api.BlkCaches(shape, [dict(K=k, V=v, Ks=ks, Vs=vs) for k, ks, v, vs in s["layers"]]) if "layers" in s else None
            ws = torch.zeros(api.kv_free_workspace_bytes(shape), dtype=torch.uint8, device=DEV)
        s["handle"] = (api, shape, caches, ws)
    return s["handle"]


def run(s):
    kind = s["kind"]
    if not own:
        return PLAIN[kind](s)
    if kind == "norm":
        from paper_2411_18077_amd import api
        c = s["case"]
        api.minikv_norm_rope(c["Hq"], c["Hkv"], c["T"], s["Q"], s["K"], s["w_q"], s["w_k"], EPS, s["inv_freq"], c["rot"], c["adjacent"], s["pos"],
                             s["q_out"], s["k_out"])
        return dict(q=s["q_out"], k=s["k_out"])
    api, shape, caches, ws = _handle(s)
    if kind == "attend":
        api.minikv_prompt_attn_blk(shape, s["T"], s["q"], caches, s["table"], s["len"], s["cu"], SM, s["out"], s["lse"], ws)
        return dict(out=s["out"], lse=s["lse"])
    if kind == "fork":
        api.kv_fork_blk(shape, s["len"], s["parent"], s["keep"], s["table"], s["ring"], s["state"], s["len_next"], s["table_next"], s["state_next"],
                        s["src"], s["dst"])
        api.kv_copy_blk(shape, caches, s["src"], s["dst"])
        return dict(len=s["len_next"], table=s["table_next"], state=s["state_next"], src=s["src"], dst=s["dst"], layers=s["layers"])
    if kind == "free":
        api.kv_free_blk(shape, s["len"], s["table"], s["ring"], s["state"], ws)
        return dict(ring=s["ring"], state=s["state"])
    api.kv_compact_blk(shape, s["len"], s["table"], s["table_next"], s["ring"], s["state"], s["src"], s["dst"], ws)
    api.kv_copy_blk(shape, caches, s["src"], s["dst"])
    return dict(table=s["table_next"], ring=s["ring"], state=s["state"], src=s["src"], dst=s["dst"], layers=s["layers"])


# ---------------------------------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "norm":
        heads = case["Hq"] + case["Hkv"]
        return {"bytes": case["T"] * heads * D * 4 + case["T"] * 4, "flops": case["T"] * heads * D * (8 if case["weights"] else 4)}
    block = case["block"]
    up = lambda n: -(-n // block)  # noqa: E731
    if kind == "attend":
        held, new = _plan(case)
        pairs = sum(h * n + n * (n + 1) // 2 for h, n in zip(held, new))
        total = [h + n if n else 0 for h, n in zip(held, new)]
        byts = sum(total) * case["Hkv"] * 2 * D + sum(new) * case["Hq"] * (4 * D + 4)
        return {"bytes": byts + sum(up(t) for t in total) * (4 + 8 * case["Hkv"]), "flops": 4 * D * case["Hq"] * pairs}
    one = case.get("layers", 0) * 2 * case.get("Hkv", 0) * (block * D + 4)             # bytes of a block in all layers
    if kind == "fork":
        held, parent, keep = _plan(case)
        if case["group"] == case["R"]:
            held = [h if r == 0 else 0 for r, h in enumerate(held)]
        keep = [min(k, held[p]) if p >= 0 else 0 for p, k in zip(parent, keep)]
        heirs, copies = set(), 0
        for r in sorted(range(case["R"]), key=lambda r: (parent[r] != r, r)):
            if keep[r] % block == 0 or parent[r] < 0:
                continue
            if keep[r] == held[parent[r]] and parent[r] not in heirs:
                heirs.add(parent[r])
            else:
                copies += 1
        return {"bytes": sum(up(k) for k in keep) * 8 + 24 * case["R"] + min(copies, max(case["R"] - case["R"] // 16, 1)) * 2 * one, "flops": 8 * case["R"]}
    held, shared = _plan(case)
    entries = sum(up(h) for h in held)
    blocks = entries - sum(s // block for s in shared)
    pool = max(case["pool"], blocks + 1)
    if kind == "free":
        return {"bytes": entries * 4 + case["R"] * 4 + (pool - blocks) * 4, "flops": entries + pool}
    moves = blocks * (pool - blocks) // pool               # of blocks spread evenly over the pool
    return {"bytes": entries * 8 + case["R"] * 4 + (pool - blocks) * 4 + moves * (8 + 2 * one), "flops": entries + pool}


# ---------------------------------------------------------------------------------------------------------
# the definition in 64 bits

def _exact_norm(s):
    case, out = s["case"], {}
    half, T = case["rot"] // 2, case["T"]
    first = torch.arange(half, device=DEV) * 2 if case["adjacent"] else torch.arange(half, device=DEV)
    second = first + (1 if case["adjacent"] else half)
    turn = torch.polar(torch.ones(T, half, dtype=torch.float64, device=DEV), s["pos"].double()[:, None] * s["inv_freq"].double())
    for name, x, w in (("q", s["Q"], s["w_q"]), ("k", s["K"], s["w_k"])):
        y = x.double()
        if w is not None:
            y = y / torch.sqrt((y * y).sum(dim=2) / D + EPS)[:, :, None] * w.double()
        z = torch.complex(y[:, :, first], y[:, :, second]) * turn[:, None]
        y = y.clone()
        y[:, :, first], y[:, :, second] = z.real, z.imag
        y[s["pos"] < 0] = 0.0                              # (as the buffers were)
        out[name] = y
    return out


def _exact_attend(s):
    case = s["case"]
    held, new = _plan(case)
    Hq, Hkv, block, T = case["Hq"], case["Hkv"], case["block"], s["T"]
    rep = Hq // Hkv
    out = torch.zeros(T, Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.zeros(T, Hq, dtype=torch.float64, device=DEV)
    at = 0
    for r, (h, n) in enumerate(zip(held, new)):
        if n == 0:
            continue
        blocks = s["table"][r, :-(-(h + n) // block)].long()
        seen = torch.ones(n, h + n, dtype=torch.bool, device=DEV).tril(h)
        for g in range(Hkv):
            k = (s["Kc"][blocks, g].double() * s["Ks"][blocks, g].double()[:, None, None]).reshape(-1, D)[:h + n]
            v = (s["Vc"][blocks, g].double() * s["Vs"][blocks, g].double()[:, None, None]).reshape(-1, D)[:h + n]
            for hq in range(g * rep, (g + 1) * rep):
                x = (s["q"][at:at + n, hq].double() @ k.t() * SM).masked_fill(~seen, float("-inf"))
                lse[at:at + n, hq] = torch.logsumexp(x, dim=1)
                out[at:at + n, hq] = torch.softmax(x, dim=1) @ v
        at += n
    return dict(out=out, lse=lse)


def _exact_pages(s):
    """Tables and rings are whole numbers; the moved blocks are what the pairs say, one after the other."""
    got = PLAIN[s["kind"]](dict(s, layers=[[t.clone() for t in layer] for layer in s["layers"]]))
    pairs = [(a, b) for a, b in zip(got["src"].tolist(), got["dst"].tolist()) if a >= 0]
    out = dict.fromkeys(got)
    out["layers"] = []
    for layer in s["layers"]:
        wide = [t.double() for t in layer]
        for t, w in zip(layer, wide):
            for a, b in pairs:
                w[b] = t[a].double()
        out["layers"].append(wide)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        return _exact_norm(s)
    if case["kind"] == "attend":
        return _exact_attend(s)
    if case["kind"] == "free" or case["layers"] * case["R"] > 4000:
        return None
    return _exact_pages(s)
