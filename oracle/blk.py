"""Plain definitions of the operators over packed prompts and the paged 8-bit cache, in 64 bits and request by request
(test infrastructure only): written from include/minikv.h, sharing nothing with the library.  Codes are uint8; tensors are CPU
tensors (prompt_attn takes them anywhere)."""
import math

import torch

E4M3_MAX = 448.0


def e4m3_values():
    """The 256 values: sign, 4 exponent bits (bias 7), 3 mantissa bits; exponent 0 is subnormal, 0x7f and 0xff are NaN."""
    out = []
    for code in range(256):
        e, m = (code >> 3) & 15, code & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        if code & 127 == 127:
            v = math.nan
        out.append(-v if code & 128 else v)
    return torch.tensor(out, dtype=torch.float64)


_VALUES = e4m3_values()
_POSITIVE = _VALUES[:127]                              # ascending; code = index


def encode(x):
    """Codes of the nearest value of x (float64, |x| <= 448 or NaN), ties to the even code."""
    mag = x.abs()
    hi = torch.searchsorted(_POSITIVE, mag).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    below, above = mag - _POSITIVE[lo], _POSITIVE[hi] - mag
    code = torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    code = torch.where(mag.isnan(), 127, code)
    return (code + 128 * torch.signbit(x)).to(torch.uint8)


def decode_codes(codes):
    return _VALUES[codes.long()]


def scale_for(amax):
    """The smallest power of two s >= 2^-126 with amax <= 448 s; 0 for 0."""
    if amax == 0:
        return 0.0
    e = -126
    while amax > E4M3_MAX * 2.0 ** e:
        e += 1
    return 2.0 ** e


def assign(q_len, n_new, table, ring, state, block, n_slots):
    """Request by request.  Lists and nested lists of ints in, a dict of them out; nothing is changed in place."""
    R, width, N = len(q_len), len(table[0]), len(ring)
    table, ring = [list(t) for t in table], list(ring)
    head, n_free = state
    blocks = lambda n: -(-n // block)  # noqa: E731
    cu, slots, length, back = [0], [-1] * n_slots, list(q_len), []
    taken, asked = 0, 0
    for r in range(R):
        add = max(n_new[r], 0)
        cu.append(cu[-1] + add)
        held, after = blocks(q_len[r]), blocks(q_len[r] + add)
        if n_new[r] < 0:
            back += table[r][:held]
            length[r] = 0
            continue
        if after > width or cu[-1] > n_slots:
            continue
        asked += after - held
        if after > held and asked > n_free:
            continue
        for b in range(held, after):
            table[r][b] = ring[(head + taken) % N]
            taken += 1
        for i in range(add):
            pos = q_len[r] + i
            b = table[r][pos // block]
            slots[cu[r] + i] = b * block + pos % block if 0 <= b <= (2 ** 31 - 1) // block else -1
        length[r] = q_len[r] + add
    for i, b in enumerate(back):
        ring[(head + n_free + i) % N] = b
    return dict(table=table, ring=ring, q_len=length, state=[(head + taken) % N, n_free - taken + len(back)], cu=cu, slots=slots)


def file_rows(x, codes, scales, slots):
    """x [T][Hkv][128] into codes uint8 [N][Hkv][block][128], scales [N][Hkv]; returns new ones."""
    codes, scales, x = codes.clone(), scales.double().clone(), x.double()
    N, Hkv, block, _ = codes.shape
    rows_of = {}
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < N * block:
            rows_of.setdefault(s // block, []).append((t, s % block))
    for b, rows in rows_of.items():
        fresh = any(off == 0 for _, off in rows)
        for h in range(Hkv):
            amax = max(float(x[t, h].abs().max()) for t, _ in rows)
            s, old = scale_for(amax), float(scales[b, h])
            if not fresh:
                s = max(s, old)
                if s != old:
                    codes[b, h] = encode(decode_codes(codes[b, h]) * old / s)
            for t, off in rows:
                codes[b, h, off] = encode(x[t, h] / s) if s else 0
            scales[b, h] = s
    return codes, scales


def decode_attn(q, Kc, Ks, Vc, Vs, table, q_len, sm):
    """out, and per output the sum of weight times |value| and the largest sum of |q k| sm of a row (what tolerances count)."""
    R, Hq, D = q.shape
    N, Hkv, block, _ = Kc.shape
    rep = Hq // Hkv
    out, mean, score = torch.zeros(R, Hq, D, dtype=torch.float64), torch.zeros(R, Hq, D, dtype=torch.float64), 0.0
    for r in range(R):
        n = max(min(int(q_len[r]), table.shape[1] * block), 0)
        at = [(int(table[r, i // block]), i % block) for i in range(n)]
        at = [(b, o) for b, o in at if 0 <= b < N]
        if not at:
            continue
        b, o = torch.tensor([p[0] for p in at]), torch.tensor([p[1] for p in at])
        for h in range(Hkv):
            k = decode_codes(Kc[b, h, o]) * Ks[b, h].double()[:, None]
            v = decode_codes(Vc[b, h, o]) * Vs[b, h].double()[:, None]
            x = q[r, h * rep:(h + 1) * rep].double()
            p = torch.softmax(x @ k.t() * sm, dim=1)
            out[r, h * rep:(h + 1) * rep], mean[r, h * rep:(h + 1) * rep] = p @ v, p @ v.abs()
            score = max(score, float((x.abs() @ k.abs().t()).max()) * abs(sm))
    return out, mean, score


def prompt_attn(Q, K, V, cu, sm):
    """X_O, LSE, A_cumul of packed prompts (LSE and A_cumul laid out prompt by prompt, a row per head), and as above."""
    T, Hq, D = Q.shape
    rep = Hq // K.shape[1]
    zeros = lambda *n: torch.zeros(*n, dtype=torch.float64, device=Q.device)  # noqa: E731  (products in 64 bits wherever the inputs are)
    X, mean, lse, A, score = zeros(T, Hq, D), zeros(T, Hq, D), zeros(T * Hq), zeros(T * Hq), 0.0
    for a, e in zip(cu[:-1], cu[1:]):
        n = e - a
        if n == 0:
            continue
        later = torch.ones(n, n, dtype=torch.bool, device=Q.device).triu(1)
        for h in range(Hq):
            q, k, v = Q[a:e, h].double(), K[a:e, h // rep].double(), V[a:e, h // rep].double()
            x = (q @ k.t() * sm).masked_fill(later, -math.inf)
            z = torch.logsumexp(x, dim=1)
            p = torch.exp(x - z[:, None])
            X[a:e, h], mean[a:e, h] = p @ v, p @ v.abs()
            f = a * Hq + h * n
            lse[f:f + n], A[f:f + n] = z, p.sum(dim=0)
            score = max(score, float((q.abs() @ k.abs().t()).max()) * abs(sm))
    return X, lse, A, mean, score
