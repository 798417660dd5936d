"""Plain definitions of what requests that share blocks of the paged 8-bit cache need, in 64 bits and request by request (test
infrastructure only): written from include/minikv.h, sharing nothing with the library.  CPU tensors, or lists of ints."""
import math

import torch

from oracle.blk import decode_codes


def norm_rope(x, w, eps, inv_freq, rot, adjacent, pos):
    """Rows x [T][H][128] normed and turned; and what a rounding of one part of a pair is measured by, |u| + |v|.  Rows with pos < 0 are x."""
    y = x.double()
    if w is not None:
        y = y * w.double() / torch.sqrt((y * y).mean(dim=2, keepdim=True) + eps)
    out, size = y.clone(), y.abs()
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + rot // 2)
        angle = pos.double() * float(inv_freq[i])
        c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        u, v = y[:, :, a], y[:, :, b]
        out[:, :, a], out[:, :, b] = u * c - v * s, v * c + u * s
        size[:, :, a] = size[:, :, b] = u.abs() + v.abs()
    keep = (pos < 0)[:, None, None]
    return torch.where(keep, x.double(), out), size


def prompt_attn(q, Kc, Ks, Vc, Vs, table, q_len, cu, sm):
    """out [T][Hq][128], lse [T][Hq] (-inf where a row sees nothing), which rows belong to a request, per output the sum of weight times
    |value|, and the largest sum of |q k| sm of a row."""
    T, Hq, D = q.shape
    N, Hkv, block, _ = Kc.shape
    rep = Hq // Hkv
    zeros = lambda *n: torch.zeros(*n, dtype=torch.float64)  # noqa: E731
    out, mean, lse, score = zeros(T, Hq, D), zeros(T, Hq, D), torch.full((T, Hq), -math.inf, dtype=torch.float64), 0.0
    live = torch.zeros(T, dtype=torch.bool)
    for r in range(len(q_len)):
        at, end = int(cu[r]), int(cu[r + 1])
        if at < 0 or end <= at or end > T:
            continue
        live[at:end] = True
        n, L = end - at, max(min(int(q_len[r]), table.shape[1] * block), 0)
        where = [(j, int(table[r, j // block]), j % block) for j in range(L)]
        where = [w for w in where if 0 <= w[1] < N]
        if not where:
            continue
        j, b, o = (torch.tensor(v) for v in zip(*where))
        hidden = j[None] > (L - n + torch.arange(n))[:, None]          # [n][tokens]
        for h in range(Hkv):
            k = decode_codes(Kc[b, h, o]) * Ks[b, h].double()[:, None]
            v = decode_codes(Vc[b, h, o]) * Vs[b, h].double()[:, None]
            for hq in range(h * rep, (h + 1) * rep):
                x = (q[at:end, hq].double() @ k.t() * sm).masked_fill(hidden, -math.inf)
                z = torch.logsumexp(x, dim=1)
                p = torch.where(z[:, None] > -math.inf, torch.exp(x - z[:, None]), 0.0)
                out[at:end, hq], mean[at:end, hq], lse[at:end, hq] = p @ v, p @ v.abs(), z
                score = max(score, float((q[at:end, hq].double().abs() @ k.abs().t()).max()) * sm)
    return out, lse, live, mean, score


def fork(q_len, parent, n_keep, table, ring, state, block):
    """A dict of the lists that kv_fork_blk writes; rows of `table` are as long as their entries."""
    R, N, width = len(q_len), len(ring), len(table[0])
    head, n_free = state
    held = [min(max(n, 0), width * block) for n in q_len]
    made, heirs = [], {}
    for r in range(R):
        p = parent[r] if 0 <= parent[r] < R else None
        k = 0 if p is None else min(max(n_keep[r], 0), held[p])
        made.append((p, k))
        if p is not None and k % block and k == held[p]:
            heirs.setdefault(p, []).append(r)
    heir = {p: p if p in rs else rs[0] for p, rs in heirs.items()}
    out = dict(q_len=[], table=[], src=[], dst=[])
    taken = 0
    for r, (p, k) in enumerate(made):
        row, src, dst = [] if p is None else list(table[p][:-(-k // block)]), -1, -1
        if k % block and heir.get(p) != r and 0 <= row[-1] < N:
            if taken < n_free:
                src, dst = row[-1], ring[(head + taken) % N]
                row[-1] = dst
                taken += 1
            else:
                row.pop()
                k -= k % block
        for name, v in (("q_len", k), ("table", row), ("src", src), ("dst", dst)):
            out[name].append(v)
    return dict(out, state=[(head + taken) % N, n_free - taken])


def named(q_len, table, N, block):
    """The blocks that the tables name."""
    return {b for n, row in zip(q_len, table) for b in row[:-(-min(max(n, 0), len(row) * block) // block)] if 0 <= b < N}


def free(q_len, table, N, block):
    """The ring's free blocks."""
    used = named(q_len, table, N, block)
    return [b for b in range(N) if b not in used]


def compact(q_len, table, N, block, n_pairs):
    """Moves [(src, dst)], table rows as long as their entries, the ring's free blocks."""
    held = named(q_len, table, N, block)
    used, holes = sorted(held), [b for b in range(N) if b not in held]
    high = [b for b in reversed(used) if b >= len(used)][:n_pairs]
    moves = list(zip(high, holes))
    to = dict(moves)
    rows = [[to.get(b, b) for b in row[:-(-min(max(n, 0), len(row) * block) // block)]] for n, row in zip(q_len, table)]
    after = {to.get(b, b) for b in used}
    return moves, rows, [b for b in range(N) if b not in after]
