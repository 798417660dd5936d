"""Causal attention of packed prompts of different lengths on the GPU: against the plain definition prompt by prompt, against the
call for prompts of one length, and in the chain that it stands in (scores -> selection; rows -> paged cache -> decode)."""
import pytest
import torch

from blk_common import HALF, SM, attn_tolerance
from oracle import blk

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def api():
    assert torch.cuda.is_available()
    from paper_2411_18077_amd import api as _api
    return _api


def fused(T, Hq, Hkv, dtype, seed, gain=1.0, pad=0):
    """Q, K, V as slices of one projection of (Hq + 2 Hkv) heads and `pad` elements more per token."""
    g = torch.Generator().manual_seed(seed)
    width = (Hq + 2 * Hkv) * 128
    x = (torch.randn(T, width + pad, generator=g) * gain).to(dtype).cuda()
    heads = lambda a, n: x[:, a * 128:(a + n) * 128].unflatten(1, (n, 128))  # noqa: E731
    return heads(0, Hq), heads(Hq, Hkv), heads(Hq + Hkv, Hkv)


def run(api, Q, K, V, cu, scores, max_len=None, sm=SM, T=None, fill=float("nan")):
    T = Q.shape[0] if T is None else T
    Hq, Hkv = Q.shape[1], K.shape[1]
    X = torch.full((T, Hq, 128), fill, dtype=Q.dtype, device="cuda")
    lse = torch.full((T * Hq,), fill, device="cuda")
    A = torch.full((T * Hq,), fill, device="cuda") if scores else None
    n = max([b - a for a, b in zip(cu[:-1], cu[1:])] + [0])
    api.selective_flash_attn_packed(len(cu) - 1, Hq, Hkv, T, n if max_len is None else max_len, Q, K, V,
                                    torch.tensor(cu, dtype=torch.int32, device="cuda"), sm, X, lse, A)
    return X, lse, A


def lse_tolerance(lse, score):
    """A score's own error (136 half steps of the sum of magnitudes, in attn_tolerance), and the roundings of the sum's logarithm and of
    its product and sum with the maximum: four half steps of the result's or the largest score's size."""
    return 137 * 2.0 ** -24 * score * 1.01 + 4 * 2.0 ** -24 * (lse.abs() + score + 1)


def check(api, lens, Hq, Hkv, dtype, scores=True, seed=1, gain=1.0, pad=0, max_len=None, sm=SM, tail=0):
    cu = [sum(lens[:i]) for i in range(len(lens) + 1)]
    T = cu[-1] + tail
    Q, K, V = fused(T, Hq, Hkv, dtype, seed, gain, pad)
    if tail:                                           # rows of no prompt: not read, and their outputs stay as they are
        for x in (Q, K, V):
            x[cu[-1]:] = float("nan")
    X, lse, A = run(api, Q, K, V, cu, scores, max_len, sm, fill=7.0)
    X0, lse0, A0, mean, score = blk.prompt_attn(Q, K, V, cu, sm)
    n, m = cu[-1], cu[-1] * Hq
    assert bool((X[n:] == 7.0).all()) and bool((lse[m:] == 7.0).all())
    tol = attn_tolerance(X0, mean, score, max(lens), float(V[:n].abs().max()), HALF[dtype], dtype)
    err = (X.double() - X0).abs()
    assert bool((err <= tol)[:n].all()), (float(err[:n].max()), float((err / tol)[:n].max()))
    ltol = lse_tolerance(lse0, score)
    err = (lse.double() - lse0).abs()[:m]
    assert bool((err <= ltol[:m]).all()), float((err / ltol[:m]).max())
    if scores:
        # a weight exp(score - LSE): the errors of both, its own rounding, and a half step per addition of up to L of them
        rel = 137 * 2.0 ** -24 * score * 1.01 + float(ltol.max()) + (max(lens) / 64 + 70) * 2.0 ** -24
        err = (A.double() - A0).abs()[:m]
        assert bool((A[m:] == 7.0).all()) and bool((err <= (A0 * rel + 1e-30)[:m]).all()), float((err / (A0 * rel + 1e-30)[:m]).max())
    again = run(api, Q, K, V, cu, scores, max_len, sm, fill=7.0)
    assert torch.equal(again[0].view(torch.int16)[:n], X.view(torch.int16)[:n]) and torch.equal(again[1][:m], lse[:m])
    return X, lse, A


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("Hq,Hkv,lens", [
    (1, 1, [1]), (4, 2, [2, 1, 64]), (2, 1, [65, 0, 63, 128, 0]), (4, 4, [129, 127]), (8, 1, [300]), (6, 2, [31, 33, 257, 1]),
    (2, 2, [640, 5, 700]), (3, 1, [1] * 9), (12, 12, [0, 200, 0]),
])
def test_packed_prompts(api, dtype, Hq, Hkv, lens):
    check(api, lens, Hq, Hkv, dtype)
    check(api, lens, Hq, Hkv, dtype, scores=False, seed=2)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_long_prompts(api, dtype):
    check(api, [1500, 40, 2100], 2, 1, dtype)
    check(api, [4200], 2, 2, dtype)
    check(api, [600, 1030, 1, 300], 32, 8, dtype)


# One shape for each form of the two passes (the rules go by the longest prompt and the number of blocks): queries per workgroup, sets of
# waves, buffers, heads of a KV head side by side in 1, 2 and 4.
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("Hq,Hkv,lens,form", [
    (64, 8, [4100, 70], "128 queries, four of eight heads side by side"), (72, 24, [4200], "128 queries, many blocks"), (8, 4, [3000, 3001], "128 queries, two sets"),
    (16, 16, [1030, 900], "64 queries, two sets, one buffer"), (24, 3, [400, 100, 450], "64 queries, two sets, one buffer, two heads side by side"),
    (4, 2, [500, 97], "64 queries, two sets, two buffers"), (32, 8, [700, 300, 1, 900, 33], "128 queries, four heads side by side"),
    (32, 16, [600, 1000, 500], "128 queries, two heads side by side"), (40, 8, [100, 90, 128, 3, 0, 64], "prompts of one block"),
    (33, 11, [200, 300, 90], "128 queries"),
])
def test_every_form(api, dtype, Hq, Hkv, lens, form):
    check(api, lens, Hq, Hkv, dtype, seed=len(form))
    check(api, lens, Hq, Hkv, dtype, scores=False, seed=len(form) + 1)


def test_many_prompts(api):
    """More prompts than a wave has lanes: their counts stand in local memory."""
    lens = [(i * 37) % 150 for i in range(200)]
    check(api, lens, 2, 1, F16)
    check(api, lens, 2, 1, BF16, max_len=1000)
    check(api, [i % 3 for i in range(1500)], 1, 1, F16, scores=False)
    check(api, [0] * 100 + [500] + [0] * 100 + [3], 2, 2, F16)


@pytest.mark.parametrize("max_len", [130, 500, 1 << 23])
def test_bound_far_above_the_lengths(api, max_len):
    check(api, [100, 130, 9], 4, 2, F16, max_len=max_len)


def test_rows_of_any_pitch(api):
    """Tokens that are not a multiple of 256 bytes apart (8 elements of something else in the projection), and rows of no prompt."""
    check(api, [70, 200], 4, 2, BF16, pad=8)
    check(api, [90, 300, 1], 2, 1, F16, pad=120, tail=33)
    check(api, [128, 16], 2, 2, F16, tail=1)


@pytest.mark.parametrize("lens,Hq,Hkv", [([100, 64], 2, 1), ([150, 60], 4, 1), ([140, 70], 64, 32)])
def test_the_largest_pitch(api, lens, Hq, Hkv):
    """Tokens 2^23 elements apart, a tile of rows nearly 2^31 bytes: the same outputs as from rows that stand together."""
    cu = [0, lens[0], sum(lens)]
    near = fused(cu[-1], Hq, Hkv, F16, 5)
    x = torch.full((cu[-1], 1 << 23), float("nan"), dtype=F16, device="cuda")
    far, at = [], 0
    for t in near:
        width = t.shape[1] * 128
        far.append(x[:, at:at + width].unflatten(1, (t.shape[1], 128)))
        far[-1].copy_(t)
        at += width
    for a, b in zip(run(api, *near, cu, True), run(api, *far, cu, True)):
        assert torch.equal(a, b)


def test_peaked_rows(api):
    check(api, [150, 260], 2, 1, F16, gain=4.0)
    check(api, [150, 260], 2, 1, BF16, gain=4.0)
    check(api, [150, 90], 2, 1, F16, sm=1e-3)


def test_prompts_that_do_not_fit_are_left_alone(api):
    Q, K, V = fused(300, 2, 1, F16, 5)
    X, lse, A = run(api, Q, K, V, [0, 100, 250, 300], True, max_len=120, fill=7.0)                # the second is longer than the bound
    ok = run(api, Q[:100], K[:100], V[:100], [0, 100], True)
    assert torch.equal(X[:100], ok[0]) and bool((X[100:250] == 7.0).all()) and bool((lse[200:500] == 7.0).all()) and bool((A[200:500] == 7.0).all())
    ok = run(api, Q[250:], K[250:], V[250:], [0, 50], True)
    assert torch.equal(X[250:], ok[0]) and torch.equal(A[500:], ok[2])
    for cu in ([0, 100, 310], [-5, 40, 300], [0, 300, 200]):                                      # outside the rows, or backwards
        X, lse, A = run(api, Q, K, V, cu, True, max_len=300, fill=7.0)
        assert bool(torch.isfinite(X).all())
    X, lse, A = run(api, Q, K, V, [0, 100, 310], True, max_len=300, fill=7.0)
    assert bool((X[100:] == 7.0).all()) and not bool((X[:100] == 7.0).all(dim=(1, 2)).any())


def test_no_rows_at_all(api):
    Q, K, V = fused(4, 2, 1, F16, 5)
    X, lse, A = run(api, Q, K, V, [0, 0, 0], True, max_len=4, fill=7.0)
    assert bool((X == 7.0).all()) and bool((lse == 7.0).all())
    run(api, Q[:0], K[:0], V[:0], [0, 0], True, max_len=4)


def test_equal_lengths_agree_with_the_dense_call(api):
    """Prompts of one length: the dense entry point's numbers, head-major against token-major."""
    for B, Hq, Hkv, L in ((2, 4, 2, 100), (3, 2, 1, 500)):
        Q, K, V = fused(B * L, Hq, Hkv, F16, 3)
        X, lse, A = run(api, Q, K, V, [L * i for i in range(B + 1)], True)
        dense = lambda x, h: x.unflatten(0, (B, L)).transpose(1, 2).contiguous()  # noqa: E731
        q, k, v = dense(Q, Hq), dense(K, Hkv), dense(V, Hkv)
        xo, l2, a2 = torch.empty_like(q), torch.empty(B, Hq, L, device="cuda"), torch.empty(B, Hq, L, device="cuda")
        ws = torch.empty(api.selective_flash_attn_workspace_bytes(B, Hkv, L), dtype=torch.uint8, device="cuda")
        api.selective_flash_attn(B, Hq, Hkv, L, q, k, v, SM, xo, l2, a2, ws)
        assert torch.allclose(X.float(), xo.transpose(1, 2).reshape(B * L, Hq, 128).float(), atol=2e-3)
        assert torch.allclose(lse, l2.reshape(-1), atol=1e-4) and torch.allclose(A, a2.reshape(-1), rtol=1e-4, atol=1e-6)


def test_captured_and_replayed(api):
    lens, Hq, Hkv = [300, 129, 40], 4, 2
    cu = [0, 300, 429, 469]
    Q, K, V = fused(469, Hq, Hkv, BF16, 8)
    want = run(api, Q, K, V, cu, True)
    c = torch.tensor(cu, dtype=torch.int32, device="cuda")
    X, lse, A = torch.zeros_like(want[0]), torch.zeros_like(want[1]), torch.zeros_like(want[2])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        api.selective_flash_attn_packed(3, Hq, Hkv, 469, 300, Q, K, V, c, SM, X, lse, A)
    for _ in range(3):
        X.zero_(), A.zero_()
        g.replay()
        assert torch.equal(X, want[0]) and torch.equal(lse, want[1]) and torch.equal(A, want[2])
    c.copy_(torch.tensor([0, 100, 100, 200], dtype=torch.int32))                                  # other lengths under the same bounds
    g.replay()
    two = run(api, Q[:200], K[:200], V[:200], [0, 100, 100, 200], True)
    assert torch.allclose(X[:200].float(), two[0].float(), atol=2e-2) and torch.allclose(A[:800], two[2], rtol=1e-4)


def test_scores_go_to_the_selection_as_they_are(api):
    """A_cumul of each prompt is what kv_select_hh_rw takes for it: kept positions equal those of the oracle's selection."""
    from oracle import ref
    lens, Hq, Hkv = [200, 333], 8, 2
    Q, K, V = fused(sum(lens), Hq, Hkv, F16, 4)
    _, _, A = run(api, Q, K, V, [0, 200, 533], True)
    at = 0
    for n in lens:
        a = A[at * Hq:(at + n) * Hq]
        hh, rw = (torch.full((Hkv,), v, dtype=torch.int32, device="cuda") for v in (32, 32))
        idx, n_tok = torch.zeros(Hkv, 64, dtype=torch.int32, device="cuda"), torch.zeros(Hkv, dtype=torch.int32, device="cuda")
        ws = torch.empty(api.kv_select_workspace_bytes(Hkv, Hq // Hkv, n), dtype=torch.uint8, device="cuda")
        api.kv_select_hh_rw(Hkv, Hq // Hkv, n, a, hh, rw, idx, 64, n_tok, ws)
        want, _ = ref.select_hh_rw(a.reshape(Hq, n).cpu().numpy(), hh.cpu().numpy(), rw.cpu().numpy(), rep=Hq // Hkv, idx_stride=64)
        assert (idx.cpu().numpy() == want).all()
        at += n


@pytest.mark.parametrize("dtype,block", [(F16, 16), (BF16, 64)])
def test_a_serving_loop(api, dtype, block):
    """The four calls as a program runs them: prompts arrive and are filed, tokens are generated, a request ends and its blocks go to a new
    one.  After every step each request's attention is checked against its own rows in 64 bits."""
    R, Hq, Hkv, width, N = 4, 8, 2, 300 // block + 2, 700 // block + 6
    shape = api.make_blk_shape(R, Hq, Hkv, 128, block, N, width, dtype)
    cache = api.BlkCache(shape)
    i = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    table, ring, cu, slots = i([[-1] * width] * R), i(list(range(N))), i([0] * (R + 1)), i([0] * 500)
    q_len, q_next, state, s_next = i([0] * R), i([0] * R), i([0, N]), i([0, 0])
    rows = [[None, None] for _ in range(R)]            # every request's own keys and values
    plans = [[150, 0, 17, 90], [1, 1, 1, 1], [1, 0, 1, 1], [-1, 200, 1, 1], [120, 1, 1, -1], [1, 1, 1, 0], [1, 1, 1, 260]]
    steps = [(k, p) for k, p in enumerate(plans)] + [(9 + k, [1] * R) for k in range(6)]
    for seed, plan in steps:
        api.kv_assign_blk(shape, q_len, i(plan), table, ring, state, q_next, s_next, cu, slots)
        q_len, q_next, state, s_next = q_next, q_len, s_next, state
        T = sum(max(n, 0) for n in plan)
        Q, K, V = fused(T, Hq, Hkv, dtype, 50 + seed)
        fresh = [n > 1 for n in plan]
        if all(n <= 0 or f for n, f in zip(plan, fresh)):                                         # prompts only: they attend to themselves
            run(api, Q, K, V, cu.tolist(), True)
        api.kv_quantize_blk(shape, K, V, slots[:T], cache)
        out = torch.zeros(R, Hq, 128, dtype=dtype, device="cuda")
        last = torch.randn(R, Hq, 128, generator=torch.Generator().manual_seed(seed)).to(dtype)
        api.minikv_decode_attn_blk(shape, last.cuda(), cache, table, q_len, SM, out)
        at = cu.tolist()
        for r, n in enumerate(plan):
            if n < 0:
                rows[r] = [None, None]
            elif n > 0:
                for j, x in enumerate((K, V)):
                    new = x[at[r]:at[r] + n].cpu().double()
                    rows[r][j] = new if rows[r][j] is None else torch.cat([rows[r][j], new])
            k, v = rows[r]
            assert int(q_len[r]) == (0 if k is None else len(k))
            if k is None:
                assert not bool(out[r].any())
                continue
            x = (last[r].double().reshape(Hkv, -1, 128) @ k.permute(1, 2, 0)) * SM
            p = torch.softmax(x, dim=2)
            want, mean = (p @ v.transpose(0, 1)).reshape(Hq, 128), (p @ v.transpose(0, 1).abs()).reshape(Hq, 128)
            # a code is within 2^-4 of its row's value (half a step of 4 bits), or within half a subnormal step of the largest one
            # of its block, 2^-10 of a scale that is at most max / 224; the scores move by sum |q| |dk|, the weights by twice that
            dk = k.abs() * 2.0 ** -4 + float(k.abs().max()) * 2.0 ** -17
            ds = float((last[r].double().abs().reshape(Hkv, -1, 128) @ dk.permute(1, 2, 0)).max()) * SM
            tol = mean * 2 * torch.expm1(torch.tensor(2 * ds)) + mean * 2.0 ** -3 + 2e-2
            assert bool(((out[r].cpu().double() - want).abs() <= tol).all())
            # and closely against the rows as they were filed
        Kc, Vc = cache.K.view(torch.uint8).cpu(), cache.V.view(torch.uint8).cpu()
        want, mean, score = blk.decode_attn(last, Kc, cache.Ks.cpu(), Vc, cache.Vs.cpu(), table.cpu(), q_len.tolist(), SM)
        tol = attn_tolerance(want, mean, score, 300, 6.0, 2.0 ** -11, dtype)
        assert bool(((out.cpu().double() - want).abs() <= tol).all())


def test_the_binding_refuses_on_the_gpu(api):
    """What is checked behind the place of the first tensor: nothing is launched."""
    Q, K, V = fused(10, 8, 2, BF16, 1)
    i = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    f = torch.zeros(80, device="cuda")
    good = dict(T=10, Q=Q, K=K, V=V, cu=i([0, 4, 10]), X=Q.contiguous(), lse=f, A=f.clone())
    for bad in (dict(T=11), dict(Q=Q[:9]), dict(K=K[:9]), dict(V=V.half()), dict(cu=good["cu"][:2]), dict(cu=good["cu"].long()), dict(K=Q[:, ::4]),
                dict(X=good["X"].half()), dict(X=Q), dict(lse=f[:79]), dict(lse=f.double()), dict(A=f[::2]), dict(V=V.cpu()), dict(A=f.cpu()),
                dict(cu=good["cu"].cpu())):
        a = {**good, **bad}
        with pytest.raises(ValueError):
            api.selective_flash_attn_packed(2, 8, 2, a["T"], 6, a["Q"], a["K"], a["V"], a["cu"], 0.1, a["X"], a["lse"], a["A"])
    shape = api.make_blk_shape(4, 8, 2, 128, 32, 10, 5, BF16)
    cache, n = api.BlkCache(shape), i([0] * 20)
    x, q = K[:4], Q[:4]
    for slots, V4, other in ((n[:3], V[:4], cache), (n.long(), V[:4], cache), (n, V[:4].cpu(), cache), (n.cpu(), V[:4], cache), (n, V[:3], cache),
                             (n, V[:4], api.BlkCache(shape, device="cpu")),
                             (n, V[:4], api.BlkCache(api.make_blk_shape(4, 8, 2, 128, 32, 9, 5, BF16))),
                             (n, V[:4], api.BlkCache(api.make_blk_shape(4, 8, 2, 128, 64, 10, 5, BF16)))):
        with pytest.raises(ValueError):
            api.kv_quantize_blk(shape, x, V4, slots, other)
    out = torch.zeros(4, 8, 128, dtype=BF16, device="cuda")
    for q4, table, lens, o, ws in ((q[:3], n, n, out, None), (q, n[:19], n, out, None), (q, n, n[:3], out, None), (q, n, n, out[:, :4], None),
                                   (q, n, n, out.half(), None), (q, n, n, out.cpu(), None), (q, n.cpu(), n, out, None), (q.half(), n, n, out, None),
                                   (q, n, n, torch.zeros(8, 4, 128, dtype=BF16, device="cuda").transpose(0, 1), None),
                                   (q, n, n, out, cache.workspace.cpu()), (q, n, n, out, torch.cat([cache.workspace] * 2)[::2])):
        with pytest.raises(ValueError):
            api.minikv_decode_attn_blk(shape, q4, cache, table, lens, SM, o, workspace=ws)
    with pytest.raises(api.MinikvError):
        api.minikv_decode_attn_blk(shape, q, cache, n, n, SM, out, workspace=cache.workspace[:1024])
    with pytest.raises(api.MinikvError):
        api.kv_quantize_blk(shape, x[:1].expand(4, 2, 128), V[:4], n, cache)         # rows on top of each other
    i9 = [i([0] * 20) for _ in range(9)]
    for k in range(9):
        for bad in (i9[0].long(), i9[0].cpu(), i9[0][::2]):
            args = list(i9)
            args[k] = bad
            with pytest.raises(ValueError):
                api.kv_assign_blk(shape, *args)
    assert not bool(out.any()) and not bool(cache.K.view(torch.uint8).any())
