"""minikv_norm_rope against its definition in 64 bits."""
import math
from fractions import Fraction

import pytest
import torch

from blk_common import HALF
from oracle import pages
from paper_2411_18077_amd import api

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def tolerance(want, size, dtype):
    """The norm (a sum of 128 squares over sixteen lanes, a reciprocal root, three products) is right to 2^-20, the angle to 2^-20 and its
    sine and cosine to 2^-24 beside that, the turn rounds three times: 2^-19 of |u| + |v|; then one rounding to the type."""
    return size * 2.0 ** -19 + want.abs() * HALF[dtype] * 1.001 + 2.0 ** -25


def run_case(T, Hq, Hkv, rot, adjacent, wq, wk, dtype, far, fused=True, inplace=False, eps=1e-6, gain=1.0, seed=0, freq=10000.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(T, Hq + 2 * Hkv, 128, generator=g) * gain).to(dtype)
    pos = torch.randint(0, far, (T,), generator=g, dtype=torch.int64).to(torch.int32)
    if T > 3:
        pos[1], pos[T - 1] = -1, far - 1
    w = [(1 + 0.3 * torch.randn(128, generator=g)).to(dtype) if on else None for on in (wq, wk)]
    inv = (freq ** (-torch.arange(rot // 2, dtype=torch.float64) / max(rot // 2, 1))).float()
    d = x.cuda()
    Q, K = d[:, :Hq], d[:, Hq:Hq + Hkv]
    if not fused:
        Q, K = Q.contiguous(), K.contiguous()
    qo, ko = (Q, K) if inplace else (torch.full((T + 2, Hq, 128), 7.0, dtype=dtype, device="cuda"), torch.full((T + 2, Hkv, 128), 7.0, dtype=dtype, device="cuda"))
    up = lambda t: None if t is None else t.cuda()  # noqa: E731
    api.minikv_norm_rope(Hq, Hkv, T, Q, K, up(w[0]), up(w[1]), eps, up(inv), rot, adjacent, up(pos), qo, ko)
    for first, H, weight, got in ((0, Hq, w[0], qo), (Hq, Hkv, w[1], ko)):
        rows = x[:, first:first + H]
        want, size = pages.norm_rope(rows, weight, eps, inv, rot, adjacent, pos)
        got = got.cpu().double()
        if not inplace:
            assert (got[T:] == 7.0).all()
            left = pos < 0
            assert (got[:T][left] == 7.0).all()
            got = torch.where(left[:, None, None], rows.double(), got[:T])
        off, tol = (got - want).abs(), tolerance(want, size, dtype)
        assert (off <= tol).all(), "off by %.3g of what is allowed" % float((off / tol).max())
    if inplace and fused:
        assert torch.equal(d[:, Hq + Hkv:].cpu(), x[:, Hq + Hkv:])


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("rot", [0, 16, 48, 64, 96, 128])
def test_rotations(rot, adjacent, dtype):
    run_case(9, 8, 2, rot, adjacent, True, True, dtype, 10000, seed=rot)


@pytest.mark.parametrize("wq,wk", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("adjacent", [False, True])
def test_rows_without_norm(wq, wk, adjacent):
    run_case(5, 6, 3, 128, adjacent, wq, wk, F16, 500, seed=2)


@pytest.mark.parametrize("T,Hq,Hkv", [(1, 1, 1), (1, 32, 8), (2, 5, 5), (3, 7, 1), (64, 32, 8), (65, 12, 4), (300, 33, 11), (700, 8, 8), (1, 200, 100),
                                      (2500, 16, 2)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_sizes(T, Hq, Hkv, dtype):
    run_case(T, Hq, Hkv, 128, False, True, True, dtype, 4096, seed=T)


@pytest.mark.parametrize("far", [1, 2, 100000, 1 << 20, 2 ** 31 - 1])
@pytest.mark.parametrize("adjacent", [False, True])
def test_far_positions(far, adjacent):
    run_case(40, 4, 2, 128, adjacent, True, True, F16, far, seed=9)


@pytest.mark.parametrize("freq", [1.5, 500000.0])
def test_frequencies(freq):
    run_case(40, 4, 2, 64, False, True, True, F16, 200000, seed=9, freq=freq)


@pytest.mark.parametrize("fused", [True, False])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("T", [1, 6, 130])
def test_in_place(fused, dtype, T):
    run_case(T, 8, 2, 96, False, True, True, dtype, 3000, fused=fused, inplace=True, seed=5)


@pytest.mark.parametrize("gain,eps", [(1e-4, 1e-6), (0.0, 1e-5), (300.0, 0.0), (1.0, 0.5)])
def test_magnitudes(gain, eps):
    run_case(6, 4, 4, 128, False, True, True, F16, 3000, eps=eps, gain=gain, seed=6)


def test_largest_rows():
    """Rows of the type's largest value: squares of fp16 sum to below 2^39."""
    x = torch.full((2, 2, 128), 65504.0, dtype=F16, device="cuda")
    w = torch.ones(128, dtype=F16, device="cuda")
    out, k = torch.zeros_like(x), torch.zeros_like(x)
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    api.minikv_norm_rope(2, 2, 2, x, x, w, None, 1e-6, None, 0, False, pos, out, k)
    assert ((out - 1).abs() <= 2.0 ** -10).all() and torch.equal(k, x)


def test_captured_and_on_another_stream():
    T, Hq, Hkv = 33, 8, 2
    g = torch.Generator().manual_seed(1)
    x = torch.randn(T, Hq + Hkv, 128, generator=g).to(BF16).cuda()
    inv = (10000.0 ** (-torch.arange(64) / 64)).cuda()
    w = torch.ones(128, dtype=BF16, device="cuda")
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    q, k = torch.zeros(T, Hq, 128, dtype=BF16, device="cuda"), torch.zeros(T, Hkv, 128, dtype=BF16, device="cuda")
    call = lambda st=None: api.minikv_norm_rope(Hq, Hkv, T, x[:, :Hq], x[:, Hq:], w, w, 1e-6, inv, 128, False, pos, q, k, stream=st)  # noqa: E731
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    s.synchronize()
    first = q.clone(), k.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):
        pos += 1
        q.zero_(), k.zero_()
        graph.replay()
        got = q.clone(), k.clone()
        q.zero_(), k.zero_()
        call()
        assert torch.equal(got[0], q) and torch.equal(got[1], k) and not torch.equal(q, first[0])


def test_many_tokens():
    """Tokens 2^23 elements apart: rows beyond 2^32 bytes."""
    T, stride = 300, 1 << 23
    buf = torch.zeros(T * stride, dtype=BF16, device="cuda")
    rows = buf.as_strided((T, 2, 128), (stride, 128, 1))
    src = torch.randn(T, 2, 128, generator=torch.Generator().manual_seed(3)).to(BF16)
    rows.copy_(src.cuda())
    inv = (10000.0 ** (-torch.arange(64) / 64)).float()
    pos = torch.arange(T, dtype=torch.int32)
    q, k = torch.zeros(T, 1, 128, dtype=BF16, device="cuda"), torch.zeros(T, 1, 128, dtype=BF16, device="cuda")
    api.minikv_norm_rope(1, 1, T, rows[:, :1], rows[:, 1:], None, None, 0.0, inv.cuda(), 128, False, pos.cuda(), q, k)
    for got, h in ((q, 0), (k, 1)):
        want, size = pages.norm_rope(src[:, h:h + 1], None, 0.0, inv, 128, False, pos)
        assert ((got.cpu().double() - want).abs() <= tolerance(want, size, BF16)).all()


def exact_turn(pos, freq):
    """cos and sin of pos * freq, the whole turns dropped in rational numbers."""
    two_pi = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459")
    a = Fraction(pos) * Fraction(freq)
    a -= two_pi * round(a / two_pi)
    return math.cos(a), math.sin(a)


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("top", [1.0, 1000.0, 2.0 ** 20, 2.0 ** 24])
def test_angles_of_any_frequency(top, adjacent):
    """Angles up to 2^31 radians are right to 2^-20: pairs (1, 0) become (cos, sin)."""
    most = int((2 ** 31 - 1) / top)
    pos = [max(most - 2 * i, 0) for i in range(6)] + [most // 175, 1, 0]
    inv = [(-1) ** i * top * (1 - i / 1024.1) for i in range(64)]
    inv = torch.tensor(inv, dtype=torch.float32)
    q = torch.zeros(len(pos), 1, 128, dtype=BF16)
    u, v = (slice(0, None, 2), slice(1, None, 2)) if adjacent else (slice(0, 64), slice(64, None))
    q[:, :, u] = 1.0
    out, ko = torch.zeros_like(q).cuda(), torch.zeros_like(q).cuda()
    api.minikv_norm_rope(1, 1, len(pos), q.cuda(), q.cuda(), None, None, 0.0, inv.cuda(), 128, adjacent, torch.tensor(pos, dtype=torch.int32).cuda(), out, ko)
    got = out.cpu().double()[:, 0]
    want = torch.tensor([[exact_turn(p, float(f)) for f in inv] for p in pos], dtype=torch.float64)
    for k, part in enumerate((u, v)):
        off = (got[:, part] - want[:, :, k]).abs()
        assert (off <= want[:, :, k].abs() * HALF[BF16] + 2.0 ** -19).all(), float(off.max())
