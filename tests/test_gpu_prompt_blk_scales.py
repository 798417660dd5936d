"""minikv_prompt_attn_blk where the blocks' scales decide: everything relative to what a row holds, nothing absolute but the output type's own
smallest step."""
import math

import pytest
import torch

from pages_common import HALF, SM, check_prompt, lse_tolerance
from oracle import pages
from test_gpu_prompt_blk import Case

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
LEAST = {F16: 2.0 ** -25, BF16: 2.0 ** -134}           # half a step of the type's subnormal numbers


def largest_products(c):
    """[T][Hq]: the largest weight times V scale that a row holds."""
    peak = torch.zeros(c.T, c.Hq, dtype=torch.float64)
    block, rep = c.Kc.shape[2], c.Hq // c.Kc.shape[1]
    for r in range(len(c.q_len)):
        at, end, L = int(c.cu[r]), int(c.cu[r + 1]), int(c.q_len[r])
        if end == at:
            continue
        j = torch.arange(L)
        b, o = c.table[r, j // block].long(), j % block
        hidden = j[None] > (L - (end - at) + torch.arange(end - at))[:, None]
        for hq in range(c.Hq):
            k = pages.decode_codes(c.Kc[b, hq // rep, o]) * c.Ks[b, hq // rep].double()[:, None]
            p = torch.softmax((c.q[at:end, hq].double() @ k.t() * SM).masked_fill(hidden, -math.inf), dim=1)
            peak[at:end, hq] = (p * c.Vs[b, hq // rep].double()).amax(dim=1)
    return peak


def check_relative(c):
    """A weight with its V scale is rounded once to 11 bits (2^-11), or below 2^-29 of the row's largest such product by at most 2^-40 of it, times
    a code of at most 448.  Its exponent is a score of 128 products, summed in fp32 (136 half steps of 2^-24 of the sum of magnitudes with
    the three roundings behind it, in numerator and denominator each) and log2 of scales and headroom: differences of numbers up to 160, each
    rounded (4 half steps of 2^-24 of them, twice).  Sums are fp32 (64 half steps counted); the result is rounded once to its type."""
    want, wlse, live, mean, score = pages.prompt_attn(c.q.cpu(), c.Kc, c.Ks, c.Vc, c.Vs, c.table, c.q_len, c.cu, SM)
    weight = 2.0 ** -11 + 2 * (136 * 2.0 ** -24 * score * 1.01) + 8 * 160 * 2.0 ** -24 + 64 * 2.0 ** -24
    small = int(c.q_len.max()) * 2.0 ** -40 * 448.0 * largest_products(c)[:, :, None]
    tol = mean * weight + small + want.abs() * HALF[c.dtype] * 1.001 + LEAST[c.dtype] * 1.01
    off = (c.out.cpu().double() - want).abs()[live]
    assert not off.isnan().any() and (off <= tol[live]).all(), "off by %.3g of what is allowed" % float((off / tol[live]).max())
    off = (c.lse.cpu().double() - wlse)[live].abs()
    assert (off <= lse_tolerance(wlse[live], score)).all()
    return want[live]


# few heads: blocks of 32 rows; many: of 128
@pytest.mark.parametrize("Hq,Hkv,n", [(4, 2, 20), (128, 128, 150)])
@pytest.mark.parametrize("block", [16, 64])
def test_small_scales_behind_blocks_of_zeros(Hq, Hkv, n, block):
    """Values of nothing (scale 0) in front: the row's products are those of the others, however small."""
    c = Case([3 * block], [n], Hq, Hkv, block, BF16, seed=50 + block)
    c.Vs[:] = 2.0 ** -60
    c.Vs[c.table[0, 0].long()] = 0.0
    c.Vs[c.table[0, 2].long()] = 0.0
    assert float(check_relative(c.run()).abs().min(dim=2).values.max()) > 0.0


@pytest.mark.parametrize("Hq,Hkv,n", [(4, 4, 3), (128, 128, 150)])
@pytest.mark.parametrize("block", [16, 32])
def test_values_of_zero_with_all_the_weight(Hq, Hkv, n, block):
    """A block of zeros whose keys win by 2^57: what is left of the row is the others', to full precision."""
    c = Case([4 * block], [n], Hq, Hkv, block, BF16, seed=60)
    c.Kc[:], c.Ks[:] = 0x38, 2.0 ** -3                 # keys of 1/8, of 1 in block 1
    c.Ks[c.table[0, 1].long()], c.Vs[c.table[0, 1].long()] = 1.0, 0.0
    x = torch.full_like(c.q, 4.0)
    c.q, c.q_dev = x, x.cuda()
    want = check_relative(c.run())
    assert 0.0 < float(want.abs().max()) < 2.0 ** -50  # (the test's own premise)


@pytest.mark.parametrize("Hq,Hkv,n", [(4, 2, 70), (128, 128, 150)])
@pytest.mark.parametrize("block", [16, 32, 64])
def test_larger_scales_behind_take_nothing_from_those_in_front(Hq, Hkv, n, block):
    """Each block's V scale 2^70 above the one before it: rows that end inside a block do not see the next one, whose values they share a tile with."""
    c = Case([0], [n], Hq, Hkv, block, BF16, seed=40 + block)
    for i, b in enumerate(c.table[0].tolist()):
        if b >= 0:
            c.Vs[b] = 2.0 ** (-100 + 70 * (i % 4))     # -100, -30, 40, 110
    want = check_relative(c.run())
    assert float(want[:16].abs().max()) < 2.0 ** -90         # (the test's own premise)


@pytest.mark.parametrize("Hq,Hkv,n", [(4, 2, 70), (128, 128, 150)])
@pytest.mark.parametrize("block", [16, 32, 64])
def test_smaller_scales_behind_that_have_all_the_weight(Hq, Hkv, n, block):
    """V scales fall by 2^70 and the keys' weights rise by 2^115: each block's values are those of the rows that end in it."""
    c = Case([0], [n], Hq, Hkv, block, BF16, seed=45 + block)
    c.Kc[:] = 0x38
    for i, b in enumerate(c.table[0].tolist()):
        if b >= 0:
            c.Vs[b], c.Ks[b] = 2.0 ** (100 - 70 * (i % 4)), 2.0 * (i % 4) + (0 if i < 4 else 8)
    x = torch.full_like(c.q, 3.5)
    c.q, c.q_dev = x, x.cuda()
    check_relative(c.run())


@pytest.mark.parametrize("held,n,Hq,Hkv", [(70, 20, 4, 2), (70, 150, 128, 128), (5000, 3, 2, 1)])
@pytest.mark.parametrize("exponent", [-112, -115, -126])
def test_the_smallest_scales(held, n, Hq, Hkv, exponent):
    """All of a row's V scales next to the smallest normal number: outputs are normal numbers of bf16 all the same."""
    c = Case([held], [n], Hq, Hkv, 32, BF16, seed=70)
    c.Vs[:] = 2.0 ** exponent
    assert float(check_relative(c.run()).abs().max()) > 2.0 ** exponent


@pytest.mark.parametrize("held,n,Hq,Hkv", [(70, 20, 4, 2), (70, 150, 128, 128)])
def test_the_largest_scales(held, n, Hq, Hkv):
    c = Case([held], [n], Hq, Hkv, 16, BF16, seed=71)
    c.Vs[:] = 2.0 ** 117                               # (times 448: below 2^126)
    check_relative(c.run())


@pytest.mark.parametrize("Hq,Hkv,n", [(4, 2, 30), (128, 128, 150)])
def test_keys_of_nothing_and_queries_of_any_size(Hq, Hkv, n):
    """Raw products of up to 2^126 with keys of scale 0: scores of 0."""
    c = Case([64], [n], Hq, Hkv, 16, BF16, seed=80, gain=2.0 ** 112)
    c.Ks *= 2.0 ** -112
    zero = c.table[0, 1].long()
    c.Kc[zero], c.Ks[zero] = 0x7e, 0.0
    check_relative(c.run())


@pytest.mark.parametrize("Hq,Hkv,n", [(4, 2, 30), (128, 128, 150)])
@pytest.mark.parametrize("block", [16, 32, 64])
@pytest.mark.parametrize("scale", [math.inf, math.nan, 3e38])
def test_absent_blocks_beside_a_free_block_of_any_scale(Hq, Hkv, n, block, scale):
    """Block 0 is in no table, and holds what its memory held."""
    c = Case([3 * block], [n], Hq, Hkv, block, F16, seed=90)
    spare = (set(range(c.N)) - set(c.table[0].tolist())).pop()
    c.table[c.table == 0] = spare
    c.table[0, 1] = -1
    c.Ks[0], c.Vs[0], c.Kc[0], c.Vc[0] = scale, scale, 0x7f, 0xff
    c.run()
    c.Ks[0], c.Vs[0] = 1.0, 1.0
    check_prompt(c.shape, c.q, (c.Kc, c.Ks, c.Vc, c.Vs), c.table, c.q_len, c.cu, c.out, c.lse)
