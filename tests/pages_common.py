"""Inputs and tolerances shared by the tests of requests that share blocks of the paged 8-bit cache."""
import math

import torch

from blk_common import HALF, SM, rand_cache, tables  # noqa: F401
from oracle import pages
from paper_2411_18077_amd import api

E4M3 = torch.float8_e4m3fn


def make_cache(shape, Kc, Ks, Vc, Vs):
    up = lambda t: t.cuda()  # noqa: E731
    return api.BlkCache(shape, K=up(Kc).view(E4M3), V=up(Vc).view(E4M3), Ks=up(Ks), Vs=up(Vs))


def ints(v):
    return torch.tensor(v, dtype=torch.int32)


def prompt_tolerance(out, mean, score, tokens, vmax, spread, dtype):
    """Per output value.  A weight with its V scale is rounded once to fp16 (2^-11; below 2^-29 of the row's largest by at most 2^-40 of it, each
    times a value of at most vmax).  Its exponent is a score of 128 products, summed in fp32 (136 half steps of 2^-24 of the sum of magnitudes
    with the three roundings behind it, in numerator and denominator each), and log2 of scales: differences of numbers up to
    `spread` (log2 of the scales and of the headroom), each rounded (4 half steps of 2^-24 of them, twice).  Sums of weights and of
    products are fp32, a half step per addition of a part of the whole (64 counted), and the result is rounded once to its type."""
    weight = 2.0 ** -11 + 2 * (136 * 2.0 ** -24 * score * 1.01) + 8 * spread * 2.0 ** -24 + 64 * 2.0 ** -24
    return mean * weight + tokens * 2.0 ** -40 * vmax + out.abs() * HALF[dtype] * 1.001 + 2.0 ** -25


def lse_tolerance(lse, score):
    """Scores as above; sum, logarithm and product round a few times."""
    return 136 * 2.0 ** -24 * score * 1.01 + 80 * 2.0 ** -24 + lse.abs() * 2.0 ** -21


def check_prompt(shape, q, cache_cpu, table, q_len, cu, out, lse, before=7.0, spread=64, sm=SM):
    """out and lse (device) against the definition; rows of no request still hold `before`."""
    Kc, Ks, Vc, Vs = cache_cpu
    want, wlse, live, mean, score = pages.prompt_attn(q.cpu(), Kc, Ks, Vc, Vs, table, q_len, cu, sm)
    got, glse = out.cpu().double(), lse.cpu().double()
    assert (got[~live] == before).all() and (glse[~live] == before).all()
    vmax = float((torch.nan_to_num(pages.decode_codes(Vc)).abs().amax(dim=(2, 3)) * Vs.double().abs()).max())
    tol = prompt_tolerance(want, mean, score, max(min(int(max(q_len)), table.shape[1] * Kc.shape[2]), 1), vmax, spread, out.dtype)
    off = (got - want).abs()[live]
    assert not off.isnan().any() and (off <= tol[live]).all(), "off by %.3g of what is allowed" % float((off / tol[live]).max())
    none = wlse == -math.inf
    assert (glse[live][none[live]] == -math.inf).all() and (got[live][none[live]] == 0).all()
    some = live[:, None] & ~none
    off = (glse - wlse)[some].abs()
    assert (off <= lse_tolerance(wlse[some], score)).all(), "lse off by %.3g" % float(off.max())
