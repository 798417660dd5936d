"""Inputs and tolerances shared by the tests of the paged 8-bit cache and of packed prompts."""
import torch

from oracle import blk

SM = 128 ** -0.5
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}          # half a step, relative


def rand_cache(N, Hkv, block, seed, spread=0, subnormal=False):
    """Codes of N(0,1) rows under their power-of-two scale, blocks times 2^(-spread .. spread); the oracle's own rounding."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(N, Hkv, block, 128, generator=g, dtype=torch.float64)
    x *= 2.0 ** torch.randint(-spread, spread + 1, (N, Hkv, 1, 1), generator=g)
    amax = x.abs().amax(dim=(2, 3))
    s = torch.tensor([[blk.scale_for(float(a)) for a in row] for row in amax], dtype=torch.float64)
    if subnormal:
        s = s * 256.0
    return blk.encode(x / s[:, :, None, None]), s.float()


def tables(lens, block, width, n_blocks, seed):
    """Disjoint shuffled blocks for every request; unused entries hold an index that must not be read."""
    order = torch.randperm(n_blocks, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    t = torch.full((len(lens), width), -7, dtype=torch.int32)
    at = 0
    for r, n in enumerate(lens):
        k = -(-n // block)
        t[r, :k] = order[at:at + k]
        at += k
    return t


def attn_tolerance(out, mean, score, tokens, vmax, weight_half, dtype):
    """Per output value: every weight is rounded once (weight_half, relative; below fp16's or bf16's normal numbers by at most
    2^-25 of the largest weight, 1 in each part of a row), the score of a weight is a sum of 128 products in fp32
    and passes three more fp32 roundings (136 half steps of 2^-24 of the sum of magnitudes, for numerator and
    denominator each), outputs and sums are fp32 (a half step per addition of at most `tokens`, each of a part of the whole: 64 of
    them counted), and the result is rounded once to its type."""
    weight = weight_half + 2 * (136 * 2.0 ** -24 * score * 1.01) + 64 * 2.0 ** -24
    return mean * weight + tokens * 2.0 ** -25 * vmax + out.abs() * HALF[dtype] * 1.001 + 2.0 ** -24
