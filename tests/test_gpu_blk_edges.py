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
