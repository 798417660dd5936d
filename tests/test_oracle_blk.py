"""Pins of the plain definitions that the paged cache and the packed prompts are checked against, and the refusals of their entry
points (no GPU needed)."""
import ctypes as C
import math

import pytest
import torch

from oracle import blk


def test_e4m3_values_and_rounding():
    v = blk.e4m3_values()
    assert v[0x7e] == 448.0 and v[0x08] == 2.0 ** -6 and v[0x01] == 2.0 ** -9 and v[0x38] == 1.0 and v[0xb8] == -1.0
    assert math.isnan(v[0x7f]) and math.isnan(v[0xff])
    torch_values = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    assert torch.equal(v.nan_to_num(nan=7e9), torch_values.nan_to_num(nan=7e9))
    good = torch.tensor([c for c in range(256) if c & 127 != 127], dtype=torch.uint8)
    assert torch.equal(blk.encode(blk.decode_codes(good)), good)                     # every value is its own nearest
    assert int(blk.encode(torch.tensor([math.nan], dtype=torch.float64))[0]) & 127 == 127
    # ties go to the even code: halfway between neighbours of either parity, subnormal ones too
    for lo in range(0, 126):
        mid = (v[lo] + v[lo + 1]) / 2
        assert int(blk.encode(mid.reshape(1))[0]) == (lo if lo % 2 == 0 else lo + 1)
    x = torch.randn(4096, generator=torch.Generator().manual_seed(1)) * 100
    x = x.clamp(-448, 448)
    assert torch.equal(blk.encode(x.double()).int(), x.to(torch.float8_e4m3fn).view(torch.uint8).int())


@pytest.mark.parametrize("amax,want", [(0.0, 0.0), (448.0, 1.0), (448.5, 2.0), (447.0, 1.0), (224.0, 0.5), (225.0, 1.0), (1e-45, 2.0 ** -126),
                                       (65504.0, 256.0), (2.0 ** -24, 2.0 ** -32)])
def test_scale_is_the_smallest_power_of_two(amax, want):
    assert blk.scale_for(amax) == want
    if amax and want > 2.0 ** -126:
        assert amax <= 448 * want and amax > 448 * want / 2


def test_filing_by_hand():
    codes, scales = torch.zeros(2, 1, 16, 128, dtype=torch.uint8), torch.zeros(2, 1)
    x = torch.zeros(1, 1, 128)
    x[0, 0, 0], x[0, 0, 1] = 448.0, 3.0
    c1, s1 = blk.file_rows(x, codes, scales, torch.tensor([16]))                     # block 1, offset 0
    assert s1.tolist() == [[0.0], [1.0]] and blk.decode_codes(c1[1, 0, 0, :3]).tolist() == [448.0, 3.0, 0.0]
    x[0, 0, 0], x[0, 0, 1] = 896.0, 2.0 ** -9                                        # offset 1: the scale doubles, row 0 keeps its values
    c2, s2 = blk.file_rows(x, c1, s1, torch.tensor([17]))
    assert s2.tolist() == [[0.0], [2.0]]
    assert (blk.decode_codes(c2[1, 0, :2, :2]) * 2).tolist() == [[448.0, 3.0], [896.0, 0.0]]    # (a tie between 0 and 2^-8: even)
    c3, s3 = blk.file_rows(x / 896, c2, s2, torch.tensor([16]))                      # offset 0 again: the block starts afresh
    assert s3[1, 0] == 2.0 ** -8 and torch.equal(c3[1, 0, 1], c2[1, 0, 1])
    c4, s4 = blk.file_rows(x, c3, s3, torch.tensor([-1]))                            # padding
    assert torch.equal(c4, c3) and torch.equal(s4, s3)


def test_assignment_by_hand():
    table = [[9, -1], [4, 5], [-1, -1], [7, -1], [-1, -1]]
    got = blk.assign([16, 20, 0, 3, 0], [1, -1, 17, 0, 1], table, [0, 1, 2, 3, 6, 8, 10, 11, 99, 99], [1, 3], 16, 40)
    assert got["cu"] == [0, 1, 1, 18, 18, 19]
    assert got["table"] == [[9, 1], [4, 5], [2, 3], [7, -1], [-1, -1]]               # the last one finds no block
    assert got["slots"] == [16] + [32 + i for i in range(16)] + [48, -1] + [-1] * 21
    assert got["q_len"] == [17, 0, 17, 3, 0]
    assert got["state"] == [4, 2] and got["ring"] == [0, 1, 2, 3, 4, 5, 10, 11, 99, 99]


def test_attention_definitions_on_cases_worked_by_hand():
    # equal keys: the mean of the values; an absent block and a request without tokens
    Kc, Vc = blk.encode(torch.ones(3, 1, 16, 128, dtype=torch.float64)), torch.zeros(3, 1, 16, 128, dtype=torch.uint8)
    Vc[2, 0] = blk.encode(torch.full((16, 128), 4.0, dtype=torch.float64))
    one = torch.ones(3, 1)
    table = torch.tensor([[1, 2], [2, 1], [-1, 2], [0, 0]])
    out, mean, _ = blk.decode_attn(torch.ones(4, 1, 128), Kc, one, Vc, one * 0.5, table, [24, 24, 32, 0], 0.1)
    assert torch.allclose(out[:, 0, 0], torch.tensor([2 * 8 / 24, 2 * 16 / 24, 2.0, 0.0], dtype=torch.float64)) and torch.equal(out, mean)
    # packed prompts: each like alone
    g = torch.Generator().manual_seed(2)
    Q, K, V = torch.randn(9, 4, 128, generator=g), torch.randn(9, 2, 128, generator=g), torch.randn(9, 2, 128, generator=g)
    X, lse, A, _, _ = blk.prompt_attn(Q, K, V, [0, 4, 4, 9], 0.1)
    X1, lse1, A1, _, _ = blk.prompt_attn(Q[4:], K[4:], V[4:], [0, 5], 0.1)
    assert torch.equal(X[4:], X1) and torch.equal(lse[16:], lse1) and torch.equal(A[16:], A1)
    assert torch.allclose(X[4], V[4].double()[[0, 0, 1, 1]]) and torch.allclose(A[:16].reshape(4, 4).sum(1), torch.full((4,), 4.0, dtype=torch.float64))


# ---------------------------------------------------------------------------------------------------------
# refusals: on the host, before anything is launched

@pytest.fixture(scope="module")
def api():
    import os
    from paper_2411_18077_amd import api as _api
    if not os.path.exists(_api.LIB_PATH):
        from paper_2411_18077_amd import build
        build.build(verbose=False)
    return _api


P = C.c_void_p
GOOD = dict(R=4, Hq=8, Hkv=2, D=128, block=32, n_blocks=100, max_blocks=20, dtype=0)


ALL = ("assign", "file", "attend")


def calls(api, shape, which=ALL, p=P(0x1000), cache=None, stride=1024, kv_stride=256, sm=0.1, wsb=1 << 30, n_slots=4, n_tok=4, nxt=P(0x2000)):
    """Status codes of the calls named (each has something wrong with it: nothing may be launched with these pointers)."""
    l, s = api.lib(), C.byref(shape)
    cache = C.byref(cache or api.MinikvBlkCache(*[0x1000] * 4))
    call = dict(assign=lambda: l.kv_assign_blk(s, p, p, p, p, p, nxt, nxt, p, p, n_slots, None),
                file=lambda: l.kv_quantize_blk(s, n_tok, p, kv_stride, p, kv_stride, p, cache, None),
                attend=lambda: l.minikv_decode_attn_blk(s, p, stride, cache, p, p, sm, p, p, wsb, None))
    return [call[w]() for w in which]


@pytest.mark.parametrize("bad,status", [
    (dict(R=0), -1), (dict(R=8193), -1), (dict(Hq=7), -1), (dict(Hkv=0), -1), (dict(Hq=18), -2), (dict(D=64), -2), (dict(block=8), -2),
    (dict(block=48), -2), (dict(block=256), -2), (dict(n_blocks=0), -1), (dict(max_blocks=0), -1), (dict(dtype=2), -2), (dict(dtype=-1), -2),
    (dict(n_blocks=1 << 26), -1), (dict(max_blocks=(1 << 25) + 1), -1), (dict(R=8192, Hq=64, Hkv=64, max_blocks=10000), -1),
])
def test_paged_shapes_are_checked_on_the_host(api, bad, status):
    shape = api.MinikvBlkShape(*{**GOOD, **bad}.values())
    assert calls(api, shape) == [status] * 3
    assert api.lib().minikv_blk_cache_bytes(C.byref(shape), 0) == 0 and api.lib().minikv_blk_workspace_bytes(C.byref(shape)) == 0


def test_paged_sizes_and_arguments_are_checked_on_the_host(api):
    l, shape = api.lib(), api.MinikvBlkShape(*GOOD.values())
    assert [l.minikv_blk_cache_bytes(C.byref(shape), i) for i in range(10)] == [100 * 2 * 32 * 128, 800, 0, 100 * 2 * 32 * 128, 800, 0, 0, 0, 0, 0]
    need = l.minikv_blk_workspace_bytes(C.byref(shape))
    assert need == 256 * (4 * 5 + 2 * 4 * 8 * 130)
    assert l.minikv_blk_cache_bytes(None, 0) == 0
    rows = ("file", "attend")
    assert calls(api, shape, p=None) == [-1] * 3 and calls(api, shape, p=P(0x1002)) == [-1] * 3
    assert calls(api, shape, rows, p=P(0x1008)) == [-1] * 2                          # rows: 16 bytes
    assert calls(api, shape, rows, cache=api.MinikvBlkCache(0x1000, 0x1008, 0x1000, 0x1000)) == [-1] * 2
    assert calls(api, shape, rows, cache=api.MinikvBlkCache(0x1000, 0x1000, 0x1000, 0)) == [-1] * 2
    for stride in (1016, 1028, -1024, 0, (1 << 23) + 8):
        assert calls(api, shape, ["attend"], stride=stride) == [-1]
    for stride in (248, 260, -256, 0, (1 << 23) + 8):
        assert calls(api, shape, ["file"], kv_stride=stride) == [-1]
    for sm in (math.nan, math.inf):
        assert calls(api, shape, ["attend"], sm=sm) == [-1]
    assert calls(api, shape, ["attend"], wsb=need - 1) == [-3]
    assert calls(api, shape, ["assign"], nxt=P(0x1000)) == [-1]                      # lengths read and written at one place
    assert calls(api, shape, ["assign"], n_slots=-1) == [-1] and calls(api, shape, ["file"], n_tok=-1) == [-1]
    assert l.kv_quantize_blk(C.byref(shape), 0, None, 0, None, 0, None, C.byref(api.MinikvBlkCache(*[0x1000] * 4)), None) == 0
    assert calls(api, shape, ["file"], n_tok=1 << 29) == [-1]                        # 2^30 rows of K and as many of V


def test_the_binding_refuses_what_a_pointer_does_not_tell(api):
    """Types, sizes, strides; and host memory, which everything is here (the checks before that one name what they refuse)."""
    shape = api.make_blk_shape(4, 8, 2, 128, 32, 10, 5, torch.float16)
    cache = api.BlkCache(shape, device="cpu")
    assert cache.K.shape == (10, 2, 32, 128) and cache.Ks.shape == (10, 2) and not bool(cache.workspace.any())
    with pytest.raises(AttributeError):
        cache.K = cache.V
    x = torch.zeros(4, 2, 128, dtype=torch.float16)
    i = torch.zeros(64, dtype=torch.int32)
    heads = "rows are"
    for K, V, slots, what in ((x.bfloat16(), x, i, "K: got"), (x, x[:3], i, "4 tokens, V 3"), (x[:, :1], x, i, heads), (x.float(), x, i, "K: got"),
                              (x.transpose(1, 2).contiguous().transpose(1, 2), x, i, heads), (torch.zeros(4, 3, 128, dtype=torch.float16), x, i, heads),
                              (x, x, i, "K is on cpu")):
        with pytest.raises(ValueError, match=what):
            api.kv_quantize_blk(shape, K, V, slots, cache, stream=0)
    q = torch.zeros(4, 8, 128, dtype=torch.float16)
    for k in range(9):
        for bad in (i.long(), i[::2], i[:0] if k < 8 else i.float()):
            args = [i] * 9
            args[k] = bad
            with pytest.raises(ValueError, match="contiguous tensor of at least" if k == 0 else "contiguous tensor|is on cpu"):
                api.kv_assign_blk(shape, *args, stream=0)
    with pytest.raises(ValueError, match="q is on cpu"):
        api.minikv_decode_attn_blk(shape, q, cache, i, i, 0.1, q.clone(), stream=0)
    with pytest.raises(ValueError, match="K: a contiguous"):
        api.BlkCache(shape, K=cache.K[:5], V=cache.V, Ks=cache.Ks, Vs=cache.Vs)
    with pytest.raises(ValueError, match="float16 or torch.bfloat16"):
        api.make_blk_shape(4, 8, 2, 128, 32, 10, 5, torch.float32)
    with pytest.raises(ValueError, match="invalid shape"):
        api.BlkCache(api.make_blk_shape(4, 8, 3, 128, 32, 10, 5, torch.float16), device="cpu")


def test_packed_prompt_arguments_are_checked_on_the_host(api):
    l = api.lib()
    good = dict(B=2, Hq=8, Hkv=2, T=100, max_len=60, dtype=1, Q=P(0x1000), qs=1536, K=P(0x1000), ks=1536, V=P(0x1000), vs=256,
                cu=P(0x1000), sm=0.1, X=P(0x1000), lse=P(0x1000), A=None)
    call = lambda **bad: l.selective_flash_attn_packed(*{**good, **bad}.values(), None)  # noqa: E731
    for bad in (dict(B=0), dict(B=8193), dict(Hq=7), dict(Hkv=0), dict(T=-1), dict(max_len=-1), dict(max_len=(1 << 23) + 1), dict(Q=None),
                dict(T=2 ** 31 // 8), dict(K=P(0x1008)), dict(V=None), dict(cu=None), dict(cu=P(0x1002)), dict(X=P(0x1004)), dict(lse=None),
                dict(lse=P(0x1001)), dict(A=P(0x1002)), dict(sm=0.0), dict(sm=-1.0), dict(sm=math.nan), dict(sm=math.inf), dict(qs=1020),
                dict(qs=1016), dict(ks=128), dict(vs=252), dict(vs=-256), dict(qs=(1 << 23) + 8)):
        assert call(**bad) == -1, bad
    assert call(B=8192, T=8192, max_len=9, Hq=4096, Hkv=4096, qs=4096 * 128, ks=4096 * 128, vs=4096 * 128) == -1      # too large a launch
    assert call(dtype=2) == -2 and call(dtype=-1) == -2
    assert call(T=0, Q=None, K=None, V=None, X=None, lse=None) == 0 and call(max_len=0) == 0                 # no rows


def test_the_binding_refuses_packed_rows_that_do_not_fit(api):
    x, kv = torch.zeros(10, 8, 128, dtype=torch.bfloat16), torch.zeros(10, 2, 128, dtype=torch.bfloat16)
    cu, f = torch.tensor([0, 4, 10], dtype=torch.int32), torch.zeros(80)
    good = dict(T=10, Q=x, K=kv, V=kv, cu=cu, X=x.clone(), lse=f, A=f.clone())
    for what, bad in (("Q: got", dict(Q=x.float())), ("rows are", dict(Q=x[:, :7])), ("Q is on cpu", dict())):
        a = {**good, **bad}
        with pytest.raises(ValueError, match=what):
            api.selective_flash_attn_packed(2, 8, 2, a["T"], 6, a["Q"], a["K"], a["V"], a["cu"], 0.1, a["X"], a["lse"], a["A"], stream=0)
