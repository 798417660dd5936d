"""What minikv_norm_rope, minikv_prompt_attn_blk, kv_fork_blk, kv_copy_blk, kv_free_blk and kv_compact_blk refuse before anything is launched,
by the library and by the binding (no GPU: every call here is refused, or has nothing to do)."""
import ctypes as C
import math
import os

import pytest
import torch


@pytest.fixture(scope="module")
def api():
    from paper_2411_18077_amd import api as _api
    if not os.path.exists(_api.LIB_PATH):
        from paper_2411_18077_amd import build
        build.build(verbose=False)
    return _api


def shape(api, **kw):
    base = dict(R=4, Hq=8, Hkv=2, D=128, block=16, n_blocks=40, max_blocks=6, dtype=torch.float16)
    base.update(kw)
    return api.make_blk_shape(**base)


BAD_SHAPES = [(dict(D=64), -2), (dict(block=8), -2), (dict(Hq=7), -1), (dict(Hq=18), -2), (dict(R=0), -1), (dict(R=8193), -1), (dict(n_blocks=0), -1),
              (dict(max_blocks=0), -1), (dict(n_blocks=1 << 28), -1)]


def call(api, name, args):
    return getattr(api.lib(), name)(*args)


def norm_args(**kw):
    a = dict(Hq=8, Hkv=2, T=5, dtype=0, Q=0x1000, qs=1280, K=0x2000, ks=1280, wq=0x3000, wk=0x3100, eps=1e-6, inv=0x4000, rot=128, adjacent=0, pos=0x5000,
             qo=0x6000, qos=1024, ko=0x7000, kos=256)
    a.update(kw)
    return list(a.values()) + [None]


@pytest.mark.parametrize("bad,status", [
    (dict(Hq=0), -1), (dict(Hkv=0), -1), (dict(T=-1), -1), (dict(T=(1 << 25) + 1), -1), (dict(dtype=2), -2), (dict(dtype=-1), -2), (dict(rot=8), -1),
    (dict(rot=144), -1), (dict(rot=-16), -1), (dict(rot=24), -1), (dict(eps=-1.0), -1), (dict(eps=math.nan), -1), (dict(eps=math.inf), -1),
    (dict(Q=None), -1), (dict(Q=0x1008), -1), (dict(K=None), -1), (dict(K=0x1002), -1), (dict(wq=0x3008), -1), (dict(wk=2), -1), (dict(inv=None), -1),
    (dict(inv=0x4002), -1), (dict(pos=None), -1), (dict(pos=0x5001), -1), (dict(qo=None), -1), (dict(qo=0x6004), -1), (dict(ko=None), -1),
    (dict(qs=1016), -1), (dict(qs=1281), -1), (dict(ks=128), -1), (dict(qos=8), -1), (dict(kos=(1 << 23) + 8), -1), (dict(qo=0x1000), -1),
    (dict(ko=0x2000), -1),
])
def test_norm_rope_refuses(api, bad, status):
    assert call(api, "minikv_norm_rope", norm_args(**bad)) == status


def test_norm_rope_without_tokens(api):
    assert call(api, "minikv_norm_rope", norm_args(T=0, Q=None, K=None, pos=None, qo=None, ko=None)) == 0


def prompt_args(api, s=None, **kw):
    a = dict(s=C.byref(s or shape(api)), T=5, q=0x1000, qs=1024, c=C.byref(api.MinikvBlkCache(*[0x1000] * 4)), table=0x1000, q_len=0x1000, cu=0x1000, sm=0.1,
             out=0x1000, lse=0x1000, ws=0x1000, n=1 << 40)
    a.update(kw)
    return list(a.values()) + [None]


@pytest.mark.parametrize("bad,status", BAD_SHAPES)
def test_shapes_are_refused(api, bad, status):
    s = shape(api, **bad)
    b = C.byref(s)
    c = api.MinikvBlkCache(*[0x1000] * 4)
    p = [0x1000 * (i + 1) for i in range(12)]
    assert call(api, "minikv_prompt_attn_blk", prompt_args(api, s)) == status
    assert call(api, "kv_fork_blk", [b, *p[:11], None]) == status
    assert call(api, "kv_copy_blk", [b, 1, C.byref(c), 3, p[0], p[1], None]) == status
    assert call(api, "kv_free_blk", [b, *p[:5], 1 << 40, None]) == status
    assert call(api, "kv_compact_blk", [b, *p[:5], 3, *p[5:8], 1 << 40, None]) == status
    assert api.kv_free_workspace_bytes(s) == 0 and api.minikv_prompt_blk_workspace_bytes(s, 5) == 0


@pytest.mark.parametrize("bad,status", [
    (dict(T=-1), -1), (dict(T=1 << 29), -1), (dict(q=None), -1), (dict(q=0x1008), -1), (dict(qs=1016), -1), (dict(qs=1028), -1), (dict(qs=(1 << 23) + 8), -1),
    (dict(c=None), -1), (dict(table=None), -1), (dict(q_len=0x1001), -1), (dict(cu=None), -1), (dict(sm=0.0), -1), (dict(sm=-1.0), -1),
    (dict(sm=math.nan), -1), (dict(sm=math.inf), -1), (dict(out=None), -1), (dict(out=0x1002), -1), (dict(lse=0x1002), -1), (dict(ws=None), -1),
    (dict(ws=0x1008), -1), (dict(n=100), -3),
])
def test_prompt_attn_refuses(api, bad, status):
    assert call(api, "minikv_prompt_attn_blk", prompt_args(api, **bad)) == status


def test_prompt_attn_without_rows(api):
    assert call(api, "minikv_prompt_attn_blk", prompt_args(api, T=0, q=None, out=None, lse=None, ws=None, n=0)) == 0


def test_prompt_attn_refuses_more_row_blocks_than_a_launch_counts(api):
    s = shape(api, Hq=512, Hkv=512, n_blocks=1000)
    T = 4000000
    assert call(api, "minikv_prompt_attn_blk", prompt_args(api, s, T=T, qs=65536)) == -1


@pytest.mark.parametrize("R,T", [(1, (1 << 26) + 1024), (1, (1 << 26) - (1 << 13)), (8192, 1 << 26)])
def test_prompt_attn_refuses_more_row_blocks_of_a_head_than_it_counts(api, R, T):
    """8 heads over one: blocks of 128 rows are T / 16, and two a request beside them; 2^22 - 512 at most."""
    s = shape(api, R=R, Hkv=1, n_blocks=1000)
    assert call(api, "minikv_prompt_attn_blk", prompt_args(api, s, T=T, out=1 << 45, lse=1 << 46)) == -1


@pytest.mark.parametrize("out,lse", [
    (0x100000, None), (0x100000 + 2032, None), (0x100000 + 4 * 8192 + 2032, None), (0x100000 + 2048, None), (0x100000 - 5 * 2048 + 16, None),
    (1 << 40, 0x100000 + 2044), (1 << 40, 0x100000 + 8192 - 156), (1 << 40, 0x100000 - 156), (1 << 40, 1 << 40), (1 << 40, (1 << 40) + 5 * 2048 - 4),
    (1 << 40, (1 << 40) - 156),
])
def test_prompt_attn_refuses_outputs_over_what_is_read(api, out, lse):
    """Five rows of 2048 bytes, 8192 apart, and outputs of five rows one behind the other; sums of 160 bytes."""
    assert call(api, "minikv_prompt_attn_blk", prompt_args(api, q=0x100000, qs=4096, out=out, lse=lse)) == -1


def test_prompt_workspace_covers_the_parts(api):
    """1024 parts of up to 128 rows: m, l and 128 sums each; fewer rows where T has fewer."""
    s = shape(api)
    assert api.minikv_prompt_blk_workspace_bytes(s, 1000) >= 1024 * 128 * 130 * 4
    assert 1024 * 4 * 130 * 4 <= api.minikv_prompt_blk_workspace_bytes(s, 1) < 1024 * 8 * 130 * 4
    assert api.minikv_prompt_blk_workspace_bytes(s, -1) == 0


@pytest.mark.parametrize("which", range(11))
def test_fork_refuses(api, which):
    p = [0x1000 * (i + 1) for i in range(11)]
    for v in (None, 0x1002):
        assert call(api, "kv_fork_blk", [C.byref(shape(api)), *p[:which], v, *p[which + 1:], None]) == -1
    if which >= 6:                                     # what is written must be nothing that is read, nor written twice
        for other in range(which):
            assert call(api, "kv_fork_blk", [C.byref(shape(api)), *p[:which], p[other], *p[which + 1:], None]) == -1


def test_copy_refuses(api):
    b, c = C.byref(shape(api)), (api.MinikvBlkCache * 2)(*[api.MinikvBlkCache(*[0x1000] * 4) for _ in range(2)])
    copy = lambda *a: call(api, "kv_copy_blk", [b, *a, None])  # noqa: E731
    assert copy(-1, c, 3, 0x1000, 0x2000) == -1 and copy(2, c, -1, 0x1000, 0x2000) == -1 and copy(2, None, 3, 0x1000, 0x2000) == -1
    assert copy(2, c, 3, None, 0x2000) == -1 and copy(2, c, 3, 0x1000, 0x2001) == -1 and copy(2, c, 3, 0x1000, 0x1000) == -1
    assert copy(2, c, 2 ** 30 + 1, 0x1000, 0x2000) == -1 and copy(2, c, 2 ** 31 - 1, 0x1000, 0x2000) == -1
    assert copy(0, None, 3, None, None) == 0 and copy(2, c, 0, None, None) == 0
    c[1].Vs = None
    assert copy(2, c, 3, 0x1000, 0x2000) == -1


@pytest.mark.parametrize("which", range(5))
def test_free_refuses(api, which):
    p = [0x1000 * (i + 1) for i in range(5)]
    for v in (None, 0x1002):
        assert call(api, "kv_free_blk", [C.byref(shape(api)), *p[:which], v, *p[which + 1:], 1 << 40, None]) == -1
    if which in (2, 3):
        for other in range(which):                     # written: nothing that is read, nothing twice
            assert call(api, "kv_free_blk", [C.byref(shape(api)), *p[:which], p[other], *p[which + 1:], 1 << 40, None]) == -1
    assert call(api, "kv_free_blk", [C.byref(shape(api)), *p, api.kv_free_workspace_bytes(shape(api)) - 1, None]) == -3


@pytest.mark.parametrize("which", range(8))
def test_compact_refuses(api, which):
    p = [0x1000 * (i + 1) for i in range(8)]
    go = lambda q, n=3, size=1 << 40: call(api, "kv_compact_blk", [C.byref(shape(api)), *q[:5], n, *q[5:], size, None])  # noqa: E731
    for v in (None, 0x1002):
        assert go(p[:which] + [v] + p[which + 1:]) == -1
    if 2 <= which <= 6:
        for other in range(which):
            assert go(p[:which] + [p[other]] + p[which + 1:]) == -1
    assert go(p, n=-1) == -1 and go(p, n=2 ** 30 + 1) == -1 and go(p, size=api.kv_free_workspace_bytes(shape(api)) - 1) == -3
    assert go(p[:2] + [p[1]] + p[3:]) == -1 and go(p[:6] + [p[5]] + p[7:]) == -1


def test_free_workspace_grows_with_the_pool(api):
    assert api.kv_free_workspace_bytes(shape(api, n_blocks=100000)) >= 128 + 100000 // 1024 * 384


# ---------------------------------------------------------------------------------------------------------
# the binding: what a raw pointer does not tell

def z(*n, dtype=torch.int32):
    return torch.zeros(*n, dtype=dtype)


def test_binding_refuses_types_sizes_and_places(api):
    s = shape(api)
    rows = z(5, 8, 128, dtype=torch.float16)
    good = dict(T=5, Q=rows, K=rows[:, :2], w_q=None, w_k=None, inv=z(64, dtype=torch.float32), pos=z(5), qo=rows.clone(), ko=rows[:, :2].clone())

    def norm(**kw):
        a = dict(good, **kw)
        api.minikv_norm_rope(8, 2, a["T"], a["Q"], a["K"], a["w_q"], a["w_k"], 1e-6, a["inv"], 128, False, a["pos"], a["qo"], a["ko"])
    half = torch.float16
    for bad in (dict(T=6), dict(Q=rows[:, :7]), dict(Q=rows.bfloat16()), dict(Q=rows.float()), dict(K=rows), dict(w_q=z(127, dtype=half)), dict(w_q=z(128)),
                dict(inv=z(63, dtype=torch.float32)), dict(inv=z(64, dtype=torch.float64)), dict(pos=z(4)), dict(pos=z(5, dtype=torch.int64)),
                dict(qo=rows[:4]), dict(Q=rows.transpose(0, 1)), dict(ko=z(5, 2, 128, dtype=torch.bfloat16)), dict()):
        with pytest.raises(ValueError):                # (the last: all is right, but in host memory)
            norm(**bad)
    for call_ in (lambda: api.kv_free_blk(s, z(4), z(4, 6), z(40), z(2), z(100)),
                  lambda: api.kv_compact_blk(s, z(4), z(4, 6), z(4, 6), z(40), z(2), z(5), z(5), z(100)),
                  lambda: api.kv_fork_blk(s, z(4), z(4), z(4), z(4, 6), z(40), z(2), z(4), z(4, 6), z(2), z(4), z(4)),
                  lambda: api.kv_copy_blk(s, api.BlkCaches(s, []), z(3), z(3)),
                  lambda: api.kv_copy_blk(s, api.BlkCaches(s, []), z(1).expand(2 ** 32 + 3), z(1).expand(2 ** 32 + 3)),
                  lambda: api.kv_compact_blk(s, z(4), z(4, 6), z(4, 6), z(40), z(2), z(1).expand(2 ** 32), z(1).expand(2 ** 32), z(64 + 2 * 16)),
                  lambda: api.kv_copy_blk(s, api.BlkCaches(s, []), z(3), z(4))):
        with pytest.raises(ValueError):
            call_()
    with pytest.raises(ValueError):
        api.BlkCaches(s, [dict(K=z(1), V=z(1), Ks=z(1), Vs=z(1))])
    with pytest.raises(ValueError):
        api.BlkCaches(shape(api, block=8), [dict(K=z(1), V=z(1), Ks=z(1), Vs=z(1))])


def test_without_the_compiled_calls(api, monkeypatch):
    """_bind.so is a quicker way to make some calls: a program runs without it, and is told why it is slower."""
    import sys
    import paper_2411_18077_amd as package
    api.lib()
    monkeypatch.setitem(sys.modules, "paper_2411_18077_amd._bind", None)
    monkeypatch.delattr(package, "_bind", raising=False)
    monkeypatch.setattr(api, "_lib", None)
    monkeypatch.setattr(api, "_bind", None)
    with pytest.warns(RuntimeWarning, match="_bind"):
        assert api.lib() is api.lib()
    assert not api._quick(0)
    assert api.kv_free_workspace_bytes(shape(api)) > 0
    with pytest.raises(ValueError):
        api.kv_fork_blk(shape(api), z(4), z(4), z(4), z(4, 6), z(40), z(2), z(4), z(4, 6), z(2), z(4), z(3))


def test_a_build_without_a_compiler_for_the_compiled_calls(monkeypatch, tmp_path):
    """The library is there before the build says that _bind.so is not."""
    from paper_2411_18077_amd import build
    monkeypatch.setattr(build, "OBJ", str(tmp_path))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libminikv.so"))
    monkeypatch.setattr(build, "BIND", str(tmp_path / "_bind.so"))
    monkeypatch.setattr(build, "SOURCES", ["scalar.hip"])
    monkeypatch.setattr(build, "_compile", lambda src: (str(empty), ""))

    def fails():
        raise RuntimeError("g++ failed for bind.cpp")
    monkeypatch.setattr(build, "_compile_bind", fails)
    empty = tmp_path / "empty.o"
    import subprocess
    subprocess.run(["gcc", "-x", "c", "-fPIC", "-c", "/dev/null", "-o", str(empty)], check=True)
    with pytest.raises(RuntimeError, match="bind.cpp"):
        build.build(verbose=False)
    assert (tmp_path / "libminikv.so").exists()


def test_compiled_calls_for_another_torch_are_not_used(api, monkeypatch):
    from paper_2411_18077_amd import build
    assert api._compiled() is not None
    monkeypatch.setattr(build, "bound_to", lambda: "torch 1.0, Python 2.7")
    with pytest.warns(RuntimeWarning, match="built for torch"):
        assert api._compiled() is None


def test_compiled_calls_that_do_not_say_what_they_are_for_are_not_used(api, monkeypatch):
    import types
    import paper_2411_18077_amd as package
    monkeypatch.setattr(package, "_bind", types.ModuleType("_bind"), raising=False)
    with pytest.warns(RuntimeWarning, match="_bind"):
        assert api._compiled() is None
