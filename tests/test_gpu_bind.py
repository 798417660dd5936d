"""The compiled calls of the binding and the interpreter's make the same calls and refuse the same ones."""
import pytest
import torch

from pages_common import E4M3, SM, ints, rand_cache
from paper_2411_18077_amd import api

pytestmark = pytest.mark.gpu
F16 = torch.float16


class Setup:
    def __init__(self):
        self.shape = api.make_blk_shape(3, 4, 2, 128, 16, 20, 5, F16)
        (Kc, Ks), (Vc, Vs) = rand_cache(20, 2, 16, 1), rand_cache(20, 2, 16, 2)
        self.cache = api.BlkCache(self.shape, K=Kc.cuda().view(E4M3), V=Vc.cuda().view(E4M3), Ks=Ks.cuda(), Vs=Vs.cuda())
        self.caches = api.BlkCaches(self.shape, [self.cache])
        g = torch.Generator().manual_seed(3)
        self.x = torch.randn(9, 8, 128, generator=g).to(F16).cuda()
        i = lambda v: ints(v).cuda()  # noqa: E731
        z = lambda *n: torch.zeros(*n, dtype=torch.int32, device="cuda")  # noqa: E731
        table = i([[0, 1, 2, 3, 4], [5, 6, 7, 8, 9], [10, 11, 12, 13, 14]])
        self.of = dict(
            norm=dict(Hq=4, Hkv=2, T=9, Q=self.x[:, :4], K=self.x[:, 4:6], w_q=torch.ones(128, dtype=F16, device="cuda"), w_k=None, eps=1e-6,
                      inv_freq=torch.ones(64, device="cuda"), rot_dim=128, adjacent=False, pos=i(range(9)),
                      Q_out=torch.zeros(9, 4, 128, dtype=F16, device="cuda"), K_out=torch.zeros(9, 2, 128, dtype=F16, device="cuda")),
            attend=dict(shape=self.shape, T=9, q=self.x[:, :4], cache=self.cache, table=table, q_len=i([70, 20, 9]), cu=i([0, 4, 5, 9]), sm_scale=SM,
                        out=torch.zeros(9, 4, 128, dtype=F16, device="cuda"), lse=torch.zeros(9, 4, device="cuda"),
                        workspace=torch.zeros(api.minikv_prompt_blk_workspace_bytes(self.shape, 9), dtype=torch.uint8, device="cuda")),
            fork=dict(shape=self.shape, q_len=i([70, 20, 9]), parent=i([0, 0, 1]), n_keep=i([70, 33, 20]), table=table, ring=i(list(range(15, 20)) + [0] * 15),
                      ring_state=i([0, 5]), q_len_next=z(3), table_next=z(3, 5), ring_state_next=z(2), src=z(3), dst=z(3)),
            copy=dict(shape=self.shape, caches=self.caches, src=i([1, -1]), dst=i([15, -1])),
            free=dict(shape=self.shape, q_len=i([70, 20, 9]), table=table, ring=z(20), ring_state=z(2),
                      workspace=torch.zeros(api.kv_free_workspace_bytes(self.shape), dtype=torch.uint8, device="cuda")),
            compact=dict(shape=self.shape, q_len=i([70, 20, 9]), table=table, table_next=z(3, 5), ring=z(20), ring_state=z(2), src=z(8), dst=z(8),
                         workspace=torch.zeros(api.kv_free_workspace_bytes(self.shape), dtype=torch.uint8, device="cuda")))


CALLS = dict(norm="minikv_norm_rope", attend="minikv_prompt_attn_blk", fork="kv_fork_blk", copy="kv_copy_blk", free="kv_free_blk", compact="kv_compact_blk")


@pytest.mark.parametrize("kind", sorted(CALLS))
def test_both_ways_give_the_same(kind, monkeypatch):
    a, b = Setup(), Setup()
    made = []
    quick = api._quick

    class Counted:
        def __getattr__(self, name):
            def f(*args):
                made.append((name, getattr(api._bind, name)(*args)))
                return made[-1][1]
            return f
    monkeypatch.setattr(api, "_quick", lambda home: Counted())
    getattr(api, CALLS[kind])(**a.of[kind])
    assert len(made) == 1 and made[0][1] == 0          # (it was the compiled call that did it)
    monkeypatch.setattr(api, "_quick", lambda home: None)
    getattr(api, CALLS[kind])(**b.of[kind])
    monkeypatch.setattr(api, "_quick", quick)
    for k, t in a.of[kind].items():
        if isinstance(t, torch.Tensor):
            assert torch.equal(t, b.of[kind][k]), k
    assert torch.equal(a.cache.K.view(torch.uint8), b.cache.K.view(torch.uint8)) and torch.equal(a.cache.Vs, b.cache.Vs)


@pytest.mark.parametrize("kind", sorted(CALLS))
def test_what_is_not_right_is_refused(kind):
    """Each tensor in turn: of another type, too short, strided, in host memory, none at all."""
    s = Setup()
    call = getattr(api, CALLS[kind])
    for name, t in s.of[kind].items():
        if not isinstance(t, torch.Tensor):
            continue
        rows = name in ("Q", "K", "Q_out", "K_out", "q")
        bad = [t.double(), t[:0] if rows or t.dim() == 1 else t[:1, :1], t.cpu(), t.transpose(0, 1) if t.dim() > 1 else t.repeat(2)[::2]]
        for x in bad:
            if kind in ("copy", "compact") and name in ("src", "dst") and x.numel() == 0 and x.dtype == torch.int32:
                continue                               # (no pairs at all are none)
            if name == "workspace" and x.dtype == torch.float64:
                continue                               # (any type will do)
            with pytest.raises((ValueError, api.MinikvError)):
                call(**dict(s.of[kind], **{name: x}))
    torch.cuda.synchronize()


def test_a_shape_of_its_own(monkeypatch):
    """A shape equal to the cache's but another object, numbers of other types: made by the interpreter's way."""
    s = Setup()
    other = api.make_blk_shape(3, 4, 2, 128, 16, 20, 5, F16)
    api.minikv_prompt_attn_blk(**s.of["attend"])
    first = s.of["attend"]["out"].clone()
    s.of["attend"]["out"].zero_()
    api.minikv_prompt_attn_blk(**dict(s.of["attend"], shape=other))
    assert torch.equal(first, s.of["attend"]["out"])
    api.minikv_norm_rope(**dict(s.of["norm"], eps=0, adjacent=1))
    with pytest.raises(ValueError):
        api.minikv_prompt_attn_blk(**dict(s.of["attend"], shape=api.make_blk_shape(3, 4, 2, 128, 16, 21, 5, F16)))
