"""Pins of the definitions in oracle/pages.py: closed forms and hand-worked cases."""
import math

import pytest
import torch

from oracle import blk, pages


def test_rotation_keeps_lengths_and_turns_by_differences():
    g = torch.Generator().manual_seed(0)
    x = torch.randn(2, 1, 128, generator=g, dtype=torch.float64)
    inv = 10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)
    for adjacent in (False, True):
        at = lambda p: pages.norm_rope(x, None, 0.0, inv, 128, adjacent, torch.tensor(p))[0]  # noqa: E731
        a, b = at([5, 9]), at([105, 109])
        assert torch.allclose((a * a).sum(), (x * x).sum()) and torch.allclose((a[0] * a[1]).sum(), (b[0] * b[1]).sum())
        assert torch.equal(at([0, 0]), x)


def test_rotation_by_hand():
    x = torch.zeros(1, 1, 128)
    x[0, 0, 0], x[0, 0, 8], x[0, 0, 100] = 3.0, 4.0, 5.0
    out, size = pages.norm_rope(x, None, 0.0, torch.full((8,), math.pi / 2, dtype=torch.float64), 16, False, torch.tensor([1]))
    assert torch.allclose(out[0, 0, [0, 8, 100]], torch.tensor([-4.0, 3.0, 5.0], dtype=torch.float64)) and float(size[0, 0, 0]) == 7.0
    x[0, 0, 1] = 2.0
    out, _ = pages.norm_rope(x, None, 0.0, torch.full((8,), math.pi, dtype=torch.float64), 16, True, torch.tensor([1]))
    assert torch.allclose(out[0, 0, [0, 1, 8, 100]], torch.tensor([-3.0, -2.0, -4.0, 5.0], dtype=torch.float64))


def test_norm_by_hand():
    x = torch.full((1, 1, 128), 2.0)
    w = torch.arange(128).float()
    out, _ = pages.norm_rope(x, w, 5.0, None, 0, False, torch.tensor([3]))
    assert torch.allclose(out[0, 0], w.double() * 2 / 3)


def test_padding_rows_stay():
    x = torch.randn(2, 3, 128)
    out, _ = pages.norm_rope(x, torch.ones(128), 1e-6, torch.ones(64), 128, False, torch.tensor([-1, 4]))
    assert torch.equal(out[0], x[0].double()) and not torch.equal(out[1], x[1].double())


def test_prompt_attention_of_single_tokens_is_decode_attention():
    g = torch.Generator().manual_seed(1)
    Kc, Vc = (torch.randint(0, 120, (6, 2, 16, 128), generator=g).to(torch.uint8) for _ in range(2))
    Ks, Vs = torch.rand(6, 2, generator=g) / 64, torch.rand(6, 2, generator=g)
    q = torch.randn(3, 4, 128, generator=g)
    table, q_len = torch.tensor([[0, 3], [5, -1], [1, 2]]), torch.tensor([20, 30, 0])
    a, mean, score = blk.decode_attn(q, Kc, Ks, Vc, Vs, table, q_len, 0.1)
    b, lse, live, mean2, score2 = pages.prompt_attn(q, Kc, Ks, Vc, Vs, table, q_len, torch.arange(4), 0.1)
    assert torch.allclose(a, b, rtol=1e-12) and live.all() and torch.allclose(mean, mean2) and (lse[2] == -math.inf).all()


def test_prompt_attention_is_causal_and_lse_adds_up():
    """Equal keys: the output is the running mean of the values, lse the score plus log of their number."""
    Kc, Vc = torch.full((2, 1, 16, 128), 0x38, dtype=torch.uint8), torch.randint(0, 120, (2, 1, 16, 128)).to(torch.uint8)
    one = torch.ones(2, 1)
    q = torch.ones(5, 1, 128)
    out, lse, _, _, _ = pages.prompt_attn(q, Kc, one, Vc, one, torch.tensor([[1, 0]]), [19], [0, 5], 0.01)
    v = blk.decode_codes(Vc[[1, 0], 0]).reshape(-1, 128)
    for i in range(5):
        n = 15 + i
        assert torch.allclose(out[i, 0], v[:n].mean(dim=0)) and abs(float(lse[i, 0]) - 1.28 - math.log(n)) < 1e-9


def test_fork_by_hand():
    got = pages.fork([20, 5, 40], [0, 0, 2], [20, 20, 36], [[7, 8, 0], [9, 0, 0], [1, 2, 3]], [4, 5, 6, 0, 0, 0, 0, 0, 0, 0], (0, 3), 16)
    assert got == dict(q_len=[20, 20, 36], table=[[7, 8], [7, 4], [1, 2, 5]], src=[-1, 8, 3], dst=[-1, 4, 5], state=[2, 1])
    got = pages.fork([20, 5, 40], [1, 2, 0], [5, 40, 18], [[7, 8, 0], [9, 0, 0], [1, 2, 3]], [4] * 10, (9, 1), 16)
    assert got == dict(q_len=[5, 40, 18], table=[[9], [1, 2, 3], [7, 4]], src=[-1, -1, 8], dst=[-1, -1, 4], state=[0, 0])
    got = pages.fork([20, 5, 40], [0, 0, -1], [20, 20, 36], [[7, 8, 0], [9, 0, 0], [1, 2, 3]], [4] * 10, (9, 0), 16)
    assert got == dict(q_len=[20, 16, 0], table=[[7, 8], [7], []], src=[-1] * 3, dst=[-1] * 3, state=[9, 0])


def test_free_and_compact_by_hand():
    q_len, table = [20, 33, 0], [[7, 2, 1], [7, 9, 5], [3, 3, 3]]
    assert pages.free(q_len, table, 10, 16) == [0, 1, 3, 4, 6, 8]
    moves, rows, ring = pages.compact(q_len, table, 10, 16, 9)
    assert moves == [(9, 0), (7, 1), (5, 3)] and rows == [[1, 2], [1, 0, 3], []] and ring == [4, 5, 6, 7, 8, 9]
    moves, rows, ring = pages.compact(q_len, table, 10, 16, 1)
    assert moves == [(9, 0)] and rows == [[7, 2], [7, 0, 5], []] and ring == [1, 3, 4, 6, 8, 9]


@pytest.mark.parametrize("seed", range(20))
def test_compaction_keeps_what_is_shared(seed):
    g = torch.Generator().manual_seed(seed)
    N, R = 30, 4
    table = torch.randint(0, N, (R, 5), generator=g).tolist()
    q_len = torch.randint(0, 81, (R,), generator=g).tolist()
    moves, rows, ring = pages.compact(q_len, table, N, 16, 100)
    used = pages.named(q_len, table, N, 16)
    after = {b for row in rows for b in row}
    assert after == set(range(len(used))) and sorted(after | set(ring)) == list(range(N))
    pair = {(a, b) for t, row in zip(table, rows) for a, b in zip(t, row)}
    assert len({a for a, _ in pair}) == len(pair) == len({b for _, b in pair})         # one to one
    assert not {a for a, _ in moves} & {b for _, b in moves}
