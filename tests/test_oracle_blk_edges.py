"""Pins of the plain definitions of the paged cache where values are out of range (no GPU needed)."""
from oracle import blk


def test_assignment_with_absent_blocks_by_hand():
    """Rows of a block outside the pool have a slot outside it; the request is accepted all the same."""
    got = blk.assign([15, 15, 0], [2, 2, 1], [[-1, -1], [1 << 28, -1], [-1, -1]], [9, 0, 7], [0, 3], 16, 6)
    assert got["slots"] == [-1, 144, -1, 0, 112, -1] and got["table"] == [[-1, 9], [1 << 28, 0], [7, -1]]
    assert got["q_len"] == [17, 17, 1] and got["state"] == [0, 0]
