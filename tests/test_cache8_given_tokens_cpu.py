"""A cache whose tokens are given (lens) without their positions, or without seen: they count as the last of
their sequences' tokens, in order."""
import pytest

from paper_2609_22158_amd import cache8 as C8

CU = [0, 5, 5, 12]


def i32(x):
    import torch

    return torch.tensor(x, dtype=torch.int32)


def made(**kw):
    return C8.Cache8(2, 3, 64, CU, device="cpu", **kw)


@pytest.mark.parametrize("weights", [True, "given"])
def test_positions_follow_from_lens_and_seen(weights):
    import torch

    kw = {} if weights is True else {"weights": torch.zeros((2, 3, 12))}
    seen = i32([4, 0, 1000])
    c = made(lens=i32([4, 0, 3]), seen=seen, **kw)
    want = i32([0, 1, 2, 3, 0] + [997, 998, 999, 0, 0, 0, 0])  # rows without a token hold 0
    assert c.positions.dtype == torch.int32 and c.positions.is_contiguous()
    assert torch.equal(c.positions, want.expand(2, 3, 12)) and c.seen is seen
    assert c.c.positions == c.positions.data_ptr()
    # past the room: the tokens of the room
    assert made(lens=i32([9, 0, 0]), seen=i32([9, 0, 0])).positions[0, 0, :5].tolist() == [0, 1, 2, 3, 4]
    assert made(lens=i32([-3, 0, 0]), seen=i32([0, 0, 0])).positions.eq(0).all()


def test_seen_follows_from_lens():
    import torch

    lens = i32([4, 0, 3])
    c = made(lens=lens)
    assert c.seen.tolist() == [4, 0, 3] and c.seen is not c.lens
    assert c.seen.data_ptr() != lens.data_ptr() and c.c.seen == c.seen.data_ptr()
    assert c.positions[1, 2].tolist() == [0, 1, 2, 3, 0, 0, 1, 2, 0, 0, 0, 0]
    assert made(lens=lens, weights=False).seen.tolist() == [4, 0, 3]
    assert torch.equal(made(lens=i32([0, 0, 0])).positions, torch.zeros((2, 3, 12), dtype=torch.int32))


def test_what_is_given_stays():
    import torch

    p, seen, lens = torch.full((2, 3, 12), 77, dtype=torch.int32), i32([9, 9, 9]), i32([5, 0, 7])
    c = made(lens=lens, seen=seen, positions=p)
    assert c.positions is p and c.seen is seen and c.lens is lens and p.eq(77).all()
    fresh = made()
    assert fresh.positions.eq(0).all() and fresh.seen.eq(0).all() and fresh.lens.eq(0).all()
