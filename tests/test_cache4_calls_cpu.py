"""Calls on the 4-bit cache that its binding has to refuse, or to keep apart from what the caller
does with its own arrays later (no GPU: nothing is launched)."""
import pytest

from paper_2609_22158_amd import cache4 as C4


# ---------------------------------------------------------------- lists of blocks
def test_refuses_an_empty_list_of_blocks():
    """No block listed is not the same as no list (which attends to every token): refused."""
    import torch

    c = C4.Cache4(2, 2, 64, [0, 100, 164], device="cpu")
    q = torch.zeros((2, 2, 8, 64), dtype=torch.bfloat16)
    some = torch.zeros((2, 2, 2, 4), dtype=torch.int32)
    for none in (some[..., :0], torch.empty((2, 2, 2, 0), dtype=torch.int32)):
        with pytest.raises(ValueError, match="blocks"):
            C4.decode_attention4(c, q, blocks=none)
    with pytest.raises(ValueError, match="blocks"):
        C4.decode_attention4(c, q, blocks=torch.zeros((), dtype=torch.int32))
