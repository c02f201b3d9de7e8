"""Calls on the 4-bit cache that its binding has to refuse, or to keep apart from what the caller
does with its own arrays later (no GPU: nothing is launched)."""
import numpy as np
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


# ---------------------------------------------------------------- row offsets
def test_a_cache_keeps_its_own_row_offsets():
    """The library reads the offsets at every call: what the caller writes into the array that the
    cache was made from changes neither them nor the device's copy nor any size."""
    for dtype in (np.int32, np.int64):
        cu = np.array([0, 100, 200], dtype=dtype)
        c = C4.Cache4(2, 2, 64, cu, device="cpu")
        before = C4.load().stepkv_cache4_decode_workspace_bytes(c._ref, 8, 0)
        cu[:] = [0, 50, 90000]
        for x in (c, c.layers(1)):
            assert [x.c.cu_rows_host[i] for i in range(3)] == [0, 100, 200]
            assert x.cu_rows.tolist() == x.cu_rows_dev.tolist() == [0, 100, 200] and x.rows == 200
        assert C4.load().stepkv_cache4_decode_workspace_bytes(c._ref, 8, 0) == before
        with pytest.raises(ValueError):
            c.cu_rows[1] = 7  # and the cache's own is not for writing
        c.cu_rows_dev[1] = 7
        assert c.c.cu_rows_host[1] == 100
