"""Calls on the 4-bit cache that its binding has to refuse, or to keep apart from what the caller
does with its own arrays later (no GPU: nothing is launched)."""
import ctypes

import numpy as np
import pytest

from paper_2609_22158_amd import binding as B
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


# ---------------------------------------------------------------- limits of a launch
FAKE = 0x10000  # placeholder device address: every call below is refused before a launch


def _cache(rooms, L=16, H=16, d=128):
    cu = np.concatenate([[0], np.cumsum(np.asarray(rooms, np.int64))]).astype(np.int32)
    c = C4.Cache4C(L, H, d, len(cu) - 1, cu.ctypes.data_as(B._i32p), *[FAKE] * 7, None)
    c._keep = cu
    return c


def _problem(c):
    return B.ProblemC(c.num_layers, c.num_kv_heads, c.num_kv_heads, c.head_dim, 1, c.num_seqs,
                      c.cu_rows_host, FAKE, c.cu_rows_host, FAKE)


ONE_LONG = [128000] + [0] * 20000  # 5 M (layer, sequence, head) rows, at 1024 threads each
TOO_LARGE = {
    # a launch of 2^32 work items or more, in each of the kernels
    "compact": ([2 ** 28], lambda lib, c: lib.stepkv_cache4_compact(
        ctypes.byref(_problem(c)), c, FAKE, FAKE, FAKE, 0, FAKE, None)),
    "append": ([2 ** 28], lambda lib, c: lib.stepkv_cache4_append(
        c, FAKE, C4._i64x3(8, 8, 8), FAKE, C4._i64x3(8, 8, 8), FAKE, 2 ** 28, None)),
    "read": ([2 ** 20], lambda lib, c: lib.stepkv_cache4_read(c, FAKE, 2 ** 24, FAKE, FAKE, None)),
    "read, one head": ([[9], 1, 1], lambda lib, c: lib.stepkv_cache4_read(
        c, FAKE, 2 ** 31 - 1, FAKE, FAKE, None)),
    "decode": ([1] * 70000, lambda lib, c: lib.stepkv_cache4_decode(
        c, 16, FAKE, None, 0, 0.0, FAKE, None, FAKE, 1 << 62, None)),
    "decode, merge": ([2 ** 17] + [0] * 70000, lambda lib, c: lib.stepkv_cache4_decode(
        c, 16, FAKE, None, 0, 0.0, FAKE, None, FAKE, 1 << 62, None)),
    "select": ([1] * 70000, lambda lib, c: lib.stepkv_cache4_select_blocks(
        c, 16, FAKE, 4, 1, 1, FAKE, FAKE, 1 << 62, None)),
    "select, wide": (ONE_LONG, lambda lib, c: lib.stepkv_cache4_select_blocks(
        c, 16, FAKE, 4, 1, 1, FAKE, FAKE, 1 << 62, None)),
    "select, scores": ([2 ** 29], lambda lib, c: lib.stepkv_cache4_select_blocks(
        c, 16, FAKE, 4, 1, 1, FAKE, FAKE, 1 << 62, None)),
    "sparse": (ONE_LONG, lambda lib, c: lib.stepkv_cache4_decode_sparse(
        c, 16, FAKE, 4, 1, 1, 0.0, FAKE, FAKE, None, FAKE, 1 << 62, None)),
}


@pytest.mark.parametrize("call", list(TOO_LARGE))
def test_refuses_more_than_a_launch_takes(call):
    """A launch has fewer than 2^32 work items, and of more runs a part without an error: larger calls
    are refused."""
    rooms, fn = TOO_LARGE[call]
    c = _cache(*rooms) if isinstance(rooms[0], list) else _cache(rooms)
    assert fn(C4.load(), c) == B.EUNSUPPORTED


# ---------------------------------------------------------------- values that would change silently
@pytest.mark.parametrize("cu", [np.array([0, 2 ** 32 + 100]), np.array([0.0, 100.5]), [0, 2 ** 33],
                                np.array([0, 10, -2 ** 32 + 64])])
def test_refuses_row_offsets_that_int32_does_not_hold(cu):
    with pytest.raises((ValueError, OverflowError)):
        C4.Cache4(1, 1, 64, cu, device="cpu")


@pytest.mark.parametrize("scale,code", [(3.0e38, B.EINVAL), (2.4e38, B.EINVAL), (2.3e38, B.EWORKSPACE),
                                        (-3.0e38, B.EWORKSPACE)])
def test_refuses_a_scale_that_overflows_in_the_log2_domain(scale, code):
    """Logits of 0 would be 0 * inf there. (A misaligned workspace ends the calls that pass.)"""
    lib, c = C4.load(), _cache([100, 3000], 2, 2)
    ws = (FAKE + 8, 1 << 40, None)
    assert lib.stepkv_cache4_decode(c, 8, FAKE, None, 0, scale, FAKE, None, *ws) == code
    assert lib.stepkv_cache4_decode_sparse(c, 8, FAKE, 4, 1, 1, scale, FAKE, FAKE, None, *ws) == code
