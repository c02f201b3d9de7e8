"""A problem's offset arrays are its own (no GPU)."""
import numpy as np
import pytest

from paper_2609_22158_amd import binding as B


def test_a_problem_keeps_its_own_offsets():
    """The library reads the host offsets at every call, beside a device copy made once: what the
    caller writes into its arrays later changes neither."""
    cu, steps = np.array([0, 100, 200], np.int32), np.array([0, 3, 5], np.int32)
    pb = B.Problem(2, 8, 2, 64, 4, cu, steps, device="cpu")
    before = pb.workspace_bytes()
    cu[:] = [0, 50, 90000]
    steps[:] = [0, 1, 2]
    assert [pb.c.cu_seqlens_host[i] for i in range(3)] == [0, 100, 200] and pb.ntot == 200
    assert [pb.c.cu_steps_host[i] for i in range(3)] == [0, 3, 5] and pb.total_steps == 5
    assert pb.cu_seqlens_dev.tolist() == [0, 100, 200] and pb.cu_steps_dev.tolist() == [0, 3, 5]
    assert pb.workspace_bytes() == before > 0
    for own in (pb.cu_seqlens, pb.cu_steps):
        with pytest.raises(ValueError):
            own[1] = 7
