"""Decode attention over the 8-bit cache, and the weights it gathers, in every form that plan_attend8 chooses
between and no case of test_gpu_attend8.py reaches; its oracle and its tolerances."""
import pytest

from paper_2609_22158_amd import cache8 as C8
from tests.gpu_cases import log
from tests.test_gpu_attend8 import Made

pytestmark = pytest.mark.gpu

LONG = [1900, 40, 0, 64, 33, 129, 1, 700]
CASES = {
    # name: (L, Hq, H, d, tokens, room past them)
    # a sequence a workgroup of 8 waves, too many logits for LDS: 32 KiB are 51 tiles of 32 tokens of 5 heads
    "memory_g5_d128": (2, 40, 8, 128, LONG, 3),
    "memory_g5_d64": (2, 40, 8, 64, LONG, 3),
    "memory_g16_d128": (1, 256, 16, 128, [900, 513], 1),
    # in LDS: groups of 6 to 16 heads at d 64, and exactly 32 KiB
    "lds_g8_d64": (1, 32, 4, 64, [500, 33, 0, 1], 5),
    "lds_g16_full_d64": (1, 32, 2, 64, [512, 17], 0),
    "lds_g16_full_d128": (1, 32, 2, 128, [512, 31], 0),
    "lds_g4_full_d128": (8, 64, 16, 128, [2047], 1),
    # more than 256 workgroups of a sequence each, 4 waves
    "many_g6_d64": (16, 48, 8, 64, [700, 1, 95], 2),
    "many_g7_d128": (16, 56, 8, 128, [600, 0, 97], 2),
    "many_g16_d64": (16, 64, 4, 64, [130, 33, 1, 0, 64], 40),
    "many_g16_d128": (16, 64, 4, 128, [129, 32, 2, 0, 300], 40),
    # splits in order of length, logits in memory, one copy of the heads
    "by_length_g7_d128": (16, 28, 4, 128, [2600, 1300, 1280, 64, 0], 9),
    "by_length_g9_d128": (16, 36, 4, 128, [128, 2500, 129], 1),
}


@pytest.mark.parametrize("cid", list(CASES))
def test_decode(cid, gpu_lib):
    import torch

    L, Hq, H, d, lens, more = CASES[cid]
    log(f"[attend8 forms {cid}] L={L} Hq={Hq} H={H} d={d} tokens={lens}")
    m = Made(cid, L, Hq, H, d, lens, [n + more for n in lens])
    before = m.cache.weights.clone()
    out, lse = C8.decode_attention8(m.cache, m.q, want_lse=True)
    m.check(out, lse)
    for times in (1, 2):
        o2, l2 = C8.decode_attention8(m.cache, m.q, want_lse=True, gather=True)
        assert torch.equal(out, o2) and torch.equal(lse, l2)
        m.check(out, lse, m.gathered(), times=times)
        if times == 1:
            once = m.cache.weights.clone()
    other = torch.ones(m.cache.rows, dtype=torch.bool, device="cuda")
    other[m.at] = False
    assert torch.equal(before.view(torch.int32)[:, :, other], m.cache.weights.view(torch.int32)[:, :, other])
    m.write()
    C8.decode_attention8(m.cache, m.q, gather=True)
    assert torch.equal(once.view(torch.int32), m.cache.weights.view(torch.int32))  # the same every time
    assert m.cache.status() == 0
