"""Eviction from a cache that was made of given tokens: as from the cache that they were appended to."""
import pytest

from paper_2609_22158_amd import cache8 as C8
from tests.gpu_cases import log
from tests.test_gpu_cache8 import dev

pytestmark = pytest.mark.gpu
BUFFERS = ("k_codes", "v_codes", "k_scales", "v_scales", "weights", "lens", "seen")


@pytest.mark.parametrize("given", [("seen",), ()], ids=["seen", "lens only"])
def test_evict(given, gpu_lib):
    import torch

    log(f"[given tokens: {given}]")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(8)
    a = C8.Cache8(2, 3, 64, [0, 200, 260, 400])
    cu = dev([0, 170, 230, 231])
    x = torch.randn((2, 231, 3, 64), generator=gen, device="cuda").bfloat16()
    C8.advance8(a, cu)
    C8.append8(a, x, x, cu)
    a.weights.uniform_(generator=gen)
    own = {n: getattr(a, n).clone() for n in BUFFERS}
    b = C8.Cache8(2, 3, 64, [0, 200, 260, 400], **{n: own[n] for n in BUFFERS if n != "seen" or n in given})
    for c in (a, b):
        C8.evict8(c, 50, first=4, recent=20)
    kept = a.positions[:, :, :50]
    assert a.lens.tolist() == [50, 50, 1]
    assert not torch.equal(kept, torch.arange(50, dtype=torch.int32, device="cuda").expand_as(kept))  # by weight
    for n in BUFFERS:
        assert torch.equal(getattr(a, n), getattr(b, n)), n
    for s0, n in ((0, 50), (200, 50), (260, 1)):
        assert torch.equal(a.positions[:, :, s0:s0 + n], b.positions[:, :, s0:s0 + n])
