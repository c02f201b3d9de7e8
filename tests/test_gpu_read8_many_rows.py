"""The largest reads of the 8-bit cache, four rows a thread: where one row a thread would take 2^32 threads
or more."""
import numpy as np
import pytest

from paper_2609_22158_amd import cache8 as C8
from tests.gpu_cases import log
from tests.test_gpu_cache8 import dev, offsets

pytestmark = pytest.mark.gpu

L, H = 16, 4
# sequences that end inside a workgroup's rows, many of them in one, empty ones, one that ends with it
LENS = [700, 1, 0, 333, 63] + [1, 2, 0, 3] * 12 + [128, 0, 65, 130]


@pytest.mark.parametrize("which", [0, 1], ids=["k", "v"])
@pytest.mark.parametrize("d", [64, 128])
def test_read_back_of_many_rows(d, which, gpu_lib):
    """Rows of a buffer of 64 GiB: what a small read gives, and every other row as it was. The sequence
    whose count is far more than it holds puts those behind it at the buffer's end."""
    import torch

    rows = (1 << 32) // (L * H * (d // 8)) + 3  # rows a read: one a thread is 2^32 threads and more
    log(f"[read8 many rows, d {d}] {rows} rows of {L * H} heads")
    cache = C8.Cache8(L, H, d, offsets(np.add(LENS, 5)))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d)
    cu = dev(offsets(LENS))
    x = [torch.randn((L, sum(LENS), H, d), generator=gen, device="cuda").bfloat16() for _ in range(2)]
    C8.advance8(cache, cu)
    C8.append8(cache, x[0], x[1], cu)
    small = C8.read8(cache, cu, sum(LENS))[which]
    far = list(LENS)
    far[3] += rows - 70 - sum(LENS)  # 70 rows past the last sequence's
    fewer = [max(n - 2, 0) for n in LENS]
    out = torch.empty((L, H, rows, d), dtype=torch.bfloat16, device="cuda")
    want = torch.empty((H, rows, d), dtype=torch.bfloat16, device="cuda")
    for counts in (LENS, far, fewer):
        at, src = [], []
        for o, s0, n, m in zip(offsets(counts)[1:], offsets(LENS)[1:], LENS, counts):
            k = min(n, m)  # the last k tokens are the last k of the count's rows
            at.append(np.arange(o - k, o))
            src.append(np.arange(s0 - k, s0))
        at, src = (torch.from_numpy(np.concatenate(y).astype(np.int64)).cuda() for y in (at, src))
        out.fill_(7.0)
        kw = {"k_out": out, "v_out": False} if which == 0 else {"k_out": False, "v_out": out}
        got = C8.read8(cache, dev(offsets(counts)), rows, **kw)
        assert got[which] is out and got[1 - which] is None
        for l in range(L):
            want.fill_(7.0)
            want[:, at] = small[l][:, src]
            assert torch.equal(out[l].view(torch.int16), want.view(torch.int16)), l
    assert cache.status() == 0
    del out, want, small
    torch.cuda.empty_cache()
