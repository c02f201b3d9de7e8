"""Values at the end of the range that the headers of the quantised caches state for decode attention:
2^111 / n over n tokens.

By arithmetic: a probability is at most 2^16 before the division by the sum (the softmax's reference stays
until a logit exceeds it by 16 in the log2 domain), so n products with values of at most 2^111 / n add
up to 2^127 at most, and every partial sum of them is smaller: the parts of a probability have one sign.
Without the 1 / n, values of 2^111 would add up to n * 2^127.

The tolerance is that of test_gpu_attend8.py: 2 (eps + 2^-19 + (2 n + 64) u) * sum p |v| with u = 2^-24; one
channel has a logit, of exact numbers, so eps = (d + 2) u |logit|. A gathered weight carries the same
factor for each head, and one rounding more for each."""
import math

import numpy as np
import pytest

from paper_2609_22158_amd import cache4 as C4
from paper_2609_22158_amd import cache8 as C8
from tests.gpu_cases import log

pytestmark = pytest.mark.gpu
U = 2.0 ** -24

# Layers, KV heads, tokens, tiles of 32 from one low tile to the next: a wave's run starts with a low one.
# One sequence a workgroup, its waves with 12 tiles each; and splits of 1024 tokens, a wave with 8 tiles.
SHAPES = {"one split": (8, 16, 2944, 12), "splits": (4, 16, 16384, 8)}


@pytest.mark.parametrize("G", [4, 8, 11])
@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("bits", [4, 8])
def test_values_of_2_to_111_over_n(bits, shape, G, gpu_lib):
    import torch

    L, H, n, period = SHAPES[shape]
    d, lag = 64, 15.9
    C, name = (C4, "4") if bits == 4 else (C8, "8")
    log(f"[range {bits} bits, {shape}, G {G}] n={n}")
    cache = getattr(C, "Cache" + name)(L, H, d, [0, n])
    low = (np.arange(n) // 32) % period == 0
    top = 2.0 ** math.floor(111 - math.log2(n))  # a power of two: exact in either format
    sign = np.where(np.arange(d) % 2 == 0, 1.0, -1.0)
    v = top * sign * np.where(low, 0.5, 1.0)[:, None]
    k = np.zeros((n, d))
    k[:, 0] = np.where(low, 0.0, 16.0)
    scale = lag * math.log(2.0) / 16.0
    k_new, v_new = (torch.from_numpy(x).cuda().bfloat16()[None, :, None].expand(L, n, H, d).contiguous() for x in (k, v))
    q = torch.zeros((L, 1, G * H, d), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    getattr(C, "advance" + name)(cache, cu)
    getattr(C, "append" + name)(cache, k_new, v_new, cu)
    back = getattr(C, "read" + name)(cache, cu, n)
    assert torch.equal(back[0][0, 0].double().cpu(), torch.from_numpy(k))  # held without a rounding
    assert torch.equal(back[1][0, 0].double().cpu(), torch.from_numpy(v))
    p = np.exp(float(np.float32(scale)) * k[:, 0])
    p /= p.sum()
    want = p @ v
    tol = 2 * ((d + 2) * U * lag + 2.0 ** -19 + (2 * n + 64) * U)
    kw = {} if bits == 4 else {"gather": True}
    out = getattr(C, "decode_attention" + name)(cache, q, scale=scale, **kw).double().cpu().numpy()
    assert (np.abs(out - want) <= tol * (p @ np.abs(v))).all()
    if bits == 8:
        w = cache.weights.double().cpu().numpy()
        assert (np.abs(w - G * p) <= (tol + G * U) * G * p).all()
    assert cache.status() == 0
