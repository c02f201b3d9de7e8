"""Weights of wide groups, from the keys read again, in long caches: every number of blocks a wave takes, up to
the greatest, and both merges whose launch does it. All heads against 64 bits, over the values that the
cache reads back.

Tolerances as in test_gpu_attend8.py (u = 2^-24): a result |error| <= 2 (eps + 2^-19 + (2 n + 64) u) * sum
p |v| with eps = (d + 2) u * scale * sum |q k|, the log-sum-exp eps + 2^-19 + (2 n + 64) u + 4 u |lse|; a
gathered weight each head's p with the first factor, 2^-40 in all for smaller ones, and G + 1 roundings
of the sum."""
import math
import zlib

import numpy as np
import pytest

from paper_2609_22158_amd import cache8 as C8
from tests.gpu_cases import log
from tests.test_gpu_cache8 import dev, offsets

pytestmark = pytest.mark.gpu
U = 2.0 ** -24

# L, Hq, H, d, tokens, room past them, blocks of 64 tokens that a wave takes, rows that the merge writes a
# sequence at a time (units times sequences >= 512) or a head at a time
CASES = {
    # runs of 512 * 5 tokens: a last one whose waves but the first have no block, one that ends with a block
    "blocks_5_d64": (2, 44, 4, 64, [200000, 0, 70007, 129, 51200, 2560 * 3 + 1], 7, 5, False),
    "blocks_3_d128": (1, 64, 4, 128, [8192 * 30 + 1, 1, 150000], 3, 3, False),
    "blocks_16_d64": (8, 40, 8, 64, [70001, 33, 0, 61100], 9, 16, False),   # groups of 5
    "blocks_16_d128": (4, 128, 8, 128, [262200], 1, 16, False),
    "blocks_16_two_tiles": (4, 136, 8, 128, [8192 * 33 + 65], 0, 16, False),  # groups of 17
    # merges of whole groups: 256 threads, runs of 256 * blocks tokens
    "batch_16_d128": (8, 80, 8, 128, [40001, 0, 4096 * 3, 1, 30000, 64, 4097, 50011], 2, 16, True),
    "batch_16_d64": (16, 40, 8, 64, [30000, 7, 4096, 35000], 1, 16, True),  # groups of 5
    "batch_7_d64": (8, 80, 8, 64, [1792 * 8, 1793, 0, 1, 20000, 129, 5000, 17011], 40, 7, True),
    "batch_1_d128": (8, 272, 8, 128, [1100, 256, 0, 257, 1000, 1], 5, 1, True),  # groups of 34: three tiles
    "batch_1_d64": (16, 88, 8, 64, [2100, 1, 0, 700], 5, 1, True),
}


def plan(L, Hq, H, rooms):
    """Blocks a wave, and whether the merge writes whole groups: plan_attend8 and merges_heads."""
    units = L * H * -(-(Hq // H) // 16)
    return min(max(L * H * sum(rooms) // (64 * 8192), 1), 16), units * len(rooms) >= 512


@pytest.mark.parametrize("cid", list(CASES))
def test_gathered_weights_of_wide_groups(cid, gpu_lib):
    import torch

    L, Hq, H, d, lens, more, blocks, whole = CASES[cid]
    G, S, rooms = Hq // H, len(lens), [n + more for n in lens]
    log(f"[attend8 sweep {cid}] L={L} Hq={Hq} H={H} d={d} tokens={lens}")
    assert plan(L, Hq, H, rooms) == (blocks, whole)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(zlib.crc32(cid.encode()))
    cache = C8.Cache8(L, H, d, offsets(rooms))
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    cu, n = dev(offsets(lens)), sum(lens)
    q = rand(L, S, Hq, d)
    cache.weights.uniform_(generator=gen)
    C8.advance8(cache, cu)
    for l in range(L):
        C8.append8(cache.layers(l), rand(1, n, H, d), rand(1, n, H, d), cu)
    held = torch.zeros(cache.rows, dtype=torch.bool, device="cuda")
    for r, m in zip(offsets(rooms), lens):
        held[int(r):int(r) + m] = True
    cache.weights[:, :, held] = torch.rand((L, H, n), generator=gen, device="cuda")
    before = cache.weights.clone()
    out, lse = C8.decode_attention8(cache, q, want_lse=True, gather=True)
    after = cache.weights.clone()
    assert torch.equal(before.view(torch.int32)[:, :, ~held], after.view(torch.int32)[:, :, ~held])
    o2, l2 = C8.decode_attention8(cache, q, want_lse=True)  # gathering changes neither result
    assert torch.equal(out, o2) and torch.equal(lse, l2)
    cache.weights.copy_(before)
    C8.decode_attention8(cache, q, gather=True)  # the same every time
    assert torch.equal(after.view(torch.int32), cache.weights.view(torch.int32))
    assert cache.status() == 0
    scale = 1.0 / math.sqrt(d)
    worst = 0.0
    for l in range(L):
        kl, vl = C8.read8(cache.layers(l), cu, n)
        for s in range(S):
            a, b, r = int(offsets(lens)[s]), int(offsets(lens)[s + 1]), int(offsets(rooms)[s])
            if a == b:
                assert (out[l, s] == 0).all() and (lse[l, s] == -math.inf).all()
                continue
            for h in range(H):
                heads = slice(h * G, (h + 1) * G)
                k, v, x = kl[0, h, a:b].double(), vl[0, h, a:b].double(), q[l, s, heads].double()
                z = torch.mm(k, x.t().contiguous()) * scale
                reach = torch.mm(k.abs(), x.abs().t().contiguous()).amax(dim=0) * scale
                top = z.amax(dim=0)
                p = torch.exp(z - top)
                total = p.sum(dim=0)
                p /= total
                pt = p.t().contiguous()
                step = (d + 2) * U * reach + 2.0 ** -19 + (2 * (b - a) + 64) * U  # per head
                err = (out[l, s, heads].double() - torch.mm(pt, v)).abs()
                assert (err <= 2 * step[:, None] * torch.mm(pt, v.abs())).all(), (l, s, h)
                want = top + torch.log(total)
                assert ((lse[l, s, heads].double() - want).abs() <= step + 4 * U * want.abs()).all(), (l, s, h)
                want = before[l, h, r:r + b - a].double() + p.sum(dim=1)
                tol = 2.0 ** -40 + (2 * step * p).sum(dim=1) + (G + 1) * U * want
                err = (after[l, h, r:r + b - a].double() - want).abs()
                assert (err <= tol).all(), (l, s, h, float((err / tol).max()))
                worst = max(worst, float((err / tol).max()))
    log(f"[attend8 sweep {cid}] the weights' greatest share of the tolerance: {worst:.3f}")
