"""Decode attention over the 4-bit cache against the fp64 oracle, over all tokens and over lists
of blocks, and the selection of those lists.

Tolerance, per output channel, derived from what is rounded (u = 2^-24, a half step of fp32):
logits are fp32 sums of exact products of bf16 pairs, off by at most eps = (d + 2) u * scale *
sum |q k|, and scaled to the log2 domain (2 u |z|, within the same sum); a probability
2^x, with x rounded to u |x|, is off by a factor of 1 +- (eps + 2^-19) while |x| <= 40, and below
2^-40 has no part in what follows; it is multiplied without a rounding (three bf16 parts); sums
over n tokens are off by n u, and as much again for the merges. Numerator and denominator both
carry it, so |error| <= 2 (eps + 2^-19 + (2 n + 64) u) * sum p |v|. The log-sum-exp: eps + 2^-19 +
(2 n + 64) u + 4 u |lse|."""
import math
import zlib

import numpy as np
import pytest

import oracle.cache4_ref as R
from oracle import decode_bf16
from paper_2609_22158_amd import binding as B
from paper_2609_22158_amd import cache4 as C4
from synth import f32_to_bf16_bits
from tests.gpu_cases import log

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


class Made:
    """A cache with random tokens and queries, and their values on the host."""

    def __init__(self, name, L, Hq, H, d, lens, rooms, kscale=1.0, shift=0.0):
        import torch

        rng = np.random.default_rng(zlib.crc32(name.encode()))
        S = len(lens)
        self.L, self.Hq, self.H, self.d, self.S, self.G = L, Hq, H, d, S, Hq // H
        cu = np.concatenate([[0], np.cumsum(rooms)]).astype(np.int32)
        self.cache = C4.Cache4(L, H, d, cu)
        for t in (self.cache.k_codes, self.cache.v_codes, self.cache.k_scales, self.cache.v_scales):
            t.fill_(0xFF)  # NaN wherever no token is
        self.q_bits = f32_to_bf16_bits(rng.standard_normal((L, S, Hq, d)).astype(np.float32) + shift)
        n = sum(lens)
        self.k_bits = f32_to_bf16_bits((rng.standard_normal((L, n, H, d)) * kscale).astype(np.float32))
        self.v_bits = f32_to_bf16_bits(rng.standard_normal((L, n, H, d)).astype(np.float32))
        self.lens, self.cu = lens, np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        self.write()

    def write(self):
        import torch

        cu = torch.from_numpy(self.cu).cuda()
        self.cache.lens.copy_(torch.tensor(self.lens, dtype=torch.int32))
        C4.append4(self.cache, B.bf16_from_bits(self.k_bits), B.bf16_from_bits(self.v_bits), cu)
        self.q = B.bf16_from_bits(self.q_bits)

    def rows(self, l, s, h):
        a, b = self.cu[s], self.cu[s + 1]
        return tuple(R.dequantise4(*R.quantise4(decode_bf16(x[l, a:b, h]))) for x in (self.k_bits, self.v_bits))

    def query(self, l, s, h):
        return decode_bf16(self.q_bits[l, s, h * self.G:(h + 1) * self.G])

    def check(self, out, lse, blocks=None, scale=None, seqs=None):
        out, lse = out.cpu().numpy(), lse.cpu().numpy()
        scale = scale or 1.0 / math.sqrt(self.d)
        for l in range(self.L):
            for s in seqs if seqs is not None else range(self.S):
                for h in range(self.H):
                    k, v = self.rows(l, s, h)
                    if blocks is not None:
                        keep = np.zeros(-(-len(k) // 64), bool)
                        keep[blocks[l][s][h]] = True
                        keep = keep.repeat(64)[:len(k)]
                        k, v = k[keep], v[keep]
                    for g, q in enumerate(self.query(l, s, h)):
                        ref, z, spread, reach = R.attend(q, k, v, scale)
                        eps = (self.d + 2) * U * reach
                        steps = 2.0 ** -19 + (2 * len(k) + 64) * U
                        tol = 2 * (eps + steps) * spread
                        got = out[l, s, h * self.G + g]
                        assert (np.abs(got - ref) <= tol).all(), (l, s, h, g, np.abs(got - ref).max(), tol.max())
                        gz = lse[l, s, h * self.G + g]
                        if len(k) == 0:
                            assert gz == -math.inf
                        else:
                            assert abs(gz - z) <= eps + steps + 4 * U * abs(z), (l, s, h, g, gz, z)


CASES = {
    # name: (L, Hq, Hkv, d, tokens, rooms[, key scale[, softmax scale[, shift of the queries]]])
    "lengths_d128": (1, 4, 2, 128, [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129],
                     [5, 1, 20, 16, 40, 31, 33, 64, 63, 64, 200, 500, 128, 130]),
    "lengths_d64": (2, 4, 1, 64, [1, 0, 31, 32, 33, 95, 96, 97, 511, 512, 513],
                    [1, 0, 31, 64, 33, 95, 96, 120, 511, 700, 513]),
    "g1": (2, 3, 3, 128, [700, 65], [700, 100]),
    "g5": (1, 10, 2, 128, [1333, 40], [1333, 40]),
    "g6_d64": (1, 12, 2, 64, [1400, 33], [1500, 33]),
    "g7_splits": (1, 14, 2, 128, [2560, 31, 900, 1300], [4000, 31, 901, 1400]),
    "g8_d64": (2, 16, 2, 64, [1100, 17, 16], [1100, 17, 20]),
    "g12": (1, 24, 2, 128, [530, 47], [600, 50]),
    "g16": (1, 32, 2, 128, [900, 3], [900, 4]),
    "g20_two_tiles": (1, 40, 2, 64, [300, 70], [300, 70]),
    "g32_two_tiles": (1, 32, 1, 128, [700, 2], [700, 2]),
    # logits over about 100 nats: the reference of each head moves within a split
    "peaky": (1, 14, 2, 128, [1400, 600], [1500, 600], 12.0),
    "scaled": (1, 4, 2, 64, [333], [333], 1.0, 0.37, 1.0),
    # far more room than tokens: the splits follow the tokens
    "roomy": (1, 8, 2, 128, [1500, 3], [40000, 30000]),
    # more splits than one pass of lanes merges, and 70 sequences
    "long_d64": (1, 2, 1, 64, [40001], [40001]),
    "many_seqs": (1, 2, 2, 64, [(37 * i) % 300 for i in range(70)], [300] * 70),
    # more sequences than a wave, or a workgroup, has lanes: many short ones and a long one among them
    "thousands": (1, 4, 2, 64, [3 + i % 5 if i != 1500 else 2500 for i in range(3000)],
                  [8 if i != 1500 else 2600 for i in range(3000)]),
    # enough (layer, head) pairs that a split is longer than a tile per wave
    "wide": (16, 16, 16, 64, [1025, 2100], [1025, 2200]),
    "wide_d128": (8, 8, 8, 128, [1700, 40, 900, 1, 0, 64, 333, 2000], [1700, 50, 900, 1, 9, 64, 400, 2000]),
    # as many, of one split each
    "wide_short": (16, 16, 16, 64, [1025, 900], [1025, 1000]),
    "wide_short_d128": (8, 16, 8, 128, [600, 1, 0, 64, 333], [600, 1, 5, 64, 400]),
}


@pytest.mark.parametrize("cid", list(CASES))
def test_decode(cid, gpu_lib):
    L, Hq, H, d, lens, rooms, *more = CASES[cid]
    kscale, scale, shift = (list(more) + [1.0, 0.0, 0.0][len(more):])
    log(f"[attend4 {cid}] L={L} Hq={Hq} H={H} d={d} tokens={lens[:6]}")
    m = Made(cid, L, Hq, H, d, lens, rooms, kscale, shift)
    out, lse = C4.decode_attention4(m.cache, m.q, scale=scale, want_lse=True)
    m.check(out, lse, scale=scale or None)
    assert m.cache.status() == 0
    import torch

    assert torch.equal(out, C4.decode_attention4(m.cache, m.q, scale=scale))  # the same every time


def test_sequence_past_its_room(gpu_lib):
    """lens beyond the room: the tokens of the room are attended to, and it is reported."""
    m = Made("past", 1, 4, 2, 128, [100, 64], [100, 64])
    m.cache.lens.add_(50)
    out, lse = C4.decode_attention4(m.cache, m.q, want_lse=True)
    m.check(out, lse)
    assert m.cache.status() == B.FLAG_OUT_ROWS


def test_not_a_number(gpu_lib):
    """A NaN in a query makes its head NaN, one in a key or a value its KV head's heads (of the
    sequence); nothing else changes."""
    import torch

    m = Made("nan", 1, 8, 2, 64, [400, 300, 200], [400, 300, 200])
    m.q_bits[0, 2, 5, 7] = 0x7FC0
    m.k_bits[0, 350, 1, 3] = 0x7F80           # an infinite key of sequence 0, KV head 1
    m.v_bits[0, 400 + 299, 0, 60] = 0xFFC0    # sequence 1, KV head 0: channels 32 .. 63
    m.write()
    out, lse = C4.decode_attention4(m.cache, m.q, want_lse=True)
    assert m.cache.status() == B.FLAG_NONFINITE
    want = torch.zeros((1, 3, 8, 64), dtype=torch.bool)
    want[0, 2, 5] = True
    want[0, 0, 4:] = True
    want[0, 1, :4, 32:] = True
    assert torch.equal(torch.isnan(out).cpu(), want)
    assert torch.isnan(lse[0, 0, 4:]).all() and torch.isnan(lse[0, 2, 5]) and torch.isfinite(lse[0, 1]).all()
    # a list without the block of the NaN key (block 5) does not see it
    some = torch.tensor([0, 1, 2, 3, 4, 6, -1], dtype=torch.int32, device="cuda").expand(1, 3, 2, 7).contiguous()
    part, _ = C4.decode_attention4(m.cache, m.q, blocks=some, want_lse=True)
    assert torch.isfinite(part[0, 0]).all()
    # and neither do rows behind the last token of a sequence that shares its last tile
    m.cache.lens.copy_(torch.tensor([350, 299, 200]))
    m.lens = [350, 299, 200]
    out, lse = C4.decode_attention4(m.cache, m.q, want_lse=True)
    assert torch.isfinite(out[0, :2]).all()


@pytest.mark.parametrize("cid", ["g7_splits", "lengths_d64", "g20_two_tiles", "many_seqs", "long_d64", "wide_short_d128"])
def test_decode_over_listed_blocks(cid, gpu_lib):
    """Lists of any blocks, one per (layer, sequence, KV head), with entries that are passed over:
    -1, ids that are no block of the sequence, repeats and entries out of order."""
    import torch

    L, Hq, H, d, lens, rooms, *_ = CASES[cid]
    m = Made(cid, L, Hq, H, d, lens, rooms)
    rng = np.random.default_rng(11)
    for n in (1, 6, 150):
        lists = np.full((L, m.S, H, n), -1, np.int32)
        taken = [[[None] * H for _ in range(m.S)] for _ in range(L)]
        for l in range(L):
            for s in range(m.S):
                nb = -(-lens[s] // 64)
                for h in range(H):
                    e = rng.integers(-2, max(nb, 1) + 2, n)
                    if rng.random() < 0.7:
                        e = np.sort(e)
                    lists[l, s, h] = e
                    got, top = [], -1
                    for x in e[:min(n, nb)]:
                        if top < x < nb:
                            got.append(int(x))
                        top = max(top, int(x))
                    taken[l][s][h] = got
        out, lse = C4.decode_attention4(m.cache, m.q, blocks=torch.from_numpy(lists).cuda(), want_lse=True)
        m.check(out, lse, blocks=taken)


SELECT = {
    # name: (L, Hq, Hkv, d, tokens, rooms)
    "d128": (2, 8, 2, 128, [5000, 64, 700, 0, 1300], [5000, 64, 800, 10, 1300]),
    "d64_g1": (1, 3, 3, 64, [9000, 1], [9100, 1]),
    "g16": (1, 16, 1, 128, [2049], [2049]),
    "long": (1, 4, 1, 64, [80000], [80000]),  # more blocks than a workgroup scores, or lists at once
}


@pytest.mark.parametrize("cid", list(SELECT))
def test_select_and_sparse_decode(cid, gpu_lib):
    import torch

    L, Hq, H, d, lens, rooms = SELECT[cid]
    m = Made(cid, L, Hq, H, d, lens, rooms)
    for n, first, last in ((1, 0, 0), (1, 1, 0), (2, 1, 1), (4, 1, 1), (20, 0, 3), (16, 5, 0), (64, 2, 2), (2000, 1, 1)):
        got = C4.select_blocks4(m.cache, m.q, n, first=first, last=last)
        host = got.cpu().numpy()
        taken = [[[None] * H for _ in range(m.S)] for _ in range(L)]
        for l in range(L):
            for s in range(m.S):
                for h in range(H):
                    k, _ = m.rows(l, s, h)
                    score = R.block_scores(m.query(l, s, h), R.block_bounds(k))
                    want = R.select_blocks(score, n, first, last)
                    assert np.array_equal(host[l, s, h], want), (n, first, last, l, s, h)
                    taken[l][s][h] = [int(x) for x in want if x >= 0]
        out, blocks, lse = C4.decode_sparse4(m.cache, m.q, n, first=first, last=last, want_lse=True)
        assert torch.equal(blocks, got)
        o2, l2 = C4.decode_attention4(m.cache, m.q, blocks=got, want_lse=True)
        assert torch.equal(out, o2) and torch.equal(lse, l2)
        if n in (1, 20, 2000):
            m.check(out, lse, blocks=taken)
    log(f"[select4 {cid}] ok")


SELECT_MANY = {
    # name: (L, H, G, d, tokens): the ways of sharing out the scores
    "alone_small_groups": (8, 8, 3, 64, [4000, 64 * 130, 64, 0, 700, 6000, 1, 9999]),
    "alone_wide": (16, 16, 1, 128, [70000, 12345]),
    "spread": (2, 3, 5, 128, [64 * 3000, 50000]),
    "spread_past_lds": (1, 2, 2, 64, [64 * 9000 - 1, 64 * 5000, 3]),
}


@pytest.mark.parametrize("cid", list(SELECT_MANY))
def test_select_many(cid, gpu_lib):
    """Selections of many blocks and rows against scores in 64 bits from the same bounds."""
    import torch

    L, H, G, d, lens = SELECT_MANY[cid]
    S = len(lens)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(9)
    x = torch.randn((L, H, int(cu[-1]) // 64 + S, 2, d), generator=gen, device="cuda")
    bounds = x.sort(dim=3).values.bfloat16()
    # buffers of no rows would do: the selection reads lens and bounds alone
    cache = C4.Cache4(L, H, d, cu, k_bounds=bounds, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    q = torch.randn((L, S, H * G, d), generator=gen, device="cuda").bfloat16()
    for n, first, last in ((7, 1, 1), (100, 0, 2)):
        got = C4.select_blocks4(cache, q, n, first=first, last=last).cpu().numpy()
        for s in range(S):
            nb, at = -(-lens[s] // 64), int(cu[s]) // 64 + s
            qs = q[:, s].double().view(L, H, G, 1, d)
            b = bounds[:, :, None, at:at + nb].double()
            score = torch.maximum(qs * b[..., 0, :], qs * b[..., 1, :]).sum(dim=(2, 4)).cpu().numpy()
            for l in range(L):
                for h in range(H):
                    want = R.select_blocks(score[l, h], n, first, last)
                    assert np.array_equal(got[l, s, h], want), (cid, n, l, s, h)
    log(f"[select4 {cid}] ok")


def test_select_ties_and_nan(gpu_lib):
    """Equal scores go to the lower block (all tokens alike, and zero queries); blocks whose
    bounds hold a NaN score as -inf, and come first of all only where forced."""
    import torch

    m = Made("ties", 1, 2, 1, 64, [64 * 40], [64 * 40])
    m.k_bits[:] = m.k_bits[:, :1]
    m.write()
    got = C4.select_blocks4(m.cache, m.q, 10, first=1, last=2).cpu().numpy()[0, 0, 0]
    assert got.tolist() == list(range(8)) + [38, 39]
    m = Made("ties2", 1, 2, 1, 64, [64 * 40 - 5], [64 * 40])
    m.k_bits[0, 64 * 7 + 3, 0, 50] = 0x7FC0
    m.k_bits[0, 64 * 20, 0, 1] = 0xFF80
    m.write()
    got = C4.select_blocks4(m.cache, m.q, 39, first=0, last=0).cpu().numpy()[0, 0, 0]
    assert got.tolist() == [b for b in range(40) if b != 20]  # the later of the two that rank last
    m.q_bits[:] = 0
    m.write()
    got = C4.select_blocks4(m.cache, m.q, 10, first=0, last=0).cpu().numpy()[0, 0, 0]
    assert got.tolist() == [b for b in range(11) if b != 7]  # 0 * NaN is NaN still
    m.q_bits[:] = 0x7FC0  # NaN queries add nothing to a score
    m.write()
    assert C4.select_blocks4(m.cache, m.q, 3, first=0, last=0).cpu().tolist()[0][0][0] == [0, 1, 2]


def test_scores_closer_than_fp32_tells(gpu_lib):
    """Blocks whose scores differ in the 30th bit rank as their exact values do."""
    import torch

    d, nb = 64, 24
    m = Made("close", 1, 1, 1, d, [64 * nb], [64 * nb])
    q = np.zeros(d, np.float32)
    q[0], q[32] = 1.0, 2.0 ** -29
    m.q_bits[0, 0, 0] = f32_to_bf16_bits(q)
    k = np.zeros((nb, 64, d), np.float32)
    k[:, :, 0] = 4.0
    level = [0.5, 1, 1.5, 2, 3, 4, 6, 0]
    order = np.random.default_rng(3).permutation(nb)
    for b in range(nb):  # 24 increasing values: 8 elements at three scales
        k[order[b], :, 32] = level[b % 8] * 8.0 ** (b // 8)
    m.k_bits[0, :, 0] = f32_to_bf16_bits(k.reshape(-1, d))
    m.write()
    score = R.block_scores(m.query(0, 0, 0), R.block_bounds(m.rows(0, 0, 0)[0]))
    for n in range(1, nb):
        got = C4.select_blocks4(m.cache, m.q, n, first=0, last=0).cpu().numpy()[0, 0, 0]
        assert np.array_equal(got, R.select_blocks(score, n, 0, 0)), n


def test_rows_past_four_gigabytes(gpu_lib):
    """Tokens whose codes and scales lie past 2^32 bytes of their buffers, and as many rows before."""
    import torch

    m = Made("far", 1, 8, 2, 128, [1, 700], [35_000_000, 900])
    assert m.cache.k_codes.numel() > 2 ** 32
    out, blocks, lse = C4.decode_sparse4(m.cache, m.q, 100, want_lse=True)
    m.check(out, lse)
    k, v = C4.read4(m.cache, torch.from_numpy(m.cu).cuda(), 701)
    for h in range(2):
        kk, vv = m.rows(0, 1, h)
        assert np.array_equal(k[0, h, 1:].float().cpu().numpy(), kk)
        assert np.array_equal(v[0, h, 1:].float().cpu().numpy(), vv)


def test_a_step_replays_in_a_hip_graph(gpu_lib):
    """advance, append, dense and sparse decode captured once: each replay takes the next token,
    as the eager calls on another cache do, with eager work between the replays."""
    import torch

    L, Hq, H, d, S = 2, 8, 2, 128, 3
    cu_rows = [0, 400, 700, 1000]
    a, b = (C4.Cache4(L, H, d, cu_rows) for _ in range(2))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    start = torch.tensor([0, 330, 340, 520], dtype=torch.int32, device="cuda")
    k, v = (torch.randn((L, 520, H, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    for c in (a, b):
        C4.advance4(c, start)
        C4.append4(c, k, v, start)
    one = torch.arange(S + 1, dtype=torch.int32, device="cuda")
    kn, vn = (torch.zeros((L, S, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros((L, S, Hq, d), dtype=torch.bfloat16, device="cuda")
    bufs = dict(out=torch.zeros((L, S, Hq, d), device="cuda"), lse=torch.zeros((L, S, Hq), device="cuda"),
                workspace=torch.zeros(1 << 24, dtype=torch.uint8, device="cuda"))
    sparse = dict(out=torch.zeros((L, S, Hq, d), device="cuda"), lse=torch.zeros((L, S, Hq), device="cuda"),
                  blocks=torch.zeros((L, S, H, 3), dtype=torch.int32, device="cuda"),
                  workspace=torch.zeros(1 << 24, dtype=torch.uint8, device="cuda"))

    def step(c, dense, sp):
        C4.advance4(c, one)
        for l in range(L):
            C4.append4(c.layers(l), kn[l:l + 1], vn[l:l + 1], one)
        return (C4.decode_attention4(c, q, want_lse=True, **dense),
                C4.decode_sparse4(c, q, 3, want_lse=True, **sp))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a, bufs, sparse)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(a, bufs, sparse)
    step(b, {}, {})  # the warm-up's token
    torch.cuda.synchronize()
    for rep in range(70):  # past a block's and a tile's end
        for t in (kn, vn, q):
            t.normal_(generator=gen)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        (out, lse), (so, blocks, sl) = step(b, {}, {})
        for x, y in ((out, bufs["out"]), (lse, bufs["lse"]), (so, sparse["out"]),
                     (blocks, sparse["blocks"]), (sl, sparse["lse"]), (a.lens, b.lens),
                     (a.k_codes, b.k_codes), (a.k_bounds, b.k_bounds)):
            assert torch.equal(x, y), rep
    log("[graph4] 70 replays match")


def test_another_stream(gpu_lib):
    """Every call on a stream that is not the current one, behind work that it has to wait for."""
    import torch

    m = Made("stream", 1, 8, 2, 64, [900, 65], [1000, 100])
    want, wl = C4.decode_attention4(m.cache, m.q, want_lse=True)
    wo, wb = C4.decode_sparse4(m.cache, m.q, 4)
    cu = torch.from_numpy(m.cu).cuda()
    wk, wv = C4.read4(m.cache, cu, 965)
    kt, vt = B.bf16_from_bits(m.k_bits), B.bf16_from_bits(m.v_bits)
    busy = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    c = C4.Cache4(1, 2, 64, m.cache.cu_rows)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            busy = busy @ busy * 1e-2
        q = m.q.clone()
    C4.advance4(c, cu, stream=side)
    C4.append4(c, kt, vt, cu, stream=side)
    out, lse = C4.decode_attention4(c, q, want_lse=True, stream=side)
    so, sb = C4.decode_sparse4(c, q, 4, stream=side)
    k, v = C4.read4(c, cu, 965, stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in ((out, want), (lse, wl), (so, wo), (sb, wb), (k, wk), (v, wv)))


def test_the_cycle_of_a_trajectory(gpu_lib):
    """A boundary (score, select, compaction into 4 bits), decoded tokens appended and attended to,
    the cache read back for the next boundary's scoring, and compacted again into a new cache: the
    rows that survive keep their codes."""
    import torch

    from tests.gpu_cases import HipRun, reduced

    w = reduced("l1_8k", seqlens=[900, 333], protected_len=40)
    g = HipRun(w, budget=200)
    L, H, Hq, d, S = w.num_layers, w.num_kv_heads, w.q_win.shape[3], w.head_dim, 2
    idx, cu_ret, _ = g.select(g.score()["scores"])
    rows = [int(x) for x in (cu_ret[1:] - cu_ret[:-1])]
    cu_rows = np.concatenate([[0], np.cumsum([n + 64 for n in rows])]).astype(np.int32)
    cache = C4.Cache4(L, H, d, cu_rows)
    C4.compact4(g.pb, cache, g.k, g.v, idx, cu_ret)
    k_hat, v_hat = g.compact(idx, cu_ret)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    q = torch.randn((L, S, Hq, d), generator=gen, device="cuda").bfloat16()
    one = torch.arange(S + 1, dtype=torch.int32, device="cuda")
    # the bf16 decode over the rows as read back agrees (it carries P to 2^-16, twice; fp32 sums)
    k4, v4 = C4.read4(cache, cu_ret, int(cu_ret[-1]))
    ref = B.decode_attention(g.pb, q, k4, v4, cu_ret, int(cu_ret[-1]))
    out = C4.decode_attention4(cache, q)
    assert (out - ref).abs().max() <= 2 * (2.0 ** -15 + 4000 * U) * 2 * v4.abs().max()
    err = float((k4.float() - k_hat.float()).norm() / k_hat.float().norm())
    assert err < 0.25  # at most half a step of 1 in 3.5 per value
    new_k, new_v = (torch.randn((30, L, S, H, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    for t in range(30):
        C4.advance4(cache, one)
        C4.append4(cache, new_k[t], new_v[t], one)
        C4.decode_sparse4(cache, q, 3)
    # the next boundary
    n2 = [n + 30 for n in rows]
    cu2 = torch.tensor([0] + list(np.cumsum(n2)), dtype=torch.int32, device="cuda")
    k2, v2 = C4.read4(cache, cu2, sum(n2))
    pb2 = B.Problem(L, Hq, H, d, w.window, cu2.cpu().numpy(), np.arange(S + 1))
    sid = torch.zeros(sum(n2), dtype=torch.int32, device="cuda")
    prot = torch.zeros(sum(n2), dtype=torch.uint8, device="cuda")
    util = torch.ones(S, device="cuda")
    res = B.score(pb2, g.q, k2, sid, prot, util, B.Params())
    idx2, cu_ret2, _ = B.select(pb2, res["scores"], prot, sid, 100)
    second = C4.Cache4(L, H, d, [0, 150, 300])
    C4.compact4(pb2, second, k2, v2, idx2, cu_ret2)
    assert second.lens.tolist() == [100, 100] and second.status() == 0 and cache.status() == 0
    for l in range(L):
        for h in range(H):
            for s in range(S):
                i = idx2[l, h, int(cu2[s]):int(cu2[s]) + 100].long() + int(cu_rows[s])
                r = 150 * s
                for a, b in ((second.k_codes, cache.k_codes), (second.k_scales, cache.k_scales),
                             (second.v_codes, cache.v_codes), (second.v_scales, cache.v_scales)):
                    assert torch.equal(a[l, h, r:r + 100], b[l, h][i])
