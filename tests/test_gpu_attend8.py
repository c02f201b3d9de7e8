"""Decode attention over the 8-bit cache, and the weights that it gathers, against the fp64 oracle.

Tolerance, per output channel, derived from what is rounded (u = 2^-24, a half step of fp32):
logits are fp32 sums of exact products of bf16 pairs, off by at most eps = (d + 2) u * scale *
sum |q k|, and scaled to the log2 domain (2 u |z|, within the same sum); a probability
2^x, with x rounded to u |x|, is off by a factor of 1 +- (eps + 2^-19) while |x| <= 40, and below
2^-40 has no part in what follows; it is multiplied without a rounding (three bf16 parts); sums
over n tokens are off by n u, and as much again for the merges. Numerator and denominator both
carry it, so |error| <= 2 (eps + 2^-19 + (2 n + 64) u) * sum p |v|. The log-sum-exp: eps + 2^-19 +
(2 n + 64) u + 4 u |lse|. A gathered weight: each head's p carries the same factor (2^-40 in all
where p is below that), and the sum over the heads with what was there G + 1 roundings of it."""
import math
import zlib

import numpy as np
import pytest

import oracle.cache8_ref as R
from oracle import decode_bf16
from oracle.cache4_ref import attend
from paper_2609_22158_amd import binding as B
from paper_2609_22158_amd import cache8 as C8
from synth import f32_to_bf16_bits
from tests.gpu_cases import log
from tests.test_gpu_attend4 import CASES
from tests.test_gpu_cache8 import dev, offsets

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


class Made:
    """A cache with random tokens and queries, and their values on the host."""

    def __init__(self, name, L, Hq, H, d, lens, rooms, kscale=1.0, shift=0.0):
        import torch

        rng = np.random.default_rng(zlib.crc32(name.encode()))
        S = len(lens)
        self.L, self.Hq, self.H, self.d, self.S, self.G = L, Hq, H, d, S, Hq // H
        self.cache = C8.Cache8(L, H, d, offsets(rooms))
        for x in ("k_codes", "v_codes", "k_scales", "v_scales", "weights"):
            if getattr(self.cache, x).numel():
                getattr(self.cache, x).view(torch.uint8).fill_(0xFF)  # NaN wherever no token is
        self.q_bits = f32_to_bf16_bits(rng.standard_normal((L, S, Hq, d)).astype(np.float32) + shift)
        n = sum(lens)
        self.k_bits = f32_to_bf16_bits((rng.standard_normal((L, n, H, d)) * kscale).astype(np.float32))
        self.v_bits = f32_to_bf16_bits(rng.standard_normal((L, n, H, d)).astype(np.float32))
        self.w = rng.random((L, H, n)).astype(np.float32)
        self.lens, self.cu, self.rows0 = lens, offsets(lens), offsets(rooms)
        self.write()

    def write(self):
        import torch

        cu = dev(self.cu)
        self.cache.lens.copy_(dev(self.lens))
        if self.cu[-1]:
            C8.append8(self.cache, B.bf16_from_bits(self.k_bits), B.bf16_from_bits(self.v_bits), cu)
        at = torch.cat([torch.arange(int(r), int(r) + n, device="cuda") for r, n in zip(self.rows0, self.lens)])
        if at.numel():
            self.cache.weights[:, :, at] = dev(self.w, torch.float32)
        self.at = at
        self.q = B.bf16_from_bits(self.q_bits)
        self.kept = {}

    def rows(self, l, s, h):
        a, b = self.cu[s], self.cu[s + 1]
        out = []
        for bits in (self.k_bits, self.v_bits):
            x = decode_bf16(bits[l, a:b, h])
            e = np.repeat([R.need(x[i:i + 64]) for i in range(0, b - a, 64)], 64)[:b - a, None] if b > a else 0
            out.append(R.round8(x / 2.0 ** e) * 2.0 ** e)
        return out

    def query(self, l, s, h):
        return decode_bf16(self.q_bits[l, s, h * self.G:(h + 1) * self.G])

    def wanted(self, l, s, h, scale):
        """A KV head's tokens, and of each query head what `attend` gives and the probabilities; kept,
        for the checks of one cache's results."""
        if (l, s, h, scale) not in self.kept:
            k, v = self.rows(l, s, h)
            heads = []
            for q in self.query(l, s, h):
                ref, z, spread, reach = attend(q, k, v, scale)
                heads.append((ref, z, spread, reach, np.exp(scale * (k @ q) - z) if len(k) else np.zeros(0)))
            self.kept[l, s, h, scale] = len(k), heads
        return self.kept[l, s, h, scale]

    def check(self, out, lse, weights=None, scale=None, seqs=None, times=1):
        """`weights`: what every token has gathered after `times` steps."""
        out, lse = out.cpu().numpy(), lse.cpu().numpy()
        scale = scale or 1.0 / math.sqrt(self.d)
        for l in range(self.L):
            for s in seqs if seqs is not None else range(self.S):
                for h in range(self.H):
                    n, heads = self.wanted(l, s, h, scale)
                    w, tol_w = np.zeros(n), np.full(n, 2.0 ** -40)
                    for g, (ref, z, spread, reach, p) in enumerate(heads):
                        eps = (self.d + 2) * U * reach
                        steps = 2.0 ** -19 + (2 * n + 64) * U
                        tol = 2 * (eps + steps) * spread
                        got = out[l, s, h * self.G + g]
                        assert (np.abs(got - ref) <= tol).all(), (l, s, h, g, np.abs(got - ref).max(), tol.max())
                        gz = lse[l, s, h * self.G + g]
                        if n == 0:
                            assert gz == -math.inf
                            continue
                        assert abs(gz - z) <= eps + steps + 4 * U * abs(z), (l, s, h, g, gz, z)
                        w += p
                        tol_w += 2 * (eps + steps) * p
                    if weights is not None and n:
                        a = self.cu[s]
                        want = self.w[l, h, a:a + n] + times * w
                        tol_w = times * tol_w + times * (self.G + 1) * U * want
                        err = np.abs(weights[l, h, a:a + n] - want)
                        assert (err <= tol_w).all(), (l, s, h, err.max(), tol_w[err.argmax()])

    def gathered(self):
        if not self.at.numel():
            return np.zeros((self.L, self.H, 0))
        return self.cache.weights[:, :, self.at].cpu().numpy().astype(np.float64)


CASES = dict(
    CASES,
    # many units, in numbers that the 8 XCDs do not share evenly, and as many sequences as a wave has lanes:
    # their splits in order of length, equal ones among them
    by_length=(11, 12, 6, 64, [(97 * i) % 700 if i % 5 else 0 for i in range(63)] + [2500], [700] * 63 + [2600]),
    by_length_equal=(16, 8, 4, 128, [1300, 1300, 1280, 128, 1300], [1400, 1300, 1300, 130, 1400]),
    # every sequence empty
    empty_splits=(16, 8, 4, 64, [0, 0, 0], [3000, 10, 0]),
    empty_split=(1, 8, 4, 128, [0], [5000]),
    empty_single=(1, 8, 4, 64, [0, 0], [100, 0]),
    # logits in memory though a sequence is one split: too many of them for LDS
    g16_memory=(1, 32, 2, 64, [700, 20], [700, 30]),
    # many workgroups of one split each, a tile past the sequence's end
    # wide groups, whose weights come from the keys read again: rooms that start inside a block, a block's
    # first row, empty sequences; several blocks a wave
    sweep_d64=(1, 10, 2, 64, [5000, 0, 70, 2113, 1], [5003, 40, 70, 2200, 9]),
    sweep_d128=(2, 44, 4, 128, [6145, 1, 0, 3000], [6150, 1, 5, 3001]),
    sweep_tiles=(1, 40, 1, 128, [4100, 129], [4100, 130]),
    sweep_blocks=(1, 80, 16, 64, [40007, 25600], [40010, 25700]),
    short_many=(6, 24, 12, 64, [33, 1, 64, 100], [40, 1, 64, 100]),
)


@pytest.mark.parametrize("cid", list(CASES))
def test_decode(cid, gpu_lib):
    import torch

    L, Hq, H, d, lens, rooms, *more = CASES[cid]
    kscale, scale, shift = (list(more) + [1.0, 0.0, 0.0][len(more):])
    log(f"[attend8 {cid}] L={L} Hq={Hq} H={H} d={d} tokens={lens[:6]}")
    m = Made(cid, L, Hq, H, d, lens, rooms, kscale, shift)
    before = m.cache.weights.clone()
    out, lse = C8.decode_attention8(m.cache, m.q, scale=scale, want_lse=True)
    m.check(out, lse, scale=scale or None, seqs=range(m.S) if m.S < 100 else [0, 1500, m.S - 1])
    assert m.cache.status() == 0
    assert torch.equal(out, C8.decode_attention8(m.cache, m.q, scale=scale))  # the same every time
    assert torch.equal(before.view(torch.int32), m.cache.weights.view(torch.int32))  # nothing gathered
    # gathering changes neither result, and no weight of a row that holds no token
    once = None
    for times in (1, 2):
        o2, l2 = C8.decode_attention8(m.cache, m.q, scale=scale, want_lse=True, gather=True)
        assert torch.equal(out, o2) and torch.equal(lse, l2)
        m.check(out, lse, m.gathered(), scale=scale or None, times=times,
                seqs=range(m.S) if m.S < 100 else [0, 1500, m.S - 1])
        once = m.cache.weights.clone() if once is None else once
    other = torch.ones(m.cache.rows, dtype=torch.bool, device="cuda")
    other[m.at] = False
    assert torch.equal(before.view(torch.int32)[:, :, other], m.cache.weights.view(torch.int32)[:, :, other])
    if m.at.numel():
        m.write()
        C8.decode_attention8(m.cache, m.q, scale=scale, gather=True)
    assert torch.equal(once.view(torch.int32), m.cache.weights.view(torch.int32))  # the same every time


def test_sequence_past_its_room(gpu_lib):
    """lens beyond the room: the tokens of the room are attended to, and it is reported."""
    m = Made("past", 1, 4, 2, 128, [100, 64], [100, 64])
    m.cache.lens.add_(50)
    out, lse = C8.decode_attention8(m.cache, m.q, want_lse=True, gather=True)
    m.check(out, lse, m.gathered())
    assert m.cache.status() == B.FLAG_OUT_ROWS


@pytest.mark.parametrize("rooms", [[400, 300, 200], [4000, 3000, 2000]], ids=["one split", "splits"])
def test_not_a_number(rooms, gpu_lib):
    """A NaN in a query makes its head NaN, one in a key or a value its KV head's heads (of the
    sequence), in a query or a key the weights too; nothing else changes."""
    import torch

    m = Made("nan", 1, 8, 2, 64, [400, 300, 200], rooms)
    m.q_bits[0, 2, 5, 7] = 0x7FC0
    m.k_bits[0, 350, 1, 3] = 0x7F80           # an infinite key of sequence 0, KV head 1
    m.v_bits[0, 400 + 299, 0, 60] = 0xFFC0    # sequence 1, KV head 0, channel 60
    m.write()
    out, lse = C8.decode_attention8(m.cache, m.q, want_lse=True, gather=True)
    assert m.cache.status() == B.FLAG_NONFINITE
    want = torch.zeros((1, 3, 8, 64), dtype=torch.bool)
    want[0, 2, 5] = True
    want[0, 0, 4:] = True
    want[0, 1, :4, 60] = True
    assert torch.equal(torch.isnan(out).cpu(), want)
    assert torch.isnan(lse[0, 0, 4:]).all() and torch.isnan(lse[0, 2, 5]) and torch.isfinite(lse[0, 1]).all()
    w = np.isnan(m.gathered())[0]
    assert w[1, :400].all() and w[1, 700:].all() and not w[1, 400:700].any() and not w[0].any()
    # rows behind the last token of a sequence that shares its last tile are not seen
    m.write()
    m.cache.lens.copy_(dev([350, 299, 200]))
    out, lse = C8.decode_attention8(m.cache, m.q, want_lse=True, gather=True)
    assert torch.isfinite(out[0, :2]).all()
    w = m.gathered()[0]
    assert np.isfinite(w[:, :700]).all()
    assert np.array_equal(w[:, 350:400], m.w[0, :, 350:400])  # nothing for them


@pytest.mark.parametrize("rooms", [[300], [3000]], ids=["one split", "splits"])
def test_logits_that_overflow(rooms, gpu_lib):
    """All to -inf: NaN, the log-sum-exp -inf, NaN weights. One to +inf: NaN. One to -inf: no weight."""
    import torch

    for sign, where, finite in ((-1, slice(0, 200), False), (1, slice(50, 51), False), (-1, slice(50, 51), True)):
        m = Made("over", 1, 2, 1, 64, [200], rooms)
        m.q_bits[:] = f32_to_bf16_bits(np.full(m.q_bits.shape, 1.0e20, np.float32))
        k = np.zeros((1, 200, 1, 64), np.float32)
        k[0, where] = sign * 1.0e20
        m.k_bits = f32_to_bf16_bits(k)
        m.write()
        out, lse = C8.decode_attention8(m.cache, m.q, want_lse=True, gather=True)
        w = torch.from_numpy(m.gathered()[0, 0])
        if not finite:
            assert torch.isnan(out).all() and torch.isnan(w).all()
            assert (lse == -math.inf).all() if sign < 0 else torch.isnan(lse).all()
        else:
            assert torch.isfinite(out).all() and w[50] == m.w[0, 0, 50]
            assert (w - torch.from_numpy(m.w[0, 0]).double() - 2 / 199).abs()[torch.arange(200) != 50].max() < 1e-6


def test_wide_groups_not_a_number_and_overflow(gpu_lib):
    """As above where the weights come from the keys read again, 11 heads beside 5 empty rows of the products."""
    import torch

    m = Made("wide nan", 1, 22, 2, 64, [400, 300, 200], [4000, 3000, 2000])
    m.q_bits[0, 2, 15, 7] = 0x7FC0            # sequence 2, KV head 1
    m.k_bits[0, 350, 1, 3] = 0x7F80           # an infinite key of sequence 0, KV head 1
    m.v_bits[0, 400 + 299, 0, 60] = 0xFFC0    # no weight depends on a value
    m.write()
    out, lse = C8.decode_attention8(m.cache, m.q, want_lse=True, gather=True)
    w = np.isnan(m.gathered())[0]
    assert w[1, :400].all() and w[1, 700:].all() and not w[1, 400:700].any() and not w[0].any()
    m.write()
    m.cache.lens.copy_(dev([350, 299, 200]))
    C8.decode_attention8(m.cache, m.q, gather=True)
    w = m.gathered()[0]
    assert np.isfinite(w[:, :700]).all() and np.array_equal(w[:, 350:400], m.w[0, :, 350:400])
    for sign, where, finite in ((-1, slice(0, 200), False), (1, slice(50, 51), False), (-1, slice(50, 51), True)):
        m = Made("wide over", 1, 11, 1, 64, [200], [3000])
        m.q_bits[:] = f32_to_bf16_bits(np.full(m.q_bits.shape, 1.0e20, np.float32))
        k = np.zeros((1, 200, 1, 64), np.float32)
        k[0, where] = sign * 1.0e20
        m.k_bits = f32_to_bf16_bits(k)
        m.write()
        C8.decode_attention8(m.cache, m.q, gather=True)
        w = torch.from_numpy(m.gathered()[0, 0])
        if not finite:
            assert torch.isnan(w).all()
        else:
            assert w[50] == m.w[0, 0, 50]
            # 11 weights of 1/199 within 2^-19 each, then 12 additions of numbers up to 1.06
            err = (w - torch.from_numpy(m.w[0, 0]).double() - 11 / 199).abs()
            assert err[torch.arange(200) != 50].max() < 11 / 199 * 2.0 ** -18 + 12 * 1.06 * U


@pytest.mark.parametrize("Hq", [8, 22], ids=["logits", "keys"])
def test_replays_as_the_cache_grows(Hq, gpu_lib):
    """A gathering step over split sequences captured once and replayed while the cache grows past the
    borders of tiles, blocks and splits, with eager work between the replays: the eager steps' bits."""
    import torch

    rng = np.random.default_rng(Hq)
    caches = [C8.Cache8(2, 2, 64, [0, 3000, 6001]) for _ in range(2)]
    first = B.bf16_from_bits(f32_to_bf16_bits(rng.standard_normal((2, 2700, 2, 64)).astype(np.float32)))
    for c in caches:
        C8.advance8(c, dev([0, 2000, 2700]))
        C8.append8(c, first, first, dev([0, 2000, 2700]))
    x, q = first[:, :61].clone(), first[:, :2].repeat(1, 1, Hq // 2, 1).contiguous()
    cu, side, outs = dev([0, 40, 61]), torch.cuda.Stream(), [None, None]

    def step(i):
        C8.advance8(caches[i], cu)
        C8.append8(caches[i], x, x, cu)
        outs[i] = C8.decode_attention8(caches[i], q, gather=True)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(1)
    for i in range(20):
        x.copy_(first[:, 100 * i:100 * i + 61])
        q.copy_(first[:, 7 * i:7 * i + 2].repeat(1, 1, Hq // 2, 1))
        graph.replay()
        step(0)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]), i
        for name in ("lens", "weights", "k_codes", "v_codes", "k_scales"):
            assert torch.equal(getattr(caches[0], name), getattr(caches[1], name)), (i, name)
    assert caches[0].lens.tolist() == [2800, 1120] and caches[0].status() == 0


def test_large_magnitudes(gpu_lib):
    """Keys near the greatest scale against tiny queries, and values at both ends of the range."""
    import torch

    for kf, qf, vf in ((2.0 ** 118, 2.0 ** -118, 2.0 ** 100), (2.0 ** -110, 2.0 ** 110, 2.0 ** -110)):
        m = Made("large", 1, 4, 1, 128, [500], [500])
        m.k_bits = f32_to_bf16_bits((decode_bf16(m.k_bits) * kf).astype(np.float32))
        m.q_bits = f32_to_bf16_bits((decode_bf16(m.q_bits) * qf).astype(np.float32))
        m.v_bits = f32_to_bf16_bits((decode_bf16(m.v_bits) * vf).astype(np.float32))
        m.write()
        out, lse = C8.decode_attention8(m.cache, m.q, want_lse=True, gather=True)
        m.check(out, lse, m.gathered())
        assert torch.isfinite(out).all()


def test_a_cache_without_rows(gpu_lib):
    """Rooms of nothing: zeros, nothing gathered, nothing to evict."""
    import torch

    for L, S in ((1, 2), (16, 3)):
        cache = C8.Cache8(L, 4, 64, [0] * (S + 1))
        q = torch.ones((L, S, 8, 64), dtype=torch.bfloat16, device="cuda")
        out, lse = C8.decode_attention8(cache, q, gather=True, want_lse=True)
        assert (out == 0).all() and (lse == -math.inf).all()
        C8.evict8(cache, 5)
        assert cache.lens.tolist() == [0] * S and cache.status() == 0


def test_buffers_and_streams(gpu_lib):
    """Given out, lse and workspace on another stream; a workspace that is too small is refused."""
    import torch

    m = Made("streams", 2, 14, 2, 128, [2600, 31, 900], [4000, 31, 901])
    out, lse = C8.decode_attention8(m.cache, m.q, want_lse=True)
    for gather in (False, True):
        n = int(gpu_lib.stepkv_cache8_decode_workspace_bytes(m.cache._ref, 14, int(gather)))
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        o, l = torch.full_like(out, math.nan), torch.full_like(lse, math.nan)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = C8.decode_attention8(m.cache, m.q, out=o, lse=l, workspace=ws, stream=side, gather=gather)
        side.synchronize()
        assert got[0] is o and torch.equal(o, out) and torch.equal(l, lse)
        with pytest.raises(B.StepKVError):
            C8.decode_attention8(m.cache, m.q, workspace=ws[:n - 256], gather=gather)
    m.check(out, lse, m.gathered())
