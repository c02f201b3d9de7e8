"""The 8-bit cache on the GPU: written by compaction and appending, read back and evicted from, all
element for element against the fp64 oracle (every step of the format is exact, so nothing has a
tolerance), and bytes that a call does not own, which stay as they were."""
import zlib

import numpy as np
import pytest

import oracle.cache8_ref as R
from oracle import decode_bf16
from paper_2609_22158_amd import binding as B
from paper_2609_22158_amd import cache8 as C8
from synth import f32_to_bf16_bits
from tests.gpu_cases import log

pytestmark = pytest.mark.gpu

FILL = 0xA5  # in every byte of a buffer before a call


def filled(cache):
    import torch

    for x in ("k_codes", "v_codes", "k_scales", "v_scales", "weights", "positions"):
        t = getattr(cache, x)
        if t is not None and t.numel():
            t.view(torch.uint8).fill_(FILL)
    return cache


def bf16(rng, shape, scale=1.0, swing=4):
    """Random bf16 bits: normal, with a few outlier channels and some rows far larger or smaller."""
    x = rng.standard_normal(shape) * scale
    x[..., rng.integers(0, shape[-1], 3)] *= 8
    x *= 2.0 ** rng.integers(-swing, swing + 1, shape[:-1] + (1,))
    return f32_to_bf16_bits(x.astype(np.float32))


def offsets(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def dev(x, dtype=None):
    import torch

    return torch.tensor(np.asarray(x), dtype=dtype or torch.int32, device="cuda")


def check(cache, heads):
    """Every head's tokens are those of heads[(l, h, s)]; all other bytes are FILL."""
    fill32 = np.frombuffer(bytes([FILL] * 4), np.uint32)[0]
    cu = cache.cu_rows
    for which, (codes, scales) in enumerate(((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales))):
        codes, scales = codes.cpu().numpy(), scales.cpu().numpy().view(np.uint32)
        left, left_s = np.ones(codes.shape[:3], bool), np.ones(scales.shape, bool)
        for (l, h, s), a in heads.items():
            r, n = int(cu[s]), len(a)
            at, nb = r // 64 + s, -(-n // 64)
            assert np.array_equal(scales[l, h, at:at + nb].view(np.float32), 2.0 ** np.array(a.exp[which])), (l, h, s)
            assert np.array_equal(R.NUMBERS[codes[l, h, r:r + n]], a.num[which], equal_nan=True), (which, l, h, s)
            left[l, h, r:r + n] = False
            left_s[l, h, at:at + nb] = False
        assert (codes[left] == FILL).all() and (scales[left_s] == fill32).all()
    if cache.weights is None:
        return
    w, p = cache.weights.cpu().numpy(), cache.positions.cpu().numpy()
    left = np.ones(w.shape, bool)
    for (l, h, s), a in heads.items():
        r, n = int(cu[s]), len(a)
        assert np.array_equal(w[l, h, r:r + n], a.weights.astype(np.float32), equal_nan=True), (l, h, s)
        assert np.array_equal(p[l, h, r:r + n], a.positions), (l, h, s)
        left[l, h, r:r + n] = False
    assert (w.view(np.uint32)[left] == fill32).all() and (p.view(np.uint32)[left] == fill32).all()


def empty_heads(L, H, S, d):
    return {(l, h, s): R.Head8(d) for l in range(L) for h in range(H) for s in range(S)}


COMPACT = {
    # name: (L, Hq, Hkv, d, source tokens, retained, room beyond retained, shared, weights)
    "d128": (2, 8, 2, 128, [700, 130, 65], [300, 64, 65], [10, 0, 7], False, True),
    "d64": (3, 4, 4, 64, [500, 33, 200], [129, 33, 1], [3, 40, 63], False, False),
    "shared": (2, 4, 2, 128, [400, 90], [191, 63], [0, 5], True, True),
    "empty": (1, 2, 1, 64, [0, 100, 0, 5], [0, 0, 0, 5], [4, 9, 0, 0], False, True),
    "one": (1, 1, 1, 128, [1], [1], [0], False, False),
    "many_seqs": (1, 2, 2, 64, [3] * 150, [2] * 150, [1] * 150, True, True),
}


@pytest.mark.parametrize("cid", list(COMPACT))
def test_compact_and_read_back(cid, gpu_lib):
    import torch

    L, Hq, H, d, src, kept, room, shared, weighted = COMPACT[cid]
    log(f"[cache8 compact {cid}] rows={kept[:5]}")
    rng = np.random.default_rng(zlib.crc32(cid.encode()))
    S, cu_seq, cu_ret = len(src), offsets(src), offsets(kept)
    n = int(cu_seq[-1])
    k, v = bf16(rng, (L, H, n, d)), bf16(rng, (L, H, n, d))
    w = rng.random((L, H, n)).astype(np.float32)
    idx = np.full((1 if shared else L * H, n), -7, np.int32)
    for r in range(idx.shape[0]):
        for s in range(S):
            idx[r, cu_seq[s]:cu_seq[s] + kept[s]] = np.sort(rng.permutation(src[s])[:kept[s]])
    pb = B.Problem(L, Hq, H, d, 1, cu_seq, np.zeros(S + 1, np.int32))
    cache = filled(C8.Cache8(L, H, d, offsets(np.add(kept, room))))
    heads = empty_heads(L, H, S, d)
    for (l, h, s), a in heads.items():
        i = idx[0 if shared else l * H + h, cu_seq[s]:cu_seq[s] + kept[s]]
        at = cu_seq[s] + i
        a.append(decode_bf16(k[l, h, at]), decode_bf16(v[l, h, at]), i, w[l, h, at] if weighted else None)
    C8.compact8(pb, cache, B.bf16_from_bits(k), B.bf16_from_bits(v),
                torch.from_numpy(idx[0] if shared else idx.reshape(L, H, n)).cuda(), dev(cu_ret),
                weights=dev(w, torch.float32) if weighted else None)
    assert cache.lens.tolist() == kept and cache.seen.tolist() == src and cache.status() == 0
    check(cache, heads)
    # whole sequences, then the last tokens of each with room to spare, one tensor at a time
    for counts, spare in ((kept, 0), ([x - x // 3 for x in kept], 9)):
        cu = offsets(counts)
        rows = int(cu[-1]) + spare
        got = C8.read8(cache, dev(cu), rows)
        only = torch.full((L, H, rows, d), 7.0, dtype=torch.bfloat16, device="cuda")
        assert C8.read8(cache, dev(cu), rows, k_out=False, v_out=only)[0] is None
        assert (only[:, :, cu[-1]:] == 7).all()
        for which, t in enumerate((got[0], only)):
            t = t.double().cpu().numpy()
            for (l, h, s), a in heads.items():
                assert np.array_equal(t[l, h, cu[s]:cu[s + 1]], a.values(which)[len(a) - counts[s]:])


APPEND = {
    # name: (L, H, d, counts of each call, room, layout)
    "token_by_token": (2, 2, 128, [[1, 0, 1]] * 70, 100, "token"),
    "ragged": (1, 2, 64, [[10, 0, 127, 64, 5], [0, 130, 2, 64, 59], [3, 1, 0, 0, 64]], 200, "head"),
    "prompt": (2, 1, 128, [[0], [777], [1], [30]], 900, "slice"),
    "past_the_room": (1, 2, 128, [[60, 10], [10, 3], [2, 51]], 64, "token"),
    "many_seqs": (1, 1, 64, [[7] * 130, [1] * 130], 9, "head"),
}


def laid_out(k, v, layout):
    import torch

    kt, vt = B.bf16_from_bits(k), B.bf16_from_bits(v)
    if layout == "head":  # [L][H][T][d] storage
        return tuple(t.transpose(1, 2).contiguous().transpose(1, 2) for t in (kt, vt))
    if layout == "slice":  # parts of a fused projection's output, every second token
        L, n, H, d = kt.shape
        fused = torch.zeros((L, 2 * n, 3 * H, d), dtype=torch.bfloat16, device="cuda")
        fused[:, ::2, H:2 * H], fused[:, ::2, 2 * H:] = kt, vt
        return fused[:, ::2, H:2 * H], fused[:, ::2, 2 * H:]
    return kt, vt


@pytest.mark.parametrize("cid", list(APPEND))
def test_append(cid, gpu_lib):
    """Calls after each other, with rows whose magnitudes swing, so that scales grow inside blocks."""
    L, H, d, calls, room, layout = APPEND[cid]
    log(f"[cache8 append {cid}]")
    rng = np.random.default_rng(zlib.crc32(cid.encode()))
    S = len(calls[0])
    cache = filled(C8.Cache8(L, H, d, np.arange(S + 1) * room))
    heads, lens, grew = empty_heads(L, H, S, d), np.zeros(S, int), 0
    cache.seen.copy_(dev(np.arange(S) * 1000))
    for i, counts in enumerate(calls):
        n = sum(counts)
        k, v = (bf16(rng, (L, n, H, d), 1.0, 12) for _ in range(2))
        cu = offsets(counts)
        kt, vt = laid_out(k, v, layout)
        if n:
            C8.advance8(cache, dev(cu))
            C8.append8(cache, kt, vt, dev(cu))
            if i % 2:
                C8.append8(cache, kt, vt, dev(cu))  # the same tokens again change nothing
        for (l, h, s), a in heads.items():
            a0, a1 = cu[s], cu[s + 1]
            a1 = min(a1, a0 + max(room - lens[s], 0))  # tokens past the room are not stored
            before = list(a.exp[0])
            a.append(decode_bf16(k[l, a0:a1, h]), decode_bf16(v[l, a0:a1, h]), s * 1000 + lens[s] + np.arange(a1 - a0))
            grew += before != a.exp[0][:len(before)]
        lens += counts
    assert cache.lens.tolist() == lens.tolist()
    assert cache.seen.tolist() == (lens + 1000 * np.arange(S)).tolist()
    assert cache.status() == (B.FLAG_OUT_ROWS if (lens > room).any() else 0)
    assert grew > 0 or cid == "many_seqs"
    check(cache, heads)


EXTREMES = [0.0, -0.0, 1.0, 3.38e38, -3.38e38, 3.0e38, 2.0 ** -126, 2.0 ** -133, -2.0 ** -120, 464.0, 465.0, 448.0,
            1e-20, 1e20, 2.0 ** -117 * 464, 2.0 ** 119 * 464, 2.0 ** 119 * 449]


@pytest.mark.parametrize("d", [64, 128])
def test_extreme_values(d, gpu_lib):
    """Each sequence one token of one extreme after another, in one block, then all at once."""
    log(f"[cache8 extremes d={d}]")
    rng = np.random.default_rng(d)
    S = len(EXTREMES)
    cache = filled(C8.Cache8(1, 1, d, np.arange(S + 2) * 70))
    heads = empty_heads(1, 1, S + 1, d)
    rows = np.zeros((S, d), np.float32)
    for s, x in enumerate(EXTREMES):
        rows[s] = np.float32(x) * (rng.random(d) < 0.5)
        rows[s, s % d] = x
    bits = f32_to_bf16_bits(rows)
    for i in range(S):  # token i of sequence s: extreme (s + i) mod S
        order = [(s + i) % S for s in range(S)]
        x = bits[order][None, :, None]
        cu = dev(offsets([1] * S + [0]))
        C8.advance8(cache, cu)
        C8.append8(cache, B.bf16_from_bits(x), B.bf16_from_bits(x[..., ::-1].copy()), cu)
        for s in range(S):
            y = decode_bf16(x[0, s:s + 1, 0])
            heads[0, 0, s].append(y, y[:, ::-1], np.array([i]))
    cu = dev(offsets([0] * S + [S]))
    C8.advance8(cache, cu)
    C8.append8(cache, B.bf16_from_bits(bits[None, :, None]), B.bf16_from_bits(bits[None, ::-1, None].copy()), cu)
    heads[0, 0, S].append(decode_bf16(bits), decode_bf16(bits)[::-1], np.arange(S))
    assert cache.status() == 0
    check(cache, heads)
    lens = [S] * (S + 1)
    k, v = C8.read8(cache, dev(offsets(lens)), sum(lens))
    for s in range(S + 1):
        for which, t in enumerate((k, v)):
            got = t[0, 0, s * S:(s + 1) * S].double().cpu().numpy()
            assert np.isfinite(got).all() and np.array_equal(got, heads[0, 0, s].values(which))


def test_not_finite(gpu_lib):
    """A NaN or an infinity is held as NaN, changes no other element, and is reported."""
    rng = np.random.default_rng(9)
    for bad in (0x7FC0, 0xFFC0, 0x7F80, 0xFF80, 0x7F81):
        for where in (0, 1):
            cache = filled(C8.Cache8(1, 2, 64, [0, 90]))
            x = [bf16(rng, (1, 80, 2, 64)) for _ in range(2)]
            x[where][0, 70, 1, 5] = bad
            heads = empty_heads(1, 2, 1, 64)
            for (l, h, s), a in heads.items():
                a.append(decode_bf16(x[0][0, :, h]), decode_bf16(x[1][0, :, h]), np.arange(80))
            cu = dev([0, 80])
            C8.advance8(cache, cu)
            C8.append8(cache, B.bf16_from_bits(x[0]), B.bf16_from_bits(x[1]), cu)
            assert np.isnan(heads[0, 1, 0].num[where]).sum() == 1
            check(cache, heads)
            assert cache.status(clear=True) == B.FLAG_NONFINITE
            # and again when the block grows
            y = bf16(rng, (1, 1, 2, 64), 2.0 ** 20)
            cu = dev([0, 1])
            C8.advance8(cache, cu)
            C8.append8(cache, B.bf16_from_bits(y), B.bf16_from_bits(y), cu)
            for (l, h, s), a in heads.items():
                a.append(decode_bf16(y[0, :, h]), decode_bf16(y[0, :, h]), np.array([80]))
            check(cache, heads)
            assert cache.status() == 0


def test_append_more_tokens_than_the_sequence_counts(gpu_lib):
    """Without advance8 the sequence has fewer tokens than are new: the last of them are its
    tokens, nothing is written before its first row; and tokens past num_new are not read, whose
    rows keep their bytes."""
    x = bf16(np.random.default_rng(5), (1, 8, 1, 64))
    t, y = B.bf16_from_bits(x), decode_bf16(x[0, :, 0])
    cache = filled(C8.Cache8(1, 1, 64, [0, 64, 128]))
    cache.lens.copy_(dev([0, 3]))
    cache.seen.copy_(dev([0, 9]))
    C8.append8(cache, t, t, dev([0, 0, 8]))
    heads = empty_heads(1, 1, 2, 64)
    heads[0, 0, 1].append(y[5:], y[5:], np.arange(6, 9))
    check(cache, heads)
    cache = filled(C8.Cache8(1, 1, 64, [0, 64, 128]))
    cache.lens.copy_(dev([6, 6]))
    cache.seen.copy_(dev([6, 6]))
    C8.append8(cache, t, t, dev([0, 6, 12]))
    heads = empty_heads(1, 1, 2, 64)
    heads[0, 0, 0].append(y[:6], y[:6], np.arange(6))
    heads[0, 0, 1].append(y[6:], y[6:], np.arange(2))
    check(cache, heads)
    assert cache.status() == B.FLAG_OUT_ROWS


@pytest.mark.parametrize("shared", [False, True])
def test_positions_outside_their_sequence(shared, gpu_lib):
    """Their rows keep their bytes; the block's scale is that of the rows that are written, and
    a block of nothing else keeps its own."""
    import torch

    rng = np.random.default_rng(6)
    L, H, d, n = 1, 2, 64, 300
    k = bf16(rng, (L, H, n, d))
    idx = np.tile(np.arange(n, dtype=np.int32), (1 if shared else L * H, 1))
    bad = [3, 70, 71] + list(range(128, 192))
    idx[:, bad] = [(-1, n, 1 << 30)[i % 3] for i in range(len(bad))]
    cache = filled(C8.Cache8(L, H, d, [0, n]))
    pb = B.Problem(L, H, H, d, 1, [0, n], [0, 0])
    kt = B.bf16_from_bits(k)
    C8.compact8(pb, cache, kt, kt, torch.from_numpy(idx[0] if shared else idx.reshape(L, H, n)).cuda(), dev([0, n]))
    assert cache.lens.tolist() == [n] and cache.status() == B.FLAG_OUT_ROWS
    good = np.array([j for j in range(n) if j not in bad])
    codes, scales = cache.k_codes.cpu().numpy(), cache.k_scales.cpu().numpy()
    for h in range(H):
        assert (codes[0, h, bad] == FILL).all()
        for b in range(5):
            rows = good[good // 64 == b]
            if b == 2:
                assert scales[0, h, b].tobytes() == bytes([FILL] * 4)
                continue
            e = R.need(decode_bf16(k[0, h, rows]))
            assert scales[0, h, b] == 2.0 ** e
            assert np.array_equal(R.NUMBERS[codes[0, h, rows]], R.round8(decode_bf16(k[0, h, rows]) / 2.0 ** e))


def test_more_retained_rows_than_the_source_has(gpu_lib):
    """A sequence gets no more tokens than its source has, whatever cu_retained counts, and that is
    reported."""
    rng = np.random.default_rng(7)
    src = [40, 0, 90]
    cu_seq = offsets(src)
    k = bf16(rng, (1, 1, 130, 64))
    cache = filled(C8.Cache8(1, 1, 64, [0, 130, 150, 250]))
    pb = B.Problem(1, 1, 1, 64, 1, cu_seq, np.zeros(4, np.int32))
    idx = dev(np.concatenate([np.arange(x) for x in src]))
    kt = B.bf16_from_bits(k)
    C8.compact8(pb, cache, kt, kt, idx, dev([0, 50, 57, 157]))
    heads = empty_heads(1, 1, 3, 64)
    for (l, h, s), a in heads.items():
        x = decode_bf16(k[0, 0, cu_seq[s]:cu_seq[s + 1]])
        a.append(x, x, np.arange(src[s]))
    check(cache, heads)
    assert cache.lens.tolist() == src and cache.status() == B.FLAG_OUT_ROWS


def test_layers_one_by_one_and_without_weights(gpu_lib):
    """Layers written through views, as a model does, and a cache that keeps no weights."""
    import torch

    L, H, d = 3, 2, 64
    whole, parts, bare = (filled(C8.Cache8(L, H, d, [0, 33, 64], weights=w)) for w in (True, True, False))
    t = B.bf16_from_bits(bf16(np.random.default_rng(6), (2, L, 7, H, d)))
    cu = dev([0, 4, 7])
    for c in (whole, parts, bare):
        C8.advance8(c, cu)
    C8.append8(whole, t[0], t[1], cu)
    C8.append8(bare, t[0], t[1], cu)
    for l in range(L):
        C8.append8(parts.layers(l), t[0, l:l + 1], t[1, l:l + 1], cu)
    for x in ("k_codes", "v_codes", "k_scales", "v_scales", "weights", "positions"):
        a = getattr(whole, x).view(torch.uint8)
        assert torch.equal(a, getattr(parts, x).view(torch.uint8))
        assert getattr(bare, x) is None or torch.equal(a, getattr(bare, x).view(torch.uint8))
    k, v = C8.read8(parts.layers(1, 2), cu, 7)
    kw, vw = C8.read8(whole, cu, 7)
    assert torch.equal(k, kw[1:]) and torch.equal(v, vw[1:])


def test_read_of_sequences_within_a_workgroup(gpu_lib):
    """Many short and empty sequences, whose rows share a workgroup, and counts past what they hold."""
    rng = np.random.default_rng(8)
    lens = [int(x) for x in rng.integers(0, 5, 300)] + [200, 0, 65]
    S, d = len(lens), 64
    cache = C8.Cache8(2, 1, d, offsets(np.add(lens, 2)))
    x = bf16(rng, (2, sum(lens), 1, d))
    cu = offsets(lens)
    C8.advance8(cache, dev(cu))
    C8.append8(cache, B.bf16_from_bits(x), B.bf16_from_bits(x), dev(cu))
    counts = [n + (i % 3 == 0) for i, n in enumerate(lens)]  # some ask for one more than there is
    co = offsets(counts)
    import torch

    out = torch.full((2, 1, int(co[-1]), d), 7.0, dtype=torch.bfloat16, device="cuda")
    C8.read8(cache, dev(co), int(co[-1]), k_out=out, v_out=False)
    out = out.double().cpu().numpy()
    for l in range(2):
        for s, n in enumerate(lens):
            a = R.Head8(d)
            y = decode_bf16(x[l, cu[s]:cu[s + 1], 0])
            a.append(y, y, np.arange(n))
            got = out[l, 0, co[s]:co[s + 1]]
            assert (got[:counts[s] - n] == 7).all() and np.array_equal(got[counts[s] - n:], a.values(0))


def test_rows_past_four_gigabytes(gpu_lib):
    """The last rows of a cache of 4.5 GB of codes a tensor: written, read back, attended to, evicted."""
    import torch

    L, H, d, R_ = 1, 9, 128, 1 << 22
    cache = C8.Cache8(L, H, d, [0, R_ - 700, R_])
    rng = np.random.default_rng(11)
    x = bf16(rng, (L, 600, H, d))
    cu = dev([0, 0, 600])
    C8.advance8(cache, cu)
    C8.append8(cache, B.bf16_from_bits(x), B.bf16_from_bits(x), cu)
    k, v = C8.read8(cache, cu, 600)
    a = R.Head8(d)
    y = decode_bf16(x[0, :, H - 1])
    a.append(y, y, np.arange(600))
    assert np.array_equal(k[0, H - 1].double().cpu().numpy(), a.values(0)) and torch.equal(k, v)
    q = torch.zeros((L, 2, H, d), dtype=torch.bfloat16, device="cuda")
    out = C8.decode_attention8(cache, q, gather=True)
    mean = k.double().mean(dim=2)  # logits of 0: every token weighs the same
    assert (out[:, 0] == 0).all()
    assert (out[:, 1].double() - mean).abs().max() <= 1e-5 * k.double().abs().max()
    w = cache.weights[:, :, R_ - 700:R_ - 100].double()
    assert (w * 600 - 1).abs().max() < 1e-5
    cache.weights[:, :, R_ - 700:R_ - 100] = torch.arange(600, device="cuda").float()
    C8.evict8(cache, 500)
    assert cache.lens.tolist() == [0, 500]
    want = torch.cat([torch.arange(500, 600), torch.arange(100, 500)]).to(cache.positions)
    assert (cache.positions[:, :, R_ - 700:R_ - 200] == want).all()
