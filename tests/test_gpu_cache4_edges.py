"""The 4-bit cache on the GPU where a call's arguments leave something out: rows without a source,
and the block bounds over them. Everything is compared bit for bit with the fp64 oracle: every step
of the format is exact, and so are least and greatest values."""
import zlib

import numpy as np
import pytest

import oracle.cache4_ref as R
from oracle import decode_bf16
from paper_2609_22158_amd import binding as B
from paper_2609_22158_amd import cache4 as C4
from tests.gpu_cases import log
from tests.test_gpu_cache4 import bf16, host

pytestmark = pytest.mark.gpu


def full_cache(rng, L, H, d, rooms, nan_rows=()):
    """A cache whose every row holds a token (some with a NaN key), and the values of its keys."""
    import torch

    n = sum(rooms)
    cu = np.concatenate([[0], np.cumsum(rooms)]).astype(np.int32)
    cache = C4.Cache4(L, H, d, cu)
    k = bf16(rng, (L, n, H, d), 4.0)
    for r in nan_rows:
        k[:, r, :, 1] = 0x7FC0
    dev = torch.from_numpy(cu).cuda()
    C4.advance4(cache, dev)
    C4.append4(cache, B.bf16_from_bits(k), B.bf16_from_bits(bf16(rng, (L, n, H, d))), dev)
    cache.status(clear=True)
    return cache, cu, stored_keys(cache)


def stored_keys(cache):
    codes, scales = host(cache)[:2]
    return R.dequantise4(codes, scales)


def check_all_bounds(cache, cu, lens):
    """Every block's bounds are the least and greatest keys of the rows that hold its tokens."""
    keys, got = stored_keys(cache), cache.k_bounds.float().cpu().numpy()
    for s, n in enumerate(lens):
        at, r = int(cu[s]) // 64 + s, int(cu[s])
        for l in range(cache.num_layers):
            for h in range(cache.num_kv_heads):
                want = R.block_bounds(keys[l, h, r:r + n])
                assert np.array_equal(got[l, h, at:at + len(want)], want, equal_nan=True), (l, h, s)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shared", [False, True])
def test_bounds_over_rows_that_a_compaction_leaves(d, shared, gpu_lib):
    """Positions outside their sequence: single ones, a whole block of them (the bounds are those of
    what its rows hold), one at a row with a NaN key, and a sequence of nothing else."""
    import torch

    log(f"[edges compact d={d} shared={shared}]")
    rng = np.random.default_rng(zlib.crc32(b"left") + d)
    L, H, src, kept, rooms = 2, 2, [700, 130, 40], [300, 65, 3], [310, 65, 64]
    cache, cu, old = full_cache(rng, L, H, d, rooms, nan_rows=(200, 310 + 64))
    cu_seq, cu_ret = (np.concatenate([[0], np.cumsum(x)]).astype(np.int32) for x in (src, kept))
    n = int(cu_seq[-1])
    k, v = bf16(rng, (L, H, n, d)), bf16(rng, (L, H, n, d))
    idx = np.full((1 if shared else L * H, n), -7, np.int32)
    bad = [(0, j) for j in [5, 200, 299] + list(range(64, 128))] + [(1, 64), (2, 0), (2, 1), (2, 2)]
    for r in range(idx.shape[0]):
        for s in range(3):
            idx[r, cu_seq[s]:cu_seq[s] + kept[s]] = np.sort(rng.permutation(src[s])[:kept[s]])
        for i, (s, j) in enumerate(bad):
            idx[r, cu_seq[s] + j] = (-1, src[s], 1 << 30)[(i + r) % 3]
    pb = B.Problem(L, H, H, d, 1, cu_seq, np.zeros(4, np.int32))
    C4.compact4(pb, cache, B.bf16_from_bits(k), B.bf16_from_bits(v),
                torch.from_numpy(idx[0] if shared else idx.reshape(L, H, n)).cuda(),
                torch.from_numpy(cu_ret).cuda())
    assert cache.lens.tolist() == kept
    now = stored_keys(cache)
    for s, j in bad:
        assert np.array_equal(now[:, :, cu[s] + j], old[:, :, cu[s] + j], equal_nan=True)
    check_all_bounds(cache, cu, kept)
    assert cache.status() == B.FLAG_OUT_ROWS


@pytest.mark.parametrize("num_new,counts", [(8, (6, 6, 0)), (1, (5, 500, 260)), (300, (300, 1, 129)),
                                            (70, (0, 69, 3))])
def test_bounds_over_rows_of_tokens_that_were_not_given(num_new, counts, gpu_lib):
    """New tokens at or past num_new: their rows stay as they were, and every block that counts them
    has bounds over what it holds, however many blocks they are."""
    import torch

    log(f"[edges append num_new={num_new} counts={counts}]")
    rng = np.random.default_rng(zlib.crc32(b"given") + num_new)
    L, H, d, rooms = 2, 1, 64, [400, 700, 261]
    cache, cu, old = full_cache(rng, L, H, d, rooms, nan_rows=(390, 400 + 650))
    cache.k_bounds.fill_(77.0)  # of nothing that the cache holds
    before = [100, 3, 0]
    first = torch.tensor(np.concatenate([[0], np.cumsum(before)]), dtype=torch.int32, device="cuda")
    x = bf16(rng, (L, 103, H, d))
    cache.lens.copy_(torch.tensor(before))
    C4.append4(cache, B.bf16_from_bits(x), B.bf16_from_bits(x), first)
    cu_new = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
    y = bf16(rng, (L, num_new, H, d))
    C4.advance4(cache, cu_new)
    C4.append4(cache, B.bf16_from_bits(y), B.bf16_from_bits(y), cu_new)
    lens = [a + b for a, b in zip(before, counts)]
    assert cache.lens.tolist() == lens
    now, at = stored_keys(cache), 0
    for s, n in enumerate(counts):
        r = cu[s] + before[s]
        got = max(0, min(n, num_new - at))  # of the sequence's new tokens, those that were given
        want = R.dequantise4(*R.quantise4(decode_bf16(y[:, at:at + got, 0])))
        assert np.array_equal(now[:, 0, r:r + got], want)
        assert np.array_equal(now[:, 0, r + got:cu[s + 1]], old[:, 0, r + got:cu[s + 1]], equal_nan=True)
        at += n
    check_all_bounds(cache, cu, lens)
    assert cache.status() == (B.FLAG_OUT_ROWS if sum(counts) > num_new else 0)


def test_more_retained_rows_than_the_source_has(gpu_lib):
    """A sequence gets no more tokens than its source has, whatever cu_retained counts, and that is
    reported: the rows behind them, which nothing wrote, are not attended to."""
    import torch

    rng = np.random.default_rng(zlib.crc32(b"retained"))
    L, H, d, src, rooms = 1, 2, 64, [40, 0, 90], [130, 20, 100]
    cache, cu, old = full_cache(rng, L, H, d, rooms, nan_rows=(45, 135, 245))
    cu_seq = np.concatenate([[0], np.cumsum(src)]).astype(np.int32)
    n = int(cu_seq[-1])
    k, v = bf16(rng, (L, H, n, d)), bf16(rng, (L, H, n, d))
    idx = np.concatenate([np.arange(x) for x in src]).astype(np.int32)
    pb = B.Problem(L, H, H, d, 1, cu_seq, np.zeros(4, np.int32))
    C4.compact4(pb, cache, B.bf16_from_bits(k), B.bf16_from_bits(v), torch.from_numpy(idx).cuda(),
                torch.tensor([0, 50, 57, 157], dtype=torch.int32, device="cuda"))
    assert cache.lens.tolist() == src
    assert cache.status(clear=True) == B.FLAG_OUT_ROWS
    check_all_bounds(cache, cu, src)
    now = stored_keys(cache)
    for s, m in enumerate(src):
        assert np.array_equal(now[:, :, cu[s] + m:cu[s + 1]], old[:, :, cu[s] + m:cu[s + 1]], equal_nan=True)
    q = torch.ones((L, 3, H, d), dtype=torch.bfloat16, device="cuda")
    out = C4.decode_attention4(cache, q)
    assert torch.isfinite(out).all() and (out[0, 1] == 0).all() and cache.status() == 0


@pytest.mark.parametrize("lens,n", [([64 * 40], 5), ([64 * 900, 3000], 7), ([64 * 5000], 100)])
@pytest.mark.parametrize("d", [64, 128])
def test_a_nan_in_one_query_of_a_group(d, lens, n, gpu_lib):
    """One NaN element of one head makes every score of its group NaN, which ranks as -inf: the lowest
    blocks beside the forced ones. Other groups, sequences and layers rank theirs as before."""
    import torch

    L, H, G, S = 2, 2, 3, len(lens)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(12)
    x = torch.randn((L, H, int(cu[-1]) // 64 + S, 2, d), generator=gen, device="cuda")
    bounds = x.sort(dim=3).values.bfloat16()
    cache = C4.Cache4(L, H, d, cu, k_bounds=bounds, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    q = torch.randn((L, S, H * G, d), generator=gen, device="cuda").bfloat16()
    q[1, 0, 4, 17] = float("nan")
    got = C4.select_blocks4(cache, q, n, first=1, last=2).cpu().numpy()
    for s in range(S):
        nb, at = -(-lens[s] // 64), int(cu[s]) // 64 + s
        for l in range(L):
            for h in range(H):
                score = R.block_scores(q[l, s, h * G:(h + 1) * G].double().cpu().numpy(),
                                       bounds[l, h, at:at + nb].double().cpu().numpy())
                assert np.isnan(score).all() == ((l, s, h) == (1, 0, 1))
                assert np.array_equal(got[l, s, h], R.select_blocks(score, n, 1, 2)), (l, s, h)
    assert got[1, 0, 1].tolist() == list(range(n - 2)) + [-(-lens[0] // 64) - 2, -(-lens[0] // 64) - 1]


LOST = {
    # name: (G, d, tokens of each sequence, which tokens have a logit of -inf)
    "one_split": (3, 64, [500, 64, 0, 33], lambda s, j: s != 3 or j < 20),
    "one_split_g7": (7, 128, [700, 65, 1], lambda s, j: s == 0 or j < 32),
    "splits": (3, 128, [6000, 2000, 0], lambda s, j: s == 0 or j < 1700),
    "splits_g7": (7, 64, [9000, 4000], lambda s, j: s == 0 or (j // 128) % 2 == 0),
    "many": (1, 64, [2100 if i % 40 == 0 else 70 for i in range(600)], lambda s, j: s % 2 == 0 or j < 64),
}


@pytest.mark.parametrize("cid", list(LOST))
def test_logits_of_minus_infinity(cid, gpu_lib):
    """Head 0's logits are 0, or overflow to -inf. A token of -inf has no weight beside others; where
    there is no other, the result is the softmax of such logits, NaN (not the zeros of a sequence
    without tokens), and the log-sum-exp -inf. Over lists of blocks alike. A mean over n values in
    fp32: off by (2 n + 64) u of the mean magnitude, as the other sums of attention's tests."""
    import torch

    from tests.test_gpu_attend4 import Made, U

    G, d, lens, gone = LOST[cid]
    log(f"[edges -inf {cid}] tokens={lens[:4]}")
    m = Made("lost " + cid, 1, G, 1, d, lens, [n + 3 for n in lens])
    S = len(lens)
    away = [np.array([gone(s, j) for j in range(n)], bool) for s, n in enumerate(lens)]
    for s in range(S):
        a = m.cu[s]
        m.k_bits[0, a:a + lens[s], 0, 0] = np.where(away[s], 0xC100, 0)  # -8, exact in 4 bits here
    m.q_bits[0, :, 0] = 0
    m.q_bits[0, :, 0, 0] = 0x7F60  # 2.98e38: times -8 past fp32's range
    m.write()
    assert all((m.rows(0, s, 0)[0][:, 0] == np.where(away[s], -8, 0)).all() for s in range(S))

    def check(out, lse, seen):
        out, lse = out.cpu().numpy()[0, :, 0], lse.cpu().numpy()[0, :, 0]
        for s, n in enumerate(lens):
            keep = seen[s] & ~away[s]
            if not seen[s].any():
                assert (out[s] == 0).all() and lse[s] == -np.inf, s
            elif not keep.any():
                assert np.isnan(out[s]).all() and lse[s] == -np.inf, s
            else:
                v = m.rows(0, s, 0)[1][keep]
                steps = 2.0 ** -19 + (2 * n + 64) * U
                assert (np.abs(out[s] - v.mean(axis=0)) <= 2 * steps * np.abs(v).mean(axis=0)).all(), s
                assert abs(lse[s] - np.log(len(v))) <= steps + 4 * U * np.log(len(v)), s

    out, lse = C4.decode_attention4(m.cache, m.q, want_lse=True)
    check(out, lse, [np.ones(n, bool) for n in lens])
    assert torch.isfinite(out[:, :, 1:]).all()
    rng = np.random.default_rng(3)
    most = max(-(-n // 64) for n in lens)
    for n in (2, most):
        lists = np.full((1, S, 1, n), -1, np.int32)
        seen = []
        for s in range(S):
            nb = -(-lens[s] // 64)
            pick = np.sort(rng.permutation(nb)[:rng.integers(0, min(n, nb) + 1)])
            lists[0, s, 0, :len(pick)] = pick
            keep = np.zeros(nb, bool)
            keep[pick] = True
            seen.append(keep.repeat(64)[:lens[s]])
        out, lse = C4.decode_attention4(m.cache, m.q, blocks=torch.from_numpy(lists).cuda(), want_lse=True)
        check(out, lse, seen)
    assert m.cache.status() == 0


def test_a_read_of_more_rows_than_one_row_a_thread_covers(gpu_lib):
    """2^28 rows and some of d 128 (64 GiB): past a launch of one row a thread. The tokens are the
    last rows; the others stay as they were."""
    import torch

    rows, n, d = 2 ** 28 + 1000, 100, 128
    if torch.cuda.mem_get_info()[0] < (rows * d * 2) + (8 << 30):
        pytest.skip("not enough memory on this GPU")
    rng = np.random.default_rng(zlib.crc32(b"read"))
    cache, cu, keys = full_cache(rng, 1, 1, d, [n])
    out = torch.empty((1, 1, rows, d), dtype=torch.bfloat16, device="cuda")
    tail = out[0, 0, -5000:]
    tail.fill_(7.0)
    C4.read4(cache, torch.tensor([0, rows], dtype=torch.int32, device="cuda"), rows, k_out=out, v_out=False)
    got = tail.float().cpu().numpy()
    del out, tail
    torch.cuda.empty_cache()
    assert (got[:-n] == 7).all() and np.array_equal(got[-n:], keys[0, 0])
