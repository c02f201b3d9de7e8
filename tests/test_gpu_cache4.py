"""The 4-bit cache on the GPU: written by compaction and appending, read back, and its block
bounds, all bit for bit against the fp64 oracle (every step of the format is exact, so nothing
has a tolerance), and bytes that a call does not own, which stay as they were."""
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

FILL = 0xA5  # in every byte of a buffer before a call


def filled(cache):
    for t in (cache.k_codes, cache.v_codes, cache.k_scales, cache.v_scales):
        t.fill_(FILL)
    return cache


def host(cache):
    """codes, scales of K and V and the bounds, as numpy arrays (bounds as float64)."""
    return [t.cpu().numpy() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)] + [
        None if cache.k_bounds is None else cache.k_bounds.float().cpu().numpy().astype(np.float64)]


def bf16(rng, shape, scale=1.0):
    """Random bf16 bits: normal, with a few outlier channels and some rows far larger or smaller."""
    x = rng.standard_normal(shape) * scale
    x[..., rng.integers(0, shape[-1], 3)] *= 8
    x *= 2.0 ** rng.integers(-4, 5, shape[:-1] + (1,))
    return f32_to_bf16_bits(x.astype(np.float32))


def check_rows(cache, want_k, want_v, rows_of):
    """The cache holds want_k/v[(l, h, s)] (values [n][d], None: untouched) in rows_of[s] and FILL
    everywhere else."""
    kc, ks, vc, vs, _ = host(cache)
    for codes, scales, want in ((kc, ks, want_k), (vc, vs, want_v)):
        ec = np.full_like(codes, FILL)
        es = np.full_like(scales, FILL)
        for (l, h, s), x in want.items():
            r = rows_of[s]
            ec[l, h, r:r + len(x)], es[l, h, r:r + len(x)] = R.quantise4(x)
        assert np.array_equal(es, scales)
        assert np.array_equal(ec, codes)


def check_bounds(cache, want_k, s, l, h):
    """The bounds of sequence s are those of its quantised keys want_k [n][d]."""
    at = int(cache.cu_rows[s]) // 64 + s
    y = R.dequantise4(*R.quantise4(want_k))
    got = cache.k_bounds[l, h].float().cpu().numpy()[at:at + -(-len(y) // 64)]
    assert np.array_equal(got, R.block_bounds(y), equal_nan=True), (l, h, s)


COMPACT = {
    # name: (L, Hq, Hkv, d, source tokens, retained, room beyond retained, shared)
    "d128": (2, 8, 2, 128, [700, 130, 65], [300, 64, 65], [10, 0, 7], False),
    "d64": (3, 4, 4, 64, [500, 33, 200], [129, 33, 1], [3, 40, 63], False),
    "shared": (2, 4, 2, 128, [400, 90], [191, 63], [0, 5], True),
    "empty": (1, 2, 1, 64, [0, 100, 0, 5], [0, 0, 0, 5], [4, 9, 0, 0], False),
    "one": (1, 1, 1, 128, [1], [1], [0], False),
    "many_seqs": (1, 2, 2, 64, [3] * 150, [2] * 150, [1] * 150, True),
}


def compaction(cid):
    import torch

    L, Hq, Hkv, d, src, kept, room, shared = COMPACT[cid]
    rng = np.random.default_rng(zlib.crc32(cid.encode()))
    S = len(src)
    cu_seq = np.concatenate([[0], np.cumsum(src)]).astype(np.int32)
    cu_ret = np.concatenate([[0], np.cumsum(kept)]).astype(np.int32)
    cu_rows = np.concatenate([[0], np.cumsum(np.add(kept, room))]).astype(np.int32)
    n = int(cu_seq[-1])
    k, v = bf16(rng, (L, Hkv, n, d)), bf16(rng, (L, Hkv, n, d))
    idx = np.full((1 if shared else L * Hkv, n), -7, np.int32)
    for r in range(idx.shape[0]):
        for s in range(S):
            idx[r, cu_seq[s]:cu_seq[s] + kept[s]] = np.sort(rng.permutation(src[s])[:kept[s]])
    pb = B.Problem(L, Hq, Hkv, d, 1, cu_seq, np.zeros(S + 1, np.int32))
    cache = filled(C4.Cache4(L, Hkv, d, cu_rows))
    want_k, want_v = {}, {}
    for l in range(L):
        for h in range(Hkv):
            for s in range(S):
                i = cu_seq[s] + idx[0 if shared else l * Hkv + h, cu_seq[s]:cu_seq[s] + kept[s]]
                want_k[l, h, s], want_v[l, h, s] = decode_bf16(k[l, h, i]), decode_bf16(v[l, h, i])
    args = dict(k=B.bf16_from_bits(k), v=B.bf16_from_bits(v),
                idx=torch.from_numpy(idx[0] if shared else idx.reshape(L, Hkv, n)).cuda(),
                cu_retained=torch.from_numpy(cu_ret).cuda())
    return pb, cache, args, want_k, want_v, kept, cu_rows


@pytest.mark.parametrize("cid", list(COMPACT))
def test_compact_and_read_back(cid, gpu_lib):
    import torch

    pb, cache, args, want_k, want_v, kept, cu_rows = compaction(cid)
    log(f"[cache4 compact {cid}] rows={kept}")
    C4.compact4(pb, cache, **args)
    assert cache.lens.tolist() == kept and cache.status() == 0
    check_rows(cache, want_k, want_v, cu_rows)
    for (l, h, s), x in want_k.items():
        if len(x):
            check_bounds(cache, x, s, l, h)
    # the whole sequences back, behind each other; rows past the last stay as they were
    total = int(args["cu_retained"][-1])
    shape = (cache.num_layers, cache.num_kv_heads, total + 3, cache.head_dim)
    ko = torch.full(shape, 7.0, dtype=torch.bfloat16, device="cuda")
    vo = torch.full(shape, 7.0, dtype=torch.bfloat16, device="cuda")
    C4.read4(cache, args["cu_retained"], total + 3, k_out=ko, v_out=vo)
    for out, want in ((ko, want_k), (vo, want_v)):
        got = out.float().cpu().numpy()
        assert (got[:, :, total:] == 7).all()
        for (l, h, s), x in want.items():
            a = int(args["cu_retained"][s])
            assert np.array_equal(got[l, h, a:a + len(x)], R.dequantise4(*R.quantise4(x)))
    # K alone, no longer than out_rows; then nothing but the last rows
    if total > 2:
        k2, none = C4.read4(cache, args["cu_retained"], total - 2, v_out=False)
        assert none is None and torch.equal(k2, ko[:, :, :total - 2])
    last = torch.tensor([0] + list(np.cumsum([min(n, 1) for n in kept])), dtype=torch.int32, device="cuda")
    k3, v3 = C4.read4(cache, last, int(last[-1]))
    rows = [int(args["cu_retained"][s]) + n - 1 for s, n in enumerate(kept) if n]
    assert torch.equal(k3, ko[:, :, rows]) and torch.equal(v3, vo[:, :, rows])
    # written again from what was read back: the same cache (nothing more is lost)
    again = filled(C4.Cache4(cache.num_layers, cache.num_kv_heads, cache.head_dim, cu_rows))
    new = [t[:, :, :total].transpose(1, 2) for t in (ko, vo)]
    again.lens.copy_(cache.lens)
    C4.append4(again, *new, args["cu_retained"])
    for s, n in enumerate(kept):
        r = int(cu_rows[s])
        for a, b in ((again.k_codes, cache.k_codes), (again.v_scales, cache.v_scales)):
            assert torch.equal(a[:, :, r:r + n], b[:, :, r:r + n])


def test_compact_without_room_and_with_bad_positions(gpu_lib):
    """More retained rows than room: the rest is dropped and reported, lens counts it. Positions
    outside their sequence leave their rows as they were."""
    import torch

    pb, cache, args, want_k, want_v, kept, cu_rows = compaction("d128")
    rooms = [250, 64, 60]
    cu_rows = np.concatenate([[0], np.cumsum(rooms)]).astype(np.int32)
    cache = filled(C4.Cache4(2, 2, 128, cu_rows))
    bad = {5: -1, 70: 700, 249: 1 << 30}  # of sequence 0, every head
    for j, pos in bad.items():
        args["idx"][:, :, j] = pos
    C4.compact4(pb, cache, **args)
    assert cache.lens.tolist() == kept
    assert cache.status(clear=True) == B.FLAG_OUT_ROWS
    kc, ks, _, _, _ = host(cache)
    for (l, h, s), x in want_k.items():
        codes, scales = R.quantise4(x[:rooms[s]])
        if s == 0:
            for j in bad:
                codes[j], scales[j] = FILL, FILL
        r = cu_rows[s]
        assert np.array_equal(kc[l, h, r:r + rooms[s]], codes)
        assert np.array_equal(ks[l, h, r:r + rooms[s]], scales)
    out = torch.full((2, 2, 429, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    C4.read4(cache, args["cu_retained"], 429, k_out=out, v_out=False)  # tokens past the room: none
    got = out.float().cpu().numpy()
    a = int(args["cu_retained"][2])
    assert (got[:, :, 250:300] == 7).all() and (got[:, :, a + 60:] == 7).all()
    assert np.array_equal(got[1, 1, a:a + 60], R.dequantise4(*R.quantise4(want_k[1, 1, 2][:60])))


def test_compact_from_no_tokens(gpu_lib):
    """A source without a token empties the cache's sequences; reads of them give nothing."""
    import torch

    cache = filled(C4.Cache4(1, 2, 64, [0, 8, 16]))
    cache.lens.fill_(5)
    pb = B.Problem(1, 2, 2, 64, 1, np.zeros(3, np.int32), np.zeros(3, np.int32))
    none = torch.empty((1, 2, 0, 64), dtype=torch.bfloat16, device="cuda")
    cu = torch.zeros(3, dtype=torch.int32, device="cuda")
    C4.compact4(pb, cache, none, none, torch.empty((1, 2, 0), dtype=torch.int32, device="cuda"), cu)
    assert cache.lens.tolist() == [0, 0]
    check_rows(cache, {}, {}, [0, 8])
    q = torch.ones((1, 2, 2, 64), dtype=torch.bfloat16, device="cuda")
    out, blocks, lse = C4.decode_sparse4(cache, q, 3, want_lse=True)
    assert (out == 0).all() and (blocks == -1).all() and (lse == -np.inf).all()


def test_append_past_a_full_room(gpu_lib):
    """New tokens that lie past the room altogether write nothing, whatever block they would be in."""
    import torch

    cache = filled(C4.Cache4(1, 1, 64, [0, 66]))
    t = B.bf16_from_bits(bf16(np.random.default_rng(8), (1, 80, 1, 64)))
    first = torch.tensor([0, 66], dtype=torch.int32, device="cuda")
    C4.advance4(cache, first)
    C4.append4(cache, t[:, :66], t[:, :66], first)
    before = [x for x in host(cache)]
    cache.lens.fill_(80)
    C4.append4(cache, t[:, 70:], t[:, 70:], torch.tensor([0, 10], dtype=torch.int32, device="cuda"))
    assert all(np.array_equal(x, y) for x, y in zip(before, host(cache)))
    assert cache.status() == B.FLAG_OUT_ROWS


def test_values_at_the_edges(gpu_lib):
    """NaN, infinities, zeros, signed zeros, the largest and the smallest magnitudes, ties."""
    import torch

    d, n = 64, 70
    x = np.zeros((n, d), np.uint16)
    x[0, :4] = [0x7FC0, 0x3F80, 0x0000, 0x8000]      # a NaN: its group reads back as NaN
    x[1, 33] = 0xFF80                                  # -inf in the second group
    x[2] = 0x8000                                      # all -0
    x[3, :3] = [0x7F7F, 0xFF7F, 0x7F00]                # the largest finite values
    x[4, :4] = [0x0001, 0x807F, 0x0080, 0x0000]        # subnormals and the least normal
    x[5, :6] = f32_to_bf16_bits(np.array([7, 0.25, 0.75, -1.25, 2.5, 3.5], np.float32))
    x[6, :3] = f32_to_bf16_bits(np.array([7.0625, 5, 0.5], np.float32))
    # every bf16 pattern of one binade and the ones around it, as a group's largest value
    x[7:, :32] = (0x3F00 + 5 * np.arange((n - 7) * 32)).reshape(-1, 32) % 0x7F80
    x[7:, 32:] = x[7:, :32] | 0x8000
    cache = filled(C4.Cache4(1, 1, d, [0, n]))
    t = B.bf16_from_bits(x)[None, :, None]
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    C4.advance4(cache, cu)
    C4.append4(cache, t, torch.zeros_like(t), cu)
    assert cache.status(clear=True) == B.FLAG_NONFINITE
    codes, scales = R.quantise4(decode_bf16(x))
    kc, ks, vc, vs, bounds = host(cache)
    assert np.array_equal(ks[0, 0], scales) and np.array_equal(kc[0, 0], codes)
    assert (vs == 3).all() and (vc == 0).all()
    y = R.dequantise4(codes, scales)
    k, _ = C4.read4(cache, cu, n)
    assert np.array_equal(k[0, 0].float().cpu().numpy(), y, equal_nan=True)
    assert np.array_equal(bounds[0, 0, :2], R.block_bounds(y), equal_nan=True)
    # more tokens do not take the NaN out of a block's bounds
    C4.append4(cache, t[:, 1:3] * 0, torch.zeros_like(t[:, :2]),
               torch.tensor([0, 2], dtype=torch.int32, device="cuda"))
    assert np.isnan(cache.k_bounds[0, 0, 0, 0, :32].float().cpu().numpy()).all()


APPEND = {
    # name: (L, Hkv, d, tokens before, new tokens, room, layout)
    "token": (2, 4, 128, [0, 63, 64, 200], [1, 1, 1, 1], 300, "token"),
    "ragged": (1, 2, 64, [10, 0, 127, 64, 5], [0, 130, 2, 64, 59], 200, "head"),
    "prompt": (2, 1, 128, [0], [777], 777, "slice"),
    "past_the_room": (1, 2, 128, [60, 10], [10, 3], 64, "token"),
    "many_seqs": (1, 1, 64, [7] * 130, [1] * 130, 9, "head"),
}


@pytest.mark.parametrize("cid", list(APPEND))
def test_append(cid, gpu_lib):
    import torch

    L, H, d, before, new, room, layout = APPEND[cid]
    rng = np.random.default_rng(zlib.crc32(cid.encode()))
    S = len(before)
    cu_rows = np.arange(S + 1, dtype=np.int32) * room
    cache = filled(C4.Cache4(L, H, d, cu_rows))

    def tokens(counts):
        n = sum(counts)
        k, v = bf16(rng, (L, n, H, d)), bf16(rng, (L, n, H, d))
        cu = torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32, device="cuda")
        kt, vt = B.bf16_from_bits(k), B.bf16_from_bits(v)
        if layout == "head":  # [L][H][T][d] storage
            kt, vt = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (kt, vt))
        elif layout == "slice":  # parts of a fused projection's output, every second token
            fused = torch.zeros((L, 2 * n, 3 * H, d), dtype=torch.bfloat16, device="cuda")
            fused[:, ::2, H:2 * H], fused[:, ::2, 2 * H:] = kt, vt
            kt, vt = fused[:, ::2, H:2 * H], fused[:, ::2, 2 * H:]
        return kt, vt, cu, decode_bf16(k), decode_bf16(v)

    log(f"[cache4 append {cid}] before={before[:5]} new={new[:5]}")
    want = {}
    for counts in (before, new):
        kt, vt, cu, k, v = tokens(counts)
        if sum(counts):
            C4.advance4(cache, cu)
            C4.append4(cache, kt, vt, cu)
            if counts is new:
                C4.append4(cache, kt, vt, cu)  # the same tokens again change nothing
        at = 0
        for s, n in enumerate(counts):
            for l in range(L):
                for h in range(H):
                    for name, x in (("k", k), ("v", v)):
                        old = want.get((name, l, h, s), np.zeros((0, d)))
                        want[name, l, h, s] = np.concatenate([old, x[l, at:at + n, h]])
            at += n
    assert cache.lens.tolist() == [a + b for a, b in zip(before, new)]
    over = any(a + b > room for a, b in zip(before, new))
    assert cache.status() == (B.FLAG_OUT_ROWS if over else 0)
    kept = {n: {(l, h, s): want[n, l, h, s][:room] for l in range(L) for h in range(H) for s in range(S)}
            for n in ("k", "v")}
    check_rows(cache, kept["k"], kept["v"], cu_rows)
    for (l, h, s), x in kept["k"].items():
        if len(x):
            check_bounds(cache, x, s, l, h)


def test_append_more_tokens_than_the_sequence_counts(gpu_lib):
    """Without advance4 the sequence has fewer tokens than are new: the last of them are its
    tokens, nothing is written before its first row; and tokens past num_new are not read."""
    import torch

    cache = filled(C4.Cache4(1, 1, 64, [0, 64, 128]))
    x = bf16(np.random.default_rng(5), (1, 8, 1, 64))
    t = B.bf16_from_bits(x)
    cache.lens.copy_(torch.tensor([0, 3]))
    C4.append4(cache, t, t, torch.tensor([0, 0, 8], dtype=torch.int32, device="cuda"))
    y = {(0, 0, 1): decode_bf16(x[0, 5:, 0])}
    check_rows(cache, y, y, [0, 64])
    cache = filled(C4.Cache4(1, 1, 64, [0, 64, 128]))
    cache.lens.copy_(torch.tensor([6, 6]))
    C4.append4(cache, t, t, torch.tensor([0, 6, 12], dtype=torch.int32, device="cuda"))
    y = {(0, 0, 0): decode_bf16(x[0, :6, 0]), (0, 0, 1): decode_bf16(x[0, 6:, 0])}
    check_rows(cache, y, y, [0, 64])


def test_layers_without_bounds(gpu_lib):
    """A cache without bounds, written layer by layer through views, as a model does."""
    import torch

    L, H, d, S = 3, 2, 64, 2
    cu_rows = [0, 33, 64]
    whole, parts = (filled(C4.Cache4(L, H, d, cu_rows, k_bounds=False)) for _ in range(2))
    t = B.bf16_from_bits(bf16(np.random.default_rng(6), (2, L, 7, H, d)))
    cu = torch.tensor([0, 4, 7], dtype=torch.int32, device="cuda")
    for c in (whole, parts):
        C4.advance4(c, cu)
    C4.append4(whole, t[0], t[1], cu)
    for l in range(L):
        C4.append4(parts.layers(l), t[0, l:l + 1], t[1, l:l + 1], cu)
    for a, b in zip(host(whole), host(parts)):
        assert a is None and b is None or np.array_equal(a, b)
    k, v = C4.read4(parts.layers(1, 2), cu, 7)
    kw, vw = C4.read4(whole, cu, 7)
    assert torch.equal(k, kw[1:]) and torch.equal(v, vw[1:])


def test_read_back_of_many_rows(gpu_lib):
    """A read of many rows of several sequences (four rows a thread) gives what reads of its layers
    one by one (one row a thread) do, across the sequences' boundaries."""
    import torch

    L, H, d, lens = 16, 16, 128, [700, 1, 0, 333, 63]
    cu_rows = np.concatenate([[0], np.cumsum([n + 5 for n in lens])]).astype(np.int32)
    cache = C4.Cache4(L, H, d, cu_rows)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    cu = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device="cuda")
    C4.advance4(cache, cu)
    k, v = (torch.randn((L, sum(lens), H, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    C4.append4(cache, k, v, cu)
    for counts in (lens, [600, 0, 5, 333, 62]):  # the second: more than the third sequence has
        co = torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32, device="cuda")
        n = sum(counts)
        whole = [torch.full((L, H, n + 70, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        C4.read4(cache, co, n + 70, k_out=whole[0], v_out=whole[1])
        for l in range(L):
            one = [torch.full((1, H, n + 70, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            C4.read4(cache.layers(l), co, n + 70, k_out=one[0], v_out=one[1])
            assert torch.equal(one[0][0], whole[0][l]) and torch.equal(one[1][0], whole[1][l])
    assert (whole[0][:, :, 600:605] == 7).all()
