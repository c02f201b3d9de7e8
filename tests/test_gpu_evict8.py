"""Eviction from the 8-bit cache against the fp64 oracle: which tokens stay, where they go and what
the cache holds afterwards, element for element (nothing has a tolerance); and decode steps that
append, attend, gather and evict, as a program runs them."""
import zlib

import numpy as np
import pytest

import oracle.cache8_ref as R
from oracle import decode_bf16
from paper_2609_22158_amd import binding as B
from paper_2609_22158_amd import cache8 as C8
from synth import f32_to_bf16_bits
from tests.gpu_cases import log
from tests.test_gpu_cache8 import bf16, check, dev, empty_heads, filled, offsets

pytestmark = pytest.mark.gpu


def weights_of(kind, rng, shape):
    if kind == "tail":
        return np.exp(2 * rng.standard_normal(shape)).astype(np.float32)
    if kind == "ties":  # a few values, zeros of both signs among them
        return rng.choice(np.array([0.0, -0.0, 1.0, 1.0, 2.5, 1e-30], np.float32), shape)
    if kind == "equal":
        return np.full(shape, 0.25, np.float32)
    if kind == "ends":  # whatever a float can hold
        x = rng.integers(0, 1 << 32, shape, dtype=np.uint64).astype(np.uint32).view(np.float32)
        return np.where(rng.random(shape) < 0.2, rng.choice(np.array([np.nan, np.inf, -np.inf, 0], np.float32), shape), x)
    return {"rising": np.arange(shape[-1], dtype=np.float32), "falling": -np.arange(shape[-1], dtype=np.float32)}[
        kind] * np.ones(shape, np.float32)


def made(rng, L, H, d, lens, rooms, kind, swing=4, shuffle=True):
    """A cache with tokens, its weights, positions in some order, and its heads in the oracle."""
    import torch

    S = len(lens)
    cache = filled(C8.Cache8(L, H, d, offsets(rooms)))
    n, cu = sum(lens), offsets(lens)
    k, v = bf16(rng, (L, n, H, d), 1.0, swing), bf16(rng, (L, n, H, d), 1.0, swing)
    cache.seen.copy_(dev([2 * x for x in lens]))
    cache.lens.copy_(dev(lens))
    C8.append8(cache, B.bf16_from_bits(k), B.bf16_from_bits(v), dev(cu))
    w = weights_of(kind, rng, (L, H, n))
    heads = empty_heads(L, H, S, d)
    pos = np.zeros((L, H, n), np.int32)
    for (l, h, s), a in heads.items():
        at = slice(cu[s], cu[s + 1])
        p = np.sort(rng.permutation(2 * lens[s])[:lens[s]])
        pos[l, h, at] = rng.permutation(p) if shuffle else p
        a.append(decode_bf16(k[l, at, h]), decode_bf16(v[l, at, h]), pos[l, h, at], w[l, h, at])
    rows = torch.cat([torch.arange(int(r), int(r) + m, device="cuda") for r, m in zip(cache.cu_rows, lens)])
    if n:
        cache.weights[:, :, rows] = dev(w, torch.float32)
        cache.positions[:, :, rows] = dev(pos)
    return cache, heads


def after(cache, heads, keeps, first, recent, lens):
    """The oracle's eviction, the rows that no longer hold a token taken as they were."""
    for (l, h, s), a in heads.items():
        a.evict(keeps[s], first, recent, 2 * lens[s])
    return heads


def checked(cache, heads, lens, keeps):
    """check(), for a cache whose rows past the kept ones still hold what they held."""
    import torch

    cu = cache.cu_rows
    for s, (n, k) in enumerate(zip(lens, keeps)):
        if n <= k:
            continue
        r = int(cu[s])
        for x in ("k_codes", "v_codes", "weights", "positions"):
            getattr(cache, x)[:, :, r + k:r + n].view(torch.uint8).fill_(0xA5)
        b0 = r // 64 + s
        for x in ("k_scales", "v_scales"):
            getattr(cache, x)[:, :, b0 - (-k // 64):b0 - (-n // 64)].view(torch.uint8).fill_(0xA5)
    check(cache, heads)


EVICT = {
    # name: (L, H, d, tokens, keep or keeps, first, recent, weights, swing of the rows' magnitudes)
    "one_of_many": (2, 2, 128, [300], 299, 4, 32, "tail", 0),
    "one_left": (1, 2, 64, [130, 1, 2], 1, 0, 0, "tail", 4),
    "ragged": (2, 2, 128, [700, 130, 0, 64, 65, 1, 513], 64, 3, 20, "tail", 4),
    "keeps": (1, 3, 64, [700, 130, 0, 64, 65, 1, 513], [650, 64, 5, 1, 65, 9, 0], 3, 20, "tail", 4),
    "half": (1, 2, 128, [1000, 999], 500, 0, 0, "tail", 0),
    "grow": (1, 2, 128, [900], 450, 0, 0, "tail", 24),  # rows into blocks whose scale is far smaller
    "grow_d64": (1, 2, 64, [900, 333], 300, 0, 10, "ties", 24),
    "within_a_block": (1, 2, 64, [60], 33, 2, 5, "tail", 12),  # rows leave and enter one block
    "rising": (1, 1, 64, [1000], 333, 0, 0, "rising", 4),   # all that stay move, past each other
    "falling": (1, 1, 64, [1000], 333, 0, 0, "falling", 4),  # nothing moves
    "ties": (2, 2, 64, [3000], 1111, 0, 0, "ties", 0),
    "equal": (1, 2, 64, [2500], 77, 0, 0, "equal", 0),
    "ends": (2, 2, 64, [1500], 700, 10, 10, "ends", 0),
    "all_stay": (1, 2, 64, [500], 200, 400, 600, "tail", 0),  # more that stay in any case than are kept
    "first": (1, 2, 64, [500], 200, 100, 0, "tail", 0),
    "recent": (1, 2, 64, [500], 200, 0, 100, "tail", 0),
    "nothing": (1, 2, 64, [500, 20], 500, 4, 4, "tail", 0),
    "long": (1, 1, 64, [140000], 70001, 64, 1000, "tail", 0),
    "long_few": (1, 1, 64, [70000], 69999, 0, 0, "tail", 0),
    "chunk_borders": (1, 1, 64, [1023, 1024, 1025, 2047, 2048, 2049, 4096, 4097], 1000, 0, 0, "ties", 0),
    "many_seqs": (1, 2, 64, [(37 * i) % 150 for i in range(150)], 70, 2, 3, "tail", 4),
    "many_heads": (24, 16, 64, [130, 90], 100, 2, 3, "tail", 4),
    # rows of every number of waves and keys a lane: 4 x 2, 8 x 5, 16 x 8 and 16 x 20 groups, and streamed
    "sizes": (1, 1, 64, [2047, 10239, 9], 1500, 4, 64, "tail", 0),
    "sizes_16": (1, 1, 64, [32767, 1], 31000, 0, 64, "ends", 0),
    "sizes_ties": (1, 1, 64, [81919], 40000, 0, 0, "ties", 0),
    "streamed_ties": (1, 1, 64, [81921 + 64, 500], 300, 2, 100, "ties", 0),
    # whole blocks replaced, 64 moves into each
    "dense": (1, 2, 128, [4000], 1000, 0, 0, "rising", 10),
    "dense_d64": (1, 1, 64, [700, 129], 64, 0, 0, "rising", 24),
}


@pytest.mark.parametrize("cid", list(EVICT))
def test_evict(cid, gpu_lib):
    L, H, d, lens, keep, first, recent, kind, swing = EVICT[cid]
    log(f"[evict8 {cid}] L={L} H={H} d={d} tokens={lens[:6]} keep={keep}")
    rng = np.random.default_rng(zlib.crc32(cid.encode()))
    cache, heads = made(rng, L, H, d, lens, [n + int(rng.integers(0, 70)) for n in lens], kind, swing)
    keeps = [max(1, k) for k in keep] if isinstance(keep, list) else [keep] * len(lens)
    if isinstance(keep, list):
        C8.evict8(cache, keeps=dev(keep), first=first, recent=recent)
    else:
        C8.evict8(cache, keep, first=first, recent=recent)
    assert cache.lens.tolist() == [min(n, k) for n, k in zip(lens, keeps)]
    assert cache.seen.tolist() == [2 * n for n in lens] and cache.status() == 0
    before = {key: [list(e) for e in a.exp] for key, a in heads.items()}
    after(cache, heads, keeps, first, recent, lens)
    if cid.startswith("grow"):
        assert any(e2 > e1 for key, a in heads.items() for w in (0, 1) for e1, e2 in zip(before[key][w], a.exp[w]))
    checked(cache, heads, lens, keeps)


def test_nothing_but_the_moved_rows_changes(gpu_lib):
    """Rows that no longer hold a token keep their bytes, and so does every block that no row moves into."""
    import torch

    rng = np.random.default_rng(1)
    cache, heads = made(rng, 2, 2, 64, [1000], [1010], "tail")
    names = ("k_codes", "v_codes", "k_scales", "v_scales", "weights", "positions")
    old = {x: getattr(cache, x).clone() for x in names}
    C8.evict8(cache, 990, recent=8)
    moved = old["positions"][:, :, :990] != cache.positions[:, :, :990]
    assert 0 < moved.sum() <= 40
    for x in names:
        a, b = old[x].view(torch.uint8), getattr(cache, x).view(torch.uint8)
        if "scales" in x:
            a, b = a.view(2, 2, -1, 4)[:, :, 16:], b.view(2, 2, -1, 4)[:, :, 16:]
            assert torch.equal(a, b)
            continue
        a, b = a.view(2, 2, 1010, -1), b.view(2, 2, 1010, -1)
        assert torch.equal(a[:, :, 990:], b[:, :, 990:])
        whole = torch.nn.functional.pad(moved, (0, 34)).view(2, 2, 16, 64).any(-1)  # blocks that rows move into
        same = ~whole.repeat_interleave(64, dim=2)[:, :, :990]
        assert same.any() and torch.equal(a[:, :, :990][same], b[:, :, :990][same])


def test_past_its_room(gpu_lib):
    """lens beyond the room: the tokens of the room are ranked, it is reported, and lens is keep."""
    rng = np.random.default_rng(2)
    cache, heads = made(rng, 1, 2, 64, [100, 50], [100, 60], "tail")
    cache.lens.copy_(dev([180, 50]))
    C8.evict8(cache, 70)
    assert cache.lens.tolist() == [70, 50] and cache.status() == B.FLAG_OUT_ROWS
    checked(cache, after(cache, heads, [70, 70], 0, 0, [100, 50]), [100, 50], [70, 70])


def test_positions_near_the_ends_of_int32(gpu_lib):
    """A recent window that reaches before the first position, and one near the greatest."""
    import torch

    for seen, recent, want in ((5, 2 ** 31 - 1, [0, 1]), (2 ** 31 - 1, 2, [3, 4]), (2 ** 31 - 1, 2 ** 31 - 1, [0, 1])):
        cache = C8.Cache8(1, 1, 64, [0, 5])
        x = torch.randn((1, 5, 1, 64), device="cuda").bfloat16()
        C8.advance8(cache, dev([0, 5]))
        cache.seen.fill_(seen)
        C8.append8(cache, x, x, dev([0, 5]))
        assert cache.positions.flatten().tolist() == list(range(seen - 5, seen))
        cache.weights.copy_(torch.arange(5, 0, -1).float())
        C8.evict8(cache, 2, recent=recent)
        assert sorted(cache.positions.flatten()[:2].tolist()) == [seen - 5 + i for i in want]


def test_workspace_and_stream(gpu_lib):
    import torch

    rng = np.random.default_rng(3)
    cache, heads = made(rng, 2, 2, 64, [400, 90], [400, 90], "tail")
    n = int(gpu_lib.stepkv_cache8_evict_workspace_bytes(cache._ref))
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    with pytest.raises(B.StepKVError):
        C8.evict8(cache, 100, workspace=ws[:n - 256])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    C8.evict8(cache, 100, workspace=ws, stream=side)
    side.synchronize()
    checked(cache, after(cache, heads, [100, 100], 0, 0, [400, 90]), [400, 90], [100, 100])


# ---------------------------------------------------------------- as a program uses them
class Program:
    """A boundary, then decode steps: tokens come, are attended to, and the least attended go."""

    def __init__(self, seed=0, L=2, Hq=8, H=2, d=64):
        import torch

        rng = np.random.default_rng(seed)
        self.L, self.Hq, self.H, self.d = L, Hq, H, d
        self.src, self.kept, self.keep = [400, 150], [200, 100], 180
        cu_seq = offsets(self.src)
        n = int(cu_seq[-1])
        self.pb = B.Problem(L, Hq, H, d, 4, cu_seq, np.array([0, 3, 5], np.int32))
        self.k, self.v = (B.bf16_from_bits(bf16(rng, (L, H, n, d), 1.0, 1)) for _ in range(2))
        self.q_win = B.bf16_from_bits(bf16(rng, (L, 2, 4, Hq, d), 1.0, 0))
        self.prot = torch.zeros(n, dtype=torch.uint8, device="cuda")
        self.steps = torch.zeros(n, dtype=torch.int32, device="cuda")
        self.util = torch.ones(5, device="cuda")
        self.budgets = dev(self.kept)
        self.tokens = [tuple(B.bf16_from_bits(bf16(rng, (L, 3, H, d), 1.0, 6)) for _ in range(2)) for _ in range(8)]
        self.queries = [B.bf16_from_bits(bf16(rng, (L, 2, Hq, d), 1.0, 0)) for _ in range(8)]
        self.cu_new = dev([0, 1, 3])

    def boundary(self):
        cache = C8.Cache8(self.L, self.H, self.d, [0, 230, 460])
        A = B.saliency(self.pb, self.q_win, self.k)
        P = B.priority(self.pb, A, self.steps, self.prot, self.util)["scores"]
        idx, cu_ret, _ = B.select(self.pb, P, self.prot, self.steps, 1, budgets=self.budgets)
        C8.compact8(self.pb, cache, self.k, self.v, idx, cu_ret, weights=A)
        return cache, A, idx

    def step(self, cache, layers, i, out, tokens=None, q=None, ws=(None, None), evict=True):
        k, v = tokens or self.tokens[i]
        q = self.queries[i] if q is None else q
        C8.advance8(cache, self.cu_new)
        for l, view in enumerate(layers):
            C8.append8(view, k[l:l + 1], v[l:l + 1], self.cu_new)
            C8.decode_attention8(view, q[l:l + 1], gather=True, out=out[l:l + 1], workspace=ws[0])
        if evict:
            C8.evict8(cache, self.keep, first=4, recent=16, workspace=ws[1])


STATE = ("k_codes", "v_codes", "k_scales", "v_scales", "weights", "positions", "lens", "seen")


def test_a_boundary_and_steps(gpu_lib):
    """The cache against the oracle's through a boundary and eight steps. The weights are the cache's
    own (they are sums of rounded numbers): each step's are checked against the softmax of what the
    cache holds, and the oracle evicts by them."""
    import torch

    p = Program()
    cache, A, idx = p.boundary()
    heads = empty_heads(p.L, p.H, 2, p.d)
    cu = offsets(p.src)
    for (l, h, s), a in heads.items():
        i = idx[l, h, cu[s]:cu[s] + p.kept[s]].cpu().numpy()
        x = [t[l, h, cu[s] + torch.from_numpy(i).long().cuda()].double().cpu().numpy() for t in (p.k, p.v)]
        a.append(*x, i, A[l, h].double().cpu().numpy()[cu[s] + i])
    layers = [cache.layers(l) for l in range(p.L)]
    out = torch.empty((p.L, 2, p.Hq, p.d), device="cuda")
    lens, seen, new = np.array(p.kept), np.array(p.src), [1, 2]
    left = 0
    for i in range(8):
        gathered = cache.weights.double().cpu().numpy()
        p.step(cache, layers, i, out, evict=False)  # to look at the weights that the eviction goes by
        weights = cache.weights.double().cpu().numpy()
        k, v = (t.double().cpu().numpy() for t in p.tokens[i])
        q = p.queries[i].double().cpu().numpy()
        for (l, h, s), a in heads.items():
            at = slice(s, s + 1) if s == 0 else slice(1, 3)
            a.append(k[l, at, h], v[l, at, h], seen[s] + np.arange(new[s]))
            n, r = len(a), 230 * s
            z = q[l, s, h * 4:h * 4 + 4] @ a.values(0).T / 8.0
            e = np.exp(z - z.max(axis=1, keepdims=True))
            e /= e.sum(axis=1, keepdims=True)
            was = np.concatenate([gathered[l, h, r:r + lens[s]], np.zeros(new[s])])
            assert np.abs(weights[l, h, r:r + n] - was - e.sum(axis=0)).max() <= 1e-4 * max(1.0, was.max())
            ref = e @ a.values(1)
            assert np.abs(out[l, s, h * 4:h * 4 + 4].double().cpu().numpy() - ref).max() <= 1e-4 * np.abs(a.values(1)).max()
            a.weights = weights[l, h, r:r + n].copy()
        lens, seen = lens + new, seen + new
        C8.evict8(cache, p.keep, first=4, recent=16)
        for (l, h, s), a in heads.items():
            a.evict(p.keep, 4, 16, seen[s])
        left += int((lens > p.keep).sum())
        lens = np.minimum(lens, p.keep)
        assert cache.lens.tolist() == lens.tolist() and cache.seen.tolist() == seen.tolist()
        codes, scales = cache.k_codes.cpu().numpy(), cache.k_scales.cpu().numpy()
        pos = cache.positions.cpu().numpy()
        for (l, h, s), a in heads.items():
            r, n = 230 * s, len(a)
            assert np.array_equal(pos[l, h, r:r + n], a.positions)
            assert np.array_equal(R.NUMBERS[codes[l, h, r:r + n]], a.num[0])
            assert np.array_equal(scales[l, h, r // 64 + s:][:-(-n // 64)], 2.0 ** np.array(a.exp[0]))
    assert left >= 8 and cache.status() == 0


def test_steps_replay_in_a_hip_graph(gpu_lib):
    """A step captured once and replayed over changing tokens and queries, with eager work between the
    replays, and a second graph that shares its workspaces: the same states as eager steps."""
    import torch

    p = Program(1)
    eager, _, _ = p.boundary()
    graphed, _, _ = p.boundary()
    other, _, _ = p.boundary()
    lib = C8.load()
    ws = tuple(torch.empty(n, dtype=torch.uint8, device="cuda") for n in (
        int(lib.stepkv_cache8_decode_workspace_bytes(eager.layers(0)._ref, p.Hq, 1)),
        int(lib.stepkv_cache8_evict_workspace_bytes(eager._ref))))
    views = {c: [c.layers(l) for l in range(p.L)] for c in (eager, graphed, other)}
    outs = {c: torch.zeros((p.L, 2, p.Hq, p.d), device="cuda") for c in (eager, graphed, other)}
    k, v, q = p.tokens[0][0].clone(), p.tokens[0][1].clone(), p.queries[0].clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graphs = {}
    for c in (graphed, other):
        graphs[c] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[c], stream=side):
            p.step(c, views[c], 0, outs[c], (k, v), q, ws)
    for i in range(24):
        j = (5 * i) % 8
        k.copy_(p.tokens[j][0])
        v.copy_(p.tokens[j][1])
        q.copy_(p.queries[j])
        for c in (graphed, other):
            graphs[c].replay()
        p.step(eager, views[eager], j, outs[eager])
        torch.cuda.synchronize()
        for c in (graphed, other):
            assert torch.equal(outs[c], outs[eager]), i
            for x in STATE:
                assert torch.equal(getattr(c, x), getattr(eager, x)), (i, x)
    assert eager.lens.tolist() == [180, 148]
    log("[graph8] 24 replays of two graphs match")
