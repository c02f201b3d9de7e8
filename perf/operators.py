"""The 4-bit cache and what reads it, as a program that serves compressed trajectories uses them.

A cache row (one token of one layer and KV head) holds its key and its value in 4 bits a channel:
an element of {0, .5, 1, 1.5, 2, 3, 4, 6} with a sign (e2m1; the even channel in the low half of
its byte) times a power of two that 32 channels share (a byte, 2^(byte - 127)). The power is the
smallest 2^e with max|x| <= 7 * 2^e, e within [-124, 125]; an element is x / 2^e rounded to the
nearest, ties to the even code. Sequence s owns rows cu_rows[s] .. cu_rows[s + 1] - 1 and holds
lens[s] tokens in the first of them. Every 64 rows of a sequence are a block, with the least and
greatest key value of each channel kept beside the cache (k_bounds, block b of sequence s at
cu_rows[s] // 64 + s + b).

* ``compact``: the retained rows of a pruning boundary are quantised into the cache and read back.
* ``append``: new tokens are quantised as the last rows of their sequences and read back.
* ``read``: the cache back in bf16, as the next boundary's scoring takes it.
* ``decode``: one decode step over every row.
* ``sparse``: one decode step over the blocks that score best for the step's queries.

A case is a dict of sizes; ``draw`` spreads them over the range the package supports.
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 64   # rows of a block
GROUP = 32   # channels that share a scale
_dev = "cuda"
_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)

# Every field of a case and its usual value (the 32-layer 8B-shaped cache).
_DEFAULTS = dict(
    op="decode",            # compact, append, read, decode or sparse
    layers=32, q_heads=32, kv_heads=8, d=128,
    seqs=1, n_min=0, n=1536,  # tokens held: one sequence of n, or a batch of n_min .. n
    room=512,               # rows that a sequence may still grow by
    source=0,               # compact: tokens of the longest sequence before the boundary
    shared=False,           # compact: one retained set for every layer and head
    new=0,                  # append: new tokens of every sequence (ragged in a batch if > 1)
    blocks=0,               # sparse: blocks attended per sequence and KV head
)


def _case(**kw):
    return dict(_DEFAULTS, **kw)


def listed():
    return [
        # the boundary of the long-horizon web agent: 1024 + 512 of 32k tokens, every layer
        _case(name="compact_l32_32k", op="compact", source=32768),
        # one layer of a small model at a short trajectory's boundary: launches count
        _case(name="compact_tiny", op="compact", layers=1, q_heads=4, kv_heads=2, d=64, n=192,
              source=1024, room=100),
        # a decode step's tokens of 28 sequences written by one layer
        _case(name="append_token", op="append", layers=1, q_heads=28, kv_heads=4, seqs=28, n_min=500,
              n=2560, new=1),
        # a step's observation of 8k tokens appended by one layer
        _case(name="append_prompt", op="append", layers=1, n=9001, room=8192, new=8100),
        # one layer read back for a boundary
        _case(name="read_layer", op="read", layers=1, n=1700),
        # a serving batch's cache read back, 16 ragged sequences
        _case(name="read_ragged16", op="read", layers=28, q_heads=28, kv_heads=4, seqs=16, n_min=700,
              n=2560),
        # one small layer's step, 300 tokens: the smallest call
        _case(name="decode_tiny", layers=1, q_heads=4, kv_heads=4, d=64, n=300, room=64),
        # a decode step of the serving batch, every layer, query groups of 7
        _case(name="decode_ragged16", layers=28, q_heads=28, kv_heads=4, seqs=16, n_min=700, n=8192),
        # a trajectory past 100k tokens, 8 layers
        _case(name="decode_long", layers=8, n=131071, room=1024),
        # one layer's sparse step at 32k tokens, as a model calls it between its layers
        _case(name="sparse_layer", op="sparse", layers=1, n=32768, blocks=32),
        # the serving batch, sparse
        _case(name="sparse_ragged16", op="sparse", layers=28, q_heads=28, kv_heads=4, seqs=16,
              n_min=700, n=8192, blocks=16),
        # 8 layers of a trajectory past 100k tokens, sparse
        _case(name="sparse_long", op="sparse", layers=8, n=131071, room=1024, blocks=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(("compact", "append", "read", "decode", "decode", "sparse", "sparse"))
        kv = rng.choice((1, 2, 4, 8))
        seqs = rng.choice((1, 1, 2, 5, 16, 28))
        n = _log_int(rng, 64, 131071)
        c = _case(op=op, layers=_log_int(rng, 1, 32), q_heads=kv * rng.choice((1, 2, 4, 7, 8, 16)),
                  kv_heads=kv, d=rng.choice((64, 128, 128)), seqs=seqs,
                  n_min=0 if seqs == 1 else max(n // 8, 1), n=n, room=_log_int(rng, 1, 2048))
        if op == "compact":
            c["source"] = int(n * rng.uniform(1.0, 8.0))
            c["shared"] = rng.random() < 0.3
        elif op == "append":
            c["new"] = 1 if rng.random() < 0.5 else _log_int(rng, 1, max(1, c["n_min"] or n))
        elif op == "sparse":
            c["blocks"] = _log_int(rng, 4, 128)
        values = c["layers"] * kv * c["d"] * max(_rows(c), _source_total(c))
        w, most = work(c), [work(x) for x in listed()]
        if (values <= 8 * 8 * 128 * (131071 + 1024) and w["bytes"] <= max(x["bytes"] for x in most)
                and w["flops"] <= max(x["flops"] for x in most)):
            return c


# ------------------------------------------------------------------------------- sizes
def _lengths(c):
    if c["seqs"] == 1:
        return [c["n"]]
    r = random.Random("%d %d %d" % (c["seqs"], c["n_min"], c["n"]))
    return [r.randint(c["n_min"], c["n"]) for _ in range(c["seqs"])]


def _new_counts(c):
    """Tokens appended to each sequence: one each, or from none to `new` in a batch."""
    if c["seqs"] == 1 or c["new"] == 1:
        return [c["new"]] * c["seqs"]
    r = random.Random("new %d %d" % (c["seqs"], c["new"]))
    return [min(n, r.randint(0, c["new"])) for n in _lengths(c)]


def _source_lengths(c):
    return [max(n, int(n * c["source"] / c["n"])) for n in _lengths(c)]


def _source_total(c):
    return sum(_source_lengths(c)) if c["op"] == "compact" else 0


def _rows(c):
    return sum(_lengths(c)) + c["seqs"] * c["room"]


def _offsets(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


# ------------------------------------------------------------------------------ inputs
def _values(gen, L, H, n, d, u=None, hot=None):
    """bf16 rows [L][H][n][d]: normal, a few outlier channels; `hot` tokens lie along u."""
    x = torch.empty((L, H, n, d), dtype=torch.bfloat16, device=_dev).normal_(generator=gen)
    x[..., torch.randint(0, d, (4,), generator=gen, device=_dev)] *= 2
    if u is not None:
        at = torch.nonzero(hot)[:, 0]
        x[:, :, at] += (hot[at, None] * math.sqrt(d) * u[:, :, None]).to(torch.bfloat16)
    return x


def _pow2(e):
    """2^e in float32, exactly, for integers e within [-126, 127]."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantise(x):
    """Codes uint8 [..][d / 2] and scale bytes uint8 [..][d / 32] of bf16 rows [..][d]."""
    g = x.float().unflatten(-1, (-1, GROUP))
    top = g.abs().amax(dim=-1, keepdim=True)
    m, e = torch.frexp(top)  # top = m 2^e, 0.5 <= m < 1; 7 2^f = 0.875 2^(f + 3)
    e = torch.where(m <= 0.875, e - 3, e - 2)
    e = torch.where(top == 0, torch.full_like(e, -124), e).clamp(-124, 125)
    y = g * _pow2(-e)
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5)
            + (a >= 3.5) + (a > 5.0))
    code = (code + 8 * torch.signbit(y)).flatten(-2).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).squeeze(-1).to(torch.uint8)


def _spread(codes, scales):
    """The float32 values [..][d] of quantised rows."""
    level = torch.tensor(_LEVELS + tuple(-x for x in _LEVELS), device=codes.device)
    code = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).int()
    x = level[code].unflatten(-1, (-1, GROUP))
    return (x * _pow2(scales.int() - 127)[..., None]).flatten(-2)


def _row_index(c, cu, counts, first):
    """For the `counts` rows of each sequence in order: its sequence, and first[s] + its number."""
    at = torch.arange(int(sum(counts)), device=_dev)
    s = torch.searchsorted(cu[1:].long(), at, right=True)
    return s, first[s] + at - cu.long()[s]


def prepare(case, seed):
    c = _case(**case)
    gen = torch.Generator(device=_dev)
    gen.manual_seed(seed)
    L, H, Hq, d, S = c["layers"], c["kv_heads"], c["q_heads"], c["d"], c["seqs"]
    held, rows = _lengths(c), _rows(c)
    cu_rows = _offsets([n + c["room"] for n in held])
    st = dict(case=c, cu_rows_host=cu_rows, cu_rows=torch.from_numpy(cu_rows).to(_dev),
              lens=torch.tensor(held, dtype=torch.int32, device=_dev), rows=rows)
    u = torch.randn((L, H, d), generator=gen, device=_dev)
    u /= u.norm(dim=-1, keepdim=True)  # the direction that the queries look along
    for name, width in (("k_codes", d // 2), ("v_codes", d // 2), ("k_scales", d // GROUP),
                        ("v_scales", d // GROUP)):
        st[name] = torch.zeros((L, H, rows, width), dtype=torch.uint8, device=_dev)
    st["k_bounds"] = torch.zeros((L, H, rows // BLOCK + S, 2, d), dtype=torch.bfloat16, device=_dev)
    if c["op"] == "compact":
        src = _source_lengths(c)
        cu_seq = _offsets(src)
        st["cu_seqlens_host"], st["cu_seqlens"] = cu_seq, torch.from_numpy(cu_seq).to(_dev)
        st["k"] = _values(gen, L, H, int(cu_seq[-1]), d)
        st["v"] = _values(gen, L, H, int(cu_seq[-1]), d)
        idx = torch.zeros((1 if c["shared"] else L * H, int(cu_seq[-1])), dtype=torch.int32, device=_dev)
        for s in range(S):  # retained positions, ascending
            pick = torch.rand((idx.shape[0], src[s]), generator=gen, device=_dev)
            pick = pick.topk(held[s], dim=1).indices.sort(dim=1).values
            idx[:, int(cu_seq[s]):int(cu_seq[s]) + held[s]] = pick.int()
        st["idx"] = idx[0] if c["shared"] else idx.view(L, H, -1)
        st["lens"].zero_()
        st["cu_out"] = torch.from_numpy(_offsets(held)).to(_dev)  # also cu_retained
        st["out_rows"] = sum(held)
    else:
        hot = (torch.rand(rows, generator=gen, device=_dev) < 0.01).float() * 0.4
        new = _new_counts(c) if c["op"] == "append" else [0] * S
        for l in range(L):
            k, v = _values(gen, 1, H, rows, d, u[l:l + 1], hot), _values(gen, 1, H, rows, d)
            for name, x in (("k", k), ("v", v)):
                st[name + "_codes"][l:l + 1], st[name + "_scales"][l:l + 1] = _quantise(x)
            _bounds_of(st, cu_rows, [n - m for n, m in zip(held, new)], l)  # before the new tokens
    if c["op"] == "append":
        st["cu_out"], st["out_rows"] = torch.from_numpy(_offsets(new)).to(_dev), sum(new)
        # as the projections of a model give them: token by token
        st["k_new"] = _values(gen, L, sum(new), H, d)
        st["v_new"] = _values(gen, L, sum(new), H, d)
    elif c["op"] == "read":
        st["cu_out"], st["out_rows"] = torch.from_numpy(_offsets(held)).to(_dev), sum(held)
    elif c["op"] in ("decode", "sparse"):
        q = torch.empty((L, S, Hq, d), dtype=torch.bfloat16, device=_dev).normal_(generator=gen)
        q += (2.0 * u).repeat_interleave(Hq // H, dim=1).to(torch.bfloat16)[:, None]
        st["q"] = q
    if own:
        st["cache"], st["problem"] = _handles(st)
    return st


def _bounds_of(st, cu_rows, held, l):
    """k_bounds of layer l from its codes, the first held[s] rows of every sequence."""
    x = _spread(st["k_codes"][l], st["k_scales"][l])
    st["k_bounds"][l] = 0
    for s, n in enumerate(held):
        if n == 0:
            continue
        a, nb = int(cu_rows[s]), -(-n // BLOCK)
        y = x[:, a + torch.arange(nb * BLOCK, device=_dev).clamp(max=n - 1)].unflatten(1, (nb, BLOCK))
        at = a // BLOCK + s
        st["k_bounds"][l, :, at:at + nb, 0] = y.amin(dim=2).to(torch.bfloat16)
        st["k_bounds"][l, :, at:at + nb, 1] = y.amax(dim=2).to(torch.bfloat16)


def _handles(st):
    """The cache and problem objects that a program keeps beside its tensors."""
    import paper_2609_22158_amd as stepkv

    c = st["case"]
    cache = stepkv.Cache4(c["layers"], c["kv_heads"], c["d"], st["cu_rows_host"], k_codes=st["k_codes"],
                          v_codes=st["v_codes"], k_scales=st["k_scales"], v_scales=st["v_scales"],
                          k_bounds=st["k_bounds"], lens=st["lens"], device=_dev)
    pb = None
    if c["op"] == "compact":
        pb = stepkv.Problem(c["layers"], c["q_heads"], c["kv_heads"], c["d"], 1, st["cu_seqlens_host"],
                            np.zeros(c["seqs"] + 1, np.int32), device=_dev)
    return cache, pb


# --------------------------------------------------------------------- the plain forms
def _plain_write(st, k, v, s, j):
    """Rows [L][H][n][d] as rows j of sequences s; the bounds of the blocks they touch."""
    at = st["cu_rows"].long()[s] + j
    for name, x in (("k", k), ("v", v)):
        codes, scales = _quantise(x)
        st[name + "_codes"][:, :, at] = codes
        st[name + "_scales"][:, :, at] = scales
    x = _spread(st["k_codes"][:, :, at], st["k_scales"][:, :, at])
    block = st["cu_rows"].long()[s] // BLOCK + s + j // BLOCK
    bounds = st["k_bounds"].float()
    opened = block[j % BLOCK == 0]  # blocks whose first row is among these
    lo = bounds[:, :, :, 0].index_fill(2, opened, math.inf).index_reduce(2, block, x, "amin")
    hi = bounds[:, :, :, 1].index_fill(2, opened, -math.inf).index_reduce(2, block, x, "amax")
    st["k_bounds"][:, :, :, 0], st["k_bounds"][:, :, :, 1] = lo.to(torch.bfloat16), hi.to(torch.bfloat16)


def _plain_read(st, n):
    """The last n_s rows of every sequence, in bf16."""
    first = st["lens"].long() - (st["cu_out"][1:] - st["cu_out"][:-1]).long()
    s, j = _row_index(st["case"], st["cu_out"], [n], first)
    at = st["cu_rows"].long()[s] + j
    return tuple(_spread(st[x + "_codes"][:, :, at], st[x + "_scales"][:, :, at]).to(torch.bfloat16)
                 for x in ("k", "v"))


def _plain_attend(st, at, seen):
    """softmax(q K^T / sqrt(d)) V over rows `at`, where `seen`: both [L or 1][S][H or 1][m]."""
    q = st["q"].float()
    L, S, Hq, d = q.shape
    H = st["k_codes"].shape[1]
    la, ha = torch.arange(L, device=_dev)[:, None, None, None], torch.arange(H, device=_dev)[None, None, :, None]
    k = _spread(st["k_codes"][la, ha, at], st["k_scales"][la, ha, at])  # [L][S][H][m][d]
    z = torch.matmul(q.view(L, S, H, Hq // H, d), k.transpose(-1, -2)) / math.sqrt(d)
    del k
    z = torch.where(seen[..., None, :], z, torch.full_like(z, -math.inf))
    p = torch.exp(z - z.amax(dim=-1, keepdim=True))
    v = _spread(st["v_codes"][la, ha, at], st["v_scales"][la, ha, at])
    out = torch.matmul(p, v) / p.sum(dim=-1, keepdim=True)
    return out.view(L, S, Hq, d)


def _plain_blocks(st, n):
    """The n blocks of every (layer, sequence, KV head): the first, the last and the best others."""
    q = st["q"].double()
    L, S, Hq, d = q.shape
    H = st["k_codes"].shape[1]
    q = q.view(L, S, H, Hq // H, d)
    zero = torch.zeros_like(q)
    up = torch.where(q > 0, q, zero).sum(dim=3)  # [L][S][H][d]
    down = torch.where(q < 0, q, zero).sum(dim=3)
    held = (st["lens"].long() + BLOCK - 1) // BLOCK
    most = max(-(-x // BLOCK) for x in _lengths(st["case"]))
    b = torch.arange(most, device=_dev)
    at = st["cu_rows"].long()[:-1] // BLOCK + torch.arange(S, device=_dev)
    at = torch.minimum(at[:, None] + b, at[:, None] + held[:, None] - 1)  # [S][most]
    x = st["k_bounds"].double()[:, :, at].transpose(1, 2)  # [L][S][H][most][2][d]
    score = (x[..., 1, :] * up[..., None, :]).sum(dim=-1) + (x[..., 0, :] * down[..., None, :]).sum(dim=-1)
    score = torch.where(torch.isnan(score), torch.full_like(score, -math.inf), score)
    there = b < held[:, None]
    always = there & ((b < 1) | (b >= held[:, None] - 1))
    rank = torch.where(always, 2, there.long())[None, :, None].expand(score.shape)
    by_score = score.sort(dim=-1, descending=True, stable=True).indices
    by_rank = rank.gather(-1, by_score).sort(dim=-1, descending=True, stable=True).indices
    order = by_score.gather(-1, by_rank)[..., :n]  # forced blocks, then by score, then none
    pick = torch.where(torch.arange(order.shape[-1], device=_dev) < held[:, None, None], order,
                       torch.full_like(order, 1 << 30)).sort(dim=-1).values
    out = torch.full((L, S, H, n), -1, dtype=torch.int32, device=_dev)
    out[..., :pick.shape[-1]] = torch.where(pick < (1 << 30), pick, torch.full_like(pick, -1)).int()
    return out


def _run_plain(st):
    c = st["case"]
    if c["op"] == "compact":
        cu, cs = st["cu_out"], st["cu_seqlens"].long()
        zero = torch.zeros(c["seqs"], dtype=torch.int64, device=_dev)
        s, j = _row_index(c, cu, [st["out_rows"]], zero)
        src = st["idx"].long()[..., cs[s] + j] + cs[s]  # [L][H][n] or [n]
        shape = st["k"].shape[:2] + (st["out_rows"], 1)
        src = src.expand(shape[:3])[..., None].expand(shape[:3] + (c["d"],))
        _plain_write(st, st["k"].gather(2, src), st["v"].gather(2, src), s, j)
        st["lens"].copy_(cu[1:] - cu[:-1])
    elif c["op"] == "append":
        first = st["lens"].long() - (st["cu_out"][1:] - st["cu_out"][:-1]).long()
        s, j = _row_index(c, st["cu_out"], [st["out_rows"]], first)
        _plain_write(st, st["k_new"].transpose(1, 2), st["v_new"].transpose(1, 2), s, j)
    if c["op"] in ("compact", "append", "read"):
        k, v = _plain_read(st, st["out_rows"])
        if c["op"] == "read":
            return {"k": k, "v": v}
        return {"k": k, "v": v, "k_bounds": st["k_bounds"], "lens": st["lens"]}
    lens = st["lens"].long()
    first = st["cu_rows"].long()[:-1]
    if c["op"] == "decode":
        j = torch.arange(max(_lengths(c)), device=_dev)
        seen = j < lens[:, None]
        at = first[:, None] + torch.minimum(j, lens[:, None] - 1)
        return {"out": _plain_attend(st, at[None, :, None], seen[None, :, None])}
    blocks = _plain_blocks(st, c["blocks"])
    j = (blocks.long()[..., None] * BLOCK + torch.arange(BLOCK, device=_dev)).flatten(-2)
    seen = (j >= 0) & (j < lens[:, None, None])
    j = torch.minimum(j.clamp(min=0), lens[:, None, None] - 1)
    return {"out": _plain_attend(st, first[:, None, None] + j, seen), "blocks": blocks}


# ------------------------------------------------------------------------------- calls
def _run_own(st):
    import paper_2609_22158_amd as stepkv

    c, cache = st["case"], st["cache"]
    if c["op"] == "compact":
        stepkv.compact4(st["problem"], cache, st["k"], st["v"], st["idx"], st["cu_out"])
    elif c["op"] == "append":
        stepkv.append4(cache, st["k_new"], st["v_new"], st["cu_out"])
    if c["op"] in ("compact", "append", "read"):
        k, v = stepkv.read4(cache, st["cu_out"], st["out_rows"])
        if c["op"] == "read":
            return {"k": k, "v": v}
        return {"k": k, "v": v, "k_bounds": st["k_bounds"], "lens": st["lens"]}
    if c["op"] == "decode":
        return {"out": stepkv.decode_attention4(cache, st["q"])}
    out, blocks = stepkv.decode_sparse4(cache, st["q"], c["blocks"])
    return {"out": out, "blocks": blocks}


def run(st):
    return _run_own(st) if own else _run_plain(st)


# -------------------------------------------------------------------- what a pass needs
def work(case):
    c = _case(**case)
    L, H, Hq, d, S = c["layers"], c["kv_heads"], c["q_heads"], c["d"], c["seqs"]
    held = _lengths(c)
    packed = 2 * (d // 2 + d // GROUP)  # bytes of a row, K and V
    bounds = 4 * d  # bytes of a block's bounds
    if c["op"] in ("compact", "append"):
        n = held if c["op"] == "compact" else _new_counts(c)
        nb = sum(-(-x // BLOCK) for x in n)
        # bf16 rows in, codes and bounds out, bf16 rows out; positions of the compaction
        nbytes = L * H * (sum(n) * (8 * d + packed) + nb * bounds)
        if c["op"] == "compact":
            nbytes += 4 * sum(n) * (1 if c["shared"] else L * H)
        return {"bytes": nbytes, "flops": 4 * L * H * sum(n) * d}
    if c["op"] == "read":
        return {"bytes": L * H * sum(held) * (packed + 4 * d), "flops": 2 * L * H * sum(held) * d}
    ends = L * S * Hq * d * 6  # queries in, outputs out
    if c["op"] == "decode":
        return {"bytes": L * H * sum(held) * packed + ends, "flops": 4 * L * Hq * sum(held) * d}
    nb = [-(-n // BLOCK) for n in held]
    scored = sum(x for x in nb if x > c["blocks"])
    # rows of the attended blocks; the last, always among them, may be short
    rows = sum(min(x, c["blocks"]) * BLOCK - (x * BLOCK - n) for x, n in zip(nb, held))
    return {"bytes": L * H * (scored * bounds + rows * packed + 4 * S * c["blocks"]) + ends,
            "flops": 4 * L * H * scored * d + 4 * L * Hq * rows * d}


# --------------------------------------------------------- in 64 bits, from the definition
def _exact_pow2(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_round(x):
    """The values that quantised float64 rows [..][d] stand for."""
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // GROUP, GROUP))
    top = g.abs().amax(dim=-1, keepdim=True)
    e = torch.full_like(top, -124.0)
    e = torch.where(top > 0, torch.ceil(torch.log2(top.clamp(min=2.0 ** -130) / 7.0)), e)
    e = torch.where(top > 7.0 * _exact_pow2(e), e + 1, e)  # a logarithm rounded the wrong way
    e = torch.where(top <= 7.0 * _exact_pow2(e - 1), e - 1, e).clamp(-124.0, 125.0)
    y = g / _exact_pow2(e)
    best, dist = torch.zeros_like(y), y.abs()
    for code in (2, 4, 6, 1, 3, 5, 7):  # the even codes first: they win ties
        t = y.abs() - _LEVELS[code]
        near = t.abs() < dist
        best, dist = torch.where(near, torch.full_like(y, _LEVELS[code]), best), torch.where(near, t.abs(), dist)
    return (torch.sign(y) * best * _exact_pow2(e)).reshape(x.shape)


def _exact_rows(st, name, l, a, b):
    """Float64 values [H][b - a][d] of cache rows a .. b - 1 of layer l."""
    codes = st[name + "_codes"][l, :, a:b].to(torch.int64)
    c = torch.stack([codes % 16, codes // 16], dim=-1).flatten(-2)
    m = c % 8
    mag = torch.where(m < 2, 0.5 * m, (2 + m % 2) * _exact_pow2(m // 2 - 2))
    sign = 1.0 - 2.0 * (c // 8).double()
    s = _exact_pow2(st[name + "_scales"][l, :, a:b].long() - 127)
    return sign * mag.double() * s.repeat_interleave(GROUP, dim=-1)


def exact(case, seed):
    c = _case(**case)
    st = prepare(case, seed)
    L, H, Hq, d, S, f64 = c["layers"], c["kv_heads"], c["q_heads"], c["d"], c["seqs"], torch.float64
    held, cu_rows = _lengths(c), [int(x) for x in st["cu_rows_host"]]
    if c["op"] in ("compact", "append", "read"):
        n = _new_counts(c) if c["op"] == "append" else held
        cu = [int(x) for x in _offsets(n)]
        k = torch.empty((L, H, cu[-1], d), dtype=f64, device=_dev)
        v = torch.empty_like(k)
        bounds = st["k_bounds"].to(f64)
        for l in range(L):
            for s in range(S):
                a, b = cu[s], cu[s + 1]
                if a == b:
                    continue
                if c["op"] == "read":
                    r = cu_rows[s]
                    k[l, :, a:b] = _exact_rows(st, "k", l, r, r + held[s])
                    v[l, :, a:b] = _exact_rows(st, "v", l, r, r + held[s])
                    continue
                for name, to in (("k", k), ("v", v)):
                    if c["op"] == "append":
                        x = st[name + "_new"][l, a:b].transpose(0, 1)
                    else:
                        q0 = int(st["cu_seqlens_host"][s])
                        i = st["idx"][..., q0:q0 + held[s]].long() + q0
                        i = i if c["shared"] else i[l]
                        x = torch.stack([st[name][l, h, i if c["shared"] else i[h]] for h in range(H)])
                    to[l, :, a:b] = _exact_round(x.to(f64))
                first = held[s] - n[s]
                for blk in range(first // BLOCK, (held[s] - 1) // BLOCK + 1):
                    lo, hi = max(first, blk * BLOCK), min(held[s], (blk + 1) * BLOCK)
                    x = k[l, :, a + lo - first:a + hi - first]
                    at = cu_rows[s] // BLOCK + s + blk
                    mn, mx = x.amin(dim=1), x.amax(dim=1)
                    if lo > blk * BLOCK:
                        mn, mx = torch.minimum(mn, bounds[l, :, at, 0]), torch.maximum(mx, bounds[l, :, at, 1])
                    bounds[l, :, at, 0], bounds[l, :, at, 1] = mn, mx
        if c["op"] == "read":
            return {"k": k, "v": v}
        return {"k": k, "v": v, "k_bounds": bounds, "lens": None}
    out = torch.empty((L, S, Hq, d), dtype=f64, device=_dev)
    for l in range(L):
        for s in range(S):
            r, n = cu_rows[s], held[s]
            k, v = _exact_rows(st, "k", l, r, r + n), _exact_rows(st, "v", l, r, r + n)
            q = st["q"][l, s].to(f64).reshape(H, Hq // H, d)
            z = torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(d)
            nb = -(-n // BLOCK)
            if c["op"] == "sparse" and nb > c["blocks"]:
                at = r // BLOCK + s
                x = st["k_bounds"][l, :, at:at + nb].to(f64)  # [H][nb][2][d]
                top = torch.maximum(q[:, :, None] * x[:, None, :, 0], q[:, :, None] * x[:, None, :, 1])
                score = top.sum(dim=3).sum(dim=1).cpu().numpy()
                score[:, 0] = score[:, -1] = math.inf
                keep = np.zeros((H, nb), bool)
                for h in range(H):
                    keep[h, np.argsort(-score[h], kind="stable")[:c["blocks"]]] = True
                seen = torch.from_numpy(keep.repeat(BLOCK, axis=1)[:, :n]).to(_dev)
                z = z.masked_fill(~seen[:, None], -math.inf)
            out[l, s] = torch.bmm(torch.softmax(z, dim=-1), v).reshape(Hq, d)
    return {"out": out} if c["op"] == "decode" else {"out": out, "blocks": None}
