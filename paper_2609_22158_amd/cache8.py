"""ctypes binding of the 8-bit cache (the C ABI declared in include/stepkv_cache8.h).

A compacted cache in half the bytes of bf16: written by ``compact8`` (the retained rows of a
pruning boundary) and ``append8`` (a step's new tokens), read back by ``read8``, attended to by
``decode_attention8``, which can add up the attention weight of every token, and kept at its
size between boundaries by ``evict8``, which gives up the tokens of least weight.

    cache = Cache8(L, Hkv, d, cu_rows)            # rows that each sequence may use
    layers = [cache.layers(l) for l in range(L)]  # once: making a view takes about 30 us
    compact8(pb, cache, k, v, idx, cu_retained)   # after select; sets cache.lens
    advance8(cache, cu_new)                       # each decode step, once:
    for l in range(L):                            # the model's layers
        append8(layers[l], k_new[l:l + 1], v_new[l:l + 1], cu_new)
        out = decode_attention8(layers[l], q[l:l + 1], gather=True)
    evict8(cache, budget, first=4, recent=128)    # the whole cache: every sequence to its budget

Argument marshalling only; there is no CPU fallback. Every tensor of a call lies on the
cache's device, and the call goes to the current stream of that device unless a stream of it
is given; buffers that a call allocates belong to the stream it runs on.
"""
from __future__ import annotations

import ctypes


from . import binding as B
from . import cache4 as C4

BLOCK = 64  # STEPKV_CACHE8_BLOCK
MAX_ROWS = (1 << 30) - (1 << 20)  # STEPKV_CACHE8_MAX_ROWS

_i32, _vp, _sz = ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t
_BUFFERS = ("k_codes", "v_codes", "k_scales", "v_scales", "weights", "positions")


class Cache8C(ctypes.Structure):
    _fields_ = [
        ("num_layers", _i32),
        ("num_kv_heads", _i32),
        ("head_dim", _i32),
        ("num_seqs", _i32),
        ("cu_rows_host", B._i32p),
        ("cu_rows", _vp),
        ("lens", _vp),
        ("seen", _vp),
        ("k_codes", _vp),
        ("v_codes", _vp),
        ("k_scales", _vp),
        ("v_scales", _vp),
        ("weights", _vp),
        ("positions", _vp),
        ("status", _vp),
    ]


_cp = ctypes.POINTER(Cache8C)
_i64p = ctypes.POINTER(ctypes.c_int64)
_SIGNATURES = {
    "stepkv_cache8_compact": (ctypes.c_int, [ctypes.POINTER(B.ProblemC), _cp, _vp, _vp, _vp, _i32,
                                             _vp, _vp, _vp]),
    "stepkv_cache8_advance": (ctypes.c_int, [_cp, _vp, _vp]),
    "stepkv_cache8_append": (ctypes.c_int, [_cp, _vp, _i64p, _vp, _i64p, _vp, _i32, _vp]),
    "stepkv_cache8_read": (ctypes.c_int, [_cp, _vp, _i32, _vp, _vp, _vp]),
    "stepkv_cache8_decode_workspace_bytes": (_sz, [_cp, _i32, _i32]),
    "stepkv_cache8_decode": (ctypes.c_int, [_cp, _i32, _vp, ctypes.c_float, _i32, _vp, _vp, _vp,
                                            _sz, _vp]),
    "stepkv_cache8_evict_workspace_bytes": (_sz, [_cp]),
    "stepkv_cache8_evict": (ctypes.c_int, [_cp, _i32, _vp, _i32, _i32, _vp, _sz, _vp]),
}

_loaded = False
torch = None  # imported with the library


def load() -> ctypes.CDLL:
    """The library with the signatures of stepkv_cache8.h declared."""
    global _loaded, torch
    lib = C4.load()
    if not _loaded:
        C4.declare(lib, _SIGNATURES)
        torch = C4.torch
        _loaded = True
    return lib


# ---------------------------------------------------------------- the cache
class Cache8:
    """An 8-bit cache of S sequences: sequence s may use rows cu_rows[s] .. cu_rows[s + 1] - 1
    (copied: what is written into the given array later changes nothing).

    The buffers are allocated (zeroed) unless given. ``weights`` and ``positions`` are what
    gathering and evicting need: ``weights=False`` keeps neither, for caches that only grow
    between boundaries. ``lens`` (int32 [S]) counts each sequence's tokens, ``seen`` those that
    came so far. Given tokens (``lens`` that are not 0) without ``seen`` are all that came, and
    without ``positions`` they are the last that came, in order: seen[s] - lens[s] + j for token j.
    Where tokens were pruned or evicted before, both have to be given."""

    def __init__(self, num_layers: int, num_kv_heads: int, head_dim: int, cu_rows, *, k_codes=None,
                 v_codes=None, k_scales=None, v_scales=None, weights=True, positions=None,
                 lens=None, seen=None, device="cuda", status: bool = True):
        import torch

        self.num_layers, self.num_kv_heads, self.head_dim = num_layers, num_kv_heads, head_dim
        self.cu_rows = C4.row_offsets(cu_rows)
        self.num_seqs = int(self.cu_rows.size - 1)
        self.rows = int(self.cu_rows[-1])
        self.device = C4._device(device)
        L, H, R, S, d, dev = (num_layers, num_kv_heads, self.rows, self.num_seqs, head_dim,
                              self.device)
        self.num_blocks = R // BLOCK + S
        self.cu_rows_dev = torch.tensor(self.cu_rows, device=dev)

        def buffer(t, dtype, shape, name):
            if t is None or t is True:
                return torch.zeros(shape, dtype=dtype, device=dev)
            C4._need(t, dtype, shape, name, dev)
            return t

        self.k_codes = buffer(k_codes, torch.uint8, (L, H, R, d), "k_codes")
        self.v_codes = buffer(v_codes, torch.uint8, (L, H, R, d), "v_codes")
        self.k_scales = buffer(k_scales, torch.float32, (L, H, self.num_blocks), "k_scales")
        self.v_scales = buffer(v_scales, torch.float32, (L, H, self.num_blocks), "v_scales")
        if weights is False or weights is None:
            if positions is not None:
                raise ValueError("positions: only of a cache with weights")
            self.weights = self.positions = None
        else:
            self.weights = buffer(weights, torch.float32, (L, H, R), "weights")
            self.positions = buffer(positions, torch.int32, (L, H, R), "positions")
        self.lens = buffer(lens, torch.int32, (S,), "lens")
        self.seen = buffer(seen, torch.int32, (S,), "seen")
        if lens is not None:
            if seen is None:
                self.seen.copy_(self.lens)
            if self.positions is not None and positions is None:
                cu = self.cu_rows_dev.long()
                s = torch.repeat_interleave(torch.arange(S, device=dev), cu[1:] - cu[:-1], output_size=R)
                j = torch.arange(R, device=dev) - cu[s]
                held = self.lens[s]
                self.positions.copy_(torch.where(j < held, self.seen[s] - held + j, 0))
        self.status_dev = torch.zeros(1, dtype=torch.int32, device=dev) if status else None
        self.whole = True  # not some layers of a cache
        load()
        self._bind()

    def _bind(self):
        def ptr(t):
            return t.data_ptr() if t is not None and t.numel() else None

        self.c = Cache8C(self.num_layers, self.num_kv_heads, self.head_dim, self.num_seqs,
                         self.cu_rows.ctypes.data_as(B._i32p), ptr(self.cu_rows_dev),
                         ptr(self.lens), ptr(self.seen), *(ptr(getattr(self, x)) for x in _BUFFERS),
                         ptr(self.status_dev))
        self._ref = ctypes.byref(self.c)
        self._sizes = {}    # workspace bytes of a call, by its shape
        self._strides = {}  # checked strides of new tokens, by their layout

    def layers(self, first: int, n: int = 1) -> "Cache8":
        """Layers first .. first + n - 1 as a cache of their own (views; lens and seen are shared).
        A view is made anew at every call: keep those of a model's layers over its steps."""
        if n < 1 or first < 0 or first + n > self.num_layers:
            raise ValueError(f"layers {first} .. {first + n - 1} of {self.num_layers}")
        v = object.__new__(Cache8)
        v.__dict__.update(self.__dict__)
        v.whole = self.whole and n == self.num_layers
        v.num_layers = n
        for name in _BUFFERS:
            t = getattr(self, name)
            setattr(v, name, None if t is None else t[first:first + n])
        v._bind()
        return v

    def status(self, clear: bool = False, stream=None) -> int:
        """stepkv_status_read: the STEPKV_FLAG_* bits reported so far (waits for the stream)."""
        flags = ctypes.c_uint32(0)
        pb = B.ProblemC(status=self.c.status)
        C4._call(self, "stepkv_status_read", stream, ctypes.byref(pb), ctypes.byref(flags),
                 int(bool(clear)))
        return int(flags.value)


# ---------------------------------------------------------------- write, read back
def compact8(pb: B.Problem, cache: Cache8, k, v, idx, cu_retained, *, weights=None,
             stream=None) -> Cache8:
    """stepkv_cache8_compact: the retained rows into the cache, quantised; sets cache.lens and
    cache.seen.

    idx is [L][Hkv][Ntot] (compact's) or [Ntot] (compact_shared's). weights (fp32 [L][Hkv][Ntot],
    e.g. the saliency) is what the source's tokens gathered so far; without it they start at 0."""
    L, H, d, dev = pb.num_layers, pb.num_kv_heads, pb.head_dim, cache.device
    if pb.cu_seqlens_dev.device != dev:
        raise ValueError(f"pb: lies on {pb.cu_seqlens_dev.device}, the cache on {dev}")
    kp = C4._need(k, torch.bfloat16, (L, H, pb.ntot, d), "k", dev)
    vp = C4._need(v, torch.bfloat16, (L, H, pb.ntot, d), "v", dev)
    shared = idx.dim() == 1
    ip = C4._need(idx, torch.int32, (pb.ntot,) if shared else (L, H, pb.ntot), "idx", dev)
    cp = C4._need(cu_retained, torch.int32, (pb.num_seqs + 1,), "cu_retained", dev)
    wp = None
    if weights is not None:
        if cache.weights is None:
            raise ValueError("weights: the cache keeps none")
        wp = C4._need(weights, torch.float32, (L, H, pb.ntot), "weights", dev)
    C4._call(cache, "stepkv_cache8_compact", stream, ctypes.byref(pb.c), cache._ref, kp, vp, ip,
             int(shared), cp, wp)
    return cache


def advance8(cache: Cache8, cu_new, *, stream=None) -> Cache8:
    """stepkv_cache8_advance: lens[s] and seen[s] += cu_new[s + 1] - cu_new[s], once for all
    layers."""
    cp = C4._need(cu_new, torch.int32, (cache.num_seqs + 1,), "cu_new", cache.device)
    C4._call(cache, "stepkv_cache8_advance", stream, cache._ref, cp)
    return cache


def append8(cache: Cache8, k_new, v_new, cu_new, *, stream=None) -> Cache8:
    """stepkv_cache8_append: new tokens bf16 [L][T][Hkv][d] (any strides over layers, tokens and
    heads; tokens cu_new[s] .. cu_new[s + 1] - 1 are sequence s's) as its last tokens. Call
    advance8 before, once for all layers."""
    kp, ks = C4._tokens(k_new, cache, "k_new")
    vp, vs = C4._tokens(v_new, cache, "v_new")
    if v_new.shape != k_new.shape:
        raise ValueError(f"v_new: shape {tuple(v_new.shape)}, expected {tuple(k_new.shape)}")
    cp = C4._need(cu_new, torch.int32, (cache.num_seqs + 1,), "cu_new", cache.device)
    C4._call(cache, "stepkv_cache8_append", stream, cache._ref, kp, ks, vp, vs, cp,
             int(k_new.shape[1]))
    return cache


def read8(cache: Cache8, cu_out, out_rows: int, *, k_out=None, v_out=None, stream=None):
    """stepkv_cache8_read: the last cu_out[s + 1] - cu_out[s] tokens of every sequence as bf16
    rows cu_out[s] .. of k, v [L][Hkv][out_rows][d]; ``k_out=False`` or ``v_out=False`` leaves
    that one out (None in the result). Rows without a token stay as they were."""
    return C4._read(cache, "stepkv_cache8_read", cu_out, out_rows, k_out, v_out, stream)


# ---------------------------------------------------------------- attention, eviction
def decode_attention8(cache: Cache8, q_dec, *, gather: bool = False, scale: float = 0.0, out=None,
                      lse=None, want_lse: bool = False, workspace=None, stream=None):
    """stepkv_cache8_decode: fp32 [L][S][Hq][d]. With ``gather`` every token's attention weight,
    summed over the query heads of its KV head, is added to cache.weights. With ``want_lse`` or an
    ``lse`` buffer also the rows' natural-log log-sum-exps [L][S][Hq]: (out, lse)."""
    qp, Hq = C4._queries(cache, q_dec)
    if gather and cache.weights is None:
        raise ValueError("gather: the cache keeps no weights")
    gather = int(bool(gather))
    out, op, lse, lp = C4._results(cache, Hq, out, lse, want_lse, stream)
    ws, wp, wn = C4._workspace(workspace, cache, stream, "stepkv_cache8_decode_workspace_bytes", Hq,
                               gather)
    C4._call(cache, "stepkv_cache8_decode", stream, cache._ref, Hq, qp, float(scale), gather, op, lp,
             wp, wn)
    return out if lse is None else (out, lse)


def evict8(cache: Cache8, keep: int = 0, *, keeps=None, first: int = 0, recent: int = 0,
           workspace=None, stream=None) -> Cache8:
    """stepkv_cache8_evict: every sequence gives up tokens until it holds ``keep`` (or its entry of
    ``keeps``, int32 [S] on the device): those of least gathered weight, apart from positions below
    ``first`` and the last ``recent`` ones. Each head its own, so this takes the whole cache, not
    some of its layers; cache.positions says which tokens stay, and cache.lens how many."""
    if not cache.whole:
        raise ValueError("evict8: takes all layers of a cache, whose lens they share")
    for name, x in (("keep", keep), ("first", first), ("recent", recent)):
        if not 0 <= x < 1 << 31:  # what the library takes; of more the lower bits would count
            raise ValueError(f"{name}: {x} is not a number of tokens")
    if cache.weights is None:
        raise ValueError("evict8: the cache keeps no weights")
    if keeps is None and keep < 1:
        raise ValueError("keep: one token at least")
    kp = None
    if keeps is not None:
        if keep:
            raise ValueError("keep, keeps: one of them")
        kp = C4._need(keeps, torch.int32, (cache.num_seqs,), "keeps", cache.device)
    ws, wp, wn = C4._workspace(workspace, cache, stream, "stepkv_cache8_evict_workspace_bytes")
    C4._call(cache, "stepkv_cache8_evict", stream, cache._ref, int(keep), kp, int(first), int(recent),
             wp, wn)
    return cache
