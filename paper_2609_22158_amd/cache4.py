"""ctypes binding of the 4-bit cache (the C ABI declared in include/stepkv_cache4.h).

A compacted cache in 17/64 of the bytes of bf16: written by ``compact4`` (the retained rows
of a pruning boundary) and ``append4`` (a step's new tokens), read back by ``read4``, attended
to by ``decode_attention4`` and, over its best-scoring blocks of 64 tokens, ``decode_sparse4``.

    cache = Cache4(L, Hkv, d, cu_rows)            # rows that each sequence may use
    layers = [cache.layers(l) for l in range(L)]  # once: making a view takes about 30 us
    compact4(pb, cache, k, v, idx, cu_retained)   # after select; sets cache.lens
    advance4(cache, cu_new)                       # each decode step, once:
    for l in range(L):                            # the model's layers
        append4(layers[l], k_new[l:l + 1], v_new[l:l + 1], cu_new)
        out = decode_attention4(layers[l], q[l:l + 1])

Argument marshalling only; there is no CPU fallback. Every tensor of a call lies on the
cache's device, and the call goes to the current stream of that device unless a stream of it
is given; buffers that a call allocates belong to the stream it runs on.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import numpy as np

from . import binding as B

BLOCK, GROUP = 64, 32  # STEPKV_CACHE4_BLOCK, STEPKV_CACHE4_GROUP
MAX_ROWS = (1 << 30) - (1 << 20)  # STEPKV_CACHE4_MAX_ROWS

_i32, _vp, _sz = ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t


class Cache4C(ctypes.Structure):
    _fields_ = [
        ("num_layers", _i32),
        ("num_kv_heads", _i32),
        ("head_dim", _i32),
        ("num_seqs", _i32),
        ("cu_rows_host", B._i32p),
        ("cu_rows", _vp),
        ("lens", _vp),
        ("k_codes", _vp),
        ("v_codes", _vp),
        ("k_scales", _vp),
        ("v_scales", _vp),
        ("k_bounds", _vp),
        ("status", _vp),
    ]


_cp = ctypes.POINTER(Cache4C)
_i64x3 = ctypes.c_int64 * 3
_SIGNATURES = {
    "stepkv_cache4_compact": (ctypes.c_int, [ctypes.POINTER(B.ProblemC), _cp, _vp, _vp, _vp, _i32,
                                             _vp, _vp]),
    "stepkv_cache4_advance": (ctypes.c_int, [_cp, _vp, _vp]),
    "stepkv_cache4_append": (ctypes.c_int, [_cp, _vp, ctypes.POINTER(ctypes.c_int64), _vp,
                                            ctypes.POINTER(ctypes.c_int64), _vp, _i32, _vp]),
    "stepkv_cache4_read": (ctypes.c_int, [_cp, _vp, _i32, _vp, _vp, _vp]),
    "stepkv_cache4_decode_workspace_bytes": (_sz, [_cp, _i32, _i32]),
    "stepkv_cache4_decode": (ctypes.c_int, [_cp, _i32, _vp, _vp, _i32, ctypes.c_float, _vp, _vp,
                                            _vp, _sz, _vp]),
    "stepkv_cache4_select_workspace_bytes": (_sz, [_cp]),
    "stepkv_cache4_select_blocks": (ctypes.c_int, [_cp, _i32, _vp, _i32, _i32, _i32, _vp, _vp, _sz,
                                                   _vp]),
    "stepkv_cache4_sparse_workspace_bytes": (_sz, [_cp, _i32, _i32]),
    "stepkv_cache4_decode_sparse": (ctypes.c_int, [_cp, _i32, _vp, _i32, _i32, _i32,
                                                   ctypes.c_float, _vp, _vp, _vp, _vp, _sz, _vp]),
}

_lib: Optional[ctypes.CDLL] = None
_fns: dict = {}  # the library's functions by name


def load() -> ctypes.CDLL:
    """The library with the signatures of stepkv_cache4.h declared."""
    global _lib
    if _lib is None:
        lib = B.load()
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
            _fns[name] = fn
        _fns["stepkv_status_read"] = lib.stepkv_status_read
        _lib = lib
    return _lib


# ---------------------------------------------------------------- the cache
class Cache4:
    """A 4-bit cache of S sequences: sequence s may use rows cu_rows[s] .. cu_rows[s + 1] - 1
    (copied: what is written into the given array later changes nothing).

    The buffers are allocated (zeroed) unless given; ``k_bounds=False`` keeps no bounds, for
    caches whose blocks are never selected. ``lens`` (int32 [S]) counts each sequence's tokens.
    Given codes that hold tokens need the bounds that go with them: zeroed ones are not theirs."""

    def __init__(self, num_layers: int, num_kv_heads: int, head_dim: int, cu_rows, *, k_codes=None,
                 v_codes=None, k_scales=None, v_scales=None, k_bounds=True, lens=None,
                 device="cuda", status: bool = True):
        import torch

        self.num_layers, self.num_kv_heads, self.head_dim = num_layers, num_kv_heads, head_dim
        self.cu_rows = np.array(cu_rows, dtype=np.int32, order="C")  # a copy: the library reads it at every call
        self.cu_rows.setflags(write=False)
        if self.cu_rows.ndim != 1 or self.cu_rows.size < 2:
            raise ValueError("cu_rows: the row offsets of one sequence or more")
        if not np.array_equal(self.cu_rows, cu_rows):
            raise ValueError("cu_rows: offsets that int32 does not hold")
        self.num_seqs = int(self.cu_rows.size - 1)
        self.rows = int(self.cu_rows[-1])
        self.device = _device(device)
        L, H, R, S, d, dev = (num_layers, num_kv_heads, self.rows, self.num_seqs, head_dim,
                              self.device)
        self.num_bounds = R // BLOCK + S
        self.cu_rows_dev = torch.tensor(self.cu_rows, device=dev)

        def buffer(t, dtype, shape, name):
            if t is None:
                return torch.zeros(shape, dtype=dtype, device=dev)
            _need(t, dtype, shape, name, dev)
            return t

        self.k_codes = buffer(k_codes, torch.uint8, (L, H, R, d // 2), "k_codes")
        self.v_codes = buffer(v_codes, torch.uint8, (L, H, R, d // 2), "v_codes")
        self.k_scales = buffer(k_scales, torch.uint8, (L, H, R, d // GROUP), "k_scales")
        self.v_scales = buffer(v_scales, torch.uint8, (L, H, R, d // GROUP), "v_scales")
        if k_bounds is True or k_bounds is False or k_bounds is None:
            k_bounds = (torch.zeros((L, H, self.num_bounds, 2, d), dtype=torch.bfloat16, device=dev)
                        if k_bounds else None)
        else:
            _need(k_bounds, torch.bfloat16, (L, H, self.num_bounds, 2, d), "k_bounds", dev)
        self.k_bounds = k_bounds
        self.lens = buffer(lens, torch.int32, (S,), "lens")
        self.status_dev = torch.zeros(1, dtype=torch.int32, device=dev) if status else None
        load()
        self._bind()

    def _bind(self):
        def ptr(t):
            return t.data_ptr() if t is not None and t.numel() else None

        self.c = Cache4C(self.num_layers, self.num_kv_heads, self.head_dim, self.num_seqs,
                         self.cu_rows.ctypes.data_as(B._i32p), ptr(self.cu_rows_dev),
                         ptr(self.lens), ptr(self.k_codes), ptr(self.v_codes), ptr(self.k_scales),
                         ptr(self.v_scales), ptr(self.k_bounds), ptr(self.status_dev))
        self._ref = ctypes.byref(self.c)
        self._sizes = {}    # workspace bytes of a call, by its shape
        self._strides = {}  # checked strides of new tokens, by their layout

    def layers(self, first: int, n: int = 1) -> "Cache4":
        """Layers first .. first + n - 1 as a cache of their own (views; lens is shared). A view is
        made anew at every call: keep those of a model's layers over its steps."""
        if n < 1 or first < 0 or first + n > self.num_layers:
            raise ValueError(f"layers {first} .. {first + n - 1} of {self.num_layers}")
        v = object.__new__(Cache4)
        v.__dict__.update(self.__dict__)
        v.num_layers = n
        for name in ("k_codes", "v_codes", "k_scales", "v_scales", "k_bounds"):
            t = getattr(self, name)
            setattr(v, name, None if t is None else t[first:first + n])
        v._bind()
        return v

    def status(self, clear: bool = False, stream=None) -> int:
        """stepkv_status_read: the STEPKV_FLAG_* bits reported so far (waits for the stream)."""
        flags = ctypes.c_uint32(0)
        pb = B.ProblemC(status=self.c.status)
        _call(self, "stepkv_status_read", stream, ctypes.byref(pb), ctypes.byref(flags),
              int(bool(clear)))
        return int(flags.value)


def _device(device):
    import torch

    dev = torch.device(device)
    if dev.type == "cuda" and dev.index is None:
        dev = torch.device("cuda", torch.cuda.current_device())
    return dev


def _need(t, dtype, shape, name, device):
    if t.dtype is dtype and t.shape == shape and t.device == device and t.is_contiguous():
        return t.data_ptr()
    if t.dtype != dtype:
        raise TypeError(f"{name}: dtype {t.dtype}, expected {dtype}")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    raise ValueError(f"{name}: must be a contiguous tensor on {device}")


def _call(cache, name, stream, *args):
    """The library's `name` on the cache's device; the stream is the last argument."""
    import torch

    dev = cache.device
    if dev.type != "cuda":
        raise ValueError(f"{name}: the cache lies on {dev}, not on a GPU")
    if stream is not None and stream.device != dev:
        raise ValueError(f"{name}: a stream of {stream.device}, the cache lies on {dev}")
    if torch.cuda.current_device() == dev.index:
        rc = _fns[name](*args, B._stream(stream))
    else:
        with torch.cuda.device(dev):
            rc = _fns[name](*args, B._stream(stream))
    if rc != B.OK:
        raise B.StepKVError(name, rc)


def _empty(shape, dtype, cache, stream):
    """A buffer for a call: of the stream that the call runs on."""
    import torch

    if stream is None:
        return torch.empty(shape, dtype=dtype, device=cache.device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=cache.device)


def _workspace(workspace, cache, stream, size, *args):
    """The caller's workspace, or one of `size`(cache, *args) bytes: that depends on the shape alone,
    which a cache keeps."""
    import torch

    if workspace is None:
        key = (size, args)
        nbytes = cache._sizes.get(key)
        if nbytes is None:
            nbytes = int(_fns[size](cache._ref, *args))
            if size == "stepkv_cache4_decode_workspace_bytes" and nbytes <= 256:
                nbytes = 0  # none is needed
            cache._sizes[key] = nbytes
        if nbytes == 0:
            return None, None, 0
        workspace = _empty((nbytes,), torch.uint8, cache, stream)
        return workspace, workspace.data_ptr(), nbytes
    if workspace.device != cache.device or not workspace.is_contiguous():
        raise ValueError(f"workspace: must be a contiguous tensor on {cache.device}")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


# ---------------------------------------------------------------- write, read back
def compact4(pb: B.Problem, cache: Cache4, k, v, idx, cu_retained, *, stream=None) -> Cache4:
    """stepkv_cache4_compact: the retained rows into the cache, quantised; sets cache.lens.

    idx is [L][Hkv][Ntot] (compact's) or [Ntot] (compact_shared's)."""
    import torch

    L, H, d, dev = pb.num_layers, pb.num_kv_heads, pb.head_dim, cache.device
    if pb.cu_seqlens_dev.device != dev:
        raise ValueError(f"pb: lies on {pb.cu_seqlens_dev.device}, the cache on {dev}")
    kp = _need(k, torch.bfloat16, (L, H, pb.ntot, d), "k", dev)
    vp = _need(v, torch.bfloat16, (L, H, pb.ntot, d), "v", dev)
    shared = idx.dim() == 1
    ip = _need(idx, torch.int32, (pb.ntot,) if shared else (L, H, pb.ntot), "idx", dev)
    cp = _need(cu_retained, torch.int32, (pb.num_seqs + 1,), "cu_retained", dev)
    _call(cache, "stepkv_cache4_compact", stream, ctypes.byref(pb.c), cache._ref, kp, vp, ip,
          int(shared), cp)
    return cache


def advance4(cache: Cache4, cu_new, *, stream=None) -> Cache4:
    """stepkv_cache4_advance: lens[s] += cu_new[s + 1] - cu_new[s], once for all layers."""
    import torch

    cp = _need(cu_new, torch.int32, (cache.num_seqs + 1,), "cu_new", cache.device)
    _call(cache, "stepkv_cache4_advance", stream, cache._ref, cp)
    return cache


def _tokens(t, cache, name):
    """Pointer and strides of new tokens bf16 [L][T][Hkv][d] whose channels are contiguous."""
    import torch

    if t.dtype != torch.bfloat16:
        raise TypeError(f"{name}: dtype {t.dtype}, expected {torch.bfloat16}")
    key = (t.shape, t.stride())
    strides = cache._strides.get(key)
    if strides is not None and t.device == cache.device and t.data_ptr() % 16 == 0:
        return t.data_ptr(), strides
    L, H, d = cache.num_layers, cache.num_kv_heads, cache.head_dim
    if t.dim() != 4 or t.shape[0] != L or t.shape[2] != H or t.shape[3] != d:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected ({L}, tokens, {H}, {d})")
    if t.device != cache.device or t.stride(3) != 1:
        raise ValueError(f"{name}: must lie on {cache.device} with contiguous channels")
    strides = _i64x3(*(t.stride(i) if t.shape[i] > 1 else 0 for i in range(3)))
    if t.numel() and (t.data_ptr() % 16 or any(x % 8 for x in strides)):
        raise ValueError(f"{name}: rows must be 16-byte aligned (strides {t.stride()})")
    if not t.numel():
        return None, strides
    if len(cache._strides) < 64:
        cache._strides[key] = strides
    return t.data_ptr(), strides


def append4(cache: Cache4, k_new, v_new, cu_new, *, stream=None) -> Cache4:
    """stepkv_cache4_append: new tokens bf16 [L][T][Hkv][d] (any strides over layers, tokens and
    heads; tokens cu_new[s] .. cu_new[s + 1] - 1 are sequence s's) as its last tokens. Call
    advance4 before, once for all layers."""
    import torch

    kp, ks = _tokens(k_new, cache, "k_new")
    vp, vs = _tokens(v_new, cache, "v_new")
    if v_new.shape != k_new.shape:
        raise ValueError(f"v_new: shape {tuple(v_new.shape)}, expected {tuple(k_new.shape)}")
    cp = _need(cu_new, torch.int32, (cache.num_seqs + 1,), "cu_new", cache.device)
    _call(cache, "stepkv_cache4_append", stream, cache._ref, kp, ks, vp, vs, cp,
          int(k_new.shape[1]))
    return cache


def read4(cache: Cache4, cu_out, out_rows: int, *, k_out=None, v_out=None, stream=None):
    """stepkv_cache4_read: the last cu_out[s + 1] - cu_out[s] tokens of every sequence as bf16
    rows cu_out[s] .. of k, v [L][Hkv][out_rows][d]; ``k_out=False`` or ``v_out=False`` leaves
    that one out (None in the result). Rows without a token stay as they were."""
    import torch

    shape = (cache.num_layers, cache.num_kv_heads, int(out_rows), cache.head_dim)
    cp = _need(cu_out, torch.int32, (cache.num_seqs + 1,), "cu_out", cache.device)

    def rows(t, name):
        if t is False:
            return None, None
        if t is None:
            t = _empty(shape, torch.bfloat16, cache, stream)
        p = _need(t, torch.bfloat16, shape, name, cache.device)
        return t, p if t.numel() else None

    (k, kp), (v, vp) = rows(k_out, "k_out"), rows(v_out, "v_out")
    _call(cache, "stepkv_cache4_read", stream, cache._ref, cp, int(out_rows), kp, vp)
    return k, v


# ---------------------------------------------------------------- attention
def _queries(cache, q_dec):
    import torch

    if q_dec.dim() != 4:
        raise ValueError(f"q_dec: shape {tuple(q_dec.shape)}, expected [L][S][Hq][d]")
    Hq = int(q_dec.shape[2])
    return _need(q_dec, torch.bfloat16, (cache.num_layers, cache.num_seqs, Hq, cache.head_dim),
                 "q_dec", cache.device), Hq


def _results(cache, Hq, out, lse, want_lse, stream):
    import torch

    L, S, d = cache.num_layers, cache.num_seqs, cache.head_dim
    if out is None:
        out = _empty((L, S, Hq, d), torch.float32, cache, stream)
    op = _need(out, torch.float32, (L, S, Hq, d), "out", cache.device)
    if lse is None and want_lse:
        lse = _empty((L, S, Hq), torch.float32, cache, stream)
    lp = None
    if lse is not None:
        lp = _need(lse, torch.float32, (L, S, Hq), "lse", cache.device)
    return out, op, lse, lp


def decode_attention4(cache: Cache4, q_dec, *, blocks=None, scale: float = 0.0, out=None, lse=None,
                      want_lse: bool = False, workspace=None, stream=None):
    """stepkv_cache4_decode: fp32 [L][S][Hq][d], over all tokens or the listed blocks (int32
    [L][S][Hkv][n], n >= 1, as select_blocks4 gives them). With ``want_lse`` or an ``lse`` buffer also
    the rows' natural-log log-sum-exps [L][S][Hq]: (out, lse)."""
    import torch

    qp, Hq = _queries(cache, q_dec)
    bp, n = None, 0
    if blocks is not None:
        n = int(blocks.shape[-1]) if blocks.dim() else 0
        if n < 1:  # the library takes a null list for none, which attends to every token
            raise ValueError("blocks: a list of one block at least")
        bp = _need(blocks, torch.int32, (cache.num_layers, cache.num_seqs, cache.num_kv_heads, n),
                   "blocks", cache.device)
    out, op, lse, lp = _results(cache, Hq, out, lse, want_lse, stream)
    ws, wp, wn = _workspace(workspace, cache, stream, "stepkv_cache4_decode_workspace_bytes", Hq, n)
    _call(cache, "stepkv_cache4_decode", stream, cache._ref, Hq, qp, bp, n, float(scale), op, lp,
          wp, wn)
    return out if lse is None else (out, lse)


def _blocks(cache, num_blocks, blocks, stream):
    import torch

    shape = (cache.num_layers, cache.num_seqs, cache.num_kv_heads, int(num_blocks))
    if num_blocks < 1:
        raise ValueError("num_blocks: one block at least")
    if blocks is None:
        blocks = _empty(shape, torch.int32, cache, stream)
    return blocks, _need(blocks, torch.int32, shape, "blocks", cache.device)


def select_blocks4(cache: Cache4, q_dec, num_blocks: int, *, first: int = 1, last: int = 1,
                   blocks=None, workspace=None, stream=None):
    """stepkv_cache4_select_blocks: int32 [L][S][Hkv][num_blocks], ascending, -1 past the last:
    the first and last blocks of every sequence and the best others for the step's queries."""
    qp, Hq = _queries(cache, q_dec)
    blocks, bp = _blocks(cache, num_blocks, blocks, stream)
    ws, wp, wn = _workspace(workspace, cache, stream, "stepkv_cache4_select_workspace_bytes")
    _call(cache, "stepkv_cache4_select_blocks", stream, cache._ref, Hq, qp, int(num_blocks),
          int(first), int(last), bp, wp, wn)
    return blocks


def decode_sparse4(cache: Cache4, q_dec, num_blocks: int, *, first: int = 1, last: int = 1,
                   scale: float = 0.0, blocks=None, out=None, lse=None, want_lse: bool = False,
                   workspace=None, stream=None):
    """stepkv_cache4_decode_sparse: select_blocks4 and attention over the selection in one call;
    (out, blocks), or (out, blocks, lse) with ``want_lse`` or an ``lse`` buffer."""
    qp, Hq = _queries(cache, q_dec)
    blocks, bp = _blocks(cache, num_blocks, blocks, stream)
    out, op, lse, lp = _results(cache, Hq, out, lse, want_lse, stream)
    ws, wp, wn = _workspace(workspace, cache, stream, "stepkv_cache4_sparse_workspace_bytes", Hq,
                            int(num_blocks))
    _call(cache, "stepkv_cache4_decode_sparse", stream, cache._ref, Hq, qp, int(num_blocks),
          int(first), int(last), float(scale), bp, op, lp, wp, wn)
    return (out, blocks) if lse is None else (out, blocks, lse)
