"""The 8-bit cache without a GPU: the oracle of its format and of its eviction, the exports, the
workspace sizes and the refusals of every entry point (validation runs on the host before anything
is launched; the device pointers below are placeholders that no call follows)."""
import ctypes
import os
import re

import numpy as np
import pytest

import oracle.cache8_ref as R
from paper_2609_22158_amd import binding as B
from paper_2609_22158_amd import cache4 as C4
from paper_2609_22158_amd import cache8 as C8

HEADER = os.path.join(os.path.dirname(os.path.dirname(__file__)), "include", "stepkv_cache8.h")
FAKE = 0x10000  # placeholder device address, 256-byte aligned


# ---------------------------------------------------------------- the format
def test_numbers_are_e4m3():
    import torch

    t = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, R.NUMBERS, equal_nan=True)


def test_rounding_by_hand():
    y = np.array([0.0, 448, 464, 500, -464.1, 1.0625, 1.1875, 1.0626, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -11,
                  17, -18.9, np.nan, np.inf])
    want = [0, 448, 448, 448, -448, 1.0, 1.25, 1.125, 0.0, 2.0 ** -8, 0.0, 16, -18, np.nan, np.nan]
    assert np.array_equal(R.round8(y), want, equal_nan=True)


def test_rounding_is_that_of_e4m3():
    import torch

    x = np.random.default_rng(0).standard_normal(20000) * 2.0 ** np.random.default_rng(1).integers(-12, 9, 20000)
    x = np.clip(x, -448, 448).astype(np.float32)
    t = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(R.round8(x.astype(np.float64)), t)


@pytest.mark.parametrize("top,e", [(464.0, 0), (464.5, 1), (232.0, -1), (232.1, 0), (0.0, -117), (1e-40, -117),
                                   (3.0e38, 119), (3.38e38, 119), (1.0, -8), (np.inf, -117)])
def test_need(top, e):
    x = np.zeros((2, 64))
    x[1, 7] = -top
    assert R.need(x) == e


def values(n, d, seed, spread=6):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, d)) * 2.0 ** rng.integers(-spread, spread, (n, 1))
    return x.astype(np.float32).astype(np.float64)


def test_quantising_again_gives_the_same_values():
    a = R.Head8(64)
    a.append(values(150, 64, 0), values(150, 64, 1), np.arange(150))
    b = R.Head8(64)
    b.append(a.values(0), a.values(1), np.arange(150))
    for w in (0, 1):
        assert np.array_equal(a.values(w), b.values(w)) and a.exp[w] == b.exp[w]


@pytest.mark.parametrize("step", [1, 3, 64, 200])
def test_error_bound_however_often_a_block_grows(step):
    """2^-4 of the element, or 2^-9 * 2^e: the bound that the header states, token by token too."""
    x = values(200, 64, 2) * 2.0 ** np.linspace(-20, 10, 200)[:, None]  # every block grows often
    a = R.Head8(64)
    for i in range(0, 200, step):
        a.append(x[i:i + step], x[i:i + step], np.arange(i, min(i + step, 200)))
    e = np.repeat(a.exp[0], 64)[:200, None]
    assert (np.abs(a.values(0) - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** (e - 9.0))).all()


def test_stay_by_hand():
    w = np.array([3.0, np.nan, 1.0, 3.0, 0.0, 9.0, -0.0, 2.0])
    pos = np.array([0, 5, 9, 2, 11, 7, 4, 12])
    kept = lambda keep, first, recent: np.nonzero(R.stay(w, pos, keep, first, recent, 13))[0].tolist()  # noqa: E731
    assert kept(3, 0, 0) == [0, 3, 5]
    assert kept(2, 0, 0) == [0, 5]                 # equal weights: the lower row
    assert kept(6, 0, 0) == [0, 2, 3, 4, 5, 7]     # 0 and -0 are equal: the lower row
    assert kept(7, 0, 0) == [0, 2, 3, 4, 5, 6, 7]  # NaN last
    assert kept(3, 1, 2) == [0, 4, 7]              # position 0, and 11 and 12
    assert kept(2, 1, 2) == [0, 4]                 # more than stay: the lower rows
    assert kept(5, 6, 0) == [0, 1, 3, 5, 6]        # positions below 6, then by weight


def test_evict_by_hand():
    a = R.Head8(64)
    a.append(values(70, 64, 4), values(70, 64, 5), np.arange(70), weights=np.arange(70.0)[::-1].copy())
    k, v = a.values(0).copy(), a.values(1).copy()
    a.evict(66, 0, 3, 70)  # 67, 68 and 69 stay; of the others 63 .. 66 weigh least
    assert a.positions.tolist() == list(range(63)) + [67, 68, 69]
    e = np.repeat(a.exp[0], 64)[:66, None]
    src = np.array(list(range(63)) + [67, 68, 69])
    assert (np.abs(a.values(0) - k[src]) <= 2.0 ** (e - 10.0)).all()
    assert np.array_equal(a.weights, 69.0 - src) and len(a.exp[0]) == 2


# ---------------------------------------------------------------- the library
@pytest.fixture(scope="module")
def lib():
    return C8.load()


def _cache(L=2, H=2, d=128, rooms=(1000, 2000), **kw):
    cu = np.concatenate([[0], np.cumsum(np.asarray(rooms, np.int64))]).astype(np.int32)
    c = C8.Cache8C(L, H, d, len(rooms), cu.ctypes.data_as(B._i32p), *[FAKE] * 9, None)
    for k, v in kw.items():
        setattr(c, k, v)
    c._keep = cu
    return c


def _problem(L=2, Hq=8, Hkv=2, d=128, cu=(0, 3000, 6000)):
    cu = np.array(cu, np.int32)
    cs = np.zeros(len(cu), np.int32)
    pb = B.ProblemC(L, Hq, Hkv, d, 1, len(cu) - 1, cu.ctypes.data_as(B._i32p), FAKE,
                    cs.ctypes.data_as(B._i32p), FAKE)
    pb._keep = (cu, cs)
    return pb


def test_exports_every_declared_function(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(stepkv_cache8_[a-z_]+)\s*\(", text))
    assert names == set(C8._SIGNATURES) and len(names) == 8
    for n in names:
        assert hasattr(lib, n), n


STRIDES = (8, 8, 8)
CALLS = {
    "compact": lambda lib, c, pb=None, k=FAKE, v=FAKE, idx=FAKE, cu=FAKE, w=FAKE: lib.stepkv_cache8_compact(
        ctypes.byref(pb or _problem()), c, k, v, idx, 0, cu, w, None),
    "advance": lambda lib, c, cu=FAKE: lib.stepkv_cache8_advance(c, cu, None),
    "append": lambda lib, c, k=FAKE, v=FAKE, ks=STRIDES, vs=STRIDES, cu=FAKE, n=4:
        lib.stepkv_cache8_append(c, k, C4._i64x3(*ks) if ks else None, v, C4._i64x3(*vs) if vs else None,
                                 cu, n, None),
    "read": lambda lib, c, cu=FAKE, n=4, k=FAKE, v=FAKE: lib.stepkv_cache8_read(c, cu, n, k, v, None),
    "decode": lambda lib, c, hq=8, q=FAKE, scale=0.0, gather=1, out=FAKE, ws=FAKE, nb=1 << 40:
        lib.stepkv_cache8_decode(c, hq, q, scale, gather, out, None, ws, nb, None),
    "evict": lambda lib, c, keep=5, keeps=None, first=0, recent=0, ws=FAKE, nb=1 << 40:
        lib.stepkv_cache8_evict(c, keep, keeps, first, recent, ws, nb, None),
}


@pytest.mark.parametrize("call", list(CALLS))
@pytest.mark.parametrize("kw,code", [
    (dict(num_layers=0), B.EINVAL), (dict(num_kv_heads=0), B.EINVAL), (dict(num_seqs=0), B.EINVAL),
    (dict(head_dim=0), B.EINVAL), (dict(head_dim=96), B.EUNSUPPORTED), (dict(lens=None), B.EINVAL),
    (dict(seen=None), B.EINVAL), (dict(cu_rows=None), B.EINVAL), (dict(cu_rows_host=None), B.EINVAL),
    (dict(k_codes=None), B.EINVAL), (dict(v_codes=FAKE + 8), B.EINVAL), (dict(k_scales=FAKE + 2), B.EINVAL),
    (dict(v_scales=None), B.EINVAL), (dict(weights=None), B.EINVAL), (dict(positions=None), B.EINVAL),
    (dict(weights=FAKE + 2), B.EINVAL), (dict(positions=FAKE + 1), B.EINVAL),
])
def test_every_call_refuses_a_bad_cache(lib, call, kw, code):
    assert CALLS[call](lib, ctypes.byref(_cache(**kw))) == code
    assert CALLS[call](lib, None) == B.EINVAL


@pytest.mark.parametrize("rooms", [(10, -5), (-1, 4)])
def test_refuses_offsets(lib, rooms):
    assert CALLS["advance"](lib, ctypes.byref(_cache(rooms=rooms))) == B.EINVAL


@pytest.mark.parametrize("call,kw,code", [
    ("compact", dict(k=None), B.EINVAL), ("compact", dict(v=FAKE + 8), B.EINVAL),
    ("compact", dict(idx=None), B.EINVAL), ("compact", dict(cu=None), B.EINVAL),
    ("compact", dict(w=FAKE + 2), B.EINVAL), ("compact", dict(pb=_problem(L=3)), B.EINVAL),
    ("compact", dict(pb=_problem(Hkv=4)), B.EINVAL), ("compact", dict(pb=_problem(d=64)), B.EINVAL),
    ("compact", dict(pb=_problem(cu=(0, 5))), B.EINVAL), ("compact", dict(pb=_problem(cu=(0, 9, 5))), B.EINVAL),
    ("advance", dict(cu=None), B.EINVAL),
    ("append", dict(k=None), B.EINVAL), ("append", dict(v=None), B.EINVAL),
    ("append", dict(n=-1), B.EINVAL), ("append", dict(cu=None), B.EINVAL),
    ("append", dict(ks=(8, 4, 8)), B.EINVAL), ("append", dict(vs=None), B.EINVAL),
    ("append", dict(k=FAKE + 2), B.EINVAL),
    ("read", dict(n=-1), B.EINVAL), ("read", dict(k=None, v=None), B.EINVAL),
    ("read", dict(cu=None), B.EINVAL), ("read", dict(v=FAKE + 4), B.EINVAL),
    ("read", dict(n=2 ** 31 - 1), B.EUNSUPPORTED),
    ("decode", dict(hq=3), B.EINVAL), ("decode", dict(hq=0), B.EINVAL), ("decode", dict(q=None), B.EINVAL),
    ("decode", dict(q=FAKE + 2), B.EINVAL), ("decode", dict(out=None), B.EINVAL),
    ("decode", dict(scale=float("nan")), B.EINVAL), ("decode", dict(scale=3.0e38), B.EINVAL),
    ("decode", dict(ws=None), B.EWORKSPACE), ("decode", dict(ws=FAKE + 128), B.EWORKSPACE),
    ("decode", dict(nb=255), B.EWORKSPACE),
    ("evict", dict(keep=0), B.EINVAL), ("evict", dict(keep=-3), B.EINVAL), ("evict", dict(first=-1), B.EINVAL),
    ("evict", dict(recent=-1), B.EINVAL), ("evict", dict(ws=None), B.EWORKSPACE),
    ("evict", dict(keep=0, keeps=FAKE, ws=None), B.EWORKSPACE),
    ("evict", dict(ws=FAKE + 8), B.EWORKSPACE), ("evict", dict(nb=256), B.EWORKSPACE),
])
def test_refuses_arguments(lib, call, kw, code):
    assert CALLS[call](lib, ctypes.byref(_cache()), **kw) == code


def test_refuses_weights_that_the_cache_does_not_keep(lib):
    c = ctypes.byref(_cache(weights=None, positions=None))
    assert CALLS["compact"](lib, c) == B.EINVAL
    assert CALLS["decode"](lib, c) == B.EINVAL
    assert CALLS["evict"](lib, c) == B.EINVAL
    assert CALLS["decode"](lib, c, gather=0, ws=None) == B.EWORKSPACE  # attended to all the same


def test_refuses_rows_past_the_limit(lib):
    c = _cache(rooms=(C8.MAX_ROWS,))
    assert lib.stepkv_cache8_evict_workspace_bytes(ctypes.byref(c)) > 0
    c = _cache(rooms=(C8.MAX_ROWS, 1))
    assert CALLS["advance"](lib, ctypes.byref(c)) == B.EUNSUPPORTED
    assert lib.stepkv_cache8_decode_workspace_bytes(ctypes.byref(c), 8, 0) == 0


def test_nothing_to_do_launches_nothing(lib):
    assert CALLS["append"](lib, ctypes.byref(_cache()), n=0, k=None, v=None) == B.OK
    assert CALLS["read"](lib, ctypes.byref(_cache()), n=0, k=None, v=None) == B.OK


TOO_LARGE = {
    # a launch of 2^32 work items or more, in each of the kernels
    "compact": ([2 ** 28], lambda lib, c: lib.stepkv_cache8_compact(
        ctypes.byref(_problem(16, 16, 16, cu=(0, 2 ** 28))), c, FAKE, FAKE, FAKE, 0, FAKE, None, None)),
    "append": ([2 ** 28], lambda lib, c: CALLS["append"](lib, c, n=2 ** 28)),
    "read": ([2 ** 20], lambda lib, c: CALLS["read"](lib, c, n=2 ** 24)),
    "decode": ([1] * 70000, lambda lib, c: CALLS["decode"](lib, c, hq=16, gather=0)),
    "decode, merge": ([2 ** 17] + [0] * 70000, lambda lib, c: CALLS["decode"](lib, c, hq=16, gather=0)),
    "decode, gather": ([2 ** 18] + [0] * 65000, lambda lib, c: CALLS["decode"](lib, c, hq=16)),
    "evict": ([1] * 20000, lambda lib, c: CALLS["evict"](lib, c)),
}


@pytest.mark.parametrize("call", list(TOO_LARGE))
def test_refuses_more_than_a_launch_takes(lib, call):
    rooms, fn = TOO_LARGE[call]
    assert fn(lib, ctypes.byref(_cache(16, 16, 128, rooms))) == B.EUNSUPPORTED


def test_workspace_sizes(lib):
    c = ctypes.byref(_cache())
    size = lib.stepkv_cache8_decode_workspace_bytes
    dense, gather = size(c, 8, 0), size(c, 8, 1)
    assert dense > 256 and dense % 256 == 0
    assert gather >= dense + 4 * 2 * 8 * 3000  # the logits
    assert size(c, 3, 0) == 0 and size(ctypes.byref(_cache(head_dim=96)), 8, 0) == 0
    # short sequences need none: the smallest size says so
    short = ctypes.byref(_cache(rooms=(64, 300)))
    assert size(short, 8, 0) == 256 and size(short, 8, 1) == 256
    # the logits of longer ones, or of many heads, need some
    assert size(ctypes.byref(_cache(rooms=(64, 700))), 32, 1) >= 4 * 2 * 32 * 764
    assert size(ctypes.byref(_cache(rooms=(64, 300))), 64, 1) >= 4 * 2 * 64 * 364
    # a cache without room still has a workspace to pass
    assert size(ctypes.byref(_cache(rooms=(0, 0))), 8, 1) >= 256
    # a move for every second row at most, a record for every (layer, head, sequence)
    assert lib.stepkv_cache8_evict_workspace_bytes(c) >= 8 * 4 * 1500 + 16 * 8
    assert lib.stepkv_cache8_evict_workspace_bytes(None) == 0


# ---------------------------------------------------------------- the Python layer
def test_python_refuses_before_the_library():
    import torch

    c = C8.Cache8(2, 2, 64, [0, 100, 164], device="cpu")
    assert c.num_blocks == 164 // 64 + 2 and c.k_codes.shape == (2, 2, 164, 64)
    cu = torch.zeros(3, dtype=torch.int32)
    q = torch.zeros((2, 2, 8, 64), dtype=torch.bfloat16)
    new = torch.zeros((2, 5, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="not on a GPU"):
        C8.advance8(c, cu)
    with pytest.raises(TypeError):
        C8.advance8(c, cu.long())
    with pytest.raises(TypeError):
        C8.append8(c, new.float(), new, cu)
    with pytest.raises(ValueError, match="shape"):
        C8.append8(c, new, new[:, :4], cu)
    with pytest.raises(ValueError, match="shape"):
        C8.append8(c, new.transpose(1, 2), new, cu)  # head-major has to be viewed token-major
    odd = torch.zeros((2, 5, 2, 68), dtype=torch.bfloat16)[..., :64]
    with pytest.raises(ValueError, match="aligned"):
        C8.append8(c, odd, new, cu)
    with pytest.raises(ValueError, match="shape"):
        C8.decode_attention8(c, q[..., :32])
    with pytest.raises(TypeError):
        C8.evict8(c, keeps=cu[:2].long())
    with pytest.raises(ValueError, match="shape"):
        C8.evict8(c, keeps=cu)
    with pytest.raises(ValueError, match="keep"):
        C8.evict8(c)
    for kw in (dict(keep=2 ** 32 + 5), dict(keep=-1), dict(keep=5, first=2 ** 31), dict(keep=5, recent=-2 ** 32 + 9)):
        with pytest.raises(ValueError, match="number of tokens"):
            C8.evict8(c, **kw)
    with pytest.raises(ValueError, match="one of them"):
        C8.evict8(c, 5, keeps=cu[:2])
    with pytest.raises(ValueError, match="layers"):
        c.layers(1, 2)
    with pytest.raises(ValueError, match="shape"):
        C8.Cache8(2, 2, 64, [0, 100, 164], k_codes=torch.zeros((2, 2, 164, 32), dtype=torch.uint8),
                  device="cpu")
    with pytest.raises(ValueError, match="cu_rows"):
        C8.Cache8(2, 2, 64, [0], device="cpu")


def test_eviction_takes_the_whole_cache():
    """lens is shared by the layers: one layer's eviction would cut the others short."""
    c = C8.Cache8(3, 2, 64, [0, 33, 64], device="cpu")
    for view in (c.layers(0), c.layers(1, 2), c.layers(0, 3).layers(2)):
        with pytest.raises(ValueError, match="all layers"):
            C8.evict8(view, 5)
    with pytest.raises(ValueError, match="not on a GPU"):
        C8.evict8(c.layers(0, 3), 5)


def test_a_cache_without_weights():
    import torch

    c = C8.Cache8(1, 1, 64, [0, 33], weights=False, device="cpu")
    assert c.weights is None and c.positions is None and c.c.weights is None
    with pytest.raises(ValueError, match="weights"):
        C8.decode_attention8(c, torch.zeros((1, 1, 2, 64), dtype=torch.bfloat16), gather=True)
    with pytest.raises(ValueError, match="weights"):
        C8.evict8(c, 5)
    with pytest.raises(ValueError, match="weights"):
        C8.Cache8(1, 1, 64, [0, 33], weights=False, positions=torch.zeros((1, 1, 33), dtype=torch.int32),
                  device="cpu")
    pb = B.Problem(1, 1, 1, 64, 1, [0, 9], [0, 0], device="cpu", status=False)
    k = torch.zeros((1, 1, 9, 64), dtype=torch.bfloat16)
    i32 = dict(dtype=torch.int32)
    with pytest.raises(ValueError, match="weights"):
        C8.compact8(pb, c, k, k, torch.zeros(9, **i32), torch.zeros(2, **i32), weights=torch.zeros((1, 1, 9)))


def test_layers_are_views():
    c = C8.Cache8(3, 2, 64, [0, 33, 64], device="cpu")
    v = c.layers(1, 2)
    assert v.lens is c.lens and v.seen is c.seen and v.k_scales.data_ptr() == c.k_scales[1].data_ptr()
    assert v.c.num_layers == 2 and v.c.k_codes == c.c.k_codes + 2 * 64 * 64
    assert v.c.weights == c.c.weights + 4 * 2 * 64


def test_a_cache_keeps_its_own_row_offsets():
    cu = np.array([0, 100, 200], dtype=np.int32)
    c = C8.Cache8(2, 2, 64, cu, device="cpu")
    cu[:] = [0, 50, 90000]
    assert [c.c.cu_rows_host[i] for i in range(3)] == [0, 100, 200] == c.cu_rows_dev.tolist()
    with pytest.raises((ValueError, OverflowError)):
        C8.Cache8(1, 1, 64, np.array([0, 2 ** 32 + 100]), device="cpu")
