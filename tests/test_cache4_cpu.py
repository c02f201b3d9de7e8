"""The 4-bit cache without a GPU: the oracle of its format, the exports, the workspace sizes and
the refusals of every entry point (validation runs on the host before anything is launched; the
device pointers below are placeholders that no call follows)."""
import ctypes
import os
import re

import numpy as np
import pytest

import oracle.cache4_ref as R
from paper_2609_22158_amd import binding as B
from paper_2609_22158_amd import cache4 as C4

HEADER = os.path.join(os.path.dirname(os.path.dirname(__file__)), "include", "stepkv_cache4.h")
FAKE = 0x10000  # placeholder device address, 256-byte aligned


# ---------------------------------------------------------------- the format
def test_quantise_by_hand():
    """One group: max 7 takes e = 0 and rounds to 6; ties go to the even code; signs are kept."""
    x = np.zeros(32)
    x[:16] = [7.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, 0.26, 0.74, 6.5, -6.9, -0.0, 5.01, 4.99]
    codes, byte = R.quantise4(x)
    assert byte.tolist() == [127]
    y = R.dequantise4(codes, byte)
    assert y[:16].tolist() == [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 0.0, 0.5, 0.5, 6.0, -6.0, 0.0, 6.0, 4.0]
    assert codes[0] == 7 and codes[6] == 0x8f  # -6 in the low half, -0 in the high half


@pytest.mark.parametrize("top,byte", [(7.0, 127), (7.0 * (1 + 2 ** -7), 128), (3.5, 126), (3.6, 127),
                                      (0.0, 3), (2.0 ** -140, 3), (3.38e38, 252), (1.0, 125)])
def test_quantise_scale_byte(top, byte):
    x = np.zeros(64)
    x[40] = -top
    _, b = R.quantise4(x)
    assert b.tolist() == [3, byte]


def test_quantise_again_gives_the_same():
    """Rows read back and quantised again give the same codes and scales, over all magnitudes."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((400, 128)) * 2.0 ** rng.integers(-133, 127, (400, 4)).repeat(32, axis=1)
    x = np.clip(x, -3.38e38, 3.38e38)
    codes, byte = R.quantise4(x)
    c2, b2 = R.quantise4(R.dequantise4(codes, byte))
    # a group that rounds to zero takes the smallest scale
    zero = (R.dequantise4(codes, byte).reshape(400, 4, 32) == 0).all(axis=-1)
    assert np.array_equal(codes, c2) and np.array_equal(np.where(zero, 3, byte), b2)


def test_quantise_not_finite():
    x = np.ones((2, 64))
    x[0, 3], x[1, 40] = np.nan, -np.inf
    codes, byte = R.quantise4(x)
    assert byte.tolist() == [[255, 125], [125, 255]]
    y = R.dequantise4(codes, byte)
    assert np.isnan(y[0, :32]).all() and (y[0, 32:] == 1).all() and np.isnan(y[1, 32:]).all()


def test_rounding_error_bound():
    """Each value is off by at most half the step at its magnitude: 2^e for the top step, and the
    top of the range (6 to 7 times 2^e) by at most 2^e."""
    x = np.random.default_rng(1).standard_normal((200, 64))
    codes, byte = R.quantise4(x)
    err = np.abs(R.dequantise4(codes, byte) - x)
    assert (err <= np.repeat(2.0 ** (byte - 127.0), 32, axis=-1)).all()


def test_score_is_the_bound_of_the_group():
    rng = np.random.default_rng(2)
    k, q = rng.standard_normal((150, 64)), rng.standard_normal((7, 64))
    s = R.block_scores(q, R.block_bounds(k))
    up, down = np.maximum(q, 0).sum(axis=0), np.minimum(q, 0).sum(axis=0)
    bb = R.block_bounds(k)
    np.testing.assert_allclose(s, bb[:, 1] @ up + bb[:, 0] @ down, rtol=1e-12)
    for b in range(3):
        assert s[b] >= (k[64 * b:64 * b + 64] @ q.T).sum(axis=1).max() - 1e-9


def test_select_by_hand():
    s = np.array([0.0, 5.0, np.nan, 5.0, 1.0, -np.inf, 2.0])
    assert R.select_blocks(s, 3, 1, 1).tolist() == [0, 1, 6]
    assert R.select_blocks(s, 4, 0, 0).tolist() == [1, 3, 4, 6]
    assert R.select_blocks(s, 6, 0, 1).tolist() == [0, 1, 2, 3, 4, 6]  # NaN as -inf, lower first
    assert R.select_blocks(s, 9, 1, 1).tolist() == [0, 1, 2, 3, 4, 5, 6, -1, -1]


# ---------------------------------------------------------------- the library
@pytest.fixture(scope="module")
def lib():
    return C4.load()


def _cache(L=2, H=2, d=128, rooms=(1000, 2000), **kw):
    cu = np.concatenate([[0], np.cumsum(rooms)]).astype(np.int32)
    c = C4.Cache4C(L, H, d, len(rooms), cu.ctypes.data_as(B._i32p), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE,
                   FAKE, None)
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
    names = set(re.findall(r"\b(stepkv_cache4_[a-z_]+)\s*\(", text))
    assert names == set(C4._SIGNATURES) and len(names) == 10
    for n in names:
        assert hasattr(lib, n), n


CALLS = {
    "compact": lambda lib, c, pb=None, k=FAKE, v=FAKE, idx=FAKE, cu=FAKE: lib.stepkv_cache4_compact(
        ctypes.byref(pb or _problem()), c, k, v, idx, 0, cu, None),
    "advance": lambda lib, c, cu=FAKE: lib.stepkv_cache4_advance(c, cu, None),
    "append": lambda lib, c, k=FAKE, v=FAKE, ks=(8, 8, 8), vs=(8, 8, 8), cu=FAKE, n=4:
        lib.stepkv_cache4_append(c, k, C4._i64x3(*ks) if ks else None, v, C4._i64x3(*vs) if vs else None,
                                 cu, n, None),
    "read": lambda lib, c, cu=FAKE, n=4, k=FAKE, v=FAKE: lib.stepkv_cache4_read(c, cu, n, k, v, None),
    "decode": lambda lib, c, hq=8, q=FAKE, blocks=None, n=0, scale=0.0, out=FAKE, ws=FAKE, nb=1 << 40:
        lib.stepkv_cache4_decode(c, hq, q, blocks, n, scale, out, None, ws, nb, None),
    "select": lambda lib, c, hq=8, q=FAKE, n=4, f=1, l=1, blocks=FAKE, ws=FAKE, nb=1 << 40:
        lib.stepkv_cache4_select_blocks(c, hq, q, n, f, l, blocks, ws, nb, None),
    "sparse": lambda lib, c, hq=8, q=FAKE, n=4, f=1, l=1, scale=0.0, blocks=FAKE, out=FAKE, ws=FAKE,
        nb=1 << 40: lib.stepkv_cache4_decode_sparse(c, hq, q, n, f, l, scale, blocks, out, None, ws, nb,
                                                    None),
}


@pytest.mark.parametrize("call", list(CALLS))
@pytest.mark.parametrize("kw,code", [
    (dict(num_layers=0), B.EINVAL), (dict(num_kv_heads=0), B.EINVAL), (dict(num_seqs=0), B.EINVAL),
    (dict(head_dim=0), B.EINVAL), (dict(head_dim=96), B.EUNSUPPORTED), (dict(lens=None), B.EINVAL),
    (dict(cu_rows=None), B.EINVAL), (dict(cu_rows_host=None), B.EINVAL), (dict(k_codes=None), B.EINVAL),
    (dict(v_codes=FAKE + 8), B.EINVAL), (dict(k_scales=FAKE + 2), B.EINVAL),
    (dict(v_scales=None), B.EINVAL), (dict(k_bounds=FAKE + 8), B.EINVAL),
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
    ("compact", dict(pb=_problem(L=3)), B.EINVAL), ("compact", dict(pb=_problem(Hkv=4)), B.EINVAL),
    ("compact", dict(pb=_problem(d=64)), B.EINVAL), ("compact", dict(pb=_problem(cu=(0, 5))), B.EINVAL),
    ("compact", dict(pb=_problem(cu=(0, 9, 5))), B.EINVAL),
    ("advance", dict(cu=None), B.EINVAL),
    ("append", dict(k=None), B.EINVAL), ("append", dict(v=None), B.EINVAL),
    ("append", dict(n=-1), B.EINVAL), ("append", dict(cu=None), B.EINVAL),
    ("append", dict(ks=(8, 4, 8)), B.EINVAL), ("append", dict(vs=None), B.EINVAL),
    ("append", dict(k=FAKE + 2), B.EINVAL),
    ("read", dict(n=-1), B.EINVAL), ("read", dict(k=None, v=None), B.EINVAL),
    ("read", dict(cu=None), B.EINVAL), ("read", dict(v=FAKE + 4), B.EINVAL),
    ("decode", dict(hq=3), B.EINVAL), ("decode", dict(hq=0), B.EINVAL), ("decode", dict(q=None), B.EINVAL),
    ("decode", dict(q=FAKE + 2), B.EINVAL), ("decode", dict(out=None), B.EINVAL),
    ("decode", dict(scale=float("nan")), B.EINVAL), ("decode", dict(n=3), B.EINVAL),
    ("decode", dict(blocks=FAKE, n=0), B.EINVAL), ("decode", dict(ws=None), B.EWORKSPACE),
    ("decode", dict(ws=FAKE + 128), B.EWORKSPACE), ("decode", dict(nb=255), B.EWORKSPACE),
    ("select", dict(n=0), B.EINVAL), ("select", dict(n=3, f=2, l=2), B.EINVAL),
    ("select", dict(f=-1), B.EINVAL), ("select", dict(l=-1), B.EINVAL),
    ("select", dict(f=2 ** 31 - 1, l=2 ** 31 - 1), B.EINVAL), ("select", dict(blocks=None), B.EINVAL),
    ("select", dict(hq=5), B.EINVAL), ("select", dict(nb=255), B.EWORKSPACE),
    ("sparse", dict(n=0), B.EINVAL), ("sparse", dict(scale=float("inf")), B.EINVAL),
    ("sparse", dict(blocks=None), B.EINVAL), ("sparse", dict(out=None), B.EINVAL),
    ("sparse", dict(nb=256), B.EWORKSPACE),
])
def test_refuses_arguments(lib, call, kw, code):
    assert CALLS[call](lib, ctypes.byref(_cache()), **kw) == code


def test_refuses_rows_past_the_limit(lib):
    c = _cache(rooms=(C4.MAX_ROWS,))
    assert lib.stepkv_cache4_select_workspace_bytes(ctypes.byref(c)) > 0
    c = _cache(rooms=(C4.MAX_ROWS, 1))
    assert CALLS["advance"](lib, ctypes.byref(c)) == B.EUNSUPPORTED
    assert lib.stepkv_cache4_decode_workspace_bytes(ctypes.byref(c), 8, 0) == 0


def test_selection_needs_bounds(lib):
    c = ctypes.byref(_cache(k_bounds=None))
    assert CALLS["select"](lib, c) == B.EINVAL and CALLS["sparse"](lib, c) == B.EINVAL


def test_nothing_to_do_launches_nothing(lib):
    assert CALLS["append"](lib, ctypes.byref(_cache()), n=0, k=None, v=None) == B.OK
    assert CALLS["read"](lib, ctypes.byref(_cache()), n=0, k=None, v=None) == B.OK


def test_workspace_sizes(lib):
    c = ctypes.byref(_cache())
    dense = lib.stepkv_cache4_decode_workspace_bytes(c, 8, 0)
    keys = lib.stepkv_cache4_select_workspace_bytes(c)
    assert dense > 0 and dense % 256 == 0 and keys >= 8 * 2 * 2 * (3000 // 64 + 2)
    sparse = lib.stepkv_cache4_sparse_workspace_bytes(c, 8, 4)
    assert sparse >= keys + 256
    assert lib.stepkv_cache4_decode_workspace_bytes(c, 3, 0) == 0
    assert lib.stepkv_cache4_decode_workspace_bytes(c, 8, -1) == 0
    assert lib.stepkv_cache4_sparse_workspace_bytes(c, 8, 0) == 0
    assert lib.stepkv_cache4_select_workspace_bytes(ctypes.byref(_cache(head_dim=96))) == 0
    # short sequences need none: the smallest size says so
    assert lib.stepkv_cache4_decode_workspace_bytes(ctypes.byref(_cache(rooms=(64, 300))), 8, 0) == 256
    # a cache without room still has a workspace to pass
    assert lib.stepkv_cache4_decode_workspace_bytes(ctypes.byref(_cache(rooms=(0, 0))), 8, 0) >= 256


# ---------------------------------------------------------------- the Python layer
def test_python_refuses_before_the_library():
    import torch

    c = C4.Cache4(2, 2, 64, [0, 100, 164], device="cpu")
    assert c.num_bounds == 164 // 64 + 2 and c.k_codes.shape == (2, 2, 164, 32)
    cu = torch.zeros(3, dtype=torch.int32)
    q = torch.zeros((2, 2, 8, 64), dtype=torch.bfloat16)
    new = torch.zeros((2, 5, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="not on a GPU"):
        C4.advance4(c, cu)
    with pytest.raises(TypeError):
        C4.advance4(c, cu.long())
    with pytest.raises(ValueError, match="shape"):
        C4.advance4(c, cu[:2])
    with pytest.raises(TypeError):
        C4.append4(c, new.float(), new, cu)
    with pytest.raises(ValueError, match="shape"):
        C4.append4(c, new, new[:, :4], cu)
    with pytest.raises(ValueError, match="shape"):
        C4.append4(c, new.transpose(1, 2), new, cu)  # head-major has to be viewed token-major
    odd = torch.zeros((2, 5, 2, 68), dtype=torch.bfloat16)[..., :64]
    with pytest.raises(ValueError, match="aligned"):
        C4.append4(c, odd, new, cu)
    with pytest.raises(ValueError, match="contiguous channels"):
        C4.append4(c, torch.zeros((2, 5, 2, 128), dtype=torch.bfloat16)[..., ::2], new, cu)
    with pytest.raises(ValueError, match="shape"):
        C4.decode_attention4(c, q, blocks=torch.zeros((2, 2, 1, 4), dtype=torch.int32))
    with pytest.raises(ValueError, match="shape"):
        C4.decode_attention4(c, q[..., :32])
    with pytest.raises(ValueError, match="num_blocks"):
        C4.select_blocks4(c, q, 0)
    with pytest.raises(ValueError, match="layers"):
        c.layers(1, 2)
    with pytest.raises(ValueError, match="shape"):
        C4.Cache4(2, 2, 64, [0, 100, 164], k_codes=torch.zeros((2, 2, 164, 64), dtype=torch.uint8),
                  device="cpu")
    with pytest.raises(ValueError, match="cu_rows"):
        C4.Cache4(2, 2, 64, [0], device="cpu")


def test_layers_are_views():
    c = C4.Cache4(3, 2, 64, [0, 33, 64], device="cpu")
    v = c.layers(1, 2)
    assert v.lens is c.lens and v.k_scales.data_ptr() == c.k_scales[1].data_ptr()
    assert v.c.num_layers == 2 and v.c.k_codes == c.c.k_codes + 2 * 64 * 32
    assert C4.Cache4(1, 1, 64, [0, 0], device="cpu", k_bounds=False).c.k_bounds is None
