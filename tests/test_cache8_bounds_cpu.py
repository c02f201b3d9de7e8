"""How far an element of the 8-bit cache may be off, as include/stepkv_cache8.h states it, on the
oracle (to which the kernels are equal bit for bit).

The bound: an element x, |x| <= 464 * 2^119, is held within max(2^-4 |x|, 2^-9 * 2^E), E the greatest
exponent of the blocks that held it. By arithmetic: a rounding to a grid changes a number only if the grid is
coarser at that number than every grid it was rounded to before (e4m3 numbers times a power of two lie
on the grid of every other power that is finer there: three bits after the leading one). So the half
steps of the roundings that change it are distinct powers of two, and add up to less than twice the last
one. In the normal range (2^-6 * 2^e and above) all grids are the same, so one rounding changes a
number there: by at most 2^-4 of it. A last one below that range has the half step 2^-10 * 2^e, e <= E."""
import numpy as np
import pytest

import oracle.cache8_ref as R

D = 64


def bound(x, E):
    return np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** (E - 9.0))


def exponents(head, which):
    """Of the blocks of the head's tokens."""
    return np.repeat(np.array(head.exp[which], np.float64), R.BLOCK)[:len(head)]


def test_a_moved_row_keeps_the_error_of_its_old_block():
    """Rows of 2.4 beside one of 448 * 2^10 are held as 2, and stay so in a block of exponent -7, where rows
    that were written into it are off by a sixteenth at most."""
    x = np.full((130, D), 2.4)
    x[64] = 448 * 2.0 ** 10
    a = R.Head8(D)
    a.append(x, x, np.arange(130), weights=np.where(np.arange(130) < 60, 0.0, 1.0) - (np.arange(130) == 64))
    a.evict(66, 0, 0, 130)
    assert 64 not in a.positions and a.exp[0] == [-7, 10]
    own = exponents(a, 0)[:, None]
    moved = a.positions >= 64
    src = x[a.positions]
    err = np.abs(a.values(0) - src)
    assert (err[~moved] <= bound(src, own)[~moved]).all()
    assert (err[moved & (own[:, 0] == -7)] > 2.6 * bound(src, own)[moved & (own[:, 0] == -7)]).all()
    assert (err <= bound(src, np.where(moved, 10.0, own[:, 0])[:, None])).all()


def test_values_past_the_greatest_scale():
    """The greatest bf16 value is held as 448 * 2^119; up to 464 * 2^119 the bound of 2^-4 holds."""
    top = 255 * 2.0 ** 120
    for x, held in ((top, 448), (464 * 2.0 ** 119, 448), (448 * 2.0 ** 119, 448), (440 * 2.0 ** 119, 448),
                    (430 * 2.0 ** 119, 416)):
        a = R.Head8(D)
        a.append(np.full((1, D), x), np.full((1, D), -x), np.zeros(1))
        assert a.exp == [[119], [119]]
        assert (a.values(0) == held * 2.0 ** 119).all() and (a.values(1) == -held * 2.0 ** 119).all()
        err = abs(a.values(0)[0, 0] - x) / x
        assert 0.1215 < err < 0.1216 if x == top else err <= 2.0 ** -4


@pytest.mark.parametrize("seed", range(8))
def test_the_bound_over_appends_and_evictions(seed):
    """Steps of appending and evicting rows of many magnitudes, in blocks that grow, are left and entered."""
    rng = np.random.default_rng(seed)
    a, came = R.Head8(D), 0
    xs = [np.zeros((0, D)), np.zeros((0, D))]
    E = [np.zeros(0), np.zeros(0)]  # by position: the greatest exponent of the blocks that held it

    def look():
        for which in (0, 1):
            E[which][a.positions] = np.maximum(E[which][a.positions], exponents(a, which))
            x = xs[which][a.positions]
            assert (np.abs(a.values(which) - x) <= bound(x, E[which][a.positions][:, None])).all(), which

    for step in range(12):
        n = int(rng.choice([1, 2, 17, 64, 100]))
        for which in (0, 1):
            x = rng.standard_normal((n, D)) * 2.0 ** rng.integers(-14, 15, (n, 1))
            x[rng.random(n) < 0.05] *= 2.0 ** 12
            xs[which] = np.concatenate([xs[which], x.astype(np.float32).astype(np.float64)])
            E[which] = np.concatenate([E[which], np.full(n, -200.0)])
        a.append(xs[0][came:], xs[1][came:], np.arange(came, came + n), weights=rng.random(n))
        came += n
        look()
        a.evict(max(1, int(len(a) * rng.choice([0.4, 0.9, 1.0]))), 2, 3, came)
        look()
