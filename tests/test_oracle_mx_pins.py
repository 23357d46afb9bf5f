"""Pins of ``oracle.mx``: the scale against a search, the elements against every representable value, blocks
written by hand, bytes there and back, the weight gradient against differences."""
import numpy as np
import pytest

from oracle import mx

FMTS = ["int8", "fp4"]
TABLE = {"int8": np.arange(-127, 128) / 64.0, "fp4": np.concatenate((-mx.GRID[:0:-1], mx.GRID))}


def samples(rng, n):
    """fp32 blocks over the whole range: ordinary, tiny, huge, at the borders of a scale and of an element."""
    x = rng.standard_normal((n, 32)) * np.exp2(rng.integers(-140, 126, (n, 1)))
    for i, m in enumerate((127.5 / 128, 127.4999 / 128, 0.875, 0.8749, 0.9999, 0.5, 0.75)):
        x[i::11, 0] = np.ldexp(m, rng.integers(-120, 127, len(x[i::11])))
        x[i::11, 1:] = x[i::11, :1] * rng.integers(-256, 257, (len(x[i::11]), 31)) / 256
    with np.errstate(over="ignore"):
        x = x.astype(np.float32).astype(np.float64)
    return np.where(np.isfinite(x), x, 1.0)


@pytest.mark.parametrize("fmt", FMTS)
def test_elements_are_the_nearest_and_the_scale_the_smallest(fmt):
    x = samples(np.random.default_rng(1), 400)
    code, s = mx.quantize(x, fmt)
    v = mx.values(code, s, 32, fmt)
    for r in range(len(x)):
        scale = 2.0 ** (int(s[r, 0]) - 127)
        most = np.abs(TABLE[fmt]).max()
        near = np.abs(TABLE[fmt][None] * scale - x[r][:, None]).min(axis=1)
        assert (np.abs(v[r] - x[r]) <= near).all()                     # exact: powers of two
        top = np.abs(x[r]).max() / scale
        step = 1 / 64 if fmt == "int8" else 2.0                        # past the largest element
        assert top < most + step / 2 or s[r, 0] == mx.TOP_SCALE[fmt]
        if s[r, 0] > 0:                                                # half the scale would round past it
            assert 2 * top >= most + step / 2


@pytest.mark.parametrize("fmt,block,s,values", [
    ("int8", [1.0, -1.0, 0.5, 1 / 128, 3 / 128, 1.984375, 0.0], 127, [1.0, -1.0, 0.5, 0.0, 2 / 64, 127 / 64, 0.0]),
    ("int8", [1.9921875, 1 / 64, 3 / 64], 128, [2.0, 0.0, 4 / 64]),    # 127.5 / 64: the next scale, steps of 2 / 64
    ("int8", [0.0, -0.0], 0, [0.0, 0.0]),
    ("int8", [2.0 ** -149], 0, [0.0]),
    ("int8", [2.0 ** -127, 2.0 ** -133, 2.0 ** -134], 0, [2.0 ** -127, 2.0 ** -133, 0.0]),
    ("int8", [3.4028234663852886e38], 254, [127 / 64 * 2.0 ** 127]),
    ("fp4", [6.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -0.25, -5.5, 6.99], 127,
     [6.0, 4.0, 4.0, 2.0, 2.0, 1.0, 1.0, 0.0, 0.0, -6.0, 6.0]),
    ("fp4", [7.0, 1.0, 0.5], 128, [8.0, 1.0, 0.0]),
    ("fp4", [0.0], 0, [0.0]),
    ("fp4", [3.4028234663852886e38], 252, [6.0 * 2.0 ** 125]),
])
def test_blocks_by_hand(fmt, block, s, values):
    code, sc = mx.quantize(np.array([block]), fmt)
    assert sc[0, 0] == s
    assert np.array_equal(mx.values(code, sc, len(block), fmt)[0], values)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_what_is_not_finite_makes_its_block_nan(fmt, bad):
    x = np.ones((2, 70))
    x[0, 33] = bad
    code, s = mx.quantize(x, fmt)
    v = mx.values(code, s, 70, fmt)
    assert np.isnan(v[0, 32:64]).all() and (v[0, :32] == 1).all() and (v[0, 64:] == 1).all() and (v[1] == 1).all()
    assert s[0, 1] == 255 and (code[0, 32:64] == 0).all()


@pytest.mark.parametrize("fmt", FMTS)
def test_bytes_there_and_back(fmt):
    x = np.random.default_rng(2).standard_normal((5, 70))
    code, s = mx.quantize(x, fmt)
    assert code.shape == (5, 96) and s.shape == (5, 3) and (code[:, 70:] == 0).all()
    Q = mx.to_bytes(code, fmt)
    assert Q.shape == (5, 96 if fmt == "int8" else 48)
    assert np.array_equal(mx.from_bytes(Q, fmt), code)
    # once held, a row is held as it is
    again, s2 = mx.quantize(mx.values(code, s, 70, fmt), fmt)
    assert np.array_equal(mx.values(again, s2, 70, fmt), mx.values(code, s, 70, fmt))


def test_every_value_is_exact_in_bf16():
    code = np.arange(-127, 128)[None]
    for s in (0, 1, 5, 6, 7, 127, 254):
        v = np.concatenate((code[0] / 64.0, mx.GRID)) * 2.0 ** (min(s, 252) - 127)
        bits = v.astype(np.float32).view(np.uint32)
        assert np.array_equal(v.astype(np.float32).astype(np.float64), v) and (bits & 0xFFFF == 0).all()


def test_gather_and_average():
    x = np.arange(6.0).reshape(3, 2)
    assert np.array_equal(mx.gather(x, [2, -1, 0, 2]), [[4, 5], [0, 0], [0, 1], [4, 5]])
    assert np.isnan(mx.gather(x, [3])).all()
    assert np.array_equal(mx.average(np.array([4.0]), np.array([8.0]), 0.75), [5.0])


def test_weight_gradient_against_differences():
    rng = np.random.default_rng(3)
    v, J, H, W = rng.standard_normal((7, 4)), rng.standard_normal((7, 3)), rng.standard_normal((7, 3)), rng.standard_normal((4, 3))
    f = lambda W: ((v @ W) * np.where(H > 0, J, 0.0)).sum()
    G = mx.wgrad(v, J, H)
    for at in np.ndindex(4, 3):
        e = np.zeros((4, 3))
        e[at] = 1e-3
        assert abs((f(W + e) - f(W - e)) / 2e-3 - G[at]) <= 1e-9
    assert np.array_equal(mx.product(v, v[:3], True), np.maximum(v @ v[:3].T, 0))
