"""The microscaled 4-bit oracle against hand-worked values and its own definition (CPU)."""
import numpy as np

from oracle import mx4_oracle as mx


def test_worked_block():
    x = np.zeros((1, 32))
    # largest magnitude 7 -> floor(log2) = 2, e = 0: the values are on the grid's own scale
    x[0, :12] = [7.0, 5.0, -5.1, 2.5, 3.5, 0.25, 0.26, -0.25, 0.75, 1.25, 1.75, -6.0]
    code, scale = mx.quantize(x)
    assert scale[0, 0] == 127
    assert mx.values(code, scale)[0, :12].tolist() == [6.0, 4.0, -6.0, 2.0, 4.0, 0.0, 0.5, -0.0, 1.0, 1.0, 2.0, -6.0]
    assert code[0, 7] == 8                                   # the sign of a value that rounds to zero is kept


def test_scale_bytes():
    x = np.zeros((6, 32))
    x[1, 3] = 2.0 ** -140                                    # below the smallest unit: clamped
    x[2, 0] = 1.0
    x[3, 31] = np.finfo(np.float32).max
    x[4, 5] = np.inf
    x[5, 9] = np.nan
    code, scale = mx.quantize(x)
    assert scale[:, 0].tolist() == [0, 0, 125, 252, 255, 255]
    assert np.isnan(mx.values(code, scale)[4:]).all() and not mx.values(code, scale)[:2].any()
    assert mx.values(code, scale)[2, 0] == 1.0


def test_layouts_are_inverse():
    rng = np.random.default_rng(0)
    code = rng.integers(0, 16, (5, 320), dtype=np.uint8)
    scale = rng.integers(0, 256, (5, 10), dtype=np.uint8)
    assert np.array_equal(mx.unpack(mx.pack(code)), code)
    p = mx.panels(scale)
    assert p.shape == (2, 5, 8) and not p[1, :, 2:].any()
    assert np.array_equal(mx.unpanels(p, 320), scale)
    assert p[1, 3, 1] == scale[3, 9]
