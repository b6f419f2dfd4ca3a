"""The oracle of the 4-bit rows and of the tokens that enter a cache, against values worked out by hand."""
import numpy as np
import pytest

from oracle import kv4 as OK


def _row(values):
    x = np.zeros(128, np.float32)
    x[:len(values)] = values
    return x


def test_codes_of_a_block_by_hand():
    # largest 6: unit 1; ties (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5) go to the even code
    x = _row([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.26, -6])
    codes, scale = OK.quantize_rows(x)
    assert scale.tolist() == [127, 2, 2, 2]
    assert [int(c) for b in codes[:5] for c in (b & 15, b >> 4)] == [7, 0, 2, 2, 4, 4, 6, 6, 9, 15]
    assert OK.dequantize_rows(codes, scale)[:10].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, -0.5, -6]


@pytest.mark.parametrize("top,byte", [(6.0, 127), (6.0001, 128), (3.0, 126), (3.0001, 127), (0.0, 2), (1e-45, 2), (2.0 ** 126, 251),
                                      (1.7e38, 252), (2.0 ** 127, 255), (np.inf, 255), (np.nan, 255)])
def test_scale_bytes(top, byte):
    codes, scale = OK.quantize_rows(_row([top]))
    assert scale[0] == byte and scale[1:].tolist() == [2, 2, 2]
    back = OK.dequantize_rows(codes, scale)
    assert np.isnan(back[:32]).all() if byte == 255 else np.isfinite(back).all()


def test_rounding_is_at_most_half_a_step():
    x = np.random.default_rng(1).standard_normal((50, 128)).astype(np.float32)
    codes, scale = OK.quantize_rows(x)
    back, unit = OK.dequantize_rows(codes, scale), np.repeat(2.0 ** (scale.astype(float) - 127), 32, axis=-1)
    y = np.abs(x) / unit
    assert (y <= 6).all()
    assert (np.abs(back - x) / unit <= np.where(y <= 2, 0.25, np.where(y <= 4, 0.5, 1.0))).all()
    again = OK.quantize_rows(back)
    assert np.array_equal(OK.dequantize_rows(*again), back)          # what fits stays


def test_rotation_and_norm_by_hand():
    x = np.zeros((1, 1, 128))
    x[0, 0, 0], x[0, 0, 64], x[0, 0, 100] = 3.0, 4.0, 2.0
    f = np.zeros(64)
    f[0] = np.pi / 2
    out, _ = OK.head_rows(x, [1], inv_freq=f)
    assert np.allclose(out[0, 0, [0, 64, 100]], [-4, 3, 2])
    x[0, 0, 1] = 5.0
    out, _ = OK.head_rows(x, [1], inv_freq=f[:8], interleaved=True)
    assert np.allclose(out[0, 0, [0, 1, 64, 100]], [-5, 3, 4, 2])
    out, _ = OK.head_rows(x, [0], weight=np.full(128, 2.0), eps=0.0)
    assert np.allclose((out / 2) ** 2 @ np.ones(128), 128) and out[0, 0, 64] == 2 * 4 / np.sqrt(54 / 128)
