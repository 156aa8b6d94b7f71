"""The oracle of caches in 8 bits (oracle/codes.py) against worked values."""
import numpy as np
import pytest

from oracle import codes as C


def test_e4m3_values():
    v = C.E4M3
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[7] == 7 * 2.0 ** -9 and v[8] == 2.0 ** -6
    assert v[0x38] == 1.0 and v[0x3C] == 1.5 and v[0x7E] == 448.0 and v[0xFE] == -448.0
    assert np.isnan(v[0x7F]) and np.isnan(v[0xFF])
    assert (np.diff(v[:127]) > 0).all()


@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_scales(code):
    m = C.LARGEST[code]
    assert C.scale_of([0.0, -m], code) == 1.0                       # (exact: nothing to round up)
    assert C.scale_of([m * 2.0 ** 10], code) == 2.0 ** 10
    s = C.scale_of([m * 1.001], code)
    assert s == 1.0 + 2.0 ** -7                                      # the next bf16 above
    assert C.scale_of([0.0], code) > 0
    assert np.isfinite(C.scale_of([np.inf], code) * np.float32(m))
    assert C.scale_of([np.nan, 2.0 * m], code) == 2.0


def test_codes():
    b, s = C.encode([127.0, -127.0, 0.4, 0.6, 1.5, 2.5, -0.5, np.nan], "int8")
    assert s == 1.0 and b.view(np.int8).tolist() == [127, -127, 0, 1, 2, 2, 0, 0]
    b, s = C.encode([448.0, 17.0, 19.0, 18.0, -1.0, 2.0 ** -10, 3 * 2.0 ** -10, np.nan], "e4m3")
    # between 16 and 20 steps are 2: 17 is halfway, to the even 16; 19 halfway, to 20
    assert s == 1.0 and C.E4M3[b].tolist() == [448, 16, 20, 18, -1, 0, 2.0 ** -8, 0]


@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_values_are_near(code):
    x = np.random.RandomState(0).randn(16, 64).astype(np.float32)
    b, s = C.encode(x, code)
    y = C.decode(b, s, code)
    if code == "int8":
        assert np.abs(x - y).max() <= s / 2 * (1 + 2.0 ** -20)
    else:
        tol = np.maximum(np.abs(x) * 2.0 ** -4, float(s) * 2.0 ** -10) * (1 + 2.0 ** -20)
        assert (np.abs(x - y) <= tol).all()


def test_attention_of_one_token():
    v = np.array([[1.0, 2.0], [3.0, 4.0]])
    assert np.array_equal(C.attend(np.ones((1, 2)), np.zeros((1, 2)), v[:1]), v[:1])
    assert np.allclose(C.attend(np.zeros((1, 2)), v, v), v.mean(0))
