"""Pins of the MX4 and norm oracle: values worked out by hand from the definitions."""
import numpy as np
import pytest

from oracle import mx_oracle as ref
from oracle import oracle as codes_ref


def _block(*v):
    x = np.zeros((1, 32))
    x[0, :len(v)] = v
    return x


@pytest.mark.parametrize("v,byte,codes", [
    # max 6: floor(log2) - 2 = 0; every magnitude of the format
    ((6, 4, 3, 2, 1.5, 1, 0.5, 0), 127, (7, 6, 5, 4, 3, 2, 1, 0)),
    # ties go to the even code, negatives alike
    ((4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -5, -0.25, -0.75), 127, (6, 0, 2, 2, 4, 4, 6, 14, 8, 10)),
    # between 6 and 8 (the next power of two) everything is 6
    ((7.9, 5.01, -7), 127, (7, 7, 15)),
    # the maximum's power of two sets the scale
    ((8, 1, 2), 128, (6, 1, 2)),
    ((0.75, 0.0625), 124, (7, 1)),
    # zeros: the smallest scale; a negative zero keeps its sign
    ((0, -0.0), 0, (0, 8)),
    # the smallest fp32 numbers: the exponent stops at -127
    ((2.0 ** -126, 2.0 ** -127, 2.0 ** -149), 0, (4, 2, 0)),
    ((2.0 ** -124, ), 1, (6, )),
    # no value of the format for these
    ((1, np.inf), 255, (0, 0)), ((np.nan, 2), 255, (0, 0))])
def test_quantize_by_hand(v, byte, codes):
    c, s = ref.quantize(_block(*v))
    assert s[0, 0] == byte
    assert tuple(c[0, :len(codes)]) == codes


def test_values_and_short_last_block():
    x = np.concatenate([np.full(32, 3.0), [0.5, -6.0, 100.0]])[None]
    c, s = ref.quantize(x)
    assert s.shape == (1, 2) and s[0].tolist() == [126, 131]  # 3 = 1.5 * 2; 100 = 1.56 * 64
    v = ref.values(c, s)
    assert v[0, :32].tolist() == [3.0] * 32 and v[0, 32:].tolist() == [0.0, -8.0, 96.0]
    assert np.isnan(ref.values(np.zeros((1, 3), np.uint8), np.array([[255]], np.uint8))).all()


def test_operand_places():
    c = np.zeros((17, 300), dtype=np.uint8)
    c[16, 256 + 33] = 5  # group 1, step 1, block 1, element 1
    s = np.zeros((17, 10), dtype=np.uint8)
    s[16, 9] = 77
    buf, written = ref.operand(c, s)
    assert buf.size == 2 * 2 * 2176 and written.sum() == 17 * 2 * (128 + 8)
    at = ((1 * 2 + 1) * 8 + 1) * 256
    assert buf[at] == 5 << 4 and buf[2 * 2 * 2048 + (1 * 2 + 1) * 128 + 64] == 77
    assert np.count_nonzero(buf) == 2


def test_bf16_rounding():
    one = np.float32(1)
    assert ref.to_bf16(one + 2.0 ** -8) == 1 and ref.to_bf16(one + 3 * 2.0 ** -8) == 1 + 2.0 ** -6
    assert ref.to_bf16(np.float32(one + 2.0 ** -8 + 2.0 ** -20)) == 1 + 2.0 ** -7


def test_norm_by_hand():
    # h = (3, 4): mean square 12.5; eps 3.5 makes 16, f = 1/4
    h, y = ref.norm(np.array([[3.0, 4.0]]), None, np.array([2.0, -1.0]), 3.5, "fp16")
    assert h.tolist() == [[3.0, 4.0]] and y.tolist() == [[1.5, -1.0]]
    h, y = ref.norm(np.array([[1.0, 4.0]]), np.array([[2.0, 0.0]]), None, 3.5, "bf16")
    assert h.tolist() == [[3.0, 4.0]] and y.tolist() == [[0.75, 1.0]]
    # the sum is rounded to the type: 2048 + 1 stays 2048 in fp16
    assert ref.norm(np.array([[2048.0]]), np.array([[1.0]]), None, 1.0, "fp16")[0][0, 0] == 2048.0


@pytest.mark.parametrize("q", [1, 2, 3, 4, 5, 6, 7, 8])
def test_codes_equal_the_fp16_quantizer(q):
    g = np.random.default_rng(q)
    x = (g.standard_normal((40, 97)) * np.exp(3 * g.standard_normal((40, 1)))).astype(np.float16)
    x[3] = 0
    x[4] = 2.0 ** -24  # a scale that rounds to a subnormal or to 0
    x[5, 1:] = 0
    c, s = ref.codes(x.astype(np.float64), q)
    want_c, want_s = codes_ref.quantize_fp16(x, q)
    assert np.array_equal(c, want_c) and np.array_equal(s, want_s.astype(np.float64))


def test_codes_of_rows_without_a_scale():
    y = np.ones((3, 5))
    y[0, 2], y[1, 0], y[2, 4] = np.nan, -np.inf, 1e9
    c, s = ref.codes(y, 4)
    assert np.isnan(s).all() and not c.any()
