"""The two 8-bit parts that bf16 activations of many rows are taken apart into: what include/lora_mx.h says of their sum, on every bf16 value and
largest values of a block all over the range that a scale has, from the kernel's steps in numpy."""
import os
import re

import numpy as np

from oracle import mx_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def e4m3(x):
    """Nearest value of the format, ties to even (|x| <= 448)."""
    a = np.abs(x)
    step = np.exp2(np.maximum(np.floor(np.log2(np.where(a > 0, a, 1.0))), -6) - 3)
    v = np.rint(x / step) * step
    assert (np.abs(v) <= 448).all()
    return v


def test_the_helper_is_the_format():
    x = np.random.default_rng(0).uniform(-448, 448, (40, 32)) * np.exp2(np.random.default_rng(1).integers(-14, 1, (40, 32)))
    x[:, 0] = 448.0  # (scale 1)
    codes, scales = ref.quantize(x, "e4m3")
    assert (scales == 127).all() and np.array_equal(ref.dequantize(codes, scales, "e4m3"), e4m3(x))


def parts(x):
    """(first, second) of values whose block has the scale 1: the second part's scale is 2^-4."""
    hi = e4m3(x)
    return hi, e4m3((x - hi) * 16) / 16


# every bf16 magnitude from 2^-20 to 448, where the largest of a block with scale 1 may be anything above 224
VALUES = np.array([(1 + m / 128) * 2.0 ** e for e in range(-20, 9) for m in range(128)])
VALUES = VALUES[VALUES <= 448]


def test_the_sum_of_the_parts():
    hi, lo = parts(VALUES)
    err = np.abs(hi + lo - VALUES)
    assert (err[VALUES >= 2.0 ** -6] == 0).all() and err[VALUES < 2.0 ** -6].max() == 2.0 ** -14
    # in terms of a block's largest value, just above 224 at the least
    for largest in (225.0, 226.0, 255.0, 256.0, 300.0, 448.0):
        mine = VALUES <= largest
        assert (err[mine & (VALUES >= 2.0 ** -13 * largest)] == 0).all()
        assert (err[mine] <= 2.0 ** -21 * largest).all()
    assert err.max() > 2.0 ** -22 * 225 and (err[VALUES >= 2.0 ** -14 * 225] > 0).any()  # (nothing tighter in powers of two holds)


def test_the_header_says_so():
    text = " ".join(open(os.path.join(ROOT, "include", "lora_mx.h")).read().replace("*", " ").split())
    said = re.search(r"exactly down to 2\^-(\d+) of the largest value of their block of 32, off by at most 2\^-(\d+) of it below", text)
    assert said and (int(said[1]), int(said[2])) == (13, 21)
