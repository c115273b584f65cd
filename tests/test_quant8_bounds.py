"""What the kernel of 8-bit codes counts on for a quotient 127 u / max, by reading the sources: how far the fp32 arithmetic may be off."""
import re
from fractions import Fraction

from test_bounded_waits import body, source


def power(text):
    return Fraction(2) ** int(re.fullmatch(r"0x1p([+-]?\d+)f?", text).group(1))


def test_roundings_of_a_quotient():
    """Rows whose maximum is between the borders go by fp32: a unit of the reciprocal (rcp.approx is off by one at most; below 2^-126 units do not
    get smaller, so they are a larger part of it) and three roundings have to stay within what the doubt about a code allows."""
    kernel = body(source("perq_quant8.cuh"), "quant8_kernel(const")
    bits = r"__float_as_uint\((%s)\)"
    lowest, highest = bits % r"0x1p-\d+f", bits % r"0x1p\d+f"
    ordinary = re.search(r"const bool odd = __float_as_uint\(all\) - \(%s \+ 1u\) >= %s - %s;" % (lowest, highest, lowest), kernel)
    assert ordinary, "no upper border"
    low, high = power(ordinary.group(1)), power(ordinary.group(2))
    assert ordinary.group(3) == ordinary.group(1)
    allowed = Fraction(re.search(r"p\.doubt = \(float\)\(1\.001 \* \(2\.0 \* e \+ (\d+)\.0 \* 0x1p-24\)\);", source("perq_matmul.cu")).group(1)) / 2 ** 24
    unit, half = Fraction(1, 2 ** 149), Fraction(1, 2 ** 24)
    for e in range(-133, 128):
        for m in (Fraction(1), Fraction(255, 256) * 2):             # the ends of a binade of bf16 values (sums lie between)
            top = m * Fraction(2) ** e
            if not low < top <= high:
                continue
            r = 1 / top
            k = -e if r >= Fraction(2) ** -e else -e - 1            # of the reciprocal's binade
            off = max(unit, Fraction(2) ** (k - 23)) / r
            assert (1 + off) * (1 + half) ** 3 - 1 <= allowed, "maximum %s 2^%d" % (float(m), e)
            # 127 times the reciprocal is finite and normal
            assert Fraction(2) ** -126 <= 127 * r < Fraction(2) ** 128
