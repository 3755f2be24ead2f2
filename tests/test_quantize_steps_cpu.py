"""The steps that hb_quantize_rows takes to an integer, fp32 operation by operation: for every largest value of a binade and every value of ten binades up to it, the integer is that of
the exact quotient, and the computed quotient is within 2^(e - 22) of it."""
import numpy as np

F = np.float32


def nearest(t):
    """A longdouble value rounded to fp32 both ways where it lies between two values, so that what a longdouble has lost below its 64 bits makes no difference."""
    r = t.astype(F)
    other = np.where(r.astype(np.longdouble) > t, np.nextafter(r, F(-np.inf)), np.nextafter(r, F(np.inf)))
    middle = (r.astype(np.longdouble) + other.astype(np.longdouble)) / 2
    return r, np.where(middle == t, other, r)


def test_integers_are_those_of_the_exact_quotients():
    assert np.finfo(np.longdouble).nmant >= 63                                # x86: products of two fp32 values are exact in it
    for top in range(1024, 2048):
        inverse = F(1.0) / F(top)                                             # correctly rounded, as the kernel's
        for shift in range(10):                                               # values `shift` binades below, as whole numbers over 2^shift
            x = np.arange(1024, 2048, dtype=np.int64)
            x = x[x <= top << shift]
            t = (127.0 * x / 2.0 ** shift).astype(F)                          # exact: 18 bits
            q = t * inverse
            rest = (t.astype(np.float64) - q.astype(np.float64) * float(top)).astype(F)          # exact in fp64 (35 bits), rounded once: fmaf(-q, top, t)
            exact = rest.astype(np.longdouble) * np.longdouble(inverse) + q.astype(np.longdouble)
            whole, left = np.divmod(127 * x, top << shift)
            want = whole + ((2 * left > top << shift) | ((2 * left == top << shift) & (whole % 2 == 1)))
            quotient = (127 * x).astype(np.longdouble) / np.longdouble(top << shift)
            binade = 2.0 ** np.floor(np.log2(quotient.astype(np.float64)))
            for r in nearest(exact):
                assert np.array_equal(np.rint(r).astype(np.int64), want), (top, shift)
                assert (np.abs(r.astype(np.longdouble) - quotient) <= binade * 2.0 ** -22).all(), (top, shift)
                half = 2 * left == top << shift
                assert np.array_equal(r[half].astype(np.float64), whole[half] + 0.5), (top, shift)
            assert want.max() <= 127


def test_quotients_are_a_half_or_well_away_from_one():
    """For all largest values: at least 2^(e - 20) away, 2^e the quotient's binade (below a quarter nothing rounds up)."""
    x = np.arange(1024, 2048, dtype=np.int64)
    for top in range(1024, 2048):
        for shift in range(10):
            den = top << shift
            away = np.abs(2 * 127 * x - (2 * (127 * x // den) + 1) * den) / (2.0 * den)
            quotient = 127 * x / den
            keep = (quotient >= 0.25) & (quotient <= 127.0)
            assert ((away == 0) | (away >= 2.0 ** (np.floor(np.log2(quotient)) - 20)))[keep].all(), (top, shift)
