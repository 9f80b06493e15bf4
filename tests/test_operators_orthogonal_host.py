"""Which coefficients the orthogonalised update takes, without a GPU: valid ones are seen to be so by the call's next check, which a stack of
no matrices passes and a workspace of NULL does not."""
import ctypes as C

import numpy as np
import pytest

from paper_2312_17530_b200 import binding
from paper_2312_17530_b200.build import build_library

P = 1 << 20  # a pointer that is never followed


@pytest.fixture(scope="module")
def takes():
    build_library()
    lib = binding.lib()

    def ask(*rows):
        coef = (C.c_float * (3 * len(rows)))(*[v for r in rows for v in r])
        return lib.rsdgc_orthogonalize(P, 40, 0, 0, P, 40, 0, 1, 0, 30, 40, coef, len(rows), 1e-7, P, None) == 0

    return ask


def largest(a, b, c, most=1.0):
    """max |s (a + b s^2 + c s^4)| and |b s^2 + c s^4| over [0, most], by sampling"""
    s = np.linspace(0.0, most, 200001)
    return np.abs(s * (a + b * s ** 2 + c * s ** 4)).max(), np.abs(b * s ** 2 + c * s ** 4).max()


@pytest.mark.parametrize("c", [0.0, 1e-45, -1e-45, 1e-20, -1e-20, 1e-16, -1e-16, 1e-12, 1e-8, -1e-8])
def test_a_fourth_power_next_to_nothing_changes_nothing(takes, c):
    """The largest value lies inside, where a + 3 b s^2 + 5 c s^4 is 0: at s^2 near -a / 3b, however small c is."""
    assert largest(8.5, -7.5, c)[0] > 3.4 and not takes((8.5, -7.5, c))
    assert largest(4.5, -3.5, c)[0] < 1.99 and takes((4.5, -3.5, c))


def test_what_is_taken_is_what_sampling_finds(takes):
    rng = np.random.default_rng(5)
    taken = 0
    for _ in range(3000):
        a, b, c = (float(np.float32(v)) for v in rng.normal(size=3) * rng.choice([1e-9, 1e-4, 1.0, 3.0], size=3))
        top, poly = largest(a, b, c)
        if abs(top - 2.0) < 1e-3 or poly > 7.4:
            continue  # next to a border, or beyond the other one
        ok = top < 2.0
        taken += ok
        assert takes((a, b, c)) == ok, (a, b, c, top, poly)
    assert taken > 500


# a schedule that begins steeply, each step's argument divided by 1.01 so that roundings do not grow
STEEP = tuple((a / 1.01, b / 1.01 ** 3, c / 1.01 ** 5) for a, b, c in (
    (8.2872, -23.5959, 17.3004), (4.1071, -2.9478, 0.5448), (3.9487, -2.9089, 0.5518), (3.3184, -2.4885, 0.51), (2.3007, -1.6689, 0.4188)))


def test_a_schedule_that_begins_steeply(takes):
    """Its first polynomial of A reaches 7.97, its singular values stay below 2."""
    top, poly = largest(*STEEP[0])
    assert 7.9 < poly < 8 and top < 2 and takes(*STEEP)
    for scale in (1.0, 1.9, 3.7):  # up to 29.9, where a makes up for it: s (a + b s^2 + c s^4) with a maximum next to 2
        a, b, c = 8.2 * scale, -23.6 * scale ** 3, 17.3 * scale ** 5
        top, poly = largest(a, b, c)
        assert takes((a, b, c)) == (top < 2 and poly < 30)


def test_polynomials_up_to_30(takes):
    """A first step that leaves singular values up to m (and 2^-7 more for roundings), of which the second one's b s^2 reaches 29.64 and 30.27."""
    for m, ok in ((0.1717, True), (0.1735, False)):
        top, poly = largest(29.0, -990.0, 0.0, m * (1 + 2.0 ** -7))
        assert top < 1.95 and (poly < 30) == ok and abs(poly - 30) > 0.2
        assert takes((m, 0.0, 0.0), (29.0, -990.0, 0.0)) == ok
