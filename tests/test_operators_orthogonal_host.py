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
        if abs(top * (1 + 2.0 ** -7) - 2.0) < 1e-3 or poly > 7.4:
            continue  # next to a border, or beyond the other one
        ok = top * (1 + 2.0 ** -7) < 2.0
        taken += ok
        assert takes((a, b, c)) == ok, (a, b, c, top, poly)
    assert taken > 500
