"""What the operands of orthogonalised momentum leave of X, in 64 bits but for their rounding: the stated figures, and that
nothing of the scheme is idle."""
import numpy as np
import pytest

from tests import muon_reference, muon_scheme

CASES = [(64, 1500), (1500, 64), (128, 128), (300, 301)]


def direction(rows, cols):
    g = np.random.default_rng(rows + cols)
    return g.standard_normal((rows, cols)) + g.standard_normal((rows, 4)) @ g.standard_normal((4, cols))


@pytest.mark.parametrize("rows,cols", CASES)
def test_errors_of_the_operands(rows, cols):
    u = direction(rows, cols)
    x = muon_reference.orthogonalise(u)
    off = lambda numbers, lost=None: np.linalg.norm(muon_scheme.orthogonalise(u, numbers, lost) - x) / np.linalg.norm(x)  # noqa: E731
    one, two = off(1), off(2)
    assert one < 1.1e-3 and two < 1e-6
    assert all(off(1, lost) > 1.7 * one for lost in muon_scheme.ONE)
    assert all(off(2, lost) > 50 * two for lost in muon_scheme.TWO)
