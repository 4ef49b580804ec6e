"""The check of codes itself, on the CPU: it takes right codes and no others."""
import numpy as np
import pytest

from tests.row_codes import off_from_definition


@pytest.fixture(params=(False, True))
def rows(request):
    rng = np.random.default_rng(3)
    y = rng.standard_normal((6, 512))
    y[4] = 0
    y[5] = np.sign(y[5])
    u = (2 * rng.integers(0, 65536, y.shape) + 1 - 65536) / 65536 if request.param else np.zeros(y.shape)
    most = np.abs(y).max(axis=1)
    most[most == 0] = 1
    q = np.rint(np.clip(127 * y / most[:, None] + u / 2, -127, 127))
    q[4] = 0
    return q, y, np.abs(y).max(axis=1), u


def test_right_codes_are_taken(rows):
    q, y, total, u = rows
    assert np.all(off_from_definition(q, y, total, u, 0) <= 0)


@pytest.mark.parametrize("wrong", (lambda q: np.full_like(q, -127), lambda q: np.where(np.abs(q) == 127, -q, q), lambda q: np.clip(np.rint(q * 1.02), -127, 127),
                                   lambda q: np.where(q == 127, 126, q), lambda q: np.concatenate([q[:, :-1], np.full((6, 1), 127)], axis=1)))
def test_wrong_codes_are_found_where_they_saturate_too(rows, wrong):
    q, y, total, u = rows
    w = wrong(q)
    w[4] = 0
    bad = off_from_definition(w, y, total, u, 0) > 0
    assert bad.any() and np.array_equal(bad.any(axis=1)[:5], (w != q).any(axis=1)[:5])
