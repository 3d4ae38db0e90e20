"""Distillation operators, what needs no GPU: the plain forms where a row has no term or no softmax."""
import numpy as np
import pytest

import distill_ref as ref


@pytest.mark.parametrize("tail_rest", [False, True])
@pytest.mark.parametrize("bad", [0.0, np.nan, np.inf, "masked"])
def test_plain_rows_without_a_term_are_zero(bad, tail_rest):
    s = np.linspace(-1.0, 2.0, 11)
    s[4] = -3.0 if bad == "masked" else s[4] + bad
    if bad == "masked":
        s[:] = -np.inf
    idx, val = np.array([1, 4]), np.array([0.0, -1.0])
    for n, soft, label in ((0, 1.0, -100), (0, 1.0, 11), (0, 1.0, None), (2, 0.0, -100)):
        loss, g, _, _ = ref.student_row(s, n, idx[:n], val[:n], 0.5, 2.0, soft, 0.3, tail_rest, label, 0.7)
        assert loss == 0.0 and np.array_equal(g, np.zeros(11)), (n, soft, label)
