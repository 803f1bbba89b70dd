"""Attention over the 4-bit cache where the arguments, not the sizes, are unusual."""
from __future__ import annotations

import numpy as np
import pytest

import kv4_util as ku
from paper_2607_11976_b200 import binding as lt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("max_new", [1, 3, 1000])
def test_a_wrong_max_new_only_costs_time(max_new, D):
    """Requests with more rows than any kernel was launched for are attended all the same."""
    s = ku.Step([100, 3, 700, 0], [1, 40, 100, 260], 16, 2, D, seed=1)
    out, lse = s.run(max_new=max_new)
    s.check(out, lse)
