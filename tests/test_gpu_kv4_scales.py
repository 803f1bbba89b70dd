"""Attention over the 4-bit cache with any finite scale: what counts is scale * q . k, however large or small its factors are."""
import numpy as np
import pytest

import kv4_util as ku
from paper_2607_11976_b200 import binding as lt

pytestmark = pytest.mark.gpu

PATHS = [("bf16", lt.LT_PATH_AUTO), ("bf16", lt.LT_PATH_GENERIC), ("f32", lt.LT_PATH_AUTO)]
IDS = ["bf16", "bf16-generic", "f32"]
# scale, size of the queries: scores of order 1 from factors at either end of fp32, and scores of zero
FACTORS = [(0.0, 1e30), (0.0, 5e37), (1e-36, 1e36), (-3e-37, 1e36), (1e-39, 1e37), (2.5e38, 1e-38), (-3.4e38, 3e-39), (3.4e38, 0.0), (1e30, 1e-31)]


def _both_forms(s, path, fused):
    s.check(*s.run(path, max_new=int(s.new.max())), fused=fused)
    idx = s.selection(70)
    s.check(*s.run(path, idx), idx, fused=fused)


@pytest.mark.parametrize("dtype,path", PATHS, ids=IDS)
@pytest.mark.parametrize("scale,gain", FACTORS)
@pytest.mark.parametrize("new,Hq", [([1, 2], 8), ([30, 70], 64)], ids=str)  # few rows and many, in both forms
@pytest.mark.parametrize("D", [64, 128])
def test_scales_and_queries_at_the_ends_of_their_range(dtype, path, scale, gain, new, Hq, D):
    s = ku.Step([300, 40], new, Hq, 1, D, dtype, seed=3, pad=1, q_gain=gain)
    s.scale = float(np.float32(scale))
    _both_forms(s, path, dtype == "bf16" and path != lt.LT_PATH_GENERIC)


@pytest.mark.parametrize("dtype,path", PATHS, ids=IDS)
@pytest.mark.parametrize("new,Hq", [([1, 2], 8), ([30, 70], 64)], ids=str)
@pytest.mark.parametrize("scale", [1e37, -3.4e38])
def test_keys_of_zero_under_a_large_scale(dtype, path, new, Hq, scale):
    """All scores are zero, although scale * q is beyond fp32."""
    s = ku.Step([300, 40], new, Hq, 1, 64, dtype, seed=5, q_gain=100.0, poison=False)
    for rows in (s.pool, s.clean):
        rows[..., :32], rows[..., 64:68] = 0x88, 0  # key codes and key scales
    s.scale = float(np.float32(scale))
    _both_forms(s, path, dtype == "bf16" and path != lt.LT_PATH_GENERIC)
