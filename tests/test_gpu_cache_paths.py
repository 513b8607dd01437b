"""Attention over the 8-bit cache where its kernels take ways of their own.  Tolerances are those of test_gpu_cache."""
import numpy as np
import pytest

from oracle import cache as C
from test_gpu_cache import K, Cache, attend, right  # noqa: F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ the largest score of a tile
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("T,page", [(1, 64), (1, 16), (20, 64), (130, 64), (130, 32)])
@pytest.mark.parametrize("dh", [16, 32, 64, 96, 128, 192, 256])
def test_largest_scores_of_the_last_columns(K, dtype, T, page, dh):  # noqa: F811
    """Every row sees whole tiles only; a tile's largest score is one token's, comes of the head's last column, which the products add last, and is 2^12 times the
    weight of the tile before: a maximum that is taken too early is too small by that."""
    c = Cache(dtype, 17, [T], [512], 1, dh, page)
    c.ks[:], c.kp[:] = 4.0, C.e4m3(c.kp * 2.0 ** -9)
    c.kp[..., dh - 1] = 0.0
    for tile in range(8):
        pos = tile * 64 + (37 * tile + 11) % 64
        c.kp[c.table[0, pos // page], 0, pos % page, dh - 1] = C.e4m3(12 * (tile + 1) * np.log(2) * np.sqrt(dh) / 4)
    c.load()
    q = c.rnd(c.rows, dh)
    q[:, dh - 1] = 1.0
    o, lse, q, _ = attend(K, c, 1, causal=0, q=q)
    right(c, 1, 0, o, lse, q)

