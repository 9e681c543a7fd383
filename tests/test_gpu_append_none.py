"""Rows with an infinite number or none on their way into caches of 4-bit groups: which scale bytes say so, with and without the norms of the heads.  Needs
an MI355X (-m gpu)."""
import numpy as np
import pytest
import torch

from oracle import cache_blocks as C
from oracle import cache_groups as G
from paper_2510_07535_amd import workloads as W
from test_gpu_append_norm import Rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("pairs", [False, True])
def test_which_groups_are_none(dtype, norm, pairs):
    """By the formula.  V: the group that has it.  K without the norm: that of its channel, and of the one that it is turned with.  With the norm: an infinite
    number makes the root mean square infinite, itself none, and all others zeros; one that is none makes all of the row none."""
    def rows(x):
        w = C.widen(x, dtype)
        w[0, 0, :, 40] = np.inf
        w[0, 1, :, 100] = np.nan
        w[0, 2, :, 0] = -np.inf
        w[0, 3, :, 70] = np.inf                          # not turned
        return C.store(w, dtype)
    a = Rows(7, dtype=dtype, cache="groups", norm=norm, Hq=2, Hkv=2, D=128, ctx=[13], n=5, rot_dim=64, pairs=pairs, rows=rows)
    a.run()
    torch.cuda.synchronize()
    least = G.ENDS[dtype][0] + 127
    turned = {0, 1} if not pairs else None               # channels 8 and 40, 0 and 32
    none = [turned or {1}, {3}, turned or {0}, {2}, set()]
    for i in range(5):
        page, slot = int(a.table[0, (13 + i) // 16]), (13 + i) % 16
        k, v = (s.cpu().numpy()[page, :, slot] for s in a.dev[2:])
        want = set(range(4)) if norm and i == 1 else none[i]
        for h in range(2):
            assert {g for g in range(4) if k[h, g] == 255} == want, (i, h)
            assert {g for g in range(4) if v[h, g] == 255} == [{1}, {3}, {0}, {2}, set()][i], (i, h)
            if norm and i in (0, 2, 3):
                assert all(k[h, g] == least for g in range(4) if g not in want), (i, h)
    a.check()
