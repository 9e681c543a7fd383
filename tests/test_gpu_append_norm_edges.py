"""Appending with the norms of the heads: rows with an infinite number or none on their way into caches of 4-bit groups, and heads and tokens about the numbers at
which the launch changes.  Needs an MI355X (-m gpu)."""
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


def _check_fp32(a, q):
    """Both sides work in 64 bits, in another order: they are apart by some 2^-51 of the greater of the two terms x cos, y sin whose difference is taken.  Where that
    moves a number over a tie of fp32 the two round to neighbours, one step of at most 2^-23 apart; for N numbers, terms k times greater than their
    difference, that is N 2 2^-51 k / 2^-23 of them, 0.02 k of 2.75 M, and k is some ten on average (one number of 36 times smaller than its terms lies 1.0e-15 from a tie)."""
    torch.cuda.synchronize()
    wq, wk, wv = a.want()
    pairs = [(d.cpu().numpy().reshape(w.shape), w) for d, w in zip(a.dev[:2], (wk, wv))]
    if q:
        pairs.append((a.q_out.cpu().numpy(), wq))
    for got, want in pairs:
        assert (np.abs(got.astype(np.float64) - want) <= 2.0 ** -23 * np.abs(want)).all() and np.sum(got != want) <= 4, np.sum(got != want)


@pytest.mark.parametrize("dtype,cache", [(W.DT_BF16, "own"), (W.DT_F16, "own"), (W.DT_F32, "own"), (W.DT_BF16, "groups"), (W.DT_F16, "groups")])
@pytest.mark.parametrize("Hq,Hkv,n,q", [(24, 4, 768, True), (28, 4, 768, True), (28, 4, 769, True), (24, 4, 769, True), (28, 4, 700, False), (16, 16, 5, True), (16, 16, 5, False)])
def test_heads_and_tokens_about_the_borders(dtype, cache, Hq, Hkv, n, q):
    """32 heads of 128 channels in 16 bits are one item a thread of 256 threads, 36 are more; without queries fewer."""
    a = Rows(n + Hq, dtype=dtype, cache=cache, norm=True, Hq=Hq, Hkv=Hkv, D=128, ctx=[5], n=n, rot_dim=128)
    a.run(q=q)
    if dtype == W.DT_F32:
        _check_fp32(a, q)
    else:
        a.check(q=q)
    assert int(a.status.item()) == 0
