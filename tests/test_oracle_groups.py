"""Pins of the oracle of 4-bit groups and of the norms of the heads (CPU)."""
import numpy as np
import pytest
import torch

from oracle import cache_blocks as C
from oracle import cache_groups as G
from paper_2510_07535_amd import workloads as W


def _rng(k):
    return np.random.Generator(np.random.Philox(key=k))


def test_worked_group():
    """max 6.9 <= 7: e = 0.  Ties go to the even code: 0.25 -> 0, 0.75 -> 1, 1.25 -> 1, 1.75 -> 2, 2.5 -> 2, 3.5 -> 4, 5 -> 4."""
    x = np.zeros(32)
    x[:12] = [6.9, 0.25, 0.75, 1.25, -1.75, 2.5, 3.5, 5.0, -5.1, 0.26, -0.2, 1.0]
    codes, s = G.group_of(x, 0)
    assert s == 127
    assert G.group_values(codes, s)[:12].tolist() == [6, 0, 1, 1, -2, 2, 4, 4, -6, 0.5, 0, 1]
    assert codes[10] == 8                                # a sign is kept at zero too


@pytest.mark.parametrize("top,e", [(7.0, 0), (7.0001, 1), (3.5, -1), (3.5001, 0), (1.0, -2), (448.0, 6)])
def test_scale_is_the_least_that_holds_the_greatest(top, e):
    x = np.zeros(32)
    x[5] = -top
    assert G.group_of(x, 0)[1] == e + 127


@pytest.mark.parametrize("dtype", [0, 2])
def test_ends_zeros_and_numbers_that_are_none(dtype):
    low, high = G.ENDS[dtype]
    assert G.group_of(np.zeros(32), dtype)[1] == low + 127
    x = np.zeros(32)
    x[0] = 65504.0 if dtype == 2 else 3.38e38
    codes, s = G.group_of(x, dtype)
    assert s == high + 127 and G.group_values(codes, s)[0] == 6.0 * 2.0 ** high
    assert np.isfinite(np.float16(6.0 * 2.0 ** high) if dtype == 2 else np.float32(6.0 * 2.0 ** high))
    for bad in (np.inf, -np.inf, np.nan):
        y = np.ones(32)
        y[31] = bad
        codes, s = G.group_of(y, dtype)
        assert s == 255 and not codes.any() and np.isnan(G.group_values(codes, s)).all()


@pytest.mark.parametrize("dtype", [0, 2])
def test_no_number_is_off_by_more_than_half_a_step_and_a_group_keeps_its_numbers(dtype):
    r = _rng(1)
    for _ in range(300):
        x = r.standard_normal(32) * 2.0 ** r.integers(-10, 10)
        codes, s = G.group_of(x, dtype)
        y = G.group_values(codes, s)
        unit = 2.0 ** (s - 127)
        step = np.where(np.abs(y) >= 4 * unit, 2.0, np.where(np.abs(y) >= 2 * unit, 1.0, 0.5)) * unit     # from y to the next greater one
        assert (np.abs(x - y) <= step / 2).all()
        again = G.group_of(y, dtype)
        assert np.array_equal(G.group_values(*again), y)


def test_codes_against_torch_comparisons():
    """Every code of every boundary, by a count of the boundaries below."""
    y = np.concatenate([np.linspace(0, 7, 2801), [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]])
    for part in np.array_split(y, 120):
        x = np.zeros(32)
        x[:len(part)], x[31] = part, 7.0                 # e = 0
        codes, s = G.group_of(x, 0)
        t = torch.from_numpy(x)
        want = (t > 0.25).int() + (t >= 0.75) + (t > 1.25) + (t >= 1.75) + (t > 2.5) + (t >= 3.5) + (t > 5.0)
        assert s == 127 and np.array_equal(codes, want.numpy())


def test_rows_commit_and_layout():
    """Codes lie two a byte, the lower channel in the lower half; a commit moves rows with their scales."""
    r = _rng(2)
    strides = (2 * 16 * 64, 16 * 64, 64)
    p = G.Groups(np.zeros((3, 2, 16, 64)), np.zeros((3, 2, 16, 4)), strides, 128, 0)
    x = r.standard_normal(128)
    p.write(2, 1, 7, x)
    codes, s = G.group_of(x[32:64], 0)
    at = 2 * strides[0] + strides[1] + 7 * 64
    assert p.flat[at + 16] == codes[0] + 16 * codes[1] and p.scale[2, 1, 7, 1] == s
    q = p.copy()
    q.commit(np.array([[1, 2]]), [16], np.array([[7, -1]]), [1])      # position 16 + 7 -> 16
    assert np.array_equal(q.row(2, 1, 0), p.row(2, 1, 7)) and np.array_equal(q.row(2, 1, 7), p.row(2, 1, 7))


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype", [W.DT_BF16, W.DT_F16, W.DT_F32])
def test_norms_against_torch(pairs, dtype):
    r = _rng(3)
    x = C.store(r.standard_normal((1, 5, 3, 64)), dtype)
    gain = (1 + 0.3 * r.standard_normal(64)).astype(np.float32)
    freq = (10000.0 ** (-np.arange(16) / 16)).astype(np.float32)
    pos = np.array([[0, 3, 77, 4000, 131071]])
    q, k, v = G.normalised_rows(x, x, x, pos, freq, 32, pairs, 1.0, dtype, gain, None, 1e-5)
    t = torch.from_numpy(C.widen(x, dtype))
    y = torch.nn.functional.rms_norm(t, (64,), torch.from_numpy(gain.astype(np.float64)), float(np.float32(1e-5)))
    a = torch.from_numpy(pos[0])[:, None].double() * torch.from_numpy(freq).double()
    z = torch.view_as_complex((y[..., :32].unflatten(-1, (-1, 2)) if pairs else torch.stack([y[..., :16], y[..., 16:32]], -1)).contiguous())
    z = torch.view_as_real(z * torch.polar(torch.ones_like(a), a)[:, None])
    z = z.flatten(-2) if pairs else torch.cat([z[..., 0], z[..., 1]], -1)
    want = torch.cat([z, y[..., 32:]], -1).numpy()
    # (both sides in 64 bits: off by the storage's rounding, half a step)
    half = {W.DT_BF16: 2.0 ** -8, W.DT_F16: 2.0 ** -11, W.DT_F32: 2.0 ** -24}[dtype]
    assert (np.abs(C.widen(q, dtype) - want) <= half * np.abs(want) * 1.000001 + 1e-30 + (2.0 ** -25 if dtype == W.DT_F16 else 0)).all()
    assert np.array_equal(v, x) and not np.array_equal(k, q)
