"""The oracles of the cache rows and of the log probabilities against independent statements of the same things (no GPU)."""
import numpy as np
import pytest
import torch

from oracle import cache_blocks as C
from oracle import logprobs as P


def _rng(k):
    return np.random.Generator(np.random.Philox(key=k))


def test_e4m3_is_the_format_that_torch_has():
    raw = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(raw).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(C.e4m3_values(raw), want, equal_nan=True)
    mid = (C.GRID[1:127] + C.GRID[:126]) / 2
    x = np.concatenate([mid, -mid, np.nextafter(mid, 1e9), np.nextafter(mid, 0), C.GRID[:127], _rng(1).uniform(-448, 448, 5000),
                        _rng(2).standard_normal(5000) * 1e-2, [np.nan]])
    assert np.array_equal(C.e4m3_bytes(x)[:-1], np.array([_nearest(v) for v in x[:-1]])) and C.e4m3_bytes(x)[-1] == 127


def _nearest(v):
    d = np.abs(C.GRID[:127] - abs(v))
    best = np.flatnonzero(d == d.min())
    byte = best[0] if len(best) == 1 or best[0] % 2 == 0 else best[1]
    return byte + (128 if np.signbit(v) else 0)


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_store_rounds_once(dtype):
    x = _rng(3).standard_normal(4000) * np.exp2(_rng(4).integers(-20, 12, 4000))
    t = torch.from_numpy(x)
    want = {0: torch.bfloat16, 1: torch.float32, 2: torch.float16}[dtype]
    near = t.float().to(want)                            # two roundings: one step apart at most, and rarely
    got = C.widen(C.store(x, dtype), dtype)
    assert np.mean(got != near.double().numpy()) < 1e-3
    step = np.abs(x) * {0: 2.0 ** -8, 1: 2.0 ** -24, 2: 2.0 ** -11}[dtype] + (2.0 ** -25 if dtype == 2 else 0)
    assert (np.abs(got - x) <= step).all()


@pytest.mark.parametrize("pairs", [False, True])
def test_rotation_is_a_rotation(pairs):
    r = _rng(5)
    x, freq = r.standard_normal((3, 2, 32)), 100.0 ** (-np.arange(8) / 8)
    freq = freq.astype(np.float32)
    pos = np.array([0, 5, 100000])
    y = C._rotate_all(x, pos, freq, 16, pairs, 1.0)
    for i in range(3):
        for h in range(2):
            one = C.rotate(x[i, h], int(pos[i]), freq, 16, pairs, 1.0)
            assert np.allclose(y[i, h], one, atol=1e-12)
    assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., 16:], x[..., 16:])
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
    # scores depend on the distance of the positions only
    a, b = C.rotate(x[0, 0], 7, freq, 16, pairs, 1.0), C.rotate(x[1, 0], 19, freq, 16, pairs, 1.0)
    c, d = C.rotate(x[0, 0], 1007, freq, 16, pairs, 1.0), C.rotate(x[1, 0], 1019, freq, 16, pairs, 1.0)
    assert np.isclose(a @ b, c @ d)


@pytest.mark.parametrize("dtype", [0, 2])
def test_blocks_hold_their_rows_to_half_a_step_and_survive_a_new_scale(dtype):
    r = _rng(6 + dtype)
    rows = C.widen(C.store(r.standard_normal((16, 64)) * np.exp2(r.integers(-4, 5, (16, 1))), dtype), dtype)
    raw, e = C.block_of(rows, dtype)
    big = np.abs(rows).max()
    assert big <= 448 * 2.0 ** e and (e == C.LEAST[dtype] or big > 224 * 2.0 ** e)
    held = C.e4m3_values(raw) * 2.0 ** e
    assert (np.abs(held - rows) <= np.maximum(np.abs(rows) * 2.0 ** -4, 2.0 ** (e - 10))).all()
    again, e2 = C.block_of(held, dtype)                  # what is in a block already stays
    assert e2 == e and np.array_equal(again, raw)
    up, e3 = C.block_of(np.vstack([held, np.full((1, 64), 4 * big)]), dtype)
    kept = C.e4m3_values(up[:16]) * 2.0 ** e3
    assert e3 >= e + 2 and (np.abs(kept - held) <= np.where(np.abs(held) >= 2.0 ** (e3 - 6), 0.0, 2.0 ** (e3 - 10))).all()


def test_blocks_of_what_is_no_number_of_zeros_and_of_the_types_ends():
    raw, e = C.block_of(np.zeros((3, 64)), 0)
    assert e == -117 and not raw.any()
    rows = np.ones((2, 64))
    rows[0, :3] = np.nan, np.inf, -np.inf
    raw, e = C.block_of(rows, 2)
    assert (raw[0, :3] == 127).all() and e == -8 and np.array_equal(C.e4m3_values(raw)[1] * 2.0 ** e, rows[1])
    raw, e = C.block_of(np.full((1, 64), 65504.0), 2)
    assert np.isfinite(np.float16(C.e4m3_values(raw)[0, 0] * 2.0 ** e)) and C.e4m3_values(raw)[0, 0] * 2.0 ** e == 61440.0


def test_append_and_commit_agree_with_each_other():
    """Rows appended at their final places give what rows appended as drafts and committed give, where no scale changes."""
    r = _rng(9)
    D, Hkv, L, n = 64, 2, 21, 20
    strides = (Hkv * 16 * D, 16 * D, D)
    table = np.array([[3, 1, 0, 2]], np.int32)
    start = C.Blocks(np.zeros((4, Hkv, 16, D)), np.full((4, Hkv), 127), strides, D, 0)
    start.append(C.store(r.choice([-1.75, 1.0, 1.5], size=(1, L, Hkv, D)), 0), table, [0], [L])
    rows = C.store(r.choice([-1.75, 1.0, 1.5], size=(1, n, Hkv, D)), 0)
    drafted = start.copy()
    drafted.append(rows, table, [L], [n])
    path = [0, 3, 4, 11, 19]
    drafted.commit(table, [L], np.array([path + [-1] * (n - 5)]), [5])
    direct = start.copy()
    direct.append(rows[:, path], table, [L], [5])
    for t in range(L + 5):
        for g in range(Hkv):
            assert np.array_equal(drafted.row(int(table[0, t // 16]), g, t % 16), direct.row(int(table[0, t // 16]), g, t % 16)), (t, g)


def test_logprobs_against_torch():
    r = _rng(10)
    x = r.standard_normal((5, 301)) * 3
    x[1, 5] = x[1, 100] = 9.0
    x[2, 10:] = -np.inf
    x[3] = -np.inf
    x[4, 7] = np.nan
    tok = r.integers(0, 301, (5, 3)).astype(np.int32)
    tok[0, 0], tok[1, 0] = -1, 400
    lp, h, ids, top = P.token_logprobs(x, tok, 12, 0.5)
    want = torch.log_softmax(torch.from_numpy(x) * 0.5, -1).numpy()
    for b in (0, 1, 2):
        known = (tok[b] >= 0) & (tok[b] < 301)
        assert np.allclose(lp[b, known], want[b, tok[b, known]])
        p = np.exp(want[b][np.isfinite(want[b])])
        assert np.isclose(h[b], -(p * np.log(p)).sum())
    assert lp[0, 0] == 0 and np.isnan(lp[1, 0])
    assert ids[1, :2].tolist() == [5, 100] and sorted(ids[2, :10]) == list(range(10)) and ids[2, 10:].tolist() == [-1, -1]
    assert h[3] == 0 and (ids[3] == -1).all() and (top[3] == -np.inf).all() and (lp[3] == -np.inf).all()
    assert np.isnan(lp[4]).all() and np.isnan(top[4]).all() and (ids[4] == -1).all()
