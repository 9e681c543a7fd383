"""CPU oracle of the rows of the paged cache: appending with the rotary position embedding, caches of 8-bit blocks, and
the commit in them.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``): plain numpy in 64 bits, one row or one block after the other,
written from the definitions in ``include/owl.h`` and sharing nothing with the HIP path.  Pools are flat arrays with
element strides (page, head, token); ``dtype`` is 0 (bf16, uint16 bits), 1 (float32) or 2 (fp16, uint16 bits).
"""
from __future__ import annotations

import numpy as np

PAGE = 16
LEAST = {0: -117, 2: -15}
TOP = {0: 1.875 * 2.0 ** 127, 2: 1.875 * 2.0 ** 15}


def _grid():
    v = np.empty(128)
    for byte in range(127):
        e, m = byte >> 3, byte & 7
        v[byte] = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
    v[127] = np.nan
    return v


GRID = _grid()                                           # the numbers of the bytes 0 .. 127


def e4m3_values(raw: np.ndarray) -> np.ndarray:
    raw = np.asarray(raw, dtype=np.uint8)
    return np.where(raw > 127, -1.0, 1.0) * GRID[raw & 127]


def e4m3_bytes(x: np.ndarray) -> np.ndarray:
    """Nearest byte, ties to the even one; |x| <= 448 or no number (0x7F)."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(np.where(np.isnan(x), 0.0, x))
    assert a.max(initial=0.0) <= 448.0
    hi = np.searchsorted(GRID[:127], a, side="left")     # GRID[hi - 1] < a <= GRID[hi]
    lo = np.maximum(hi - 1, 0)
    up, down = GRID[hi] - a, a - GRID[lo]
    byte = np.where((up < down) | ((up == down) & (hi % 2 == 0)) | (hi == 0), hi, lo)
    byte = np.where(np.isnan(x), 127, byte)
    return (byte + np.where(np.signbit(x) & ~np.isnan(x), 128, 0)).astype(np.uint8)


def widen(x: np.ndarray, dtype: int) -> np.ndarray:
    if dtype == 0:
        return (x.astype(np.uint32) << np.uint32(16)).view(np.float32).astype(np.float64)
    return x.view(np.float16).astype(np.float64) if dtype == 2 else x.astype(np.float64)


def store(x: np.ndarray, dtype: int) -> np.ndarray:
    """64 bits -> storage, rounded once, to nearest even."""
    x = np.asarray(x, dtype=np.float64)
    if dtype == 1:
        return x.astype(np.float32)
    if dtype == 2:
        with np.errstate(over="ignore"):
            return x.astype(np.float16).view(np.uint16)
    _, e = np.frexp(np.where(np.isfinite(x), x, 1.0))    # the step of the eight bits of x's binade
    step = np.exp2(np.maximum(e - 1, -126) - 7.0)
    with np.errstate(over="ignore", invalid="ignore"):
        f = np.where(np.isfinite(x), np.rint(x / step) * step, x).astype(np.float32)
    return (f.view(np.uint32) >> np.uint32(16)).astype(np.uint16)


def rotate(x: np.ndarray, pos: int, inv_freq: np.ndarray, rot_dim: int, pairs: bool, scale: float) -> np.ndarray:
    """One head's channels [D] (64 bits) at position id ``pos``."""
    y = np.array(x, dtype=np.float64)
    for f in range(rot_dim // 2):
        a = float(pos) * float(inv_freq[f])
        i, j = (2 * f, 2 * f + 1) if pairs else (f, f + rot_dim // 2)
        c, s = np.cos(a), np.sin(a)
        y[i] = (x[i] * c - x[j] * s) * float(scale)
        y[j] = (x[j] * c + x[i] * s) * float(scale)
    return y


def _rotate_all(x, pos, inv_freq, rot_dim, pairs, scale):
    """x [n][heads][D], pos [n]: as ``rotate``, for all of them at once."""
    y = np.array(x, dtype=np.float64)
    h = rot_dim // 2
    a = np.asarray(pos, dtype=np.float64)[:, None] * np.asarray(inv_freq, dtype=np.float32).astype(np.float64)[None, :h]
    c, s = np.cos(a)[:, None], np.sin(a)[:, None]
    i, j = (slice(0, rot_dim, 2), slice(1, rot_dim, 2)) if pairs else (slice(0, h), slice(h, rot_dim))
    with np.errstate(invalid="ignore"):                  # (an infinite channel turns into no number)
        y[..., i] = (x[..., i] * c - x[..., j] * s) * float(np.float32(scale))
        y[..., j] = (x[..., j] * c + x[..., i] * s) * float(np.float32(scale))
    return y


def _page(page_table, b, t):
    return t // PAGE if page_table is None else int(page_table[b, t // PAGE])


def rotated_rows(q, k, v, pos, inv_freq, rot_dim, pairs, scale, dtype):
    """Stored forms of the rotated q and k and of v: [B][n][heads][D] each."""
    B, n = pos.shape
    out = []
    for x, turn in ((q, True), (k, True), (v, False)):
        if x is None or not turn or rot_dim == 0:
            out.append(None if x is None else np.array(x))
            continue
        y = np.array(x)
        for b in range(B):
            turned = store(_rotate_all(widen(x[b], dtype), pos[b], inv_freq, rot_dim, pairs, scale), dtype)
            y[b, :, :, :rot_dim] = turned[..., :rot_dim]
        out.append(y)
    return out


def append(pool, rows, page_table, ctx_lens, counts, strides):
    """A copy of the flat pool with rows[b][i] at position ctx_lens[b] + i, i < counts[b]."""
    flat = np.array(pool, copy=True).reshape(-1)
    sp, sh, st = strides
    for b, L in enumerate(ctx_lens):
        for i in range(int(counts[b])):
            t = int(L) + i
            for g in range(rows.shape[2]):
                at = _page(page_table, b, t) * sp + g * sh + t % PAGE * st
                flat[at:at + rows.shape[3]] = rows[b, i, g]
    return flat.reshape(np.asarray(pool).shape)


def block_of(rows, dtype):
    """Rows [r][D] in 64 bits -> (bytes [r][D], exponent)."""
    rows = np.asarray(rows, dtype=np.float64)
    finite = np.isfinite(rows)
    rows = np.where(finite, np.clip(np.where(finite, rows, 0.0), -TOP[dtype], TOP[dtype]), np.nan)
    big = np.abs(rows[finite]).max(initial=0.0)
    e = LEAST[dtype]
    while big > 448.0 * 2.0 ** e:
        e += 1
    return e4m3_bytes(rows * 2.0 ** -e), e


class Blocks:
    """A cache of 8-bit blocks, K or V: flat bytes, scales [pages][Hkv], byte strides."""

    def __init__(self, raw, scale, strides, D, dtype):
        self.flat = np.array(raw, dtype=np.uint8, copy=True).reshape(-1)
        self.shape = np.asarray(raw).shape
        self.scale = np.array(scale, dtype=np.uint8, copy=True)
        self.strides, self.D, self.dtype = strides, D, dtype

    def copy(self):
        return Blocks(self.flat.reshape(self.shape), self.scale, self.strides, self.D, self.dtype)

    def _at(self, page, g, slot):
        sp, sh, st = self.strides
        at = page * sp + g * sh + slot * st
        return slice(at, at + self.D)

    def row(self, page, g, slot):
        return e4m3_values(self.flat[self._at(page, g, slot)]) * 2.0 ** (int(self.scale[page, g]) - 127)

    def write(self, page, g, rows):
        """The block's rows from slot 0 on, in 64 bits; later slots stay."""
        raw, e = block_of(rows, self.dtype)
        for slot in range(len(rows)):
            self.flat[self._at(page, g, slot)] = raw[slot]
        self.scale[page, g] = e + 127

    def values(self):
        """The flat pool as numbers, in the pool's layout."""
        out = np.full(self.flat.shape, np.nan)
        for page in range(self.scale.shape[0]):
            for g in range(self.scale.shape[1]):
                for slot in range(PAGE):
                    out[self._at(page, g, slot)] = self.row(page, g, slot)
        return out.reshape(self.shape)

    def append(self, rows, page_table, ctx_lens, counts):
        """rows [B][n][Hkv][D] as stored 16-bit numbers."""
        for b, L in enumerate(ctx_lens):
            L, n = int(L), int(counts[b])
            new = widen(rows[b], self.dtype)
            for block in range(L // PAGE, (L + n + PAGE - 1) // PAGE if n else L // PAGE):
                page = _page(page_table, b, block * PAGE)
                for g in range(rows.shape[2]):
                    values = [self.row(page, g, t % PAGE) if t < L else new[t - L, g]
                              for t in range(block * PAGE, min((block + 1) * PAGE, L + n))]
                    self.write(page, g, np.stack(values))

    def commit(self, page_table, ctx_lens, accepted, n_accept):
        before = self.copy()
        for b, L in enumerate(ctx_lens):
            L = int(L)
            to = {L + i: L + int(accepted[b, i]) for i in range(int(n_accept[b]))}
            for block in sorted({t // PAGE for t, s in to.items() if t != s}):
                page = _page(page_table, b, block * PAGE)
                for g in range(self.scale.shape[1]):
                    values = []
                    for t in range(block * PAGE, min((block + 1) * PAGE, L + int(n_accept[b]))):
                        s = to.get(t, t)
                        values.append(before.row(_page(page_table, b, s), g, s % PAGE))
                    self.write(page, g, np.stack(values))


def same_bytes(a: np.ndarray, b: np.ndarray) -> bool:
    """Equal bytes; the two that are no number are alike."""
    a, b = np.asarray(a, dtype=np.uint8), np.asarray(b, dtype=np.uint8)
    return bool(np.array_equal(np.where(a & 127 == 127, 127, a), np.where(b & 127 == 127, 127, b)))
