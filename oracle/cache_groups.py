"""CPU oracle of caches of 4-bit groups and of the norms of the heads.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``): plain numpy in 64 bits, one group after the other, written from the
definitions in ``include/owl.h`` and sharing nothing with the HIP path.  ``dtype`` is 0 (bf16) or 2 (fp16), for the norms 1 (float32) too.
"""
from __future__ import annotations

import numpy as np

from .cache_blocks import PAGE, _page, _rotate_all, store, widen

GROUP = 32
ENDS = {0: (-125, 125), 2: (-23, 13)}
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
NONE = 255


def group_of(x, dtype):
    """32 numbers in 64 bits -> (codes [32], scale byte)."""
    x = np.asarray(x, dtype=np.float64)
    assert x.shape == (GROUP,)
    if not np.isfinite(x).all():
        return np.zeros(GROUP, np.uint8), NONE
    low, high = ENDS[dtype]
    e = low
    while np.abs(x).max() > 7.0 * 2.0 ** e and e < high:
        e += 1
    codes = []
    for v in x:
        y = abs(v) * 2.0 ** -e
        off = np.abs(MAGNITUDES - y)
        best = np.flatnonzero(off == off.min())
        code = int(best[0]) if len(best) == 1 or best[0] % 2 == 0 else int(best[1])      # a tie goes to the even code
        codes.append(code + (8 if np.signbit(v) else 0))
    return np.array(codes, np.uint8), e + 127


def group_values(codes, s):
    codes = np.asarray(codes, np.uint8)
    if s == NONE:
        return np.full(codes.shape, np.nan)
    return np.where(codes > 7, -1.0, 1.0) * MAGNITUDES[codes & 7] * 2.0 ** (int(s) - 127)


class Groups:
    """A cache of 4-bit groups, K or V: flat bytes, scales [pages][Hkv][16][D / 32], byte strides."""

    def __init__(self, raw, scale, strides, D, dtype):
        self.flat = np.array(raw, dtype=np.uint8, copy=True).reshape(-1)
        self.shape = np.asarray(raw).shape
        self.scale = np.array(scale, dtype=np.uint8, copy=True)
        self.strides, self.D, self.dtype = strides, D, dtype

    def copy(self):
        return Groups(self.flat.reshape(self.shape), self.scale, self.strides, self.D, self.dtype)

    def at(self, page, g, slot):
        sp, sh, st = self.strides
        at = page * sp + g * sh + slot * st
        return slice(at, at + self.D // 2)

    def row(self, page, g, slot):
        raw = self.flat[self.at(page, g, slot)]
        codes = np.empty(self.D, np.uint8)
        codes[0::2], codes[1::2] = raw & 15, raw >> 4
        return np.concatenate([group_values(codes[i:i + GROUP], int(self.scale[page, g, slot, i // GROUP])) for i in range(0, self.D, GROUP)])

    def write(self, page, g, slot, row):
        for i in range(0, self.D, GROUP):
            codes, s = group_of(row[i:i + GROUP], self.dtype)
            begin = self.at(page, g, slot).start + i // 2
            self.flat[begin:begin + GROUP // 2] = codes[0::2] | codes[1::2] << 4
            self.scale[page, g, slot, i // GROUP] = s

    def append(self, rows, page_table, ctx_lens, counts):
        """rows [B][n][Hkv][D] as stored 16-bit numbers."""
        for b, L in enumerate(ctx_lens):
            new = widen(rows[b], self.dtype)
            for i in range(int(counts[b])):
                t = int(L) + i
                for g in range(rows.shape[2]):
                    self.write(_page(page_table, b, t), g, t % PAGE, new[i, g])

    def commit(self, page_table, ctx_lens, accepted, n_accept):
        before = self.copy()
        for b, L in enumerate(ctx_lens):
            for i in range(int(n_accept[b])):
                s, t = int(L) + int(accepted[b, i]), int(L) + i
                sp, tp = _page(page_table, b, s), _page(page_table, b, t)
                for g in range(self.scale.shape[1]):
                    self.flat[self.at(tp, g, t % PAGE)] = before.flat[before.at(sp, g, s % PAGE)]
                    self.scale[tp, g, t % PAGE] = before.scale[sp, g, s % PAGE]


def normalised_rows(q, k, v, pos, inv_freq, rot_dim, pairs, scale, dtype, q_gain, k_gain, eps):
    """Stored forms of the normalised and rotated q and k and of v: [B][n][heads][D] each."""
    out = []
    for x, gain in ((q, q_gain), (k, k_gain)):
        if x is None:
            out.append(None)
            continue
        y = np.array(x)
        for b in range(len(pos)):
            w = widen(x[b], dtype)
            with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
                w = w / np.sqrt(np.mean(w * w, axis=-1, keepdims=True) + float(np.float32(eps)))
                if gain is not None:
                    w = w * np.asarray(gain, np.float32).astype(np.float64)
                y[b] = store(_rotate_all(w, pos[b], inv_freq, rot_dim, pairs, scale) if rot_dim else w, dtype)
        out.append(y)
    return *out, np.array(v)
