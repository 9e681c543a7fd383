"""CPU oracle of the log probabilities of given tokens, the entropy and the top alternatives of rows of logits.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``): numpy in 64 bits, row by row, from the definition in
``include/owl.h``.
"""
from __future__ import annotations

import numpy as np


def token_logprobs(logits: np.ndarray, tokens, n_top: int, scale: float):
    """logits [rows][vocab] (64 bits), tokens [rows][n_given] -> logprob, entropy, top_ids, top_logprobs."""
    rows, vocab = logits.shape
    tokens = np.zeros((rows, 0), np.int32) if tokens is None else np.asarray(tokens)
    logprob = np.full(tokens.shape, np.nan)
    entropy = np.full(rows, np.nan)
    ids = np.full((rows, n_top), -1, np.int32)
    top = np.full((rows, n_top), np.nan)
    scale = float(np.float32(scale))
    for r in range(rows):
        x = logits[r].astype(np.float64)
        logprob[r, tokens[r] == -1] = 0.0
        if np.isnan(x).any() or (x == np.inf).any():
            continue
        seen = x > -np.inf
        logp = np.full(vocab, -np.inf)
        if seen.any():
            y = scale * x[seen]
            y = y - y.max()
            total = np.exp(y).sum()
            logp[seen] = y - np.log(total)
            entropy[r] = np.log(total) - (np.exp(y) * y).sum() / total
        else:
            entropy[r] = 0.0
        for j, t in enumerate(tokens[r]):
            if 0 <= t < vocab:
                logprob[r, j] = logp[t]
        order = sorted(np.flatnonzero(seen), key=lambda t: (-x[t], t))[:n_top] if vocab < 5000 else \
            [t for t in np.lexsort((np.arange(vocab), -x))[:n_top] if seen[t]]
        top[r] = -np.inf
        ids[r, :len(order)] = order
        top[r, :len(order)] = logp[order]
    return logprob, entropy, ids, top
