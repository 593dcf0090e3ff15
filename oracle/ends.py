"""The two ends of a pipeline in 64 bits (numpy): the definitions that include/dpo.h
states for dpo_embed, dpo_dropout, dpo_logprobs, dpo_head and their backward passes, written
from the formulas. Test infrastructure; shares no code with the package.
"""
from __future__ import annotations

import numpy as np

M32 = 0xFFFFFFFF


# ------------------------------------------------------------- embedding ----

def embed(ids, table, scale=1.0):
    ids = np.asarray(ids)
    out = np.zeros(ids.shape + (table.shape[1],))
    real = (ids >= 0) & (ids < table.shape[0])
    out[real] = scale * table[ids[real]]
    return out


def embed_backward(dy, ids, vocab, scale=1.0):
    """(the gradient, the sum of the terms' magnitudes, the number of terms of each row)."""
    ids, dy = np.asarray(ids).ravel(), dy.reshape(-1, dy.shape[-1])
    g, mag, count = np.zeros((vocab, dy.shape[1])), np.zeros((vocab, dy.shape[1])), np.zeros(vocab)
    real = (ids >= 0) & (ids < vocab)
    np.add.at(g, ids[real], scale * dy[real])
    np.add.at(mag, ids[real], np.abs(scale * dy[real]))
    np.add.at(count, ids[real], 1)
    return g, mag, count


# --------------------------------------------------------------- dropout ----

def philox(counter, key):
    """Philox4x32-10: four words from four words of counter and two of key (Python integers)."""
    c, k = list(counter), list(key)
    for _ in range(10):
        p, q = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(q >> 32) ^ c[1] ^ k[0], q & M32, (p >> 32) ^ c[3] ^ k[1], p & M32]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    return c


def kept_mask(rows, cols, p, seed, site):
    """(mask of kept elements, the dropped share p')."""
    cut = int(np.floor(65536 * p + 0.5))
    key = (seed & M32, seed >> 32 & M32)
    bits = np.zeros((rows, -(-cols // 8) * 8), dtype=np.int64)
    for r in range(rows):
        for g in range(bits.shape[1] // 8):
            words = philox((g, r & M32, r >> 32, site), key)
            for e in range(8):
                bits[r, 8 * g + e] = words[e // 2] >> 16 * (e % 2) & 0xFFFF
    return bits[:, :cols] >= cut, cut / 65536


def dropout(x, residual, mask, share):
    y = np.where(mask, x / (1 - share), 0.0)
    return y if residual is None else residual + y


# ------------------------------------------------------ log probabilities ----

def distribution(z):
    """(log p, p, entropy) of rows of scaled logits; -inf is masked."""
    m = z.max(1, keepdims=True)
    with np.errstate(invalid="ignore", divide="ignore"):
        d = z - m
        e = np.exp(d)
        s = e.sum(1, keepdims=True)
        logs = d - np.log(s)
        p = e / s
        h = np.log(s[:, 0]) - np.where(e > 0, e * d, np.where(np.isnan(e), np.nan, 0.0)).sum(1) / s[:, 0]
    return logs, p, h


def logprobs(z, ids):
    logs, _, h = distribution(z)
    real = (ids >= 0) & (ids < z.shape[1])
    r = np.arange(len(ids))
    return np.where(real, logs[r, np.where(real, ids, 0)], 0.0), h


def top(z, k):
    """Ids of the k largest, ties to the lowest id, NaN last, behind -inf."""
    nan = np.isnan(z)
    return np.lexsort((np.where(nan, 0.0, -z), nan), axis=1)[:, :k]


def logits_gradient(z, ids, dlogp, dentropy=None):
    """The gradient of the scaled logits."""
    logs, p, h = distribution(z)
    real = (ids >= 0) & (ids < z.shape[1])
    a = np.where(real, dlogp, 0.0)
    b = np.zeros(len(ids)) if dentropy is None else dentropy
    with np.errstate(invalid="ignore"):
        g = -a[:, None] * p - b[:, None] * np.where(p > 0, p * (logs + h[:, None]), 0.0)
    g[np.arange(len(ids))[real], ids[real]] += a[real]
    g[(a == 0) & (b == 0)] = 0.0
    return g
