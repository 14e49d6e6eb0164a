"""The *_latent calls in NumPy, 64 bits, from their definitions; shares no code with the library.

A cached row is 576 values, a latent c (512) and a rotated key part r (64). Caches come as fp64 arrays [pages][16][576].
The attention functions return, beside each result, how far a kernel may be from it whose probabilities are rounded to bf16
(a half step: 2^-8 of each) and whose sums are fp32.
"""
from __future__ import annotations

import numpy as np

from . import q4

LATENT, ROPE, ROW, HEAD, PAGE = 512, 64, 576, 128, 16
BF16 = 2.0 ** -8


def rows_of(pages, table_row, n):
    """The first n cached rows of a sequence."""
    ids = np.asarray(table_row[:-(-n // PAGE)], np.int64)
    return pages[ids].reshape(-1, ROW)[:n] if n else np.zeros((0, ROW))


def append_rows(kv_new, weight, eps, positions, freq, axis, rot, adjacent, magnitude=1.0):
    """(rows, tolerance): what a token's row of kv_new becomes, before its one rounding to bf16. fp32 errors: the mean square and
    the products of the normalisation stay below 2^-20 of the value, the rotation within q4.rope's bound."""
    c = kv_new[:, :LATENT]
    tol = np.zeros_like(c)
    if weight is not None:
        c = c / np.sqrt((c * c).mean(-1, keepdims=True) + eps) * weight
        tol = 2.0 ** -20 * np.abs(c)
    r, rtol = q4.rope(kv_new[:, None, LATENT:], positions, freq, axis, rot, adjacent, magnitude)
    return np.concatenate([c, r[:, 0]], 1), np.concatenate([tol, np.broadcast_to(rtol, r.shape)[:, 0]], 1)


def _weights(logits, size):
    """Softmax over the last axis, its log of the sum, and the largest change of a logit: 36 accumulations of 16 products
    in fp32, each off by less than 2^-20 of the sum of magnitudes seen so far."""
    top = logits.max(-1, keepdims=True)
    e = np.exp(logits - top)
    total = e.sum(-1, keepdims=True)
    return e / total, (top + np.log(total))[..., 0], 36 * 2.0 ** -20 * size.max(-1)


def _attend(p, v, shift, own_sum):
    """sum p v and its bound. Rounded weights p (1 + d), |d| <= 2^-8, move the result by sum p d v: at most 2^-8 of sum p |v|
    where the unrounded weights' sum normalises it; where the rounded ones' does (`own_sum`), sum p d (v - out) / sum p (1 + d): at most
    1.01 * 2^-8 of sum p |v - out|. A change of every logit by at most `shift` moves it by 2 shift (1 + shift) sum p |v - out|; fp32 sums
    by 2^-22 per 16 tokens of sum p |v|; then one rounding to bf16."""
    out = p @ v
    spread = np.empty_like(out)
    for i in range(out.shape[0]):
        spread[i] = p[i] @ np.abs(v - out[i])
    size = p @ np.abs(v)
    err = 1.02 * BF16 * (spread if own_sum else size) + 2.1 * shift[:, None] * spread + (v.shape[0] / 16 + 32) * 2.0 ** -22 * size
    return out, err + BF16 * (np.abs(out) + err)


def decode(q, pages, table, lens, scale):
    """(out, lse, out bound, lse bound) of absorbed queries q [B][H][576]."""
    b, h, _ = q.shape
    out, bound = np.zeros((b, h, LATENT)), np.zeros((b, h, LATENT))
    lse, lbound = np.full((b, h), -np.inf), np.zeros((b, h))
    for i, n in enumerate(lens):
        if n == 0:
            continue
        x = rows_of(pages, table[i], int(n))
        p, lse[i], shift = _weights(scale * (q[i] @ x.T), scale * (np.abs(q[i]) @ np.abs(x).T))
        out[i], bound[i] = _attend(p, x[:, :LATENT], shift, True)
        lbound[i] = shift + 2.0 ** -18 + 2.0 ** -21 * np.abs(lse[i])
    return out, lse, bound, lbound


def expand(w, pages, table, lens, first=None):
    """Per sequence (first token, K [n][H][128], V, K bound, V bound): 32 accumulations of 16 products, one rounding."""
    done = []
    for i, n in enumerate(lens):
        lo = 0 if first is None else int(first[i])
        c = rows_of(pages, table[i], int(n))[lo:, :LATENT]
        flat, shape = w.reshape(-1, LATENT), (len(c), w.shape[0], 2 * HEAD)
        kv = (c @ flat.T).reshape(shape)
        tol = 32 * 2.0 ** -20 * (np.abs(c) @ np.abs(flat).T).reshape(shape)
        tol = tol + BF16 * (np.abs(kv) + tol)
        done.append((lo, kv[..., :HEAD], kv[..., HEAD:], tol[..., :HEAD], tol[..., HEAD:]))
    return done


def prefill(q, indptr, k_pages, v_pages, kv_table, pages, table, lens, scale):
    """(out, lse, out bound, lse bound) of queries q [T][H][192] over expanded pages [pages][H][16][128] and rotated parts."""
    t, h, _ = q.shape
    out, bound = np.zeros((t, h, HEAD)), np.zeros((t, h, HEAD))
    lse, lbound = np.zeros((t, h)), np.zeros((t, h))
    for i, n in enumerate(lens):
        lo, hi = int(indptr[i]), int(indptr[i + 1])
        if lo == hi:
            continue
        n = int(n)
        ids = np.asarray(kv_table[i][:-(-n // PAGE)], np.int64)
        r = rows_of(pages, table[i], n)[:, LATENT:]
        seen = np.arange(n)[None, :] <= (n - (hi - lo) + np.arange(hi - lo))[:, None]
        for j in range(h):
            k = np.concatenate([k_pages[ids, j].reshape(-1, HEAD)[:n], r], 1)
            v = v_pages[ids, j].reshape(-1, HEAD)[:n]
            z = np.where(seen, scale * (q[lo:hi, j] @ k.T), -np.inf)
            p, lse[lo:hi, j], shift = _weights(z, np.where(seen, scale * (np.abs(q[lo:hi, j]) @ np.abs(k).T), 0.0))
            out[lo:hi, j], bound[lo:hi, j] = _attend(p, v, shift, False)
            lbound[lo:hi, j] = shift + 2.0 ** -18 + 2.0 ** -21 * np.abs(lse[lo:hi, j])
    return out, lse, bound, lbound
