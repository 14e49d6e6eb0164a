"""fp64 oracle of the 4-bit KV cache and of rotary positions (NumPy, index order, no shared code with the library).

TEST INFRASTRUCTURE ONLY. bf16 tensors travel as ``uint16`` bit patterns, 4-bit pools as ``uint8``
``[num_pages, num_kv_heads, 18 * head_dim]``; the format is the one ``include/pd.h`` states.
"""
from __future__ import annotations

import numpy as np

from . import bf16_bits_to_f64, f32_to_bf16_bits

PAGE = 16
GROUP = 64


def quantize_group(bits):
    """bits uint16 [64] -> (codes uint8 [64], scale bits, min bits, all values read back as NaN)."""
    x = bf16_bits_to_f64(np.asarray(bits, np.uint16))
    x = np.where(np.abs(x) < 2.0 ** -126, 0.0, x)  # NaN compares false and stays
    if not np.all(np.isfinite(x)):
        return np.zeros(GROUP, np.uint8), 0x7FC0, 0, True
    lo, hi = x.min(), x.max()
    with np.errstate(over="ignore"):
        span = np.float32(hi - lo)
        if not np.isfinite(span):
            return np.zeros(GROUP, np.uint8), 0x7FC0, 0, True
        s = np.float32(np.float64(span) / 15.0)
    if s < 2.0 ** -100:
        scale_bits, scale = 0, 0.0
    else:
        scale_bits = int((int(np.float32(s).view(np.uint32)) + 0xFFFF) >> 16)  # up to the next bf16
        scale = float(bf16_bits_to_f64(np.array([scale_bits], np.uint16))[0])
        if 15 * scale + lo >= 511 * 2.0 ** 119:  # would round past bf16's largest value, 255 * 2^120: the bf16 below
            scale_bits = int(np.float32(s).view(np.uint32)) >> 16
            scale = float(bf16_bits_to_f64(np.array([scale_bits], np.uint16))[0])
    d = (x - lo).astype(np.float32).astype(np.float64)
    codes = np.rint(d / scale).astype(np.uint8) if scale > 0 else np.zeros(GROUP, np.uint8)
    assert codes.max() <= 15
    return codes, scale_bits, int(f32_to_bf16_bits(np.array([lo + 0.0], np.float32))[0]), False


def nibble_at(d, slot, i):
    """(byte offset within the 16 rows of one tensor, shift) of value i of a slot."""
    piece = i // 32
    pos = piece ^ ((slot >> 1) & 3) if d == 128 else piece ^ ((slot >> 2) & 1)
    return slot * (d // 2) + pos * 16 + (i % 32) // 2, 4 * (i & 1)


def record_at(d, slot, group, which, entry):
    """Byte offset within the block of record entry 0 (scale) or 1 (min) of K (which 0) or V (1)."""
    return 16 * d + ((slot * (d // GROUP) + group) * 4 + which * 2 + entry) * 2


_AT = {}


def _tables(d):
    if d not in _AT:
        byte = np.zeros((PAGE, d), np.int64)
        shift = np.zeros((PAGE, d), np.int64)
        for slot in range(PAGE):
            for i in range(d):
                byte[slot, i], shift[slot, i] = nibble_at(d, slot, i)
        _AT[d] = byte, shift
    return _AT[d]


def store_row(block, which, slot, bits):
    """Quantises one row (uint16 [d]) into a block (uint8 [18 d]) in place."""
    d = len(bits)
    byte, shift = _tables(d)
    for g in range(d // GROUP):
        codes, s, m, bad = quantize_group(bits[g * GROUP:(g + 1) * GROUP])
        for k in range(GROUP):
            i = g * GROUP + k
            o = 8 * d * which + byte[slot, i]
            block[o] = (int(block[o]) & (0xF0 if shift[slot, i] == 0 else 0x0F)) | (int(codes[k]) << int(shift[slot, i]))
        for e, v in enumerate((s, m)):
            o = record_at(d, slot, g, which, e)
            block[o], block[o + 1] = v & 255, v >> 8


def append_tokens(k_new, v_new, q_indptr, kv4, page_table, ctx_lens):
    """uint16 [total, Hkv, d] rows into kv4 in place; returns the grown lengths."""
    lens = np.array(ctx_lens, np.int32)
    for b in range(len(lens)):
        n = int(q_indptr[b + 1] - q_indptr[b])
        for i in range(n):
            pos = int(ctx_lens[b]) + i
            page = int(page_table[b, pos // PAGE])
            for h in range(k_new.shape[1]):
                for which, src in ((0, k_new), (1, v_new)):
                    store_row(kv4[page, h], which, pos % PAGE, src[int(q_indptr[b]) + i, h])
        lens[b] += n
    return lens


def block_values(block, d):
    """(K, V) float64 [16, d] of one block."""
    byte, shift = _tables(d)
    out = []
    for which in range(2):
        codes = (block[8 * d * which + byte].astype(np.int64) >> shift) & 15
        rec = np.ascontiguousarray(block[16 * d:]).view(np.uint16).reshape(PAGE, d // GROUP, 4)
        s, m = bf16_bits_to_f64(rec[:, :, 2 * which]), bf16_bits_to_f64(rec[:, :, 2 * which + 1])
        out.append((codes.reshape(PAGE, d // GROUP, GROUP) * s[:, :, None] + m[:, :, None]).reshape(PAGE, d))
    return out


def block_steps(block, d):
    """(15 * v_scale, |v_min|, 15 * k_scale, |k_min|) float64 [16, groups] of one block, for error bounds."""
    rec = np.ascontiguousarray(block[16 * d:]).view(np.uint16).reshape(PAGE, d // GROUP, 4)
    f = bf16_bits_to_f64(rec)
    return 15 * f[..., 2], np.abs(f[..., 3]), 15 * f[..., 0], np.abs(f[..., 1])


def sequence_values(kv4, page_table, b, n, h, d):
    """(K, V, steps) of the first n tokens of sequence b, KV head h."""
    k, v, st = np.zeros((n, d)), np.zeros((n, d)), np.zeros((4, n, d // GROUP))
    for t in range(0, n, PAGE):
        blk = kv4[int(page_table[b, t // PAGE]), h]
        m = min(PAGE, n - t)
        bk, bv = block_values(blk, d)
        k[t:t + m], v[t:t + m] = bk[:m], bv[:m]
        for i, x in enumerate(block_steps(blk, d)):
            st[i, t:t + m] = x[:m]
    return k, v, st


def decode_attn(q, kv4, page_table, ctx_lens, sm_scale):
    """softmax(scale q K^T) V in fp64 with, beside (out, lse), the bounds an fp16 / fp32 kernel is held to:

    tol_out  2^-8 |out| (one rounding to bf16)
             + 2^-11 sum p 15 v_scale (the weights p * v_scale rounded to fp16, codes up to 15)
             + (2^-18 + 2 delta) sum p (15 v_scale + |v_min|) (fp32 sums; error of the logits)
    tol_lse  delta + 4e-6 (1 + |lse|)
    with delta = 2^-19 max_t sm_scale sum |q| (15 k_scale + |k_min|), the fp32 sums of the logits.
    """
    B, Hq, d = q.shape
    Hkv = kv4.shape[1]
    G = Hq // Hkv
    scale = float(np.float32(sm_scale))
    out, lse = np.zeros((B, Hq, d)), np.full((B, Hq), -np.inf)
    tol_out, tol_lse = np.zeros((B, Hq, d)), np.zeros((B, Hq))
    qf = bf16_bits_to_f64(q)
    for b in range(B):
        n = int(ctx_lens[b])
        if n == 0:
            continue
        for h in range(Hkv):
            k, v, (vs, vm, ks, km) = sequence_values(kv4, page_table, b, n, h, d)
            for hq in range(h * G, (h + 1) * G):
                z = scale * (k @ qf[b, hq])
                with np.errstate(invalid="ignore"):
                    p = np.exp(z - z.max())
                    total = p.sum()
                    p = p / total
                out[b, hq] = p @ v
                lse[b, hq] = z.max() + np.log(total)
                qa = np.abs(qf[b, hq]).reshape(d // GROUP, GROUP).sum(1)
                delta = 2.0 ** -19 * scale * float(((ks + km) @ qa).max())
                spread, size = np.repeat(p @ vs, GROUP), np.repeat(p @ (vs + vm), GROUP)
                tol_out[b, hq] = 2.0 ** -8 * np.abs(out[b, hq]) + 2.0 ** -11 * spread + (2.0 ** -18 + 2 * delta) * size
                tol_lse[b, hq] = delta + 4e-6 * (1 + abs(lse[b, hq]))
    return out, lse, tol_out, tol_lse


def rope(x, positions, inv_freq, axis_of_pair, rot_dim, adjacent, magnitude=1.0):
    """x float64 [rows, heads, d], positions int [axes, rows] -> (rotated float64, bound of an fp32 kernel before its
    rounding): angles in extended precision, reduced by whole turns before the sine."""
    y, tol = np.array(x, np.float64), np.zeros_like(x, dtype=np.float64)
    two_pi = 2 * np.arctan2(np.longdouble(0), np.longdouble(-1))
    for i in range(rot_dim // 2):
        a, c = (2 * i, 2 * i + 1) if adjacent else (i, i + rot_dim // 2)
        turns = positions[axis_of_pair[i]].astype(np.longdouble) * np.longdouble(np.float32(inv_freq[i])) / two_pi
        angle = ((turns - np.rint(turns)) * two_pi).astype(np.float64)[:, None]
        u, w = np.array(x[..., a], np.float64), np.array(x[..., c], np.float64)
        y[..., a] = magnitude * (u * np.cos(angle) - w * np.sin(angle))
        y[..., c] = magnitude * (u * np.sin(angle) + w * np.cos(angle))
        tol[..., a] = tol[..., c] = 2.0 ** -21 * abs(magnitude) * (np.abs(u) + np.abs(w))
    return y, tol
