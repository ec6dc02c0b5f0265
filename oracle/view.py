"""Oracle: bounded views of the prefix cache -- a sliding window with sinks, and a
cache held in 4-bit blocks.

TEST INFRASTRUCTURE ONLY (see the package docstring). Float64 numpy.

A window bounds what a token sees by its place in the committed order (prefix row
j has place j, draft token t the place P + t): of the keys that the pass shows to a
token at place i, those at places j > i - window and those at places j < sinks.

The 4-bit cache holds blocks of 32 neighbouring elements of a row: codes e2m1 and
one scale byte, an element's value being its magnitude times 2^(byte - 127), a byte
of 255 a block without values.  A block's scale is the smallest power of two for
which its largest magnitude rounds to at most 6.
"""

from __future__ import annotations

import numpy as np

from .attention import prefix_lengths, visibility

Q4_BLOCK = 32
Q4_MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def window_visibility(prefix_len, n_slots, slot_len, pass_, cross_slot, slot_pass, window, sinks):
    """Boolean mask [T, P + T] of :func:`visibility` under a window (None: no window)."""
    mask = visibility(prefix_len, n_slots, slot_len, pass_, cross_slot, slot_pass)
    if window is not None:
        i = prefix_len + np.arange(n_slots * slot_len)[:, None]
        j = np.arange(mask.shape[1])[None, :]
        mask = mask & ((j > i - window) | (j < sinks))
    return mask


def view_attention(q, k_cache, v_cache, k_slot, v_slot, prefix_len, n_slots, slot_len, scale, pass_, cross_slot=0,
                   slot_pass=None, window=None, sinks=0):
    """Masked softmax attention over the visible keys alone (an invisible key's values
    are never multiplied).  Returns (O, LSE, A), A = sum_j p_j |v_j|, the size that
    roundings of the probabilities are relative to."""
    q = np.asarray(q, dtype=np.float64)
    B, Hq, T, D = q.shape
    Hkv = k_slot.shape[1]
    G = Hq // Hkv
    plens = prefix_lengths(prefix_len, B)
    out, size, lse = np.empty((B, Hq, T, D)), np.empty((B, Hq, T, D)), np.empty((B, Hq, T))
    for b in range(B):
        P = plens[b]
        mask = window_visibility(P, n_slots, slot_len, pass_, cross_slot,
                                 None if slot_pass is None else np.asarray(slot_pass)[b], window, sinks)
        for g in range(Hkv):
            slot = (np.asarray(k_slot[b, g], np.float64), np.asarray(v_slot[b, g], np.float64))
            keys = np.concatenate([np.asarray(k_cache[b, g, :P], np.float64), slot[0]]) if P else slot[0]
            vals = np.concatenate([np.asarray(v_cache[b, g, :P], np.float64), slot[1]]) if P else slot[1]
            for h in range(g * G, (g + 1) * G):
                for t in range(T):
                    seen = np.flatnonzero(mask[t])
                    z = scale * (keys[seen] @ q[b, h, t])
                    m = z.max()
                    p = np.exp(z - m)
                    lse[b, h, t] = m + np.log(p.sum())
                    p /= p.sum()
                    out[b, h, t] = p @ vals[seen]
                    size[b, h, t] = p @ np.abs(vals[seen])
    return out, lse, size


def q4_quantize(x):
    """(codes [..., D/2] uint8, scales [..., D/32] uint8) of rows x [..., D]."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(x.shape[:-1] + (x.shape[-1] // Q4_BLOCK, Q4_BLOCK))
    finite = np.isfinite(blocks).all(-1)
    safe = np.where(finite[..., None], blocks, 0.0)
    top = np.abs(safe).max(-1)
    exponent = np.full(top.shape, -127)
    for e in range(-126, 126):  # the smallest scale 2^e with top / 2^e < 7
        exponent = np.where(top >= 7.0 * 2.0 ** (e - 1), e, exponent)
    a = np.abs(safe) / 2.0 ** exponent[..., None].astype(np.float64)
    # nearest magnitude; halfway between two, the one whose code is even
    dist = np.abs(a[..., None] - Q4_MAGNITUDES)
    best = dist.min(-1, keepdims=True)
    near = dist == best
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    code = code + 8 * (safe < 0)
    code = np.where(finite[..., None], code, 0).reshape(x.shape).astype(np.uint8)
    scales = np.where(finite, exponent + 127, 255).astype(np.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), scales


def q4_dequantize(codes, scales):
    """float64 values [..., D]; NaN in blocks whose scale is 255."""
    codes, scales = np.asarray(codes), np.asarray(scales)
    code = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (2 * codes.shape[-1],))
    value = np.where(code & 8, -1.0, 1.0) * Q4_MAGNITUDES[code & 7]
    factor = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return value * np.repeat(factor, Q4_BLOCK, -1)
