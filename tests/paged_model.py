"""The paged cache in 4 bits, the norms and the attention over it in 64 bits on the CPU, written from their definitions (include/cascade_kv.h),
one token and one byte at a time where that is simplest."""
import math

import numpy as np
import torch

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
VALUES = np.concatenate([MAGNITUDES, -MAGNITUDES])
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # largest relative error of one rounding


def bf16(x):
    """float64 array -> rounded to float32 and then to bfloat16, as float64."""
    return torch.from_numpy(np.asarray(x, dtype=np.float32).copy()).bfloat16().double().numpy()


def rotate(x, positions, base):
    """x [tokens, heads, d] float64."""
    d = x.shape[-1]
    angle = np.asarray(positions, dtype=np.float64)[:, None, None] * base ** (-2.0 * np.arange(d // 2) / d)
    lo, hi = x[..., :d // 2], x[..., d // 2:]
    return np.concatenate([lo * np.cos(angle) - hi * np.sin(angle), hi * np.cos(angle) + lo * np.sin(angle)], -1)


def nearest_codes(y):
    """Codes of y by the distance to every value, ties to the even code; at most 6."""
    dist = np.abs(np.abs(y)[..., None] - MAGNITUDES)
    best = dist.min(-1, keepdims=True)
    cand = dist == best
    even = cand & (np.arange(8) % 2 == 0)
    code = np.where(cand.sum(-1) > 1, even.argmax(-1), cand.argmax(-1))
    return (code + 8 * (y < 0)).astype(np.uint8)


def quantise_k(k):
    """Rows [..., d] float64 -> codes [..., d], exponent bytes [..., d / 32]."""
    blocks = k.reshape(k.shape[:-1] + (-1, 32))
    byte = np.zeros(blocks.shape[:-1], np.uint8)
    codes = np.zeros(blocks.shape, np.uint8)
    for at in np.ndindex(byte.shape):
        x = blocks[at]
        if not np.isfinite(x).all():
            byte[at] = 255
            codes[at] = 8 * (x < 0)
            continue
        top = np.abs(x).max()
        if top == 0.0:
            continue
        e = -126
        while e < 127 and top > 7.0 * 2.0 ** e:
            e += 1
        byte[at] = e + 127
        codes[at] = nearest_codes(x / 2.0 ** e)
    return codes.reshape(k.shape), byte


def quantise_v(v):
    """Rows [..., d] float64 (of float32 or bfloat16 numbers) -> codes [..., d], scales [...] float64."""
    scale = np.zeros(v.shape[:-1])
    codes = np.zeros(v.shape, np.uint8)
    for at in np.ndindex(scale.shape):
        x = v[at]
        if not np.isfinite(x).all():
            scale[at] = math.nan
            codes[at] = 8 * (x < 0)
            continue
        s32 = np.float32(np.abs(x).max()) / np.float32(6.0)
        s = float(bf16(s32)) if s32 >= 2.0 ** -100 else 0.0
        scale[at] = s
        if s:
            codes[at] = nearest_codes(x / s)      # the quotient is rounded, but a border has three bits and s eight: on which side x / s lies survives
    return codes, scale


def k_values(codes, byte):
    scale = np.where(byte == 255, math.nan, np.where(byte == 0, 0.0, 2.0 ** (byte.astype(np.float64) - 127)))
    return (VALUES[codes].reshape(codes.shape[:-1] + (-1, 32)) * scale[..., None]).reshape(codes.shape)


def v_values(codes, scale):
    return VALUES[codes] * scale[..., None]


def group_bytes(d):
    return -(-(33 * d + 64) // 128) * 128


def put_token(group, r, k_codes, k_byte, v_codes, v_scale):
    """Token r of one group (uint8 array of group_bytes(d)) for one KV head."""
    d = len(k_codes)
    for c in range(0, d, 2):
        group[c // 32 * 512 + r * 16 + c % 32 // 2] = k_codes[c] | k_codes[c + 1] << 4
    for c in range(d):
        if c // 16 % 2 == 0:
            group[16 * d + c // 64 * 1024 + r // 4 % 4 * 256 + c % 16 * 16 + c // 32 % 2 * 8 + r // 16 * 4 + r % 4] = v_codes[c] | v_codes[c + 16] << 4
    for b in range(d // 32):
        group[32 * d + b * 32 + r % 16 * 2 + r // 16] = k_byte[b]
    bits = 0x7FC0 if math.isnan(v_scale) else int(np.float32(v_scale).view(np.uint32)) >> 16
    at = 33 * d + 2 * (r // 4 % 4 * 8 + r // 16 * 4 + r % 4)
    group[at], group[at + 1] = bits & 255, bits >> 8


def append(pages, table, lengths, offsets, page, hkv, k, v, max_length, rope_base=None):
    """pages [n_pages, page bytes] uint8, changed in place; k, v [tokens, hkv, d] float64; returns nothing.  Positions behind max_length, the table
    or on pages that do not exist are left out."""
    d = k.shape[-1]
    size = group_bytes(d)
    for s in range(len(lengths)):
        for t in range(offsets[s], offsets[s + 1]):
            p = lengths[s] + t - offsets[s]
            if p >= max_length or p // page >= table.shape[1] or not 0 <= table[s, p // page] < len(pages):
                continue
            row = rotate(k[t:t + 1], [p], rope_base)[0] if rope_base else k[t]
            kc, kb = quantise_k(row)
            vc, vs = quantise_v(v[t])
            for h in range(hkv):
                at = (h * (page // 32) + p % page // 32) * size
                put_token(pages[table[s, p // page], at:at + size], p % 32, kc[h], kb[h], vc[h], vs[h])


def norm_rope(x, weight, eps, norm, positions, base):
    """x [tokens, heads, d] float64."""
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if weight is None else weight)
    return rotate(x, positions, base) if positions is not None else x


def attend(q, k, v, seen, scale):
    """q [rows, d], k, v [keys, d], seen [rows, keys] -> output and the sums that bound its error: sum p |v| and the largest logit
    error per unit of relative error of a product."""
    s = (q @ k.T) * scale
    s = np.where(seen, s, -math.inf)
    top = s.max(-1, keepdims=True) if s.shape[1] else np.full((len(q), 1), -math.inf)
    p = np.exp(s - np.where(np.isfinite(top), top, 0.0))
    p = np.where(seen, p, 0.0)
    total = p.sum(-1, keepdims=True)
    p = p / np.where(total == 0, 1.0, total)
    spread = np.where(seen, (np.abs(q) @ np.abs(k).T) * scale, 0.0).max(-1, initial=0.0)
    with np.errstate(invalid="ignore"):
        return np.where(seen.any(-1, keepdims=True), p @ np.where(seen.any(0)[:, None], v, 0.0), 0.0), p @ np.abs(np.where(seen.any(0)[:, None], v, 0.0)), spread


def attend_tolerance(dtype, out, weighted, spread, d, keys):
    """How far an output may be off: its own rounding; the rounding of every probability to the products' type (bf16: 2^-8; fp32: 2^-24); the
    relative error of a probability from its logit (a sum of d products in 32 bits, its scaling: d + 4 roundings of the
    terms' size, for the probability and its part of the sum) and its exponential (2^-22); the sum over the keys in 32 bits."""
    u = 2.0 ** -24
    logit = (d + 4) * u * spread
    rel = HALF_STEP[dtype] + 2.0 * (logit + 2.0 ** -22) + (keys + 8) * u
    return HALF_STEP[dtype] * np.abs(out) + rel[:, None] * weighted * 1.01 + 1e-30
