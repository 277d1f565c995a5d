"""Plain 64-bit forms of the operators around the generation step, on the host.  The generation step itself is compared with
the oracle, which is given the rows that a 4-bit cache stands for."""
from __future__ import annotations

import math

import numpy as np

GROUP = 32


def half_down(x):
    """The largest binary16 number not above x >= 0 (float64 array)."""
    h = x.astype(np.float16)
    over = h.astype(np.float64) > x
    return np.where(over, np.nextafter(h, np.float16(-np.inf)), h).astype(np.float16)


def pack_rows(x):
    """float16 [..., d] -> (codes uint8 [..., d], scale float16 [..., d/32], minimum float16 [..., d/32])."""
    g = x.astype(np.float32).reshape(*x.shape[:-1], -1, GROUP)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        low, high = g.min(-1), g.max(-1)                    # NaN wins
        span = (high - low).astype(np.float32)
        ok = np.isfinite(span)
        scale = np.where(ok, half_down((np.where(ok, span, 0) / np.float32(15)).astype(np.float32)), np.float16(np.nan)).astype(np.float16)
        inverse = np.where(scale > 0, np.float32(1) / scale.astype(np.float32), np.float32(0)).astype(np.float32)
        code = np.rint((g - low[..., None]) * inverse[..., None])
        code = np.clip(np.where(ok[..., None], code, 0), 0, 15).astype(np.uint8)
        low = np.where(ok, low, np.float32(np.nan)).astype(np.float16)
    return code.reshape(x.shape), scale, low


def slots_of(K, V):
    """float16 K, V [..., d] -> slots uint8 [..., 5d/4]."""
    parts = []
    packed = [pack_rows(K), pack_rows(V)]
    for code, _, _ in packed:
        parts.append(code[..., 0::2] | (code[..., 1::2] << 4))
    for _, scale, low in packed:
        parts.append(np.ascontiguousarray(np.stack([scale, low], -1).reshape(*scale.shape[:-1], -1)).view(np.uint8))
    return np.concatenate(parts, -1)


def rows_of(slots, d):
    """Slots uint8 [..., 5d/4] -> float16 K, V [..., d]: code * scale + minimum, rounded once."""
    out = []
    for i in range(2):
        codes = slots[..., i * d // 2:(i + 1) * d // 2]
        code = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], d // GROUP, GROUP)
        params = np.ascontiguousarray(slots[..., d + i * d // 8:d + (i + 1) * d // 8]).view(np.float16).reshape(*codes.shape[:-1], d // GROUP, 2)
        with np.errstate(invalid="ignore", over="ignore"):
            value = code.astype(np.float64) * params[..., :1].astype(np.float64) + params[..., 1:].astype(np.float64)
            out.append(value.astype(np.float16).reshape(*codes.shape[:-1], d))
    return out


def norm_rotate(x, n_heads, n_kv, d, positions, qw, kw, norm, eps, R, base, halves):
    """x float64 [B, n, (H + 2 Hkv) d] -> q, k, v float64, head-major."""
    B, n, _ = x.shape
    x = x.reshape(B, n, n_heads + 2 * n_kv, d).transpose(0, 2, 1, 3).copy()
    for part, w in ((slice(0, n_heads), qw), (slice(n_heads, n_heads + n_kv), kw)):
        if norm:
            x[:, part] *= (1.0 if w is None else w) / np.sqrt((x[:, part] ** 2).mean(-1, keepdims=True) + eps)
        for i in range(R // 2):
            a, b = (i, i + R // 2) if halves else (2 * i, 2 * i + 1)
            # whole turns are taken off in extended precision
            turns = positions.astype(np.longdouble) * np.longdouble(base) ** (np.longdouble(-2 * i) / R) / (2 * np.longdouble("3.14159265358979323846264338"))
            angle = ((turns - np.rint(turns)) * 2).astype(np.float64) * math.pi
            c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
            xa, xb = x[:, part, :, a].copy(), x[:, part, :, b].copy()
            x[:, part, :, a], x[:, part, :, b] = xa * c - xb * s, xa * s + xb * c
    return x[:, :n_heads], x[:, n_heads:n_heads + n_kv], x[:, n_heads + n_kv:]


def beam_values(logits, scores, finished, pad):
    """logits float64 [beams, V], scores float64 [beams] of one request -> float64 [beams * V]."""
    out = np.full(logits.shape, -np.inf)
    for w in range(logits.shape[0]):
        if not np.isfinite(scores[w]):
            continue
        if finished is not None and finished[w]:
            out[w, pad] = scores[w]
            continue
        x = np.where(np.isfinite(logits[w]), logits[w], -np.inf)
        if np.isfinite(x.max()):
            out[w] = scores[w] + (x - x.max() - math.log(np.exp(x - x.max()).sum()))
    return out.reshape(-1)
