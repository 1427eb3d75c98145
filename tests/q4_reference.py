"""Plain fp64 restatements of the 4-bit cache, of attention over it and of eviction (tests only, no code of the CUDA path)."""
from __future__ import annotations

import numpy as np

GROUP = 32


def frequencies(d, base=10000.0):
    i = np.arange(d // 2)
    axis = i % 3
    n_axis = np.array([(axis == a).sum() for a in range(3)])
    return axis, base ** (-(i // 3) / n_axis[axis])


def turn(x, pos, shift=0, sign=1.0):
    """x [n][heads][d] turned by the rotary embedding at (t + shift, h, w), as complex numbers"""
    x = np.asarray(x, np.float64)
    axis, freq = frequencies(x.shape[-1])
    p = np.asarray(pos)[:, :3].astype(np.float64)
    p = p + np.array([shift, 0, 0])
    z = (x[..., 0::2] + 1j * x[..., 1::2]) * np.exp(1j * sign * p[:, axis] * freq)[:, None, :]
    out = np.empty_like(x)
    out[..., 0::2], out[..., 1::2] = z.real, z.imag
    return out


def quantise(x):
    """(codes [..., d], steps, lows [..., d / 32] as fp64) of rows in fp64"""
    g = np.clip(np.nan_to_num(np.asarray(x, np.float64), nan=0.0, posinf=np.inf, neginf=-np.inf), -65504.0, 65504.0)
    g = g.reshape(*x.shape[:-1], -1, GROUP)
    low = g.min(-1).astype(np.float16).astype(np.float64)
    step = ((g.max(-1) - low) / 15.0).astype(np.float16).astype(np.float64)
    c = np.divide(g - low[..., None], step[..., None], out=np.zeros_like(g), where=step[..., None] > 0)
    return np.clip(np.rint(c), 0, 15).reshape(x.shape), step, low


def decode(rows, d):
    """Rows as they lie in memory, [n][Hkv * 5 d / 4] bytes -> two (codes, steps, lows), of keys and of values"""
    rows = np.ascontiguousarray(rows)
    n = len(rows)
    hkv, ng = rows.shape[1] * 4 // (5 * d), d // GROUP
    sl = np.ascontiguousarray(rows[:, hkv * d:]).view(np.float16).astype(np.float64).reshape(n, hkv, 4, ng)
    out = []
    for kv in range(2):
        byte = rows[:, kv * hkv * d // 2:(kv + 1) * hkv * d // 2].reshape(n, hkv, d // 2)
        nib = np.empty((n, hkv, d), np.uint8)
        nib[..., 0::2], nib[..., 1::2] = byte & 15, byte >> 4                                     # nibbles in memory order
        if kv == 0:
            codes = nib.reshape(n, hkv, 4, ng, 8).transpose(0, 1, 3, 2, 4)                    # word (t, g) = channels 32 g + 8 t ..
        else:
            codes = nib                                                                       # channel by channel
        out.append((codes.reshape(n, hkv, d).astype(np.float64), sl[:, :, 2 * kv], sl[:, :, 2 * kv + 1]))
    return out


def values(q):
    c, step, low = q
    return (low[..., None] + step[..., None] * c.reshape(*c.shape[:-1], c.shape[-1] // GROUP, GROUP)).reshape(c.shape)


def spread(q):
    """Channel by channel, what a sum over codes and a sum over lows are made of: step * code + |low|"""
    c, step, low = q
    return (np.abs(low)[..., None] + step[..., None] * c.reshape(*c.shape[:-1], c.shape[-1] // GROUP, GROUP)).reshape(c.shape)


def attend(q, q_pos, parts, valid=None):
    """parts: [(key codes, value codes, t_shift)] of anchors and history (quantise's triples); valid: of the last part.
    Returns out, lse, the mean probability of every key, and what tolerances are made of: the largest sum |q| (step code + |low|) / sqrt(d)
    of a row's visible keys, and sum p (step code + |low|) of the values."""
    n_q, hq, d = q.shape
    hkv = parts[0][0][0].shape[1]
    g = hq // hkv
    n = [len(p[0][0]) for p in parts]
    out, mag_v = np.zeros((n_q, hq, d)), np.zeros((n_q, hq, d))
    lse, mag_l = np.full((n_q, hq), -np.inf), np.zeros((n_q, hq))
    mass = np.zeros(sum(n))
    ok = np.ones(sum(n), bool)
    if valid is not None:
        ok[sum(n[:-1]):] = np.asarray(valid) != 0
    if ok.any():
        with np.errstate(invalid="ignore"):
            rq = [turn(q, q_pos, sh) for _, _, sh in parts]
            for h in range(hq):
                cat = lambda f, i: np.concatenate([f(p[i])[:, h // g] for p in parts])[ok]          # noqa: E731
                k, v, sk, sv = cat(values, 0), cat(values, 1), cat(spread, 0), cat(spread, 1)
                rows = np.repeat(np.arange(len(parts)), n)[ok]
                x = np.concatenate([r[:, h] @ k[rows == i].T for i, r in enumerate(rq)], 1) / np.sqrt(d)
                m = x.max(1, keepdims=True)
                e = np.exp(x - m)
                p = e / e.sum(1, keepdims=True)
                out[:, h], mag_v[:, h] = p @ v, p @ sv
                lse[:, h] = m[:, 0] + np.log(e.sum(1))
                mag_l[:, h] = max((np.abs(r[:, h]) @ sk[rows == i].T).max() if (rows == i).any() else 0.0 for i, r in enumerate(rq)) / np.sqrt(d)
                mass[ok] += p.sum(0)
    return out, lse, mass / (n_q * hq), mag_l, mag_v


def evict(weight, keep, recent, valid=None):
    n = len(weight)
    keep = min(keep, n)
    recent = min(recent, keep)
    old = n - recent
    w = np.asarray(weight[:old], np.float64) + 0.0
    masked = np.zeros(old, bool) if valid is None else np.asarray(valid[:old]) == 0
    w = np.where(masked, 0.0, w)
    best = np.lexsort((np.arange(old), -w, masked))[: keep - recent]
    return np.concatenate([np.sort(best), np.arange(old, n)]).astype(np.int32)
