"""Oracle of the operators of a layer held in 8 bits (include/spec_layer8.h), in numpy float64, from their definitions."""
from __future__ import annotations

import math

import numpy as np

EXP_LEAST = -100


def exponent(block: np.ndarray) -> int:
    """The least e >= -100 with amax <= 448 * 2^e, amax over the block's finite values."""
    a = np.abs(block[np.isfinite(block)])
    amax = float(a.max()) if a.size else 0.0
    e = EXP_LEAST
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return e


def e4m3(x: np.ndarray) -> np.ndarray:
    """Values rounded to the grid of e4m3 (|x| <= 448), ties to even; what is not finite becomes NaN."""
    with np.errstate(invalid="ignore"):
        step = np.exp2(np.maximum(np.frexp(x)[1] - 1, -6).astype(np.float64) - 3)
        return np.where(np.isfinite(x), np.round(x / step) * step, np.nan)   # (np.round: ties to even)


def held(block: np.ndarray) -> np.ndarray:
    """What the 8-bit form of one block stands for."""
    b = np.asarray(block, dtype=np.float64)
    e = exponent(b)
    return e4m3(b * 2.0 ** -e) * 2.0 ** e


def held_rows(x: np.ndarray) -> np.ndarray:
    """[rows, in], a block per row and 128 of in."""
    x = np.asarray(x, dtype=np.float64)
    out = np.empty_like(x)
    for i in range(x.shape[0]):
        for c in range(0, x.shape[1], 128):
            out[i, c:c + 128] = held(x[i, c:c + 128])
    return out


def gemm8(x: np.ndarray, w: np.ndarray) -> np.ndarray:
    return held_rows(x) @ held_rows(w).T


def held_kv(k: np.ndarray, hkv: int, hd: int) -> np.ndarray:
    """[64 n, hkv * hd], a block per 64 tokens and head."""
    x = np.asarray(k, dtype=np.float64).reshape(-1, 64, hkv, hd)
    out = np.empty_like(x)
    for b in range(x.shape[0]):
        for h in range(hkv):
            out[b, :, h] = held(x[b, :, h])
    return out.reshape(-1, hkv * hd)


def seen(i: int, base: int, n8: int, depth, anc, win_rows: int):
    """What row i attends to: a list of (in the blocks?, row)."""
    if depth[i] < 0:
        return None
    out = []
    for p in range(base + depth[i] + 1):
        if p < n8:
            out.append((True, p))
            continue
        r = p - n8 if p < base or anc is None else base - n8 + int(anc[i][p - base])
        if 0 <= r < win_rows:
            out.append((False, r))
    return out


def attention8(q, k8, v8, kwin, vwin, base, depth, anc, hq, hkv, hd):
    """k8, v8: the blocks' values [n8, hkv * hd] (after held_kv).  Returns (out [rows, hq * hd], NaN for padding rows; spread: the sum of
    weight * |value| of each output; delta: the largest sum |q| |k| / sqrt(hd) over the keys of each row and head; qk: the same with max |q|)."""
    rows, n8 = q.shape[0], k8.shape[0]
    out = np.full((rows, hq, hd), np.nan)
    spread, delta, qk = np.zeros((rows, hq, hd)), np.zeros((rows, hq, 1)), np.zeros((rows, hq, 1))
    ks = np.concatenate([k8, np.asarray(kwin, np.float64)]).reshape(-1, hkv, hd)
    vs = np.concatenate([v8, np.asarray(vwin, np.float64)]).reshape(-1, hkv, hd)
    for i in range(rows):
        at = seen(i, base, n8, depth, anc, kwin.shape[0])
        if at is None:
            continue
        idx = np.array([r if blocks else n8 + r for blocks, r in at], dtype=np.int64)
        for h in range(hq):
            if idx.size == 0:
                out[i, h] = 0.0
                continue
            kk, vv, qq = ks[idx, h * hkv // hq], vs[idx, h * hkv // hq], np.asarray(q[i].reshape(hq, hd)[h], np.float64)
            s = kk @ qq / math.sqrt(hd)
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h], spread[i, h] = p @ vv, p @ np.abs(vv)
            delta[i, h] = (np.abs(kk) @ np.abs(qq)).max() / math.sqrt(hd)
            qk[i, h] = np.abs(kk).sum(1).max() * np.abs(qq).max() / math.sqrt(hd)
    return out.reshape(rows, -1), spread.reshape(rows, -1), np.repeat(delta, hd, 2).reshape(rows, -1), np.repeat(qk, hd, 2).reshape(rows, -1)


def rope_frequencies(rot, theta, scaling="none", factor=1.0, trained_len=0, low_freq=1.0, high_freq=4.0, beta_fast=32.0, beta_slow=1.0):
    """(frequencies [rot / 2] in radians per position, mscale)."""
    f = np.array([theta ** (-2.0 * j / rot) for j in range(rot // 2)])
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "llama3":
        out = []
        for w in f:
            turns = trained_len * w / (2 * math.pi)
            if turns >= high_freq:
                out.append(w)
            elif turns <= low_freq:
                out.append(w / factor)
            else:
                s = (turns - low_freq) / (high_freq - low_freq)
                out.append((1 - s) * w / factor + s * w)
        return np.array(out), 1.0
    if scaling == "yarn":
        def place(times):
            return rot * math.log(trained_len / (times * 2 * math.pi)) / (2 * math.log(theta))
        lo, hi = max(math.floor(place(beta_fast)), 0), min(math.ceil(place(beta_slow)), rot - 1)
        ramp = np.clip((np.arange(rot // 2) - lo) / max(hi - lo, 0.001), 0, 1)
        return f * (1 - ramp) + f / factor * ramp, 0.1 * math.log(factor) + 1
    return f, 1.0


def rotary(x, pos, freq, mscale, rot, layout, adjoint=False):
    """x [rows, heads, hd] at positions pos [rows]."""
    x = np.array(x, dtype=np.float64)
    t = np.asarray(pos, np.float64)[:, None] * np.asarray(freq)[None]
    c, s = np.cos(t)[:, None] * mscale, np.sin(t)[:, None] * (-mscale if adjoint else mscale)
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    u, v = x[..., a].copy(), x[..., b].copy()
    x[..., a], x[..., b] = u * c - v * s, v * c + u * s
    return x
