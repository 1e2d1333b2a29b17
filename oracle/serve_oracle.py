"""Float64 definitions of the serving operators (numpy, sharing no code with the GPU path): rotary positions, a paged key-value cache as
a dictionary from (sequence, position) to a place, attention over it, and verification from given probabilities.  Each also gives
what its result's error can be measured by (`scale` of a sum of products)."""
from __future__ import annotations

import math
from typing import List, Optional, Tuple

import numpy as np


def rope_frequencies(theta: float, rot: int, scaling: str = "plain", factor: float = 1.0, low: float = 0.0, high: float = 0.0,
                     original: float = 0.0) -> np.ndarray:
    """Angle per position of pairs 0 .. rot/2 - 1."""
    out = []
    for i in range(rot // 2):
        f = float(theta) ** (-2.0 * i / rot)
        if scaling == "linear":
            f /= factor
        elif scaling == "bands":
            turns = original * f / (2 * math.pi)
            if turns <= low:
                f /= factor
            elif turns < high:
                w = (turns - low) / (high - low)
                f = w * f + (1 - w) * f / factor
        elif scaling == "ramp":
            at = lambda turns: rot * math.log(original / (2 * math.pi * turns)) / (2 * math.log(theta))
            i0, i1 = max(math.floor(at(high)), 0), min(math.ceil(at(low)), rot - 1)
            w = min(max((i - i0) / max(i1 - i0, 1e-3), 0.0), 1.0)
            f = (1 - w) * f + w * f / factor
        out.append(f)
    return np.array(out)


def rotate(x: np.ndarray, positions: np.ndarray, freq: np.ndarray, layout: str, magnitude: float = 1.0) -> Tuple[np.ndarray, np.ndarray]:
    """x [..][H][D] at positions [..]; (result, |a| + |b| of the pair every element comes from)."""
    rot = 2 * len(freq)
    y, size = np.array(x, dtype=np.float64), np.abs(np.array(x, dtype=np.float64))
    first = np.arange(rot // 2) if layout == "half" else np.arange(0, rot, 2)
    second = first + (rot // 2 if layout == "half" else 1)
    angle = np.asarray(positions, dtype=np.float64)[..., None, None] * freq
    c, s = np.cos(angle) * magnitude, np.sin(angle) * magnitude
    a, b = y[..., first].copy(), y[..., second].copy()
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    size[..., first] = size[..., second] = (np.abs(a) + np.abs(b)) * magnitude
    return y, size


def place(table: np.ndarray, n_pages: int, page_size: int, b: int, slot: int) -> Optional[Tuple[int, int]]:
    """(page, position in it) of a slot, None where it has none."""
    if slot < 0 or slot // page_size >= table.shape[1]:
        return None
    page = int(table[b, slot // page_size])
    return (page, slot % page_size) if 0 <= page < n_pages else None


def attend(q: np.ndarray, keys: List[np.ndarray], values: List[np.ndarray], scale: float):
    """q [Hq][D] over a list of keys [Hkv][D] and values: (output [Hq][D], sum_j p_j |v_j|, lse [Hq], largest scale sum_d |q_d k_d|)."""
    hq, d = q.shape
    if not keys:
        return np.zeros((hq, d)), np.zeros((hq, d)), np.full(hq, -np.inf), 0.0
    k, v = np.stack(keys).astype(np.float64), np.stack(values).astype(np.float64)       # [n][Hkv][D]
    group = hq // k.shape[1]
    with np.errstate(invalid="ignore", over="ignore"):
        out, size, lse, most = [], [], [], 0.0
        for h in range(hq):
            kk, vv = k[:, h // group], v[:, h // group]
            s = scale * (kk @ q[h].astype(np.float64))
            most = max(most, float((abs(scale) * (np.abs(kk) @ np.abs(q[h].astype(np.float64)))).max()))
            m = s.max()
            p = np.exp(s - m)
            lse.append(m + math.log(p.sum()))
            p = p / p.sum()
            out.append(p @ vv)
            size.append(p @ np.abs(vv))
    return np.array(out), np.array(size), np.array(lse), most


def verify_probs(target: np.ndarray, draft: Optional[np.ndarray], spec: np.ndarray, u_accept: np.ndarray, u_bonus: float,
                 drafted: Optional[int] = None) -> Tuple[int, int]:
    """One sequence: target [K+1][V], draft [K][V] or None (certain tokens), spec and u_accept [K]: (accepted tokens, bonus)."""
    K, V = len(spec), target.shape[1]
    n = K if drafted is None else min(max(int(drafted), 0), K)

    def one_hot(t):
        z = np.zeros(V)
        z[t] = 1.0
        return z

    k = 0
    while k < n:
        t = int(spec[k])
        if not 0 <= t < V:
            break
        q = 1.0 if draft is None else float(draft[k, t])
        if not float(u_accept[k]) * q < float(target[k, t]):
            break
        k += 1

    def clean(x):
        return np.where((x > 0) & np.isfinite(x), x, 0.0)

    p = target[k].astype(np.float64)
    with np.errstate(invalid="ignore"):
        if k < n and draft is not None:
            mass = clean(p - draft[k].astype(np.float64))
        elif k < n and 0 <= int(spec[k]) < V:
            mass = clean(np.where(one_hot(int(spec[k])) > 0, 0.0, p))
        else:
            mass = clean(p)
    if not mass.sum() > 0:
        mass = clean(p)
    total = math.fsum(mass)
    if not total > 0:
        return k, -1
    u = float(u_bonus)
    u = min(u, 1.0 - 2.0 ** -24) if u > 0 else 0.0
    upto = np.cumsum(mass)
    hit = np.flatnonzero((upto > u * upto[-1]) & (mass > 0))
    return k, int(hit[0]) if len(hit) else int(np.flatnonzero(mass > 0)[-1])
