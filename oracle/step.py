"""Oracle for the rest of a decode step around the 8-bit paged cache, in float64: heads normed
and rotated with their gradient, attention added up for each token, eviction by it, sampling.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``).
"""
from __future__ import annotations

import math
from typing import Optional, Sequence, Tuple

import numpy as np

from . import kv8, rope


def norm_mrope(x, weight, positions, sections, theta, eps, order="sectioned", pairing="halves") -> np.ndarray:
    """R (x r w) of rows [rows][heads][d], r = 1 / sqrt(mean x^2 + eps)."""
    x = np.asarray(x, np.float64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return rope.rotate(x * r * np.asarray(weight, np.float64), positions, sections, theta, order, pairing)


def norm_mrope_grad(x, dy, weight, positions, sections, theta, eps, order="sectioned",
                    pairing="halves") -> Tuple[np.ndarray, np.ndarray]:
    """(dx, dw) for the output's gradient dy."""
    x, w = np.asarray(x, np.float64), np.asarray(weight, np.float64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r
    g = rope.rotate(np.asarray(dy, np.float64), positions, sections, theta, order, pairing, inverse=True)
    h = g * w
    return r * (h - n * (h * n).mean(-1, keepdims=True)), (g * n).sum((0, 1))


def weigh(codes, scale, table, lens, rows, q, lse, weights, softmax_scale: Optional[float] = None,
          causal: bool = True) -> np.ndarray:
    """weights [n_pages][Hkv][page] after a step: codes, scale of the keys, q [rows][Hq][d], lse [rows][Hq]."""
    n_pages, Hkv, page, d = codes.shape
    G = q.shape[1] // Hkv
    s = 1.0 / math.sqrt(d) if softmax_scale is None else softmax_scale
    out = np.asarray(weights, np.float64).copy()
    K = kv8.VALUE[codes] * scale[:, :, None, None].astype(np.float64)
    at = 0
    for r, (length, m) in enumerate(zip(lens, rows)):
        for g in range(Hkv if length else 0):
            t = np.arange(length)
            ids = np.asarray(table[r])[t // page]
            k = K[ids, g, t % page]
            A = np.zeros(length)
            for i in range(m):
                sees = length - m + i + 1 if causal else length
                if sees <= 0 or m > length and i < m - length:
                    continue
                for j in range(g * G, (g + 1) * G):
                    if lse[at + i, j] != -np.inf:
                        A[:sees] += np.exp(k[:sees] @ np.asarray(q[at + i, j], np.float64) * s - lse[at + i, j])
            was = out[ids, g, t % page]
            out[ids, g, t % page] = np.where(t < length - m, was, 0.0) + A
        at += m
    return out


def evict(codes: Sequence[np.ndarray], scale: Sequence[np.ndarray], table, lens, weights, keep, sink: int, recent: int,
          kept: np.ndarray) -> list:
    """In place on codes, scale (keys, values), weights and kept [n_req][Hkv][max_keep]; returns the new lengths."""
    n_pages, Hkv, page, d = codes[0].shape
    new_lens = []
    for r, length in enumerate(lens):
        new = min(length, keep[r])
        new_lens.append(new)
        for g in range(Hkv):
            t = np.arange(length)
            at = np.asarray(table[r])[t // page], np.full(length, g), t % page
            w = weights[at].astype(np.float64)
            w[np.isnan(w)] = -np.inf
            last = np.isnan(weights[at])                 # behind -inf itself
            w[:sink] = np.inf
            w[max(0, length - recent):] = np.inf
            last[:sink] = False
            last[max(0, length - recent):] = False
            order = sorted(range(length), key=lambda i: (last[i], -w[i], i))
            stay = np.array(sorted(order[:new]), np.int64)
            kept[r, g, :new] = stay
            if new == length:
                continue
            gap = next((i for i, x in enumerate(stay) if i != x), new)
            held = [kv8.VALUE[c[at][stay]] * s[at[0][stay], g][:, None].astype(np.float64) for c, s in zip(codes, scale)]
            moved = weights[at][stay]
            for j in range(gap // page, -(-new // page)):
                a, b, p = j * page, min(new, (j + 1) * page), table[r][j]
                weights[p, g, :b - a] = moved[a:b]
                for x, c, s in zip(held, codes, scale):
                    x = x[a:b]
                    now = kv8.scale_of(float(np.abs(x[np.isfinite(x)]).max(initial=0.0)))
                    c[p, g, :b - a] = kv8.encode(x / (now if now > 0 else 1.0))
                    s[p, g] = now
    return new_lens


def sample(x, u: float, T: float, top_k: int = 0, top_p: float = 1.0, min_p: float = 0.0) -> Tuple[int, float]:
    """(token, logprob) of one row of logits."""
    x = np.asarray(x, np.float64).copy()
    x[np.isnan(x)] = -np.inf
    M = x.max()
    if M == -np.inf:
        return -1, math.nan
    if not T > 0:
        return int(np.argmax(x)), 0.0
    T = max(T, 2.0 ** -127)                                         # (no less counts)
    with np.errstate(invalid="ignore"):
        w = np.where(x == M, 1.0, np.exp((x - M) / T))
    w[(x == -np.inf) | ((M == np.inf) & (x != M))] = 0.0            # whatever T is
    order = np.argsort(-x, kind="stable")
    n = len(x)
    if top_k > 0:
        n = min(n, top_k)
    if top_p < 1:
        c = np.cumsum(w[order[:n]])
        n = min(n, int((c < top_p * c[-1]).sum()) + 1)
    if min_p > 0:
        n = min(n, max(1, int((w >= min(min_p, 1.0)).sum())))
    kept = np.sort(order[:n])
    c = np.cumsum(w[kept])
    u = 0.0 if not u > 0 else u
    i = int((c <= u * c[-1]).sum())
    i = min(i, int(np.flatnonzero(w[kept])[-1]))
    return int(kept[i]), float(np.log(w[kept[i]] / c[-1]))
