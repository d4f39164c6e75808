"""Plain definitions of the group-scaled 4-bit layers and of the operators on tokens sorted by expert, in numpy: quantizers in fp32, one
IEEE operation a step (they are compared bit for bit), everything else in 64 bits.  Shares nothing with the library."""
from __future__ import annotations

import numpy as np

SYM, ZERO = 0, 1


def round_to(x, scale_type: str):
    """fp32 -> fp32 value of the nearest fp16 / bf16 number, ties to even, overflow to the largest finite one."""
    x = np.asarray(x, np.float32)
    if scale_type == "f16":
        return np.minimum(x, np.float32(65504)).astype(np.float16).astype(np.float32)
    x = np.minimum(x, np.float32(3.3895313892515355e38))
    b = x.view(np.uint32).astype(np.uint64)
    return (((b + 0x7FFF + ((b >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32)


def quantize(W, group: int, mode: int, scale_type: str):
    """W [..., M, K] fp32 -> codes uint8 [..., M, K], scales fp32 [..., M, G], zeros uint8 [..., M, G]."""
    W = np.asarray(W, np.float32)
    K = W.shape[-1]
    G = -(-K // group)
    codes = np.empty(W.shape, np.uint8)
    scale = np.empty(W.shape[:-1] + (G,), np.float32)
    zero = np.full(W.shape[:-1] + (G,), 8, np.uint8)
    for g in range(G):
        w = W[..., g * group:(g + 1) * group]
        lo, hi = np.minimum(w.min(-1), 0), np.maximum(w.max(-1), 0)
        s = round_to(np.maximum(hi, -lo) / np.float32(7) if mode == SYM else (hi - lo) / np.float32(15), scale_type)
        safe = np.where(s > 0, s, np.float32(1))
        q = np.rint((w / safe[..., None]).astype(np.float32))
        if mode == SYM:
            u = 8 + np.clip(q, -7, 7)
        else:
            z = np.where(s > 0, np.clip(np.rint((-lo / safe).astype(np.float32)), 0, 15), 0).astype(np.float32)
            u = np.clip(q + z[..., None], 0, 15)
            zero[..., g] = z.astype(np.uint8)
        codes[..., g * group:(g + 1) * group] = np.where(s[..., None] > 0, u, zero[..., g, None]).astype(np.uint8)
        scale[..., g] = s
    return codes, scale, zero


def weights(codes, scale, zero, group: int):
    at = np.arange(codes.shape[-1]) // group
    return (codes.astype(np.float64) - zero.astype(np.float64)[..., at]) * scale.astype(np.float64)[..., at]


def product(W, x):
    """([N, M] y, [N, M] sums of the absolute products, which rounding errors go by)."""
    x = np.asarray(x, np.float64)
    return x @ W.T, np.abs(x) @ np.abs(W).T


def sort_pairs(ids, E: int):
    T, k = ids.shape
    flat = ids.reshape(-1)
    lists = [[] for _ in range(E)]
    for i, e in enumerate(flat):
        if 0 <= e < E:
            lists[e].append(i)
    offsets = np.cumsum([0] + [len(q) for q in lists]).astype(np.int32)
    order = [i for q in lists for i in q]
    rows = np.full(T * k, -1, np.int32)
    place = np.full(T * k, -1, np.int32)
    rows[:len(order)] = np.asarray(order, np.int32) // k
    place[order] = np.arange(len(order), dtype=np.int32)
    return offsets, rows, place.reshape(T, k)


def combine(ys, place, w):
    """w None: ones.  Returns (y, sums of absolute terms)."""
    ys = np.asarray(ys, np.float64)
    T, k = place.shape
    y, a = np.zeros((T, ys.shape[1])), np.zeros((T, ys.shape[1]))
    for t in range(T):
        for j in range(k):
            p = place[t, j]
            if 0 <= p < ys.shape[0]:
                term = (1.0 if w is None else float(w[t, j])) * ys[p]
                y[t] += term
                a[t] += np.abs(term)
    return y, a


def combine_backward(dy, ys, place, w):
    """(dys [R][H] with NaN in rows that no pair has, dw [T][k], sums of absolute terms of dw)."""
    dy, ys = np.asarray(dy, np.float64), np.asarray(ys, np.float64)
    T, k = place.shape
    dys = np.full(ys.shape, np.nan)
    dw, a = np.zeros((T, k)), np.zeros((T, k))
    for t in range(T):
        for j in range(k):
            p = place[t, j]
            if 0 <= p < ys.shape[0]:
                dys[p] = (1.0 if w is None else float(w[t, j])) * dy[t]
                dw[t, j] = dy[t] @ ys[p]
                a[t, j] = np.abs(dy[t]) @ np.abs(ys[p])
    return dys, dw, a
