"""The operators around the cache in plain numpy, in 64 bits, from their formulas: what the GPU tests compare with."""
import math

import numpy as np

import lamps_workloads as W


def f64(a):
    """Arrays of the workloads (float32, or uint16 bf16 bits) as float64."""
    return (W.bf16_bits_to_f32(a) if a.dtype == np.uint16 else a).astype(np.float64)


def seen(p, count, window, sinks):
    """Which of positions 0 .. count - 1 the token at position p sees."""
    t = np.arange(count)
    return (t <= p) & ((t > p - window) | (t < sinks))


def window_attn(q, K, V, first, window, sinks, scale=None):
    """q [n][H][D] at positions first and up over K, V [C][H_kv][D]: outputs, and the sums of weight times |value| that a rounding of
    the weights is scaled by."""
    n, H, D = q.shape
    G = H // K.shape[1]
    scale = scale or 1.0 / math.sqrt(D)
    out, size = np.zeros((n, H, D)), np.zeros((n, H, D))
    for i in range(n):
        on = seen(first + i, K.shape[0], window, sinks)
        if not on.any():
            continue
        k, v = K[on], V[on]
        for h in range(H):
            s = k[:, h // G] @ q[i, h] * scale
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h] = w @ v[:, h // G]
            size[i, h] = w @ np.abs(v[:, h // G])
    return out, size


def turned(x, p, freq, neighbours=False, amplitude=1.0, eps=None, weight=None):
    """Heads x [..][D] at positions p (an array of x's leading shape but the heads)."""
    x = x.copy()
    if eps is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if weight is not None:
            x = x * weight
    n = 2 * len(freq)
    if n:
        a, b = (x[..., 0:n:2].copy(), x[..., 1:n:2].copy()) if neighbours else (x[..., :n // 2].copy(), x[..., n // 2:n].copy())
        u = np.asarray(p, dtype=np.float64)[..., None, None] * np.asarray(freq)
        ya, yb = amplitude * (a * np.cos(u) - b * np.sin(u)), amplitude * (a * np.sin(u) + b * np.cos(u))
        if neighbours:
            x[..., 0:n:2], x[..., 1:n:2] = ya, yb
        else:
            x[..., :n // 2], x[..., n // 2:n] = ya, yb
    return x


def tables(cached, new, ids, grow, table, block_size, total):
    """Table, lengths, first rows, slots and report of a batch, request by request."""
    table, row = table.copy(), table.shape[1] * block_size
    ctx, start, slots, taken, at, lost, counted, stop = [], [0], [], 0, 0, [], 0, False
    for r, (a, b) in enumerate(zip(cached, new)):
        good = a >= 0 and b >= 0 and a + b <= row
        held = -(-a // block_size) if good and grow else 0
        need = -(-(a + b) // block_size) - held if good else 0
        first, at = at, at + need
        served = good and (need == 0 or at <= len(ids))
        if served:
            counted += b
            if b and counted > total:
                served = False
        if not served:
            lost.append(r)
            ctx.append(0)
            start.append(start[-1])
            continue
        table[r, held:held + need] = ids[first:first + need]
        table[r, held + need:] = -1
        taken += need
        ctx.append(a + b)
        start.append(start[-1] + b)
        slots += [(int(table[r, p // block_size]), p % block_size) for p in range(a, a + b)]
    return table, ctx, start, slots, [taken, len(lost), lost[0] if lost else -1, start[-1]]
