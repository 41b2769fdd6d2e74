"""Float64 CPU oracle for what follows the compression: rotary positions, the cache, attention over a shared prefix and the cache, eviction.
TEST INFRASTRUCTURE ONLY: shares no code with the HIP library and never imports it.

Everything is numpy float64, one sequence and one head at a time, each function its definition:
  * rotary positions: pair (a, b) of a row, as the complex number a + i b, times exp(i pos theta);
  * a cache holds, per sequence and key/value head, rows of keys and values in slots, with the position and the weight of each; slots 0 .. n-1 are
    in use; the rows of a call are its last ones;
  * attention: row t of m sees every key of the prefix and the slots 0 .. n - m + t; a row that sees nothing is zero; the weight of a slot
    grows by the probabilities of all rows of the heads that share it;
  * eviction: protected slots (position below `sink`, or above newest - recent) before the others, these by weight descending (NaN last), equal
    ones by slot; the first `budget` stay.  Those in slots below the budget stay where they are, the others take the freed slots, both in
    ascending order.
"""
import numpy as np

PLAIN, LINEAR, BASE, BANDS = 0, 1, 2, 3


def rope_theta(r, base=10000.0, scaling=PLAIN, factor=1.0, original_len=0, low=0.0, high=0.0):
    k = np.arange(r // 2, dtype=np.float64)
    if scaling == BASE:
        base = base * factor ** (r / (r - 2.0))
    theta = float(base) ** (-2.0 * k / r)
    if scaling == LINEAR:
        theta = theta / factor
    if scaling == BANDS:
        turns = original_len * theta / (2.0 * np.pi)
        g = np.clip((turns - low) / (high - low), 0.0, 1.0)
        theta = theta * (g + (1.0 - g) / factor)
    return theta


def rope_tables(pos, theta, magnitude=1.0):
    angle = np.asarray(pos, np.float64)[..., None] * theta
    return magnitude * np.cos(angle), magnitude * np.sin(angle)


def rope_apply(x, cos, sin, interleaved=False, transposed=False):
    """x [..., d]; cos, sin [..., r/2] of the same rows."""
    y = np.array(x, np.float64)
    r = 2 * cos.shape[-1]
    a = slice(0, r, 2) if interleaved else slice(0, r // 2)
    b = slice(1, r, 2) if interleaved else slice(r // 2, r)
    z = (y[..., a] + 1j * y[..., b]) * (cos + 1j * (-sin if transposed else sin))
    y[..., a], y[..., b] = z.real, z.imag
    return y


def append(K, V, slot_pos, weight, k, v, pos, n):
    """Rows k, v [heads, m, d] at positions pos [m] become the last of the n slots in use of K, V [heads, capacity, d], in place."""
    m = k.shape[1]
    for t in range(m):
        s = n - m + t
        if 0 <= s < K.shape[1]:
            K[:, s], V[:, s], slot_pos[:, s], weight[:, s] = k[:, t], v[:, t], pos[t], 0.0


def attention(q, K, V, n, m, Kp=None, Vp=None, scale=None):
    """One sequence: q [heads, T, d], K, V [kv_heads, capacity, d], Kp, Vp [kv_heads, P, d].  Returns (O [T, heads, d], what the weights
    [kv_heads, capacity] grow by)."""
    H, T, d = q.shape
    Hk, cap, _ = K.shape
    O, W = np.zeros((T, H, d)), np.zeros((Hk, cap))
    P = 0 if Kp is None else Kp.shape[1]
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    for h in range(H):
        j = h // (H // Hk)
        for t in range(m):
            end = min(max(n - m + t + 1, 0), n)
            if P + end == 0:
                continue
            keys = K[j, :end] if P == 0 else np.concatenate([Kp[j], K[j, :end]])
            vals = V[j, :end] if P == 0 else np.concatenate([Vp[j], V[j, :end]])
            s = scale * (keys @ q[h, t])
            p = np.exp(s - s.max())
            p /= p.sum()
            O[t, h] = p @ vals
            W[j, :end] += p[P:]
    return O, W


def evict(slot_pos, weight, n, budget, sink, recent):
    """One sequence and head: where the rows of the first min(n, budget) slots come from."""
    newest = max((int(x) for x in slot_pos[:n]), default=0)

    def order(s):
        safe = int(slot_pos[s]) < sink or int(slot_pos[s]) > newest - recent
        w = float(weight[s])
        return (not safe, 0.0 if safe else (np.inf if w != w else -w), s)

    kept = set(sorted(range(n), key=order)[:budget])
    freed = [s for s in range(min(n, budget)) if s not in kept]
    moved = sorted(s for s in kept if s >= budget)
    source = list(range(min(n, budget)))
    for to, come in zip(freed, moved):
        source[to] = come
    return source
