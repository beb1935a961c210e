"""Float64 definitions of the operators around the paged cache (numpy, one sequence or one row at a time; no code in common with
the CUDA library).  `positions`, `lens` and tables are plain integer arrays; caches come as lists of [tokens, h_kv, d] arrays."""
from __future__ import annotations

import numpy as np

PI = np.longdouble("3.14159265358979323846264338327950288")     # numpy's own pi is a double


def rotate(x, positions, inv_freq, axis, interleaved=False, inverse=False):
    """x [tokens, heads, d], positions [axes, tokens]: pair i turns by positions[axis[i]] * inv_freq[i]."""
    x = np.asarray(x, dtype=np.float64)
    out = x.copy()
    pairs = len(inv_freq)
    for i in range(pairs):
        # whole turns are taken off in exact integer / long double arithmetic, so that far positions keep their angle
        turns = np.asarray(positions[axis[i]], dtype=np.longdouble) * (np.longdouble(inv_freq[i]) / (2 * PI))
        theta = np.asarray(2 * PI * (turns - np.floor(turns)), dtype=np.float64)
        c, s = np.cos(theta)[:, None], np.sin(theta)[:, None]
        if inverse:
            s = -s
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        out[..., a] = x[..., a] * c - x[..., b] * s
        out[..., b] = x[..., a] * s + x[..., b] * c
    return out


def slots(q_len, kv_len):
    """Slots of a sequence's new tokens."""
    return np.arange(q_len) + (kv_len - q_len)


def chunk_attention(Q, K, V, q_len, kv_len):
    """Q [q_len, h_q, d], K / V [kv_len, h_kv, d] -> (O, lse [q_len, h_q], P-weighted |v| [q_len, h_q, d])."""
    Q, K, V = (np.asarray(t, dtype=np.float64) for t in (Q, K, V))
    h_q, d = Q.shape[1:]
    g = h_q // K.shape[1]
    O, A = np.zeros(Q.shape), np.zeros(Q.shape)
    lse = np.full((q_len, h_q), -np.inf)
    at = slots(q_len, kv_len)
    for i in range(q_len):
        n = min(int(at[i]) + 1, K.shape[0])
        if n <= 0:
            continue
        for h in range(h_q):
            s = K[:n, h // g] @ Q[i, h] / np.sqrt(d)
            m = s.max()
            w = np.exp(s - m)
            lse[i, h] = m + np.log(w.sum())
            w /= w.sum()
            O[i, h] = w @ V[:n, h // g]
            A[i, h] = w @ np.abs(V[:n, h // g])
    return O, lse, A


def key_mass(Q, K, lse, q_len, kv_len, mass_in=None, decay=1.0):
    """[h_kv, kv_len]: decayed old weights of the slots before the chunk plus the weights that the rows give."""
    Q, K, lse = (np.asarray(t, dtype=np.float64) for t in (Q, K, lse))
    h_q, d = Q.shape[1:]
    h_kv = K.shape[1]
    g = h_q // h_kv
    out = np.zeros((h_kv, kv_len))
    old = max(kv_len - q_len, 0)
    if mass_in is not None:
        out[:, :old] = decay * np.asarray(mass_in, dtype=np.float64)[:, :old]
    at = slots(q_len, kv_len)
    for i in range(q_len):
        n = min(int(at[i]) + 1, kv_len)
        if n <= 0:
            continue
        for h in range(h_q):
            out[h // g, :n] += np.exp(K[:n, h // g] @ Q[i, h] / np.sqrt(d) - lse[i, h])
    return out


def evicted(mass, n, keep, sinks, recent):
    """Kept slots, ascending, of one (sequence, KV head) with n tokens: first, last, and the largest in between; equal mass the lower
    slot, NaN below everything."""
    if n <= keep:
        return np.arange(n)
    mass = np.asarray(mass, dtype=np.float64)[:n]
    always = [t for t in range(n) if t < sinks or t >= n - recent]
    rest = [t for t in range(n) if sinks <= t < n - recent]
    rest.sort(key=lambda t: (1 if np.isnan(mass[t]) else 0, 0.0 if np.isnan(mass[t]) else -mass[t], t))
    return np.array(sorted(always + rest[:keep - len(always)]), dtype=np.int64)
