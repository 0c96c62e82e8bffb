"""fp64 reference for caches of pages: rotary positions, appending, chunk attention, attention weights, eviction.

TEST INFRASTRUCTURE, like seka_oracle: plain numpy loops over requests and heads, no code shared with the kernels.  New tokens
are packed rows [total, heads, D], request b owning rows cu[b] .. cu[b + 1] - 1; they are the last ones of its lens[b] cached
tokens, and token j of request b lies in page table[b, j // ps] at slot j % ps.
"""
import math

import numpy as np


def rope_frequencies(dim, base, scaling="plain", stretch=1.0, original=4096.0, fast=32.0, slow=1.0):
    """Radians per position, one pair at a time."""
    out = []
    if scaling == "base":
        base = base * stretch ** (dim / (dim - 2))

    def index_of(turns):                   # the (fractional) pair that makes so many turns over the original context
        return dim * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))

    for i in range(dim // 2):
        f = base ** (-2 * i / dim)
        if scaling == "linear":
            f /= stretch
        elif scaling == "parts":
            lo, hi = max(math.floor(index_of(fast)), 0), min(math.ceil(index_of(slow)), dim - 1)
            share = min(max((i - lo) / max(hi - lo, 1e-3), 0.0), 1.0)
            f = (1 - share) * f + share * f / stretch
        elif scaling == "turns":
            t = original * f / (2 * math.pi)
            keep = 1.0 if t >= fast else 0.0 if t <= slow else (t - slow) / (fast - slow)
            f = keep * f + (1 - keep) * f / stretch
        out.append(f)
    return out


def rotary(x, positions, freq, interleaved=False, factor=1.0):
    """x [..., heads, D], positions [...]."""
    y = np.array(x, np.float64)
    n = len(freq)
    for i, f in enumerate(freq):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, n + i)
        angle = np.asarray(positions, np.float64)[..., None] * f
        c, s = np.cos(angle) * factor, np.sin(angle) * factor
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def cached(pool, table, b, n):
    """Rows of tokens 0 .. n - 1 of request b: [n, Hkv, D]."""
    ps = pool.shape[1]
    j = np.arange(n)
    return pool[table[b, j // ps], j % ps]


def cached_weights(W, table, b, n):
    """[n, Hkv]."""
    ps = W.shape[2]
    j = np.arange(n)
    return W[table[b, j // ps], :, j % ps]


def append(pool, rows, table, lens, cu):
    """A copy of the pool with the packed rows at their places."""
    out = np.array(pool)
    ps = pool.shape[1]
    for b in range(len(lens)):
        n = cu[b + 1] - cu[b]
        for i in range(n):
            j = lens[b] - n + i
            if j >= 0:
                out[table[b, j // ps], j % ps] = rows[cu[b] + i]
    return out


def chunk_attention(Q, K, V, table, lens, cu, scale=None):
    """Outputs [total, Hq, D], lse [Hq, total], and what tolerances are made of: sum_j p_j |v_j| and the largest sum of |q_d k_d| scale of a
    row's visible keys."""
    total, Hq, D = Q.shape
    G = Hq // K.shape[2]
    scale = 1 / math.sqrt(D) if scale is None else scale
    O, L = np.zeros((total, Hq, D)), np.full((Hq, total), -np.inf)
    spread, size = np.zeros((total, Hq, D)), np.zeros((Hq, total))
    for b in range(len(lens)):
        k, v = cached(K, table, b, lens[b]), cached(V, table, b, lens[b])
        n = cu[b + 1] - cu[b]
        first = max(0, n - lens[b])                        # new tokens before it see nothing
        if first >= n:
            continue
        rows = slice(cu[b] + first, cu[b] + n)
        hidden = np.arange(lens[b])[None] > (lens[b] - n + np.arange(first, n))[:, None]
        for hq in range(Hq):
            h = hq // G
            s = np.where(hidden, -np.inf, scale * (Q[rows, hq] @ k[:, h].T))
            top = s.max(1, keepdims=True)
            p = np.exp(s - top)
            total_p = p.sum(1, keepdims=True)
            L[hq, rows] = (top + np.log(total_p))[:, 0]
            p /= total_p
            O[rows, hq], spread[rows, hq] = p @ v[:, h], p @ np.abs(v[:, h])
            size[hq, rows] = np.where(hidden, 0.0, scale * (np.abs(Q[rows, hq]) @ np.abs(k[:, h]).T)).max(1)
    return O, L, spread, size


def attention_weights(Q, L, K, W_out, W_in, table, lens, cu, window, decay, scale=None):
    """A copy of W_out with the cached tokens' new weights; and, of every one of them, the sum alone [num_pages, Hkv, ps]."""
    total, Hq, D = Q.shape
    Hkv, ps = K.shape[2], K.shape[1]
    G = Hq // Hkv
    scale = 1 / math.sqrt(D) if scale is None else scale
    out, sums = np.array(W_out, np.float64), np.zeros(W_out.shape)
    for b in range(len(lens)):
        k = cached(K, table, b, lens[b])
        n = cu[b + 1] - cu[b]
        got = np.zeros((lens[b], Hkv))
        first = max(0, n - window)
        hidden = np.arange(lens[b])[None] > (lens[b] - n + np.arange(first, n))[:, None]
        for hq in range(Hq):
            lse = L[hq, cu[b] + first:cu[b] + n, None]
            s = scale * (Q[cu[b] + first:cu[b] + n, hq] @ k[:, hq // G].T)
            got[:, hq // G] += np.where(hidden | np.isneginf(lse), 0.0, np.exp(s - np.where(np.isneginf(lse), 0.0, lse))).sum(0)
        for j in range(lens[b]):
            page, slot = table[b, j // ps], j % ps
            sums[page, :, slot] = got[j]
            out[page, :, slot] = got[j] + (decay * W_in[page, :, slot] if W_in is not None and decay != 0 else 0.0)
    return out, sums


def kept_tokens(w, n, budget, recent):
    """Indices of the tokens that one head keeps of its n (weights w [n])."""
    if n <= budget:
        return list(range(n))
    order = sorted(range(n - recent), key=lambda j: (not np.isnan(w[j]), w[j] if not np.isnan(w[j]) else 0.0, -j), reverse=True)
    return sorted(order[:budget - recent]) + list(range(n - recent, n))


def evict(K, V, W, K_to, V_to, W_to, table, table_to, lens, budget, recent):
    """Copies of the destination pools with the kept tokens, kept [B, Hkv, budget], new lengths."""
    K_to, V_to, W_to = np.array(K_to), np.array(V_to), np.array(W_to)
    Hkv, ps, pt = K.shape[2], K.shape[1], K_to.shape[1]
    kept = np.full((len(lens), Hkv, budget), -1, np.int32)
    for b, n in enumerate(lens):
        for h in range(Hkv):
            stay = kept_tokens(cached_weights(W, table, b, n)[:, h], n, budget, recent)
            kept[b, h, :len(stay)] = stay
            for k, j in enumerate(stay):
                a, i, c, x = table[b, j // ps], j % ps, table_to[b, k // pt], k % pt
                K_to[c, x, h], V_to[c, x, h], W_to[c, h, x] = K[a, i, h], V[a, i, h], W[a, h, i]
    return K_to, V_to, W_to, kept, np.minimum(lens, budget)
