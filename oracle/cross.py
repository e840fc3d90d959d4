"""Float64 oracle of attention to keys of another length, with a bias by relative position,
and of a decode step behind a shared prefix.

With r = j - (start_b + i), the place of key j relative to query i:
  x_ij = scale q_i . k_j + bias[rows[clamp(r - first)], h], -inf where j >= len_b or (causal) r > 0
  L = ln sum exp x, P = exp(x - L), O = P V; a row without keys: O = 0, L = -inf, no gradient
  dV = P^T dO, dP = dO V^T, dS = P (dP - D), D = sum_j P dP, dQ = scale dS K, dK = scale dS^T Q,
  dbias[c, h] = the sum of dS over the pairs whose row is c
K, V, dK and dV of a cache head belong to the query heads h with h // (Hq / Hkv) = it.
"""
from __future__ import annotations

import numpy as np


def bias_at(bias, rows, first, start, nq, nk, h):
    """The bias [nq, nk] of head h; buckets that the table does not have stand for none, entries below
    -2^16 for -inf."""
    r = np.arange(nk)[None, :] - (np.arange(nq)[:, None] + start)
    k = np.asarray(rows)[np.clip(r - first, 0, len(rows) - 1)]
    inside = (k >= 0) & (k < bias.shape[0])
    x = np.where(inside, bias[np.where(inside, k, 0), h], 0.0)
    return np.where(x < -65536.0, -np.inf, x), np.where(inside, k, -1)


def head(q, k, v, scale, n, start, causal, b=None):
    """One head: (O, L, P, x) from q [nq, d] and k, v [nk, d], of which n keys are there."""
    nq, nk = q.shape[0], k.shape[0]
    k, v = k.copy(), v.copy()
    k[n:], v[n:] = 0.0, 0.0   # what is not there may hold anything
    x = scale * (q @ k.T) + (0.0 if b is None else b)
    seen = np.broadcast_to(np.arange(nk)[None, :] < n, (nq, nk))
    if causal:
        seen = seen & (np.arange(nk)[None, :] <= np.arange(nq)[:, None] + start)
    x = np.where(seen, x, -np.inf)
    top = x.max(axis=1, keepdims=True) if nk else np.full((nq, 1), -np.inf)
    safe = np.where(np.isfinite(top), top, 0.0)
    e = np.exp(x - safe)
    z = e.sum(axis=1, keepdims=True)
    with np.errstate(divide="ignore"):
        L = (safe + np.log(z))[:, 0]
    P = e / np.where(z > 0, z, 1.0)
    return P @ v, L, P, x


def attention(q, k, v, scale, do=None, causal=False, start=0, starts=None, k_lens=None, bias=None, rows=None, first=0):
    """All outputs as a dict: O, L and, given do, dQ, dK, dV (and dBias)."""
    B, Hq, nq, d = q.shape
    Hkv, nk = k.shape[1], k.shape[2]
    G = Hq // Hkv
    out = {"O": np.zeros((B, Hq, nq, d)), "L": np.zeros((B, Hq, nq))}
    if do is not None:
        out.update(dQ=np.zeros((B, Hq, nq, d)), dK=np.zeros((B, Hkv, nk, d)), dV=np.zeros((B, Hkv, nk, d)))
        if bias is not None:
            out["dBias"] = np.zeros(bias.shape)
    for b in range(B):
        n = nk if k_lens is None else int(np.clip(k_lens[b], 0, nk))
        s = start if starts is None else int(starts[b])
        for h in range(Hq):
            kk, vv = k[b, h // G].copy(), v[b, h // G].copy()
            kk[n:], vv[n:] = 0.0, 0.0
            t, at = (None, None) if bias is None else bias_at(bias, rows, first, s, nq, nk, h)
            O, L, P, _ = head(q[b, h], kk, vv, scale, n, s, causal, t)
            out["O"][b, h], out["L"][b, h] = O, L
            if do is None:
                continue
            dP = do[b, h] @ vv.T
            dS = P * (dP - (P * dP).sum(axis=1, keepdims=True))
            out["dV"][b, h // G] += P.T @ do[b, h]
            out["dQ"][b, h] = scale * (dS @ kk)
            out["dK"][b, h // G] += scale * (dS.T @ q[b, h])
            if bias is not None:
                np.add.at(out["dBias"][:, h], at[at >= 0], dS[at >= 0])
    return out


def prefix_decode(q, k_prefix, v_prefix, k_cache, v_cache, lens, scale, k_new=None, v_new=None):
    """(O, L, k_cache, v_cache) of one step: q [B, Hq, d], prefix [Hkv, np, d], caches [B, Hkv, n_cap, d]."""
    B, Hq, d = q.shape
    G = Hq // k_prefix.shape[0]
    k_cache, v_cache = k_cache.copy(), v_cache.copy()
    O, L = np.zeros((B, Hq, d)), np.zeros((B, Hq))
    for b in range(B):
        n = int(lens[b])
        if k_new is not None:
            k_cache[b, :, n], v_cache[b, :, n] = k_new[b], v_new[b]
            n += 1
        for h in range(Hq):
            g = h // G
            k = np.concatenate((k_prefix[g], k_cache[b, g, :n]))
            v = np.concatenate((v_prefix[g], v_cache[b, g, :n]))
            o, l, _, _ = head(q[b, h][None], k, v, scale, len(k), 0, False)
            O[b, h], L[b, h] = o[0], l[0]
    return O, L, k_cache, v_cache
