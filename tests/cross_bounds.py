"""Elementwise error bounds for attn_cross_fwd / attn_cross_bwd and attn_prefix_decode, from the
number formats (shared by their GPU tests).

u is half a step of the outputs' type relative to a value (2^-8 bfloat16, 2^-24 float32), f that of
float32, r the rounding of P and dS before they multiply (2^-8 with bfloat16, none with float32).
  score     a product of d terms in float32, and the shift by the maximum or L:
            dx = f ((d + 4) scale |q|.|k| + 8 (|x| + max |x|))
  P         dx of the score and of the largest (through the sum), the exponential's and the
            sum's roundings: e = dx + max dx + (n + 8) f
  O         sum (e + r + n f) P |v|, and its last rounding u |O|
  L         max dx + (n + 8) f + 4 f |L|
and in the backward, with P = exp(x - L): e' = dx + dL + 4 f (1 + |x| + |L|),
  D         from the rounded O: sum |dO| dO_err + (d + 2) f |dO|.|O|
  dP        (d + 2) f |dO|.|v|
  dS        E = (e' + 4 f) |dS| + P (dP's + D's)
  dQ        scale sum (E + r |dS| + n f |dS|) |k| + u |dQ|; dK likewise; dV as O
  dBias     as sums of dS, but D's error is taken out through the row sums of dS, which are off by
            R = sum_j ((e' + 4 f + n f) |dS| + P dP's + n f P D's): sum of (e' + 4 f) |dS| + P (dP's + R +
            e' D's), 64 f |dS| for adding, and u |dBias|
Products of such errors are covered by a factor 1.02."""
import numpy as np

from oracle import cross

F = 2.0 ** -24


def bounds(q, k, v, scale, bf16, ref, do=None, causal=False, start=0, starts=None, k_lens=None, bias=None, rows=None, first=0):
    u, r, f = (2.0 ** -8, 2.0 ** -8, F) if bf16 else (F, 0.0, F)
    B, Hq, nq, d = q.shape
    Hkv, nk = k.shape[1], k.shape[2]
    G = Hq // Hkv
    out = {name: np.zeros(x.shape) for name, x in ref.items()}
    for b in range(B):
        n = nk if k_lens is None else int(np.clip(k_lens[b], 0, nk))
        s = start if starts is None else int(starts[b])
        for h in range(Hq):
            kk, vv = k[b, h // G].copy(), v[b, h // G].copy()
            kk[n:], vv[n:] = 0.0, 0.0
            qq = q[b, h]
            t, at = (None, None) if bias is None else cross.bias_at(bias, rows, first, s, nq, nk, h)
            O, L, P, x = cross.head(qq, kk, vv, scale, n, s, causal, t)
            seen = np.isfinite(x)
            ax = np.where(seen, np.abs(x), 0.0)
            top = ax.max(axis=1, keepdims=True)
            dx = np.where(seen, f * ((d + 4) * abs(scale) * (np.abs(qq) @ np.abs(kk).T) + 8 * (ax + top)), 0.0)
            worst = dx.max(axis=1, keepdims=True)
            e = dx + worst + (nk + 8) * f
            aL = np.where(np.isfinite(L), np.abs(L), 0.0)[:, None]
            o_err = ((e + r + nk * f) * P) @ np.abs(vv) + u * np.abs(O)
            l_err = worst + (nk + 8) * f + 4 * f * aL
            out["O"][b, h], out["L"][b, h] = o_err, l_err[:, 0]
            if do is None:
                continue
            g = do[b, h]
            e = dx + l_err + 4 * f * (1 + ax + aL)
            dP = g @ vv.T
            dS = np.abs(P * (dP - (P * dP).sum(axis=1, keepdims=True)))
            p_err = (d + 2) * f * (np.abs(g) @ np.abs(vv).T)
            d_err = (np.abs(g) * o_err).sum(axis=1, keepdims=True) + (d + 2) * f * (np.abs(g) * np.abs(O)).sum(axis=1, keepdims=True)
            E = (e + 4 * f) * dS + P * (p_err + d_err)
            out["dQ"][b, h] = abs(scale) * ((E + (r + nk * f) * dS) @ np.abs(kk)) + u * np.abs(ref["dQ"][b, h])
            out["dK"][b, h // G] += abs(scale) * ((E + (r + G * nq * f) * dS).T @ np.abs(qq))
            out["dV"][b, h // G] += ((e + r + G * nq * f) * P).T @ np.abs(g)
            if bias is not None:
                R = ((e + 4 * f + nk * f) * dS + P * p_err + nk * f * P * d_err).sum(axis=1, keepdims=True)
                E = (e + 68 * f) * dS + P * (p_err + R + e * d_err)
                np.add.at(out["dBias"][:, h], at[at >= 0], E[at >= 0])
    for name in ("dK", "dV", "dBias"):
        if name in out:
            out[name] += u * np.abs(ref[name])
    return {name: 1.02 * x + 1e-37 for name, x in out.items()}


def check(got, ref, bound, what=""):
    """`got` (float64 arrays) within the bounds; infinities (L of empty rows) equal."""
    for name, y in ref.items():
        x = got[name]
        assert x.shape == y.shape, (what, name, x.shape, y.shape)
        fine = np.isfinite(y)
        assert np.array_equal(x[~fine], y[~fine]), (what, name, "infinite values")
        assert np.isfinite(x[fine]).all(), (what, name, "not finite", int((~np.isfinite(x[fine])).sum()))
        over = np.abs(x - np.where(fine, y, 0.0))[fine] / bound[name][fine]
        assert over.size == 0 or over.max() <= 1.0, (what, name, float(over.max()), int((over > 1).sum()), over.size)
