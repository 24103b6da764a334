"""Plain 64-bit references of the operators around a training step, with the room that 32-bit arithmetic needs.

Each function returns the values and, where it is asked to, a bound on how far 32-bit sums of them may be off, from the
number of roundings: U is half a step of a 32-bit float.
"""
import numpy as np

U = 2.0 ** -24


REF = 8 * np.log(2.0)   # how far the reference of a sum may be below the row's maximum


def _chain(V):
    """Roundings a sum over V elements may pass.  64 threads share a row of at most 4096, 256 or more a longer one; a thread
    adds pieces of at most 16 elements (8 of four bytes), and a piece and up to eight short ones more may each change the
    sum's reference, six roundings; trees over the threads and the parts of a row."""
    pieces = 8 + V / (64 if V <= 4096 else 256) / 8
    return 16 + pieces + 6 * pieces + 36


def token_logprobs(z, target, scale, top=0):
    """z [n,V] float64, target [n] int or None.  dict of logp, entropy, stats, top_logp, top_id and tol_* bounds."""
    n, V = z.shape
    scale = float(np.float32(scale))
    out = {"logp": np.zeros(n), "entropy": np.zeros(n), "stats": np.zeros((n, 2)),
           "top_logp": np.full((n, top), -np.inf), "top_id": np.full((n, top), -1, dtype=np.int64),
           "tol_logp": np.zeros(n), "tol_entropy": np.zeros(n), "tol_S": np.zeros(n), "tol_top": np.zeros((n, top))}
    for i in range(n):
        t = 0 if target is None else int(target[i])
        if t < 0 or t >= V:
            continue
        r = z[i]
        if np.isnan(r).any() or (r == np.inf).any():
            out["logp"][i] = out["entropy"][i] = np.nan
            out["stats"][i] = np.nan
            out["top_logp"][i] = np.nan
            continue
        m = r.max()
        if m == -np.inf:
            out["logp"][i] = -np.inf
            out["stats"][i] = (-np.inf, 0.0)
            continue
        x = scale * (r - m)
        e = np.exp(x)
        S = e.sum()
        p = e / S
        x0 = np.where(p > 0, x, 0.0)
        ls = np.log(S)
        out["logp"][i] = x[t] - ls
        out["entropy"][i] = ls - (p * x0).sum()
        out["stats"][i] = (m, S)
        # x carries three roundings, its exponential the relative error ln-wise plus two; sums as above.  The entropy's sum of
        # e x has x relative to the reference, so that its terms are larger by REF until it is referred to the maximum.
        A, A2, L = (p * -x0).sum(), (p * x0 * x0).sum(), _chain(V)
        ts = U * (L + 3 * A + 4)
        out["tol_S"][i] = ts
        lp = lambda v: ts + U * (3 * abs(v) + 4 * abs(ls) + abs(v - ls))  # noqa: E731
        out["tol_logp"][i] = lp(x[t]) if np.isfinite(x[t]) else 0.0
        out["tol_entropy"][i] = ts + U * (3 * A2 + (2 * L + 16) * (A + REF) + 4 * ls)
        if top:
            r0 = r + 0.0
            order = np.lexsort((np.arange(V), -r0))[:top]
            order = order[np.isfinite(r0[order])]
            k = len(order)
            out["top_id"][i, :k] = order
            out["top_logp"][i, :k] = x[order] - ls
            out["tol_top"][i, :k] = [lp(v) for v in x[order]]
    return out


def token_logprobs_backward(z, target, scale, dlogp, dentropy, half_step):
    """d(sum dlogp logp + dentropy entropy)/dz and its bound; dlogp, dentropy: [n] or None."""
    n, V = z.shape
    f = token_logprobs(z, target, scale)
    scale = float(np.float32(scale))
    dz, tol = np.zeros((n, V)), np.zeros((n, V))
    for i in range(n):
        t = 0 if target is None else int(target[i])
        if t < 0 or t >= V or f["stats"][i, 1] == 0.0:
            continue
        m, S = f["stats"][i]
        x = scale * (z[i] - m)
        p = np.exp(x) / S
        lp = np.where(p > 0, x - np.log(S), 0.0)
        x = np.where(p > 0, x, 0.0)
        dl = 0.0 if dlogp is None else float(dlogp[i])
        dh = 0.0 if dentropy is None else float(dentropy[i])
        H = f["entropy"][i]
        g = -p * (dl + dh * (lp + H))
        size = p * (abs(dl) + abs(dh) * (np.abs(x) + 2 * np.log(S) + H))
        tol[i] = size * (f["tol_S"][i] + U * (3 * np.abs(x) + 12)) + p * abs(dh) * (f["tol_entropy"][i] + f["tol_S"][i])
        if dlogp is not None:
            g[t] += dl
            tol[i, t] += 2 * U * abs(dl)
        dz[i] = scale * g
        tol[i] *= scale
        tol[i] += half_step * (np.abs(dz[i]) + tol[i]) + 1e-37
    return dz, tol


def combine_backward(dy, Yp, gates, inv_perm, half_step):
    """dy [T,d], Yp [T*K,d], gates [T,K], inv_perm [T*K] (rows out of range are left out)."""
    T, d = dy.shape
    K = gates.shape[1]
    S = T * K
    rows = inv_perm.reshape(T, K)
    ok = (rows >= 0) & (rows < S)
    at = np.where(ok, rows, 0)
    dYp, tol_dYp = np.full((S, d), np.nan), np.zeros((S, d))
    dg, tg = np.zeros((T, K)), np.zeros((T, K))
    chain = d / 64 + 24
    for j in range(K):
        v = dy * gates[:, j:j + 1]
        dYp[at[ok[:, j], j]] = v[ok[:, j]]
        tol_dYp[at[ok[:, j], j]] = (half_step + 2 * U) * np.abs(v[ok[:, j]]) + 1e-37
        dg[:, j] = np.where(ok[:, j], (Yp[at[:, j]] * dy).sum(1), 0.0)
        tg[:, j] = np.where(ok[:, j], U * chain * np.abs(Yp[at[:, j]] * dy).sum(1), 0.0)
    mix = (gates * dg).sum(1, keepdims=True)
    dz = gates * (dg - mix)
    tz = gates * (tg + (gates * tg).sum(1, keepdims=True) + 12 * U * (gates * np.abs(dg)).sum(1, keepdims=True)
                  + 3 * U * np.abs(dg)) + 1e-37
    return {"dYp": dYp, "tol_dYp": tol_dYp, "dgates": dg, "tol_dgates": tg + 1e-37, "dz": dz, "tol_dz": tz}


def permute_backward(dXp, inv_perm, add, T, half_step):
    S, d = dXp.shape
    K = S // T
    rows = inv_perm.reshape(T, K)
    dx = np.zeros((T, d)) if add is None else add.copy()
    size = np.abs(dx)
    for j in range(K):
        ok = (rows[:, j] >= 0) & (rows[:, j] < S)
        v = np.where(ok[:, None], dXp[np.where(ok, rows[:, j], 0)], 0.0)
        dx += v
        size += np.abs(v)
    t = U * (K + 1) * size
    return dx, t + half_step * (np.abs(dx) + t) + 1e-37
