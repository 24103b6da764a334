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


def _f16(x):
    return x.astype(np.float16).astype(np.float64)


def _pair(x):
    h = _f16(x)
    return h + _f16(x - h)


QUINTIC = (3.4445, -4.775, 2.0315)


def orthogonalize(G, steps=5, coef=QUINTIC, eps=1e-7, scale=1.0, to="f32"):
    """One matrix G: (the result in 64 bits, a bound on the 2-norm of the error).  The bound is three times what the roundings of
    the documented number formats do to this matrix (X as pairs of f16, A and its polynomial as f16 or, for f32 results, as
    pairs; all times 2^12), the chains of f32 sums, and the result's rounding."""
    a, b, c = (float(np.float32(v)) for v in coef)
    eps, scale = float(np.float32(eps)), float(np.float32(scale))
    X = G if G.shape[0] <= G.shape[1] else G.T
    n = np.linalg.norm(X) + eps
    X = X / n if n > 0 else X
    unit, small = 4096.0, _pair if to == "f32" else _f16
    q, r = (lambda v: _pair(v * unit) / unit), (lambda v: small(v * unit) / unit)
    Y, I = q(X), np.eye(len(X))
    for k in range(steps):
        apart = a + b + c if k >= steps - 2 else a
        A = X @ X.T
        X = a * X + (b * A + c * (A @ A)) @ X
        H = r(Y)
        A = r(H @ H.T)
        Y = apart * Y + r((a - apart) * I + b * A + c * (A @ A)) @ H
        Y = q(Y) if k + 1 < steps else Y
    size, half = np.linalg.norm(X), 2.0 ** -8 if to == "bf16" else U
    # 32 products to a rounding of a sum, the worst of a chain's roundings in one direction, for the three products of a step and
    # growth by the quintic's steepest slope
    chain = U * steps * 3 * (8 + max(G.shape) / 32) * abs(a)
    tol = abs(scale) * (3 * np.linalg.norm(Y - X) + chain * size + half * size * 1.01 + 1e-30)
    out = scale * (X if G.shape[0] <= G.shape[1] else X.T)
    return out, tol


def spans(starts, n):
    """[begin, end) of each sequence; one of everything without starts."""
    return [(0, n)] if starts is None else [(int(a), int(b)) for a, b in zip(starts, starts[1:])]


def policy_loss(logp, adv, old=None, infer=None, ref=None, entropy=None, target=None, starts=None, ratio="token", norm="tokens", adv_seq=False,
                clip_low=0.2, clip_high=0.2, dual_clip=0.0, weight_cap=np.inf, kl_coef=0.0, entropy_coef=0.0, scale=1.0):
    """stats [8], dlogp, dentropy [n] and their bounds."""
    n = len(logp)
    lo, hi, dual, cap, beta, gamma, scale = (float(np.float32(v)) for v in (clip_low, clip_high, dual_clip, weight_cap, kl_coef, entropy_coef, scale))
    live = np.zeros(n, dtype=bool)
    seqs = spans(starts, n)
    for a, b in seqs:
        live[a:b] = True
    if target is not None:
        live &= target >= 0
    groups = [np.arange(a, b)[live[a:b]] for a, b in seqs]
    N, S = sum(len(g) for g in groups), sum(len(g) > 0 for g in groups)
    dl, dh, tl, th = np.zeros(n), np.zeros(n), np.zeros(n), np.zeros(n)
    parts, room, cuts, weights, wroom = np.zeros(3), np.zeros(3), 0, 0.0, 0.0
    with np.errstate(all="ignore"):
        borders = np.log1p(hi), np.log1p(-lo), np.log(dual) if dual else np.inf
        for q, g in enumerate(groups):
            m = len(g)
            if m == 0:
                continue
            nu = scale / N if norm == "tokens" else scale / (S * m) if norm == "sequences" else scale
            x = logp[g]
            A = np.full(m, adv[q]) if adv_seq else adv[g]
            o = x if old is None else old[g]
            d = x - o
            # the ratio's exponent is rounded once; exp by three roundings
            if ratio == "sequence":
                d = np.full(m, d.mean())
            r = np.exp(d)
            tr = U * (np.abs(d) + 6)
            lw = np.zeros(m) if infer is None else o - infer[g]
            w = np.minimum(np.exp(lw), cap) if infer is not None else np.ones(m)
            tw = U * (np.abs(lw) + 6)
            up, down, over = d > borders[0], d < borders[1], d > borders[2]
            used = np.where(A > 0, np.where(up, 1 + hi, r), np.where(over, dual, np.where(down, 1 - lo, r)))
            cut = np.where(A > 0, up, np.where(A < 0, down | over, False)).astype(bool)
            part = np.where(cut, 0.0, -w * A * r)
            part[A == 0] = 0.0
            l = np.where(A == 0, 0.0, -w * A * used)
            tpart = np.abs(part) * (tr + tw + 8 * U)
            if ratio == "sequence":
                part, tpart = np.full(m, part.mean()), np.full(m, tpart.mean() + 4 * U * np.abs(part).mean())
            tl[g] = tpart
            dl[g] = part
            parts[0] += nu * l.sum()
            room[0] += abs(nu) * (np.abs(l) * (tr + tw + 12 * U)).sum()
            if ref is not None:
                k = ref[g] - x
                if beta:      # (a term with coefficient 0 is a statistic alone)
                    dl[g] -= beta * np.expm1(k)
                tl[g] += abs(beta) * U * (8 * np.abs(np.expm1(k)) + np.exp(k) * np.abs(k))
                parts[1] += nu * (np.expm1(k) - k).sum()
                room[1] += abs(nu) * U * (12 * np.abs(np.expm1(k) - k) + 2 * np.abs(np.expm1(k) * k) + 4 * np.abs(k) * (np.abs(k) > 0.12)).sum()
            if entropy is not None:
                parts[2] += nu * entropy[g].sum()
                room[2] += abs(nu) * 4 * U * np.abs(entropy[g]).sum()
            dl[g] *= nu
            tl[g] = abs(nu) * tl[g] + 4 * U * np.abs(dl[g])
            dh[g] = -gamma * nu
            th[g] = 4 * U * np.abs(dh[g])
            cuts += cut.sum()
            weights += w.sum()
            wroom += (w * tw).sum()
    one = max(N, 1)
    inv = 1 / scale if scale else 0.0
    loss = parts[0] + (beta * parts[1] if beta else 0.0) - (gamma * parts[2] if gamma else 0.0)
    stats = np.array([loss, parts[0], parts[1] * inv, parts[2] * inv, cuts / one, weights / one, N, S])
    tol = np.array([room[0] + abs(beta) * room[1] + abs(gamma) * room[2], room[0], room[1] * abs(inv), room[2] * abs(inv), 0.0, wroom / one, 0.0, 0.0])
    tol += 2 * U * np.abs(stats) + 1e-37
    return {"stats": stats, "dlogp": dl, "dentropy": dh, "tol_stats": tol, "tol_dlogp": tl + 1e-37, "tol_dentropy": th + 1e-37}


def balance_loss(z, idx, starts=None, alpha=0.01, zeta=0.0):
    """z [T,E], idx [T,K].  stats [3], counts, probs [groups,E], dlogits [T,E] and bounds."""
    T, E = z.shape
    K = idx.shape[1]
    alpha, zeta = float(np.float32(alpha)), float(np.float32(zeta))
    groups = spans(starts, T)
    some, N = max(1, sum(b > a for a, b in groups)), max(1, sum(b - a for a, b in groups))
    out = {"counts": np.zeros((len(groups), E), dtype=np.int64), "probs": np.zeros((len(groups), E)), "dlogits": np.zeros((T, E)),
           "tol_probs": np.zeros((len(groups), E)), "tol_dlogits": np.zeros((T, E))}
    bal = zl = tb = tz = 0.0
    C = 16 + E / 8              # sums over a row, by 2 to 64 lanes
    with np.errstate(all="ignore"):
        for g, (a, b) in enumerate(groups):
            if a >= b:
                continue
            n = b - a
            ids = idx[a:b].reshape(-1)
            c = np.bincount(ids[ids < E], minlength=E)
            out["counts"][g] = c
            f = c * E / (K * n)
            m = z[a:b].max(1, keepdims=True)
            empty = m[:, 0] == -np.inf
            x = np.where(empty[:, None], -np.inf, z[a:b] - np.where(empty[:, None], 0.0, m))
            e = np.exp(x)
            S = e.sum(1, keepdims=True)
            p = np.where(empty[:, None], 0.0, e / np.where(empty[:, None], 1.0, S))
            ax = np.where(p > 0, -x, 0.0)
            lse = np.where(empty, 0.0, np.where(empty, 0.0, m[:, 0]) + np.log(np.where(empty, 1.0, S[:, 0])))
            ts = U * (C + 3 * (p * ax).sum(1, keepdims=True))       # S, relative
            tp = p * (U * (3 * ax + 8) + ts)
            mean = (f * p).sum(1, keepdims=True)
            tm = (f * tp).sum(1, keepdims=True) + U * C * mean
            tlse = ts[:, 0] + 3 * U * (np.abs(lse) + np.log(np.where(empty, 1.0, S[:, 0])))
            ga, gz = alpha / (some * n), 2 * zeta / N
            out["dlogits"][a:b] = ga * p * (f - mean) + gz * lse[:, None] * p
            out["tol_dlogits"][a:b] = (tp * (abs(ga) * np.abs(f - mean) + np.abs(gz * lse)[:, None]) + p * (abs(ga) * (tm + 4 * U * (f + mean))
                                       + np.abs(gz) * tlse[:, None] + 4 * U * np.abs(gz * lse)[:, None])) + 1e-37
            out["probs"][g] = p.mean(0)
            out["tol_probs"][g] = tp.mean(0) + U * (200 + T / 1000) * p.mean(0) + 1e-37
            bal += mean.sum() / n
            tb += tm.sum() / n
            zl += (lse ** 2).sum()
            tz += (2 * np.abs(lse) * tlse + tlse ** 2).sum()
    bal, zl = bal / some, zl / N
    out["stats"] = np.array([alpha * bal + zeta * zl, bal, zl])
    out["tol_stats"] = np.array([abs(alpha) * tb / some + abs(zeta) * tz / N, tb / some, tz / N]) + 2 * U * (
        np.abs(out["stats"]) + np.array([abs(alpha * bal) + abs(zeta * zl), 0, 0])) + 1e-37
    return out
