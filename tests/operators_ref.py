"""64-bit references of the operators around the layer (numpy, written from
the definitions in include/pmpe.h, token by token), and error bounds."""
import numpy as np

E4M3_MAX = 448.0
FLT_MAX = float(np.finfo(np.float32).max)


def rms_norm(h, weight, eps):
    """(y, rstd) of the (already rounded) rows h."""
    rstd = 1.0 / np.sqrt((h * h).mean(1) + eps)
    return h * rstd[:, None] * weight, rstd


def rms_norm_backward(dy, h, weight, rstd, d_h):
    """(dx, dw) and the magnitudes their errors are relative to."""
    n = h * rstd[:, None]
    g = dy * weight
    m = (g * n).mean(1, keepdims=True)
    dx = rstd[:, None] * (g - n * m)
    size = rstd[:, None] * (np.abs(g) + np.abs(n) * np.abs(g * n).mean(1, keepdims=True))
    if d_h is not None:
        dx, size = dx + d_h, size + np.abs(d_h)
    return dx, (dy * n).sum(0), size, np.abs(dy * n).sum(0)


def pool_of(t, policy, E_pub, E_priv):
    return (E_pub, E_pub + E_priv) if policy is not None and policy[t] == 1 else (0, E_pub)


def scores(z, sigmoid):
    """Scores of one pool's logits; -1 where an expert is not eligible."""
    ok = z > -np.inf
    s = np.full(z.shape, -1.0)
    c = np.minimum(z[ok], FLT_MAX)
    if ok.any():
        with np.errstate(over="ignore"):
            if sigmoid:
                s[ok] = 1.0 / (1.0 + np.exp(-c))
            else:
                e = np.exp(c - c.max())
                s[ok] = e / e.sum()
    return s


def route(logits, policy, E_pub, E_priv, k, sigmoid=False, renorm=True, scale=1.0, bias=None, groups=(1, 1),
          groups_priv=(1, 1), top2=False):
    """(idx, w) token by token."""
    T = logits.shape[0]
    idx, w = np.full((T, k), -1, np.int32), np.zeros((T, k))
    for t in range(T):
        lo, hi = pool_of(t, policy, E_pub, E_priv)
        z = logits[t, lo:hi].astype(np.float64)
        s = scores(z, sigmoid)
        value = s + (bias[lo:hi] if bias is not None else 0.0)
        choice = value if bias is not None else np.minimum(z, FLT_MAX)
        cand = [e for e in range(hi - lo) if s[e] >= 0 and choice[e] > -np.inf]
        n, top = groups_priv if lo else groups
        size = (hi - lo) // n
        if top < n:
            rank = []
            for g in range(n):
                inside = [e for e in cand if e // size == g]
                if not inside:
                    continue
                v = max(choice[e] for e in inside)
                if top2:
                    v = sum(sorted((value[e] for e in inside), reverse=True)[:2])
                rank.append((-v, g))
            kept = {g for _, g in sorted(rank)[:top]}
            cand = [e for e in cand if e // size in kept]
        sel = sorted(cand, key=lambda e: (-choice[e], e))[:k]
        wt = np.array([s[e] for e in sel])
        if renorm and sel:
            wt = wt / (wt.sum() + 1e-20) if sigmoid else wt / wt.sum()
        idx[t, :len(sel)] = np.array(sel, dtype=np.int32) + lo
        w[t, :len(sel)] = wt * scale
    return idx, w


def weights(z, picks, sigmoid, renorm, scale):
    """Weights of the picks of one token's pool (positions in z)."""
    s = scores(z, sigmoid)[picks]
    if renorm:
        s = s / (s.sum() + 1e-20) if sigmoid else s / s.sum()
    return s * scale


def route_backward(logits, policy, idx, dw, E_pub, E_priv, sigmoid=False, renorm=True, scale=1.0):
    """d_logits and the magnitudes its errors are relative to."""
    d, size = np.zeros(logits.shape), np.zeros(logits.shape)
    for t in range(logits.shape[0]):
        lo, hi = pool_of(t, policy, E_pub, E_priv)
        s = scores(logits[t, lo:hi].astype(np.float64), sigmoid)
        js = [j for j in range(idx.shape[1]) if lo <= idx[t, j] < hi and s[idx[t, j] - lo] >= 0]
        if not js:
            continue
        e = idx[t, js] - lo
        D, sj = dw[t, js] * scale, s[e]
        if renorm:
            S = sj.sum() + 1e-20
            ds, ads = (D - (D * sj).sum() / S) / S, (np.abs(D) + np.abs(D * sj).sum() / S) / S
        else:
            ds, ads = D, np.abs(D)
        if sigmoid:
            for i, x in enumerate(e):
                d[t, lo + x] += ds[i] * sj[i] * (1 - sj[i])
                size[t, lo + x] += ads[i] * sj[i] * (1 - sj[i])
        elif renorm:
            # w_j = p_j / sum of the chosen p: dz_j = w_j (D_j - sum_i D_i w_i) and
            # nothing elsewhere (p_e (ds_e - sum_i ds_i p_i) is the same, but its
            # zeros are differences that only cancel to 2^-53)
            wj = sj / sj.sum()
            mean, amean = (D * wj).sum(), np.abs(D * wj).sum()
            for i, x in enumerate(e):
                d[t, lo + x] += wj[i] * (D[i] - mean)
                size[t, lo + x] += wj[i] * (np.abs(D[i]) + amean)
        else:
            p = np.maximum(s, 0.0)
            g, a = np.zeros(hi - lo), np.zeros(hi - lo)
            for i, x in enumerate(e):
                g[x] += D[i]
                a[x] += np.abs(D[i])
            d[t, lo:hi] = p * (g - (p * g).sum())
            size[t, lo:hi] = p * (a + (p * a).sum())
    return d, size


def global_norm(grads):
    return float(np.sqrt(sum((g.astype(np.float64) ** 2).sum() for g in grads)))
