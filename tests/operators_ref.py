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


def e4m3(v):
    """v rounded to the nearest e4m3 value, ties to even."""
    _, ex = np.frexp(v)
    step = np.exp2(np.maximum(ex - 1, -6) - 3.0)
    return np.clip(np.round(v / step) * step, -E4M3_MAX, E4M3_MAX)


def kv_entries(table, lengths, cu, rows, pages, page_size):
    """(page, place) of each row's entry in the cache, None for a row that has none."""
    B, width = table.shape
    found = []
    for r in range(rows):
        at = None
        for b in range(B):
            first, last = (b, b + 1) if cu is None else (int(cu[b]), int(cu[b + 1]))
            if first <= r < last:
                pos = int(lengths[b]) - last + r
                if 0 <= pos < width * page_size:
                    page = int(table[b, pos // page_size])
                    at = (page, pos % page_size) if 0 <= page < pages else None
                break
        found.append(at)
    return found


def kv_seen(table, length, window, pages, page_size):
    """Pages and places of the positions that one sequence's query sees."""
    n = min(max(int(length), 0), len(table) * page_size)
    pos = np.arange(max(0, n - window) if window else 0, n)
    page = np.asarray(table)[pos // page_size]
    ok = (page >= 0) & (page < pages)
    return page[ok], pos[ok] % page_size


def attend(q, k, v, scale):
    """(out, lse, size, scores) of one sequence: q [heads, D], k and v [n,
    kv_heads, D]; size: the magnitude that errors of out are relative to, scores:
    the largest sum of |q k| scale of each head."""
    heads, n, group = q.shape[0], k.shape[0], q.shape[0] // k.shape[1]
    if n == 0:
        return np.zeros_like(q), np.full(heads, -np.inf), np.zeros_like(q), np.zeros(heads)
    k, v = np.repeat(k, group, 1), np.repeat(v, group, 1)
    s = np.einsum("hd,nhd->hn", q, k) * scale
    top = s.max(1, keepdims=True)
    e = np.exp(s - top)
    a = e / e.sum(1, keepdims=True)
    size = np.einsum("hn,nhd->hd", a, np.abs(v))
    scores = np.einsum("hd,nhd->hn", np.abs(q), np.abs(k)).max(1) * abs(scale)
    return np.einsum("hn,nhd->hd", a, v), (top + np.log(e.sum(1, keepdims=True)))[:, 0], size, scores


def sample_row(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, prob, kept ids) of one row, in 64 bits."""
    z = np.asarray(z, np.float64)
    ids = np.flatnonzero(z > -np.inf)
    if len(ids) == 0:
        return -1, 0.0, ids
    z = np.minimum(z, FLT_MAX)
    ids = ids[np.lexsort((ids, -z[ids]))]
    if not temperature > 0:
        return int(ids[0]), 1.0, ids[:1]
    x = (z[ids[0]] - z[ids]) / np.float64(temperature)
    r = np.exp(-x)
    n = int((r >= 2.0 ** -40).sum())
    if top_k > 0:
        n = min(n, top_k)
    ids, r, x = ids[:n], r[:n], x[:n]
    if not top_p >= 1:
        below = np.cumsum(r) - r
        n = max(1, int((below < np.float64(top_p if top_p > 0 else 0.0) * r.sum()).sum()))
        ids, r, x = ids[:n], r[:n], x[:n]
    if min_p > 0:
        keep = x <= -np.log(min(float(min_p), 1.0))  # (exp rounds to 1 what is next to it)
        ids, r = ids[keep], r[keep]
    order = np.argsort(ids)
    ids, r = ids[order], r[order]
    total = np.cumsum(r)
    u = min(max(u, 0.0), 1.0 - 2.0 ** -24) if u == u else 0.0
    at = min(int((total <= u * total[-1]).sum()), len(ids) - 1)
    return int(ids[at]), r[at] / total[-1], ids
