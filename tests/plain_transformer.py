"""Plain numpy forms, in 64 bits, of attention, of the norm and rotation of queries and keys and of gradient clipping, with the magnitudes
that their rounding errors scale with."""
import numpy as np

U = 2.0 ** -24           # half a step of fp32
TINY = 2.0 ** -125       # fp32 numbers, and factors of products on the matrix cores, below 2^-126 may count as 0: an exponential (2^-126 off),
                         # its product with dP - D (as much, and 2^-126 times the factor) and each term of a sum (2^-126)


# ---- attention, one sequence: q [Lq, H, D], k and v [Lk, Hkv, D] --------------------------------------------------------
def seen(Lq, Lk, window):
    """Which keys a query sees, [Lq, Lk]."""
    c = np.arange(Lq)[:, None] + Lk - Lq
    j = np.arange(Lk)[None, :]
    out = np.ones((Lq, Lk), bool)
    if window[0] >= 0:
        out &= j >= c - window[0]
    if window[1] >= 0:
        out &= j <= c + window[1]
    return out


def attention(q, k, v, scale, window):
    """o, lse, and sum_j p |v| (what o's error scales with), max_j scale sum_d |q k| (the scores')."""
    Lq, H, D = q.shape
    Lk, Hkv = k.shape[:2]
    o, lse = np.zeros((Lq, H, D)), np.full((H, Lq), -np.inf)
    size, score = np.zeros((Lq, H, D)), np.zeros((H, Lq))
    see = seen(Lq, Lk, window)
    for h in range(H):
        kh, vh = k[:, h // (H // Hkv)], v[:, h // (H // Hkv)]
        for i in range(Lq):
            js = np.flatnonzero(see[i])
            if not len(js):
                continue
            x = scale * (kh[js] @ q[i, h])
            top = x.max()
            e = np.exp(x - top)
            lse[h, i] = top + np.log(e.sum())
            p = e / e.sum()
            o[i, h], size[i, h] = p @ vh[js], p @ np.abs(vh[js])
            score[h, i] = scale * (np.abs(kh[js]) @ np.abs(q[i, h])).max()
    return o, lse, size, score


def attention_backward(q, k, v, o, lse, do, scale, window, half):
    """dq, dk, dv from the given o and lse, and bounds on the errors that a product of operands rounded by `half` (relative) and fp32
    sums leave."""
    Lq, H, D = q.shape
    Lk, Hkv = k.shape[:2]
    out = [np.zeros(q.shape), np.zeros(k.shape), np.zeros(k.shape)]
    tol = [np.zeros(q.shape), np.zeros(k.shape), np.zeros(k.shape)]
    see = seen(Lq, Lk, window)
    n = Lq * (H // Hkv) / 2 + 64           # length of a chain of sums over queries (a wave's MFMA adds two or more terms at a time)
    for h in range(H):
        kv = h // (H // Hkv)
        kh, vh, qh, gh, oh = k[:, kv], v[:, kv], q[:, h], do[:, h], o[:, h]
        rows = np.isfinite(lse[h])
        with np.errstate(invalid="ignore", over="ignore"):
            p = np.where(see & rows[:, None], np.exp(scale * qh @ kh.T - np.where(rows, lse[h], 0.0)[:, None]), 0.0)
        dp, delta = gh @ vh.T, (gh * oh).sum(1)[:, None]
        ds = p * (dp - delta)
        # relative error of p: the score's sum of D products, the product with 1 / ln 2, lse / ln 2, the exponential
        dev = (D + 8) * U * scale * (np.abs(qh) @ np.abs(kh).T) + 8 * U * (1 + np.abs(np.where(rows, lse[h], 0.0))[:, None])
        ep = p * (dev + half) + TINY
        es = np.abs(ds) * (dev + half + 4 * U) + TINY * (1 + np.abs(dp - delta)) + p * (D + 4) * U * (np.abs(gh) @ np.abs(vh).T + (np.abs(gh) * np.abs(oh)).sum(1)[:, None])
        out[0][:, h] += scale * ds @ kh
        out[1][:, kv] += scale * ds.T @ qh
        out[2][:, kv] += p.T @ gh
        tol[0][:, h] += scale * (es + (Lk / 2 + 64) * U * np.abs(ds)) @ np.abs(kh) + (1 + scale) * Lk * TINY
        tol[1][:, kv] += scale * (es + n * U * np.abs(ds)).T @ np.abs(qh) + (1 + scale) * Lq * TINY
        tol[2][:, kv] += (ep + n * U * p).T @ np.abs(gh) + Lq * TINY
    return out, tol


# ---- norm and rotation, x [T, H, D], positions [T, A] -------------------------------------------------------------------
def angles(positions, frequencies, sections):
    """[T, pairs]; frequencies are fp32 numbers, so that the products have at most 55 bits: formed in long double."""
    axis = np.repeat(np.arange(len(sections)), sections)
    w = np.asarray(positions, np.longdouble)[:, axis] * np.asarray(frequencies, np.longdouble)
    return np.asarray(np.remainder(w, 2 * np.longdouble("3.14159265358979323846264338327950288")), np.float64)


def _places(D, pairs, halves):
    p = np.arange(pairs)
    return (p, p + pairs) if halves else (2 * p, 2 * p + 1)


def turned(n, w, halves, back=False):
    """The pairs of n [T, H, D] turned by w [T, pairs], and |a| + |b| of each element's pair."""
    out, size = n.copy(), np.abs(n)
    a, b = _places(n.shape[-1], w.shape[1], halves)
    c, s = np.cos(w)[:, None], np.sin(w)[:, None] * (-1 if back else 1)
    out[..., a] = n[..., a] * c - n[..., b] * s
    out[..., b] = n[..., a] * s + n[..., b] * c
    size[..., a] = size[..., b] = np.abs(n[..., a]) + np.abs(n[..., b])
    return out, size


def norm_rotary(x, gamma, w, halves, eps, norm=True):
    """y and the magnitudes its errors scale with."""
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if gamma is None else gamma)
    return turned(x, w, halves)


def norm_rotary_backward(x, dy, gamma, w, halves, eps, norm=True):
    """dx, dgamma and the magnitudes their errors scale with."""
    dn, size = turned(dy, w, halves, back=True)
    if not norm:
        return dn, None, size, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xhat, g = x * r, np.ones(x.shape[-1]) if gamma is None else gamma
    h, hs = dn * g, size * np.abs(g)
    dx = r * (h - xhat * (h * xhat).mean(-1, keepdims=True))
    dx_size = r * (hs + np.abs(xhat) * (hs * np.abs(xhat)).mean(-1, keepdims=True))
    return dx, (dn * xhat).sum((0, 1)), dx_size, (size * np.abs(xhat)).sum((0, 1))


# ---- clipping ------------------------------------------------------------------------------------------------------------
def clip(tensors, largest):
    norm = np.sqrt(sum((np.asarray(t, np.float64) ** 2).sum() for t in tensors))
    c = largest / norm if norm > largest else 1.0
    return norm, [np.asarray(t, np.float64) * c for t in tensors], c
