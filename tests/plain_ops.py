"""Plain numpy forms, in 64 bits, of the group norm, label log probability and AdamW calls, and the 8-bit moment format."""
import numpy as np

F32 = np.float32
U = 2.0 ** -24           # half a step of fp32


# ---- group norm -------------------------------------------------------------------------------------------------------
def gn_stats(x, groups, eps):
    B, C = x.shape[0], x.shape[-1]
    xg = np.asarray(x, np.float64).reshape(B, -1, groups, C // groups)
    mean, var = xg.mean(axis=(1, 3)), xg.var(axis=(1, 3))
    return mean, 1.0 / np.sqrt(var + eps)


def _spread(s, C):
    return np.repeat(s, C // s.shape[1], axis=1)[:, None, None, :]


def gn_z32(x, gamma, beta, mean, rstd):
    """z as the fp32 number that one rounding per operation gives."""
    C = x.shape[-1]
    xhat = (np.asarray(x, F32) - _spread(np.asarray(mean, F32), C)) * _spread(np.asarray(rstd, F32), C)
    return xhat * np.asarray(gamma, F32) + np.asarray(beta, F32)


def gn_act(z, act):
    if act == 1:
        return np.where(z > 0, z, 0.0)
    if act == 2:
        with np.errstate(over="ignore"):
            return z / (1.0 + np.exp(-z))
    return z


def gn_forward(x, gamma, beta, groups, act, eps):
    mean, rstd = gn_stats(x, groups, eps)
    C = x.shape[-1]
    xhat = (np.asarray(x, np.float64) - _spread(mean, C)) * _spread(rstd, C)
    return gn_act(xhat * gamma + beta, act), mean, rstd, xhat


def gn_backward(x, dy, gamma, beta, mean, rstd, groups, act):
    """dx, dgamma, dbeta and the magnitudes their rounding errors scale with: (dz, h, xhat)."""
    B, C = x.shape[0], x.shape[-1]
    x, dy, gamma, beta, mean, rstd = (np.asarray(a, np.float64) for a in (x, dy, gamma, beta, mean, rstd))
    xhat = (x - _spread(mean, C)) * _spread(rstd, C)
    z = xhat * gamma + beta
    if act == 1:
        dz = np.where(gn_z32(x, gamma, beta, mean, rstd) > 0, dy, 0.0)
    elif act == 2:
        s = 1.0 / (1.0 + np.exp(-z))
        dz = dy * s * (1.0 + z * (1.0 - s))
    else:
        dz = dy
    h = dz * gamma

    def group_mean(v):
        return _spread(v.reshape(B, -1, groups, C // groups).mean(axis=(1, 3)), C)

    dx = _spread(rstd, C) * (h - group_mean(h) - xhat * group_mean(h * xhat))
    size = _spread(rstd, C) * (np.abs(h) + group_mean(np.abs(h)) + np.abs(xhat) * group_mean(np.abs(h * xhat)))
    return dx, (dz * xhat).sum(axis=(0, 1, 2)), dz.sum(axis=(0, 1, 2)), size, np.abs(dz * xhat).sum(axis=(0, 1, 2)), np.abs(dz).sum(axis=(0, 1, 2))


# ---- log probabilities ---------------------------------------------------------------------------------------------
def log_probs(x, labels, top):
    """logp, entropy, lse, top_logp, top_index in 64 bits, with the rules for masked, empty and non-finite rows."""
    x = np.asarray(x, np.float64)
    N, V = x.shape
    logp, H, lse = np.full(N, np.nan), np.full(N, np.nan), np.full(N, np.nan)
    tl, ti = np.full((N, top), np.nan), np.full((N, top), -1, np.int32)
    for n in range(N):
        r = x[n]
        if np.isnan(r).any() or (r == np.inf).any():
            continue
        tl[n] = -np.inf
        ok = 0 <= labels[n] < V
        if (r == -np.inf).all():
            lse[n], H[n] = -np.inf, 0.0
            logp[n] = -np.inf if ok else np.nan
            continue
        m = r.max()
        e = np.exp(r - m)
        lse[n] = m + np.log(e.sum())
        q = (r - m) - np.log(e.sum())          # (not r - lse: log V is lost beside logits of 1e38)
        p = np.exp(q)
        H[n] = -np.sum(p[p > 0] * q[p > 0])
        if ok:
            logp[n] = q[labels[n]]
        order = np.lexsort((np.arange(V), -r))[:top]
        order = order[r[order] > -np.inf]
        tl[n, :len(order)], ti[n, :len(order)] = q[order], order
    return logp, H, lse, tl, ti


def log_probs_backward(x, labels, lse, H, a, b):
    x, lse = np.asarray(x, np.float64), np.asarray(lse, np.float64)
    N, V = x.shape
    out, size = np.zeros((N, V)), np.zeros((N, V))
    for n in range(N):
        if lse[n] == -np.inf:
            continue
        q = x[n] - lse[n]
        p = np.exp(q)
        hot = (np.arange(V) == labels[n]).astype(float)
        fine = np.where(p > 0, q, 0.0)
        out[n] = a[n] * (hot - p) - b[n] * p * (fine + H[n])
        size[n] = abs(a[n]) * (hot + p) * (1 + np.abs(fine)) + abs(b[n]) * p * (np.abs(fine) + H[n]) * (1 + np.abs(fine))
    return out, size


def softmax_gradient(x, labels, a, b):
    """a ([i = y] - p) - b p (log p + H) of the rows' own softmax in 64 bits: (gradient, p, log p, H)."""
    x = np.asarray(x, np.float64)
    N, V = x.shape
    out, ps, qs, hs = np.full((N, V), np.nan), np.zeros((N, V)), np.zeros((N, V)), np.zeros(N)
    for n in range(N):
        r = x[n]
        if np.isnan(r).any() or (r == np.inf).any():
            continue
        out[n] = 0.0
        if (r == -np.inf).all():
            continue
        q = r - r.max()
        q = q - np.log(np.exp(q).sum())
        p = np.exp(q)
        fine = np.where(p > 0, q, 0.0)
        H = -(p * fine).sum()
        out[n] = a[n] * ((np.arange(V) == labels[n]) - p) - b[n] * p * (fine + H)
        ps[n], qs[n], hs[n] = p, q, H
    return out, ps, qs, hs


# ---- AdamW ---------------------------------------------------------------------------------------------------------
def philox(counter, seed, stream):
    """Words [n, 4] of Philox4x32-10 for uint64 counters."""
    c = np.asarray(counter, np.uint64)
    low = np.uint64(0xFFFFFFFF)
    x = [c & low, c >> np.uint64(32), np.full_like(c, stream), np.zeros_like(c)]
    ka, kb = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    for _ in range(10):
        p0, p1 = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(p1 >> np.uint64(32)) ^ x[1] ^ np.uint64(ka), p1 & low, (p0 >> np.uint64(32)) ^ x[3] ^ np.uint64(kb), p0 & low]
        ka, kb = (ka + 0x9E3779B9) & 0xFFFFFFFF, (kb + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(x, 1).astype(np.uint32)


def adamw_places(offsets):
    """Slot and place in the block of every element."""
    offsets = np.asarray(offsets, np.int64)
    n = np.diff(offsets)
    t = np.repeat(np.arange(len(n)), n)
    local = np.arange(offsets[-1]) - offsets[t]
    return offsets[t] // 256 + t + local // 256, local % 256


def adamw_decode(code, scale, offsets, top):
    slot, _ = adamw_places(offsets)
    s = np.asarray(scale, np.int64)[slot]
    c = np.asarray(code, np.int64)
    t = (c & top) + s - top
    x = np.where(((c & top) > 0) & (t > 0), t << 20, 0).astype(np.uint32).view(F32)
    return np.where(s < 0, np.nan, np.where(c > top, -x, x)).astype(F32)


def adamw_encode(x, r16, offsets, slots, top, old_scale):
    """Codes and the slots' scales (those of slots without elements stay)."""
    slot, _ = adamw_places(offsets)
    bits = np.abs(np.asarray(x, F32)).view(np.uint32).astype(np.int64)
    largest = np.full(slots, -1, np.int64)
    np.maximum.at(largest, slot, bits)
    scale = np.where(largest < 0, old_scale, np.where(largest >= 0x7F800000, -1, (largest >> 20) + 1))
    t = np.minimum((bits + 16 * r16.astype(np.int64) + 8) >> 20, 0x7F7)
    c = np.maximum(t - scale[slot] + top, 0)
    c = np.where(bits > 0, np.maximum(c, 1), c) if top == 255 else c | np.where(x < 0, 128, 0)
    return c.astype(np.uint8), scale.astype(np.int16)


def adamw_step(theta, g, m, v, wd, lr, b1, b2, eps, t):
    """One step in fp32, one rounding per operation; m and v fp32."""
    lr, b1, b2, eps = F32(lr), F32(b1), F32(b2), F32(eps)
    om1, om2 = F32(1.0 - float(b1)), F32(1.0 - float(b2))
    c1, c2 = F32(1.0 / (1.0 - float(b1) ** t)), F32(1.0 / (1.0 - float(b2) ** t))
    with np.errstate(all="ignore"):
        m = b1 * m + om1 * g
        v = b2 * v + om2 * (g * g)
        u = (m * c1) / (np.sqrt(v * c2) + eps)
        return theta - lr * (u + np.asarray(wd, F32) * theta), m, v


def bf16_round(x):
    b = np.asarray(x, F32).view(np.uint32).astype(np.uint64)
    return ((b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(F32)
