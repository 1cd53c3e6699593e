"""Plain float64 forms of the operators around the MoC layer in training: layer norm and RMSNorm with their gradients, the 8-bit
stored set, and the softmax router.  Written from the definitions in include/moc.h; shares no code with the HIP path."""
import numpy as np


# ------------------------------------------------------------------------------------------------------------- norms
def norm_forward(h, gain, bias, eps, rms):
    """(out, n, r): n the normalised rows, r [T,1] what they were multiplied with."""
    mean = np.zeros((h.shape[0], 1)) if rms else h.mean(axis=1, keepdims=True)
    r = 1.0 / np.sqrt(((h - mean) ** 2).mean(axis=1, keepdims=True) + eps)
    n = (h - mean) * r
    return n * gain + (0.0 if bias is None else bias), n, r


def norm_backward(h, gain, eps, dy, dres, rms):
    """(dh, dgain, dbias)."""
    _, n, r = norm_forward(h, gain, None, eps, rms)
    p = dy * gain
    dh = p - n * (p * n).mean(axis=1, keepdims=True)
    if not rms:
        dh = dh - p.mean(axis=1, keepdims=True)
    return r * dh + (0.0 if dres is None else dres), (dy * n).sum(axis=0), dy.sum(axis=0)


# ---------------------------------------------------------------------------------------------------- 8-bit stored set
def pack8(v):
    """(q int8 [T,n], e uint8 [T, ceil(n/32)]) of float32 values v [T,n], block by block."""
    v = np.asarray(v, dtype=np.float32)
    T, n = v.shape
    q = np.zeros((T, n), dtype=np.int8)
    e = np.zeros((T, -(-n // 32)), dtype=np.uint8)
    for t in range(T):
        for b in range(e.shape[1]):
            blk = v[t, 32 * b:32 * b + 32]
            if not np.all(np.isfinite(blk)):
                e[t, b] = 255
                continue
            top = np.max(np.abs(blk))
            field = int(np.float32(top).view(np.uint32)) >> 23
            if field < 8:
                continue
            e[t, b] = field
            q[t, 32 * b:32 * b + 32] = np.clip(np.rint(blk.astype(np.float64) * 2.0 ** (133 - field)), -127, 127).astype(np.int8)
    return q, e


def unpack8(q, e):
    out = np.zeros(q.shape)
    for b in range(e.shape[1]):
        ex = e[:, b:b + 1].astype(np.float64)
        step = np.where(ex == 255, np.nan, np.where(ex < 8, 0.0, 2.0 ** (ex - 133)))
        out[:, 32 * b:32 * b + 32] = q[:, 32 * b:32 * b + 32] * step
    return out


def pack_mask(idx, F):
    words = np.zeros((idx.shape[0], -(-F // 32)), dtype=np.uint32)
    for t in range(idx.shape[0]):
        for j in idx[t]:
            words[t, j // 32] |= np.uint32(1 << (int(j) % 32))
    return words


def unpack_mask(words, F):
    """Rows of the set channels below F, ascending."""
    return [[j for j in range(F) if int(words[t, j // 32]) >> (j % 32) & 1] for t in range(words.shape[0])]


# ------------------------------------------------------------------------------------------------------------- router
def route(logits, k, valid=None, renorm=True):
    """Token by token.  Returns a dict: ids, weights, counts, order, loss, coef, p (zero rows for tokens without a slot)."""
    T, E = logits.shape
    ids = np.full((T, k), -1, dtype=np.int32)
    weights = np.zeros((T, k))
    p = np.zeros((T, E))
    for t in range(T):
        if valid is not None and not valid[t]:
            continue
        row = logits[t]
        ranked = sorted((e for e in range(E) if row[e] > -np.inf), key=lambda e: (-row[e], e))[:k]
        if not ranked:
            continue
        ex = np.exp(row - row[ranked[0]])
        p[t] = ex / ex.sum()
        ids[t, :len(ranked)] = ranked
        w = p[t, ranked]
        weights[t, :len(ranked)] = w / w.sum() if renorm else w
    counts = np.array([(ids == e).sum() for e in range(E)], dtype=np.int32)
    order = np.full(T * k, -1, dtype=np.int32)
    listed = [t * k + j for e in range(E) for t in range(T) for j in range(k) if ids[t, j] == e]
    order[:len(listed)] = listed
    A, N = counts.sum(), (ids[:, 0] >= 0).sum()
    coef = E * counts / (A * N) if A else np.zeros(E)
    return dict(ids=ids, weights=weights, counts=counts, order=order, coef=coef, loss=float((coef * p.sum(axis=0)).sum()), p=p)


def route_backward(r, dweights, dloss, renorm):
    """dlogits from what route() gave; dweights may be None."""
    ids, w, p, coef = r["ids"], r["weights"], r["p"], r["coef"]
    T, E = p.shape
    dl = dloss * p * (coef - (p * coef).sum(axis=1, keepdims=True))
    for t in range(T):
        live = ids[t] >= 0
        if dweights is None or not live.any():
            continue
        e, wt, dw = ids[t, live], w[t, live], dweights[t, live]
        base = np.zeros(E)
        if renorm:
            base[e] = wt
        else:
            base = p[t].copy()
        dl[t, e] += wt * dw
        dl[t] -= base * (wt * dw).sum()
    return dl
