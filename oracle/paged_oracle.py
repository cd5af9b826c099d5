"""Float64 CPU oracle of the paged routed cache, written from the formulas in
include/rolesub.h. A cache is a dict of numpy arrays K [n,H,P,dh], V [n,H,vcap,ds],
mask [n,P], slot [n,P]; every step is a plain loop over tokens."""
import numpy as np


def rotary(x, positions, inv_freq, axis=None, interleaved=False, inverse=False):
    """x [B,T,H,dh], positions [B,T,A]."""
    y = np.array(x, dtype=np.float64)
    n, A = len(inv_freq), positions.shape[2]
    for i in range(n):
        ax = 0 if axis is None else int(axis[i])
        if ax >= A:
            continue
        a = positions[:, :, ax].astype(np.longdouble) * np.longdouble(inv_freq[i])
        c = np.cos(a).astype(np.float64)[:, :, None]
        s = (np.sin(a).astype(np.float64) * (-1.0 if inverse else 1.0))[:, :, None]
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, n + i)
        u, v = y[..., p].copy(), y[..., q].copy()
        y[..., p], y[..., q] = u * c - v * s, u * s + v * c
    return y


def kept(mask, G):
    return [g for g in range(G) if int(mask) >> g & 1]


def cell(cache, row, t):
    """(page, row in it) of token t, or None where its page is not one."""
    P, n = cache["K"].shape[2], cache["K"].shape[0]
    if t // P >= len(row):
        return None
    page = int(row[t // P])
    return (page, t % P) if 0 <= page < n else None


def place(cache, at, slot, key, groups, mask, G):
    """One token's key, kept groups ([H, G, ds]) and metadata."""
    page, r = at
    cache["K"][page, :, r] = key
    cache["mask"][page, r] = mask
    cache["slot"][page, r] = slot
    for i, g in enumerate(kept(mask, G)):
        if 0 <= slot + i < cache["V"].shape[2]:
            cache["V"][page, :, slot + i] = groups[:, g]


def append(cache, k, z, mask, table, lens, n_new=None):
    """Writes into the cache in place."""
    B, T, H, dh = k.shape
    P, G = cache["K"].shape[2], dh // cache["V"].shape[3]
    cap = table.shape[1] * P
    for b in range(B):
        n0 = min(max(int(lens[b]), 0), cap)
        for j in range(T if n_new is None else min(max(int(n_new[b]), 0), T)):
            at = cell(cache, table[b], n0 + j)
            if at is None:
                continue
            slot = 0
            if at[1] > 0:
                slot = int(cache["slot"][at[0], at[1] - 1]) + len(kept(cache["mask"][at[0], at[1] - 1], G))
            place(cache, at, slot, k[b, j], z[b, j].reshape(H, G, -1), mask[b, j], G)


def token(cache, row, t):
    """Key [H,dh], groups [H,G,ds] (dropped ones zero) and mask of a cached token, or None."""
    at = cell(cache, row, t)
    if at is None:
        return None
    H, dh = cache["K"].shape[1], cache["K"].shape[3]
    ds, vcap = cache["V"].shape[3], cache["V"].shape[2]
    G = dh // ds
    z = np.zeros((H, G, ds))
    m, s = cache["mask"][at], int(cache["slot"][at])
    for i, g in enumerate(kept(m, G)):
        if 0 <= s + i < vcap:
            z[:, g] = cache["V"][at[0], :, s + i]
    return np.asarray(cache["K"][at[0], :, at[1]], dtype=np.float64), z, m


def attend(q, cache, table, lens, R=None, scale=0.0, visible=None, max_len=0, mass=None, decay=1.0):
    """out [B,Tq,Hq,dh], the accumulated weight [B,L] (mass None: from zero), and
    per output the sum of |R| P |z| that its error is measured by."""
    B, Tq, Hq, dh = q.shape
    H, P = cache["K"].shape[1], cache["K"].shape[2]
    rep, cap = Hq // H, table.shape[1] * P
    cap = min(cap, max_len) if max_len else cap
    scale = scale or dh ** -0.5
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    w = np.zeros((B, cap)) if mass is None else np.array(mass, dtype=np.float64)
    logit = 0.0  # largest sum of |q k| scale
    for b in range(B):
        n = min(max(int(lens[b]), 0), cap)
        toks = [(t, token(cache, table[b], t)) for t in range(n)]
        toks = [(t, x) for t, x in toks if x is not None]
        if mass is not None:
            w[b, :n] *= decay
        for j in range(Tq):
            see = n if visible is None else min(n, int(visible[b, j]))
            mine = [(t, x) for t, x in toks if t < see]
            if not mine:
                continue
            ts = [t for t, _ in mine]
            for h in range(Hq):
                K = np.stack([x[0][h // rep] for _, x in mine])
                Z = np.stack([x[1][h // rep].reshape(-1) for _, x in mine])
                qv = np.asarray(q[b, j, h], dtype=np.float64)
                s = K @ qv * scale
                logit = max(logit, float(np.max(np.abs(K) @ np.abs(qv))) * abs(scale))
                e = np.exp(s - s.max())
                p = e / e.sum()
                u, a = p @ Z, p @ np.abs(Z)
                if R is not None:
                    Rh = np.asarray(R[h // rep], dtype=np.float64)
                    u, a = Rh @ u, np.abs(Rh) @ a
                out[b, j, h], size[b, j, h] = u, a
                w[b, ts] += p
    return out, w, size, logit


def evict(mass, lens, keep, first=0, recent=0):
    B = mass.shape[0]
    idx, n = np.full((B, keep), -1, dtype=np.int32), np.zeros(B, dtype=np.int32)
    for b in range(B):
        ln = min(max(int(lens[b]), 0), mass.shape[1])
        stay = list(range(ln))
        if ln > keep:
            safe = [t for t in stay if t < first or t >= ln - recent]
            rest = np.arange(first, ln - recent)
            # a larger value first, NaN last, then the lower index
            m = mass[b, first:ln - recent]
            rest = rest[np.lexsort((rest, np.where(np.isnan(m), 0.0, -m), np.isnan(m)))]
            stay = sorted(safe + rest[: keep - len(safe)].tolist())
        n[b] = len(stay)
        idx[b, : len(stay)] = stay
    return idx, n


def compact(src, table, keep_idx, n_keep, dst, dst_table):
    """Writes into dst in place."""
    G = src["K"].shape[3] // src["V"].shape[3]
    P = dst["K"].shape[2]
    for b in range(table.shape[0]):
        slot = 0
        for j in range(min(max(int(n_keep[b]), 0), keep_idx.shape[1])):
            t = int(keep_idx[b, j])
            x = token(src, table[b], t) if t >= 0 else None
            if x is None:
                x = (np.zeros(src["K"].shape[1::2]), np.zeros((src["K"].shape[1], G, src["V"].shape[3])), 0)
            slot = 0 if j % P == 0 else slot
            at = cell(dst, dst_table[b], j)
            if at is not None:
                place(dst, at, slot, x[0], x[1], x[2], G)
            slot += len(kept(x[2], G))
