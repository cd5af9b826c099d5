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


# ---- normed heads, drafted tokens, few pages ------------------------------

def norm(x, weight, eps):
    """x [..,dh] over its root mean square, weighted."""
    x = np.asarray(x, dtype=np.longdouble)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + np.longdouble(eps)) * np.asarray(weight, dtype=np.longdouble)
    return y.astype(np.float64)


def norm_rotary(x, weight, eps, positions, inv_freq, axis=None, interleaved=False):
    return rotary(x if weight is None else norm(x, weight, eps), positions, inv_freq, axis, interleaved)


def tree_masks(parents):
    """Ancestors of each drafted token, itself among them, as sets; and how many others."""
    sets = []
    for row in np.asarray(parents).tolist():
        mine = []
        for j, p in enumerate(row):
            mine.append((mine[p] if 0 <= p < j else set()) | {j})
        sets.append(mine)
    return sets, [[len(s) - 1 for s in row] for row in sets]


def tree_words(sets, T):
    """The same as words [.., T, ceil(T / 32)]."""
    w = np.zeros((len(sets), T, -(-T // 32)), dtype=np.uint32)
    for b, row in enumerate(sets):
        for j, s in enumerate(row):
            for i in s:
                w[b, j, i // 32] |= np.uint32(1 << (i % 32))
    return w


def attend_over(q, cache, sees, R=None, scale=0.0):
    """q [B,Tq,Hq,dh] over the cells (page, row) that sees(b, j, key head) lists. As `attend`: out, and what its error is
    measured by."""
    B, Tq, Hq, dh = q.shape
    H, vcap, ds = cache["K"].shape[1], cache["V"].shape[2], cache["V"].shape[3]
    rep, G = Hq // H, dh // ds
    scale = scale or dh ** -0.5
    out, size, logit = np.zeros(q.shape), np.zeros(q.shape), 0.0
    for b in range(B):
        for j in range(Tq):
            for g in range(H):
                cells = sees(b, j, g)
                if not cells:
                    continue
                K = np.stack([np.asarray(cache["K"][p, g, r], dtype=np.float64) for p, r in cells])
                Z = np.zeros((len(cells), G, ds))
                for t, (p, r) in enumerate(cells):
                    for i, x in enumerate(kept(cache["mask"][p, r], G)):
                        s = int(cache["slot"][p, r]) + i
                        if 0 <= s < vcap:
                            Z[t, x] = cache["V"][p, g, s]
                Z = Z.reshape(len(cells), dh)
                for h in range(g * rep, (g + 1) * rep):
                    qv = np.asarray(q[b, j, h], dtype=np.float64)
                    s = K @ qv * scale
                    logit = max(logit, float(np.max(np.abs(K) @ np.abs(qv))) * abs(scale))
                    e = np.exp(s - s.max())
                    p = e / e.sum()
                    u, a = p @ Z, p @ np.abs(Z)
                    if R is not None:
                        Rh = np.asarray(R[g], dtype=np.float64)
                        u, a = Rh @ u, np.abs(Rh) @ a
                    out[b, j, h], size[b, j, h] = u, a
    return out, size, logit


def tree_sees(cache, table, lens, sets, Tq, n_new=None, max_len=0):
    """What rows of drafted tokens see, for attend_over."""
    cap = table.shape[1] * cache["K"].shape[2]
    cap = min(cap, max_len) if max_len else cap

    def sees(b, j, g):
        n = Tq if n_new is None else min(max(int(n_new[b]), 0), Tq)
        if j >= n:
            return []
        base = max(int(lens[b]), 0)
        mine = sets[b if len(sets) > 1 else 0][j]
        ts = list(range(min(base, cap))) + [base + i for i in sorted(mine) if i < n and base + i < cap]
        return [x for x in (cell(cache, table[b], t) for t in ts) if x is not None]
    return sees


def accept(cache, table, lens, sets, leaf):
    """Moves the paths in place and returns the new lengths."""
    P = cache["K"].shape[2]
    G = cache["K"].shape[3] // cache["V"].shape[3]
    old = {x: cache[x].copy() for x in cache}
    new = []
    for b in range(table.shape[0]):
        base = min(max(int(lens[b]), 0), table.shape[1] * P)
        rows = sets[b if len(sets) > 1 else 0]
        path = sorted(rows[int(leaf[b])]) if 0 <= int(leaf[b]) < len(rows) else []
        new.append(base + len(path))
        slot = 0
        first = cell(old, table[b], base - 1) if base % P else None
        if first is not None:
            slot = int(old["slot"][first]) + len(kept(old["mask"][first], G))
        for j, i in enumerate(path):
            t = base + j
            if t % P == 0:
                slot = 0
            src, dst = cell(old, table[b], base + i), cell(cache, table[b], t)
            x = token(old, table[b], base + i)
            if x is None:
                x = (np.zeros(old["K"].shape[1::2]), np.zeros((old["K"].shape[1], G, old["V"].shape[3])), 0)
            mask = 0 if src is None else old["mask"][src]
            if dst is not None:
                place(cache, dst, slot, x[0], x[1], mask, G)
            slot += len(kept(mask, G))
    return np.array(new)


def page_bounds(cache, table, lens, bounds, T):
    """Writes into bounds [n,H,2,dh] in place."""
    P = cache["K"].shape[2]
    n = [min(max(int(x), 0), table.shape[1] * P) for x in lens]
    for b in range(table.shape[0]):
        for i in range(max(n[b] - T, 0) // P, -(-n[b] // P)):
            pg = int(table[b, i])
            if T > 0 and 0 <= pg < cache["K"].shape[0]:
                held = max(n[x] - i * P for x in range(table.shape[0]) if int(table[x, i]) == pg)  # of those that share it
                k = cache["K"][pg, :, :min(P, held)]
                bounds[pg, :, 0] = np.fmin.reduce(np.where(np.isnan(k), np.inf, k), axis=1)
                bounds[pg, :, 1] = np.fmax.reduce(np.where(np.isnan(k), -np.inf, k), axis=1)


def select_pages(q, cache, bounds, table, lens, n_sel, first=0, recent=0, visible=None, max_len=0):
    B, Tq, Hq, dh = q.shape
    n_pages, H, P = cache["K"].shape[:3]
    rep, cap = Hq // H, table.shape[1] * P
    cap = min(cap, max_len) if max_len else cap
    sel = np.full((B, Tq, H, n_sel), -1, dtype=np.int32)
    for b in range(B):
        for j in range(Tq):
            n = min(max(int(lens[b]), 0), cap)
            n = n if visible is None else min(n, max(int(visible[b, j]), 0))
            m = -(-n // P)
            for g in range(H):
                score = np.full(m, np.nan, dtype=np.float32)
                for i in range(m):
                    pg = int(table[b, i])
                    if not 0 <= pg < n_pages:
                        continue
                    lo, hi = bounds[pg, g]
                    best = []
                    for h in range(g * rep, (g + 1) * rep):
                        x = np.asarray(q[b, j, h], dtype=np.float64)
                        with np.errstate(invalid="ignore"):
                            best.append(np.float32(np.where(x < 0, x * lo, x * hi).sum()))
                    score[i] = np.nan if np.isnan(best).any() else max(best)
                if m <= n_sel:
                    mine = list(range(m))
                else:
                    safe = [i for i in range(m) if i < first or i >= m - recent]
                    free = np.array([i for i in range(m) if first <= i < m - recent], dtype=int)
                    s = score[free]
                    order = np.lexsort((free, np.where(np.isnan(s), 0.0, -s), np.isnan(s)))
                    mine = sorted(safe + free[order][: n_sel - len(safe)].tolist())
                sel[b, j, g, : len(mine)] = mine
    return sel


def selected_sees(cache, table, lens, sel, visible=None):
    """What rows see of listed pages, for attend_over."""
    P = cache["K"].shape[2]

    def sees(b, j, g):
        n = min(max(int(lens[b]), 0), table.shape[1] * P)
        n = n if visible is None else min(n, int(visible[b, j]))
        ts = [i * P + r for i in sel[b, j, g].tolist() if 0 <= i < table.shape[1] for r in range(P) if i * P + r < n]
        return [x for x in (cell(cache, table[b], t) for t in ts) if x is not None]
    return sees
