"""Plain CPU definitions of the calls on single cached tokens for the tests, in float64 NumPy,
written per sequence and KV head from include/locks_tokens.h."""
import numpy as np
import torch

D = 128


def rows_of(cache, table, h, L, P):
    """cache [blocks][H][P][128] (torch) -> float64 [L][128]: the sequence's rows of head h."""
    out = np.zeros((L, D))
    for t in range(L):
        out[t] = cache[int(table[t // P]), h, t % P].double().numpy()
    return out


def sees(n, L, mask):
    """bool [n][L]: what each of the n newest tokens sees; mask int [n][words] or None."""
    first = L - n
    ok = np.zeros((n, max(L, 0)), bool)
    for i in range(n):
        for t in range(L):
            j = t - first
            if j < 0:
                ok[i, t] = True
            elif mask is None:
                ok[i, t] = j <= i
            else:
                ok[i, t] = j < 32 * mask.shape[1] and bool(int(mask[i, j // 32]) >> (j % 32) & 1)
    return ok


def attend(q, K, V, ok):
    """q [n][G][128], K / V [L][128], ok [n][L].  Returns out, lse, and for the bounds the
    largest sum |q k| / sqrt d over seen pairs."""
    n, G = q.shape[:2]
    out, lse, big = np.zeros((n, G, D)), np.full((n, G), -np.inf), 0.0
    for i in range(n):
        if not ok[i].any():
            continue
        k, v = K[ok[i]], V[ok[i]]
        z = q[i] @ k.T / np.sqrt(D)
        big = max(big, float((np.abs(q[i]) @ np.abs(k).T).max() / np.sqrt(D)))
        m = z.max(1, keepdims=True)
        p = np.exp(z - m)
        l = p.sum(1, keepdims=True)
        out[i], lse[i] = p @ v / l, (m + np.log(l))[:, 0]
    return out, lse, big


def weights(q, K, ok, lse):
    """What token_mass adds: [L], and the largest |z - lse|."""
    L = K.shape[0]
    add, far = np.zeros(L), 0.0
    for i in range(q.shape[0]):
        for g in range(q.shape[1]):
            if np.isneginf(lse[i, g]):
                continue
            d = q[i, g] @ K[ok[i]].T / np.sqrt(D) - lse[i, g]
            add[ok[i]] += np.exp(d)
            far = max(far, float(np.abs(d).max(initial=0)))
    return add, far


def pick(mass, L, n_keep, n_sink, n_recent):
    """mass [width] float32 -> the kept tokens, ascending."""
    if L <= n_keep:
        return list(range(L))
    sure = set(range(n_sink)) | set(range(L - n_recent, L))
    x = np.where(np.isnan(mass[:L]), -np.inf, mass[:L]).astype(np.float64)
    nan = np.isnan(mass[:L])
    rest = sorted((t for t in range(L) if t not in sure), key=lambda t: (nan[t], -x[t], t))
    return sorted(sure | set(rest[:n_keep - len(sure)]))


def keep(kept, start, caches, mass, table, P):
    """One sequence: kept [heads][n], caches (k, v) torch [blocks][H][P][128], mass [H][width]
    or None, all changed in place.  Returns the new length."""
    H = caches[0].shape[1]
    count = 0
    for h in range(H):
        ids = kept[h if len(kept) > 1 else 0]
        old = [c.clone() for c in caches]
        was = None if mass is None else mass[h].clone()
        n = next((i for i, t in enumerate(ids) if t < 0), len(ids))
        for i, t in enumerate(ids[:n]):
            if t < start + i:
                continue
            a, b = (int(table[x // P]) for x in (t, start + i))
            for c, o in zip(caches, old):
                c[b, h, (start + i) % P] = o[a, h, t % P]
            if mass is not None:
                mass[h, start + i] = was[t]
        if h == 0:
            count = n
    return start + count


def table_of(lens, P, gen, spare=3, extra=1):
    pages = [max(1, -(-L // P)) for L in lens]
    nb = sum(pages) + spare
    perm = torch.randperm(nb, generator=gen).int()
    table = torch.full((len(lens), max(pages) + extra), -1, dtype=torch.int32)
    off = 0
    for s, n in enumerate(pages):
        table[s, :n] = perm[off:off + n]
        off += n
    return table, nb
