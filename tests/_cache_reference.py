"""Plain CPU definitions of the paged-cache operators for the tests, written per token and
page from include/locks_cache.h: the appends in float32 NumPy, whose every operation is
the one rounding that the header names (so codes and scales can be compared bit for bit),
and everything in float64 for the bounds."""
import numpy as np
import torch

D = 128
QMAX = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


def angles(n_pos, rot, base=10000.0):
    a = np.arange(n_pos)[:, None] * base ** (-2.0 * np.arange(rot // 2) / rot)
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def pairs(rot, interleaved):
    half = rot // 2
    i = np.arange(half)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + half)


def rotate(x, table, interleaved, axis_pairs, pos, dtype):
    """x [heads][128] of one token, pos [n_axes]; every operation in `dtype`."""
    rot, half = table.shape[1], table.shape[1] // 2
    axis = np.repeat(np.arange(len(axis_pairs)), axis_pairs)
    at = np.asarray(pos)[axis]
    c, s = (table[at, np.arange(half) + o].astype(dtype) for o in (0, half))
    a, b = pairs(rot, interleaved)
    y = x.astype(dtype).copy()
    xa, xb = y[:, a].copy(), y[:, b].copy()
    y[:, a] = xa * c - xb * s
    y[:, b] = xb * c + xa * s
    return y


def rotate_bound(x, table, interleaved, axis_pairs, pos):
    """|a c| + |b s| of every element (0 where nothing is rotated): three float32 roundings
    are off by less than 2^-22 of it."""
    rot, half = table.shape[1], table.shape[1] // 2
    axis = np.repeat(np.arange(len(axis_pairs)), axis_pairs)
    at = np.asarray(pos)[axis]
    c, s = (np.abs(table[at, np.arange(half) + o].astype(np.float64)) for o in (0, half))
    a, b = pairs(rot, interleaved)
    x = np.abs(x.astype(np.float64))
    y = np.zeros_like(x)
    y[:, a] = x[:, a] * c + x[:, b] * s
    y[:, b] = x[:, b] * c + x[:, a] * s
    return y


def page_scale(amax, code):
    """float32 scale of a page whose largest finite magnitude is amax (float32)."""
    if not amax >= np.float32(2.0 ** -100):
        return np.float32(0)
    if code == torch.int8:
        return np.float32(amax) / np.float32(127)
    m, e = np.frexp(np.float64(amax))          # amax = m 2^e, m in [0.5, 1)
    return np.float32(2.0 ** (int(e) - 9 + (m > 0.875)))


def to_codes(x, code):
    """float32 -> codes (as a torch tensor), nearest, ties to even, saturating, NaN -> 0 (int8)."""
    x = np.asarray(x, np.float32)
    if code == torch.int8:
        y = np.clip(np.rint(x), -127, 127)
        return torch.from_numpy(np.where(np.isnan(x), 0, y).astype(np.int8))
    return torch.from_numpy(np.clip(x, -448, 448)).to(code)


def code_values(codes):
    return codes.float().numpy()


def q8_append_page(codes, scale, rows, earlier, code):
    """One page, KV head and tensor.  codes [B][128] (torch, changed in place), its scale,
    rows {page row: float32 [128]} new this call, `earlier` rows written by earlier calls.
    Returns the page's new scale."""
    if not rows:
        return scale
    x = np.stack(list(rows.values())).astype(np.float32)
    mag = np.abs(x)
    amax = np.float32(np.max(np.where(np.isfinite(x), mag, 0)))
    new = page_scale(amax, code)
    if earlier > 0 and not new > scale:
        new = np.float32(scale)
    with np.errstate(all="ignore"):
        inv = np.float32(1) / new if new > 0 else np.float32(0)
        if earlier > 0 and new > scale:
            old = code_values(codes[:earlier])
            codes[:earlier] = to_codes(old * np.float32(scale) * inv, code)
        for i, r in rows.items():
            codes[i] = to_codes(r.astype(np.float32) * inv, code)
    return new


def attend(q, codes_k, codes_v, ks, vs, table, ids, L, P):
    """float64 attention of q [G][128] over the tokens < L of pages `ids`; one KV head:
    codes [nb][P][128] (torch), scales [nb].  Returns out [G][128], lse [G], and for the
    bounds: the largest sum |q k| sk / sqrt d, and max |v| per channel."""
    K, V = [], []
    for j in ids:
        for t in range(P):
            if j * P + t < L:
                b = int(table[j])
                K.append(code_values(codes_k[b, t]).astype(np.float64) * np.float64(ks[b]))
                V.append(code_values(codes_v[b, t]).astype(np.float64) * np.float64(vs[b]))
    G = q.shape[0]
    if not K:
        return np.zeros((G, D)), np.full(G, -np.inf), 0.0, np.zeros(D)
    K, V, q = np.stack(K), np.stack(V), q.astype(np.float64)
    z = q @ K.T / np.sqrt(D)
    m = z.max(1, keepdims=True)
    p = np.exp(z - m)
    l = p.sum(1, keepdims=True)
    big = float((np.abs(q) @ np.abs(K).T).max() / np.sqrt(D))
    return p @ V / l, (m + np.log(l))[:, 0], big, np.abs(V).max(0)
