"""Oracle of include/cnnk_rel.h in numpy float64: the counter-based generator, dropout, and self-attention with a relative
position bias, forward and backward, written out with whole score matrices."""
import numpy as np

M0, M1, W0, W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85
LOW = np.uint64(0xFFFFFFFF)


def philox(ctr, key, rounds=7):
    """Philox4x32: four 32-bit words (arrays or numbers) from a counter of four and a key of two."""
    c = [np.asarray(x, dtype=np.uint64) for x in ctr]
    k = [int(x) for x in key]
    s = np.uint64(32)
    for _ in range(rounds):
        a, b = c[0] * np.uint64(M0), c[2] * np.uint64(M1)
        c = [(b >> s) ^ c[1] ^ np.uint64(k[0]), b & LOW, (a >> s) ^ c[3] ^ np.uint64(k[1]), a & LOW]
        k = [(k[0] + W0) & 0xFFFFFFFF, (k[1] + W1) & 0xFFFFFFFF]
    return c


def site_key(seed, step, site):
    lo, hi = 0xFFFFFFFF, 32
    w = philox((step & lo, step >> hi, site, 0), (seed & lo, seed >> hi))
    return int(w[0]), int(w[1])


def share(p):
    """(threshold of the 16-bit draws, factor of what is kept)"""
    q = int(np.floor(float(np.float32(p)) * 65536.0 + 0.5))
    return q, 65536.0 / (65536.0 - q)


def pieces(words):
    """[..., 8] 16-bit draws of four words, low halves first."""
    w = np.stack(words, -1)
    return np.stack((w & np.uint64(0xFFFF), w >> np.uint64(16)), -1).reshape(w.shape[:-1] + (8,))


def keep_elements(n, p, key, tag=0):
    q, f = share(p)
    i = np.arange((n + 7) // 8, dtype=np.uint64)
    z = np.zeros_like(i)
    return np.where(pieces(philox((i & LOW, i >> np.uint64(32), z, z + np.uint64(tag)), key)).reshape(-1)[:n] >= q, f, 0.0)


def keep_dropout(rows, C, p, span, key):
    """Factor of every element, [rows][C]."""
    if span == 0:
        return keep_elements(rows * C, p, key).reshape(rows, C)
    g = keep_elements((rows + span - 1) // span, p, key, tag=1)
    return np.broadcast_to(g[np.arange(rows) // span][:, None], (rows, C))


def keep_pairs(B, heads, T, p, key):
    """Factor of every probability, [B][heads][T][T]."""
    q, f = share(p)
    bh, t, u = np.arange(B * heads, dtype=np.uint64), np.arange(T, dtype=np.uint64), np.arange(T, dtype=np.uint64)
    c = np.broadcast_arrays(u[None, None, :] // np.uint64(2), t[None, :, None] // np.uint64(4), bh[:, None, None])
    w = philox((c[0], c[1], c[2], np.full_like(c[0], 2)), key)
    word = np.choose((t % np.uint64(4)).astype(np.int64)[None, :, None], w)
    draw = (word >> (np.uint64(16) * (u % np.uint64(2)))[None, None, :]) & np.uint64(0xFFFF)
    return np.where(draw >= q, f, 0.0).reshape(B, heads, T, T)


def grid_buckets(gh, gw, cls):
    T, n = gh * gw + (1 if cls else 0), (2 * gh - 1) * (2 * gw - 1)
    m = np.zeros((T, T), dtype=np.int32)
    for t in range(T):
        for u in range(T):
            a, b = t - (1 if cls else 0), u - (1 if cls else 0)
            if a < 0 or b < 0:
                m[t, u] = n + 2 if a < 0 and b < 0 else n if a < 0 else n + 1
            else:
                m[t, u] = (a // gw - b // gw + gh - 1) * (2 * gw - 1) + a % gw - b % gw + gw - 1
    return m


def attention(qkv, heads, table=None, bucket=None, lens=None, keep=None, d_o=None):
    """qkv [B][T][3 * heads * dh]; table [buckets][heads]; keep [B][heads][T][T] or None.  A dict: o, top, log (statistics of the
    rows), and with d_o dqkv, dtable; also the absolute sums that bound what rounding can do (bound_*)."""
    B, T, w = qkv.shape
    dh = w // 3 // heads
    q, k, v = (np.ascontiguousarray(qkv.reshape(B, T, 3, heads, dh)[:, :, i].transpose(0, 2, 1, 3)) for i in range(3))
    ok = np.ones((B, 1, T, T), dtype=bool)
    if lens is not None:
        n = np.clip(np.asarray(lens), 0, T)
        inside = np.arange(T)[None, :] < n[:, None]
        ok = ok & inside[:, None, :, None] & inside[:, None, None, :]
        q, k, v = (np.where(inside[:, None, :, None], a, 0.0) for a in (q, k, v))
    bias = 0.0
    if bucket is not None:
        seen = (bucket >= 0) & (bucket < table.shape[0])
        ok = ok & seen[None, None]
        bias = np.where(seen[..., None], table[np.where(seen, bucket, 0)], 0.0).transpose(2, 0, 1)[None]
    s = 1.0 / np.sqrt(dh)
    kt = k.transpose(0, 1, 3, 2)
    x = np.where(ok, q @ kt * s + bias, -np.inf)
    top = x.max(-1, keepdims=True)
    empty = np.isneginf(top)
    e = np.where(np.isneginf(x), 0.0, np.exp(np.where(np.isneginf(x), 0.0, x) - np.where(empty, 0.0, top)))
    total = e.sum(-1, keepdims=True)
    P = e / np.where(empty, 1.0, total)
    keep = np.ones_like(P) if keep is None else keep
    D = P * keep
    O = D @ v
    back = lambda a: a.transpose(0, 2, 1, 3).reshape(B, T, heads * dh)
    r = dict(o=back(O), top=top[..., 0], log=np.where(empty, 0.0, np.log(np.where(empty, 1.0, total)))[..., 0], scores=np.abs(q) @ np.abs(kt) * s,
             bound_o=back(D @ np.abs(v)), probs=P)
    if d_o is None:
        return r
    g = np.ascontiguousarray(d_o.reshape(B, T, heads, dh).transpose(0, 2, 1, 3))
    if lens is not None:
        g = np.where(inside[:, None, :, None], g, 0.0)
    vt = v.transpose(0, 1, 3, 2)
    dP = (g @ vt) * keep
    dx = P * (dP - (P * dP).sum(-1, keepdims=True))
    size = P * (keep * (np.abs(g) @ np.abs(vt)) + (np.abs(g) * (D @ np.abs(v))).sum(-1, keepdims=True))      # of the terms of dx, delta's among them
    t = lambda a: a.transpose(0, 1, 3, 2)
    three = lambda a, b, c: np.stack([z.transpose(0, 2, 1, 3) for z in (a, b, c)], 2).reshape(B, T, 3 * heads * dh)
    r["dqkv"] = three(dx @ k * s, t(dx) @ q * s, t(D) @ g)
    r["bound_dqkv"] = three(np.abs(dx) @ np.abs(k) * s, np.abs(t(dx)) @ np.abs(q) * s, t(D) @ np.abs(g))          # roundings of dx and D
    r["size_dqkv"] = three(size @ np.abs(k) * s, t(size) @ np.abs(q) * s, t(D) @ np.abs(g))                       # errors of dx's terms
    if bucket is not None:
        dt, st = np.zeros(table.shape), np.zeros(table.shape)
        ids = np.where(seen, bucket, 0)[seen]
        np.add.at(dt, ids, dx.sum(0).transpose(1, 2, 0)[seen])
        np.add.at(st, ids, size.sum(0).transpose(1, 2, 0)[seen])
        r["dtable"], r["size_dtable"] = dt, st
    return r
