"""Plain NumPy statement of the attention operators: softmax attention over packed sequences in float64, and the 4-bit
key/value cache (rotation, codes, scales, page layout)."""

import numpy as np


def rotate_f32(x):
    """x . H / sqrt(D) over the last axis in float32, butterflies of distance 1, 2, 4, ... and the factor last; each
    butterfly output is one float32 sum or difference, so the result is fixed to the bit."""
    y = np.array(x, dtype=np.float32)
    dim, h = y.shape[-1], 1
    while h < dim:
        z = y.reshape(*y.shape[:-1], dim // (2 * h), 2, h)
        a, b = z[..., 0, :], z[..., 1, :]
        y = np.stack((a + b, a - b), axis=-2).reshape(y.shape)
        h *= 2
    return y * np.float32(1.0 / np.sqrt(dim))


def hadamard(dim):
    m = np.ones((1, 1))
    while m.shape[0] < dim:
        m = np.block([[m, m], [m, -m]])
    return m / np.sqrt(dim)


def quantize_heads(x, rotate):
    """Codes int8 [..., D] and float32 scales [...] of heads x: scale max |y| / 7, round half to even on the exact quotient
    (that of two float32 numbers is decided by a float64 one); a head with a NaN or an infinity has a NaN scale."""
    with np.errstate(all="ignore"):
        y = rotate_f32(x) if rotate else np.array(x, dtype=np.float32)
        top = np.abs(y).max(-1)
        d = (top / np.float32(7.0)).astype(np.float32)
        d = np.where(np.isfinite(top), d, np.float32(np.nan))
        t = y.astype(np.float64) / d[..., None].astype(np.float64)
        codes = np.where((d > 0)[..., None], np.clip(np.rint(t), -7, 7), 0.0)
    return np.nan_to_num(codes).astype(np.int8), d


def pack_nibbles(codes):
    c = codes.astype(np.uint8) & 15
    return c[..., 0::2] | (c[..., 1::2] << 4)


def unpack_nibbles(b):
    b = np.asarray(b, dtype=np.uint8)
    c = np.stack((b & 15, b >> 4), -1).reshape(*b.shape[:-1], 2 * b.shape[-1]).astype(np.int8)
    return np.where(c > 7, c - 16, c).astype(np.int8)


def pool_parts(pool, page, dim):
    """Views of a uint8 pool [pages, kv_heads, page * (dim + 8)]: key codes, value codes [..., page, dim / 2], key scales,
    value scales [..., page]."""
    n = page * dim // 2
    codes = pool[..., : 2 * n].reshape(*pool.shape[:-1], 2, page, dim // 2)
    scales = pool[..., 2 * n:].view(np.float32).reshape(*pool.shape[:-1], 2, page)
    return codes[..., 0, :, :], codes[..., 1, :, :], scales[..., 0, :], scales[..., 1, :]


def cached_heads(pool, page, dim, table_row, n, first=0):
    """The first n tokens' (from position `first`) keys and values of one sequence as the cache holds them: code times scale in
    float32 (exactly rounded products), [n, kv_heads, dim] each, in the cache's basis."""
    kc, vc, ks, vs = pool_parts(pool, page, dim)
    pos = np.arange(first, first + n)
    at, slot = np.asarray(table_row)[pos // page], pos % page
    k = unpack_nibbles(kc[at, :, slot]).astype(np.float32) * ks[at, :, slot][..., None]
    v = unpack_nibbles(vc[at, :, slot]).astype(np.float32) * vs[at, :, slot][..., None]
    return k, v


def read_back(codes, scales, rotate):
    """Heads as the cache gives them back, float32: the integers codes . H (exact) times float32(scale / sqrt(D)) -- one
    float32 product with the factor float32(1 / sqrt(D)), one with the integer; without rotation, code times scale."""
    if not rotate:
        return codes.astype(np.float32) * scales[..., None]
    dim = codes.shape[-1]
    sums = np.rint(codes.astype(np.float64) @ (hadamard(dim) * np.sqrt(dim)))
    return sums.astype(np.float32) * (scales * np.float32(1.0 / np.sqrt(dim)))[..., None]


def cached_read_back(pool, page, dim, table_row, n, first, rotate):
    """read_back of the n tokens from position `first` of one sequence: keys and values [n, kv_heads, dim]."""
    kc, vc, ks, vs = pool_parts(pool, page, dim)
    pos = np.arange(first, first + n)
    at, slot = np.asarray(table_row)[pos // page], pos % page
    return tuple(read_back(unpack_nibbles(c[at, :, slot]), s[at, :, slot], rotate) for c, s in ((kc, ks), (vc, vs)))


def attention(q, k, v, scale, causal):
    """One sequence, float64: q [n, heads, D], k and v [m, kv_heads, D].  Returns o and, for error bounds, the largest |score|
    and the largest sum of |terms| of a score, per query and head, and sum_j p_j |v_j|."""
    n, heads, dim = q.shape
    m, kv = k.shape[0], k.shape[1]
    o = np.zeros((n, heads, dim))
    mag = np.zeros((n, heads, dim))
    top = np.zeros((n, heads))
    terms = np.zeros((n, heads))
    if m == 0 or n == 0:
        return o, mag, top, terms
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    see = np.arange(m)[None] <= (m - n + np.arange(n))[:, None] if causal else np.ones((n, m), bool)
    for h in range(heads):
        g = h // (heads // kv)
        with np.errstate(all="ignore"):
            s = scale * (q[:, h] @ k[:, g].T)
            a = scale * (np.abs(q[:, h]) @ np.abs(k[:, g]).T)
        s = np.where(see, s, -np.inf)
        for i in range(n):
            js = np.nonzero(see[i])[0]
            if len(js) == 0:
                continue
            p = np.exp(s[i, js] - s[i, js].max())
            p /= p.sum()
            o[i, h] = p @ v[js, g]
            mag[i, h] = p @ np.abs(v[js, g])
            top[i, h] = np.abs(s[i, js]).max()
            terms[i, h] = a[i, js].max()
    return o, mag, top, terms
