"""Plain 64-bit forms of the calls around the prefill (numpy, loops where they are clearer): norm and rotation, the 4-bit cache
with the bytes of its blocks, attention over it."""
import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK, BLOCK_BYTES = 64, 8704


def norm_rope(x, w, eps, freq, positions, pairing, magnitude=1.0):
    """x [..., rows, 128] float64, positions [rows]."""
    y = x if w is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    half = len(freq)
    p = np.arange(half)
    i, j = (2 * p, 2 * p + 1) if pairing == 0 else (p, p + half)
    t = np.asarray(positions, dtype=np.float64)[:, None] * freq
    c, s = np.cos(t) * magnitude, np.sin(t) * magnitude
    out = y.copy()
    out[..., i] = y[..., i] * c - y[..., j] * s
    out[..., j] = y[..., i] * s + y[..., j] * c
    return out


def quantise(x):
    """x [..., 128] float64 -> codes [..., 128] and scale bytes [..., 4] (uint8)."""
    g = x.reshape(x.shape[:-1] + (4, 32))
    bad = ~np.isfinite(g).all(-1)
    a = np.abs(np.where(np.isfinite(g), g, 0.0))
    top = a.max(-1)
    e = np.full(top.shape, 2)
    for b in range(2, 252):                                  # the smallest scale that reaches the largest element
        e = np.where(top > 7.0 * 2.0 ** (b - 127), b + 1, e)
    y = a / 2.0 ** (e - 127.0)[..., None]
    d = np.abs(y[..., None] - E2M1)
    best = d.min(-1, keepdims=True)
    # of two as near the even one
    code = np.where(d == best, np.arange(8) % 2 * 16 + np.arange(8), 99).min(-1) % 16
    code = code + 8 * np.signbit(g)
    dead = bad | (top == 0)
    code = np.where(dead[..., None], 0, code)
    e = np.where(bad, 255, np.where(top == 0, 0, e))
    return code.reshape(x.shape).astype(np.uint8), e.astype(np.uint8)


def values(code, e):
    s = np.where(e == 255, np.nan, 2.0 ** (e.astype(np.float64) - 127.0))
    x = np.where(code >= 8, -1.0, 1.0) * E2M1[code & 7]
    return (x.reshape(x.shape[:-1] + (4, 32)) * s[..., None]).reshape(x.shape)


def put(block, token, kc, ke, vc, ve):
    """One token's codes [128] and scale bytes [4] into a block [8704] of bytes, as the layout says it."""
    for ch in range(128):
        nibble(block, 64 * token + ch // 2, ch & 1, kc[ch])
        at, half = v_place(ch, token)
        nibble(block, at, half, vc[ch])
    for g in range(4):
        block[8192 + 4 * (16 * g + token % 16) + token // 16] = ke[g]
        block[8448 + 16 * (4 * (token // 4 % 4) + g) + 4 * (token // 16) + token % 4] = ve[g]


def v_place(ch, token):
    u, f, c, i = token // 32, token // 16 % 2, token // 4 % 4, token % 4
    p, b, m = ch // 32, ch // 16 % 2, ch % 16
    place = 4 * f + i                                        # nibble of the word
    return 4096 + 1024 * p + 16 * (16 * c + m) + 8 * b + 4 * u + place // 2, place & 1


def nibble(block, at, high, code):
    block[at] = (block[at] & 0x0f) | (code << 4) if high else (block[at] & 0xf0) | code


def attend(q, k, v, limits, scale):
    """q [rows, 128], k, v [n, 128], limits [rows]: row i sees the keys 0 .. limits[i] -> o, lse, sum of weights times |v|."""
    o, lse, size = np.zeros(q.shape), np.full(len(q), -np.inf), np.zeros(q.shape)
    for i, last in enumerate(limits):
        if last < 0:
            continue
        s = k[:last + 1] @ q[i] * scale
        m = s.max()
        p = np.exp(s - m)
        lse[i] = m + np.log(p.sum())
        o[i] = p @ v[:last + 1] / p.sum()
        size[i] = p @ np.abs(v[:last + 1]) / p.sum()
    return o, lse, size
