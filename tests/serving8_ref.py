"""Plain 64-bit forms of rotary positions and of the 8-bit cache's operators, for the tests, and the bounds that results are
held to."""
import numpy as np

import serving_ref as R

TURN = 2.0 * np.pi

# magnitudes of the codes 0 .. 126 (127 is the format's NaN)
CODES = np.array([m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])


def angles(turns, position):
    """Radians of position * turns 2^-64 turns, from exact integers, within half a turn."""
    out = np.empty((len(position), len(turns)))
    for i, p in enumerate(position.tolist()):
        for j, t in enumerate(turns.tolist()):
            a = (int(t) * int(p)) % (1 << 64)
            out[i, j] = (a - (1 << 64) if a >> 63 else a) * 2.0 ** -64 * TURN
    return out


def rotate(x, angle, interleaved=False, magnitude=1.0, inverse=False):
    """y of x [T][heads][dim], and the bound of an fp32 evaluation's error before y is rounded to its type.

    The cosine and sine are off by at most 2^-22: two units (2^-23 each) of the functions, half a unit of the argument, at
    most pi / 4, and 2^-29 of the angle's own rounding; the products, the sum and the magnitude add 2^-24 each."""
    n = 2 * angle.shape[1]
    a, b = (x[..., 0:n:2], x[..., 1:n:2]) if interleaved else (x[..., :n // 2], x[..., n // 2:n])
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None] * (-1.0 if inverse else 1.0)
    y, e = x.copy(), np.zeros_like(x)
    u, v, size = (a * c - b * s) * magnitude, (b * c + a * s) * magnitude, (np.abs(a) + np.abs(b)) * abs(magnitude) * (2.0 ** -22 + 2.0 ** -22)
    if interleaved:
        y[..., 0:n:2], y[..., 1:n:2] = u, v
        e[..., 0:n:2], e[..., 1:n:2] = size, size
    else:
        y[..., :n // 2], y[..., n // 2:n] = u, v
        e[..., :n // 2], e[..., n // 2:n] = size, size
    return y, e


def step(dtype, y):
    """Half a step of a 16-bit type at y: relative, and its least."""
    return R.UNIT[dtype] * np.abs(y) + (2.0 ** -25 if dtype == "fp16" else 2.0 ** -134)


def least_scale(amax):
    """The least power of two s >= 2^-100 with amax <= 448 s, by trial."""
    out = np.full(np.shape(amax), 2.0 ** -100)
    while (big := amax > 448 * out).any():
        out[big] *= 2
    return out


def code_of(x):
    """x rounded to the values of the codes, to the nearest, ties to the even code."""
    mag = np.abs(x)
    hi = np.clip(np.searchsorted(CODES, mag), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = mag - CODES[lo], CODES[hi] - mag
    pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.where(x < 0, -1.0, 1.0) * CODES[pick]


def append8(x, slot, cache, scale):
    """Values of the codes and scales after x [T][heads][dim] went into cache [block][token][heads][dim] (values of codes):
    new numbers rounded in 64 bits.  Run by run, by the definition."""
    cache, scale = cache.copy(), scale.copy()
    bs, t = cache.shape[1], 0
    while t < len(slot):
        if slot[t] < 0 or slot[t] >= cache.shape[0] * bs:
            t += 1
            continue
        n = 1
        while t + n < len(slot) and slot[t + n] == slot[t] + n and slot[t + n] % bs:
            n += 1
        block, at = slot[t] // bs, slot[t] % bs
        s = least_scale(np.abs(x[t:t + n]).max((0, 2)))
        if at:
            grown = scale[block] < s
            old = cache[block, :at]
            again = code_of(old * (scale[block] / s)[None, :, None])
            cache[block, :at] = np.where(grown[None, :, None], again, old)
            s = np.maximum(s, scale[block])
        cache[block, at:at + n] = code_of(x[t:t + n] / s[None, :, None])
        scale[block] = s
        t += n
    return cache, scale


def attention8(q, k, v, k_scale, v_scale, table, query_start, kv_len, scale, dtype, **kw):
    """serving_ref.attention over codes' values [block][token][heads][dim] and scales [block][heads].

    Its bound with probabilities rounded to fp16, and the output to `dtype`; a probability times its scale below fp16's normal
    numbers is off by 2^-25 of 2^-7 of the largest scale, times its code."""
    K, V = k * k_scale[:, None, :, None], v * v_scale[:, None, :, None]
    o, z, e_out, e_lse = R.attention(q, K, V, table, query_start, kv_len, scale, unit=R.UNIT["fp16"], **kw)
    e_out = e_out + (R.UNIT[dtype] - R.UNIT["fp16"]) * np.abs(o) + (2.0 ** -25 if dtype == "fp16" else 0.0)
    for r in range(len(kv_len)):
        ids = table[r, :-(-int(kv_len[r]) // k.shape[1])]
        if len(ids):
            G = q.shape[1] // k.shape[2]
            small = 2.0 ** -32 * v_scale[ids].max(0)[:, None] * np.abs(v[ids]).sum((0, 1))
            e_out[int(query_start[r]):int(query_start[r + 1])] += np.repeat(small, G, 0)
    return o, z, e_out, e_lse
