"""Plain 64-bit forms of the serving step's operators, for the tests, and the error bounds that their results are held to."""
import numpy as np

# unit roundoffs of the stored types: half a step of a significand of 11 and of 8 bits
UNIT = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}


def tables(cached, new, table, bs, n_blocks, free, n_tokens):
    """scoot_kv_tables, request by request and token by token."""
    table, free = table.copy(), list(free)
    width = table.shape[1]
    start, kv = [0], []
    slot, pos = np.full(n_tokens, -1, np.int64), np.zeros(n_tokens, np.int32)
    lacked = taken = refused = 0
    for r, (c, n) in enumerate(zip(cached.tolist(), new.tolist())):
        bad = c < 0 or n < 0 or c + n > width * bs
        n = max(n, 0)
        held, need = (0, 0) if bad else (-(-c // bs), -(-(c + n) // bs) + -c // bs)
        ok = not bad and (need == 0 or lacked + need <= len(free))
        if ok:
            table[r, held:held + need] = free[lacked:lacked + need]
            taken += need
        refused += not ok
        lacked += need
        for j in range(n):
            t, p = start[-1] + j, c + j
            if t < n_tokens:
                pos[t] = max(p, 0)
                if ok and 0 <= table[r, p // bs] < n_blocks:
                    slot[t] = int(table[r, p // bs]) * bs + p % bs
        start.append(start[-1] + n)
        kv.append(c + n if ok else 0)
    return table, np.array(start, np.int32), np.array(kv, np.int32), slot, pos, np.array([taken, refused], np.int32)


def attention(q, k_cache, v_cache, table, query_start, kv_len, scale, causal=True, window=0, unit=UNIT["bf16"]):
    """out, lse and the bounds of their errors, in float64 (arrays of values, cache [block][token][head][dim]).

    A kernel that holds scores and sums in fp32, rounds the probabilities to the cache's type for the product with the
    values and rounds its result once is off by at most
      unit |out|  +  (unit + 2 ds + 2^-18) sum_i p_i |v_i|  +  2^-25 sum_i |v_i| / z
    with p the exact probabilities, ds = 2^-20 scale max_i sum_d |q_d k_id| the rounding of a score (2^-24 per addition,
    of which 128 in a row lose at most 2^-17 and a tensor core's, truncated in groups of sixteen, about 2^-20; the sums
    of terms of both signs are far below the sum of their magnitudes) and z = sum_i exp(s_i - max s), whose last term
    is the 16-bit type's smallest step for probabilities that underflow it."""
    T, H, D = q.shape
    bs, Hkv = k_cache.shape[1], k_cache.shape[2]
    G = H // Hkv
    out, lse = np.zeros((T, H, D)), np.full((T, H), -np.inf)
    e_out, e_lse = np.zeros((T, H, D)), np.zeros((T, H))
    for r in range(len(kv_len)):
        q0, q1, kv = int(query_start[r]), int(query_start[r + 1]), int(kv_len[r])
        for t in range(q0, q1):
            p = kv - (q1 - q0) + t - q0
            end = min(kv, p + 1) if causal else kv
            begin = max(0, p + 1 - window) if window else 0
            if end <= begin:
                continue
            i = np.arange(begin, end)
            ids, at = table[r, i // bs], i % bs
            K, V = k_cache[ids, at].astype(np.float64), v_cache[ids, at].astype(np.float64)  # [n][Hkv][D]
            for h in range(H):
                k, v, qv = K[:, h // G], V[:, h // G], q[t, h].astype(np.float64)
                s = scale * (k @ qv)
                ds = 2.0 ** -20 * scale * np.max(np.abs(k) @ np.abs(qv))
                m = s.max()
                e = np.exp(s - m)
                z = e.sum()
                pr = e / z
                out[t, h] = pr @ v
                lse[t, h] = m + np.log(z)
                e_out[t, h] = unit * np.abs(out[t, h]) + (unit + 2 * ds + 2.0 ** -18) * (pr @ np.abs(v)) + 2.0 ** -25 * np.abs(v).sum(0) / z
                e_lse[t, h] = ds + 2.0 ** -18 + 2.0 ** -22 * abs(lse[t, h])
    return out, lse, e_out, e_lse
