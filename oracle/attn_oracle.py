"""The attention operators' definition in 64 bits: plain loops over requests, tokens and heads, on the CPU.

Shares no code with the GPU path.  Pools are NumPy arrays [pool_blocks, block_tokens, kv_heads, head_dim] of doubles, 8-bit ones of
uint8 codes with [pool_blocks, kv_heads] scales.
"""
import numpy as np

#: the values of e4m3's codes 0 .. 126 (0 .. 448); code 127 is NaN, codes from 128 on are the negative ones
E4M3 = np.array([(m / 8.0) * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7) for e in range(16) for m in range(8)])[:127]


def e4m3_values(codes):
    table = np.concatenate([E4M3, [np.nan], -E4M3, [np.nan]])
    return table[np.asarray(codes)]


def e4m3_code(x):
    """Nearest code, ties to the even one; beyond 448 the largest; 127 for what is not finite."""
    if not np.isfinite(x):
        return 127
    size = min(abs(x), 448.0)
    up = int(np.searchsorted(E4M3, size))
    if E4M3[up] != size:
        down = up - 1
        over, under = E4M3[up] - size, size - E4M3[down]
        if under < over or (under == over and down % 2 == 0):
            up = down
    return up + (128 if x < 0 or (x == 0 and np.signbit(x)) else 0)


def rotate(x, table, position, pairs):
    """One head's elements at one position; table: [positions, rope_dim / 2, 2], pairs: "halves" or "neighbours"."""
    y = np.array(x, dtype=np.float64)
    if table is None:
        return y
    n = table.shape[1]
    for j in range(n):
        a, b = (j, j + n) if pairs == "halves" else (2 * j, 2 * j + 1)
        c, s = float(table[position, j, 0]), float(table[position, j, 1])
        y[a], y[b] = x[a] * c - x[b] * s, x[b] * c + x[a] * s
    return y


def least_scale(most):
    e = -32
    while e < 63 and most > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def taken_scale(s):
    """A stored scale as both operators take it."""
    return min(max(s, 2.0 ** -32), 2.0 ** 63) if s == s else 2.0 ** -32


def append(hit, app, tables, block_tokens, new, pool, scales=None):
    """new: [tokens, kv_heads, head_dim] (rotated already) into the pool, in place."""
    done = 0
    for h, n, table in zip(hit, app, tables):
        for t0 in range(int(h) // block_tokens * block_tokens, int(h + n), block_tokens):
            lo, hi = max(int(h), t0), min(int(h + n), t0 + block_tokens)
            if lo >= hi:
                continue
            block, row = int(table[t0 // block_tokens]), lo - t0
            x = new[done + lo - int(h):done + hi - int(h)]
            if scales is None:
                pool[block, row:row + hi - lo] = x
                continue
            for head in range(x.shape[1]):
                v = np.abs(x[:, head])
                v = v[np.isfinite(v)]
                s = least_scale(v.max() if v.size else 0.0)
                if row:
                    old = taken_scale(float(scales[block, head]))
                    s = max(s, old)
                    if s != old:
                        was = e4m3_values(pool[block, :row, head]) * (old / s)
                        pool[block, :row, head] = np.vectorize(e4m3_code)(was)
                scales[block, head] = s
                pool[block, row:row + hi - lo, head] = np.vectorize(e4m3_code)(x[:, head] / s)
        done += int(n)


def attend(hit, app, tables, block_tokens, q, k_pool, v_pool, scale, keys="all", window=0, sinks=0):
    """q: [tokens, q_heads, head_dim]; pools of doubles.  Returns out, lse, and for each output what the rounding of softmax weights
    can move: sum_t p_t |V_t|, and of each row the largest sum of |q K| over the keys."""
    tokens, q_heads, dim = q.shape
    kv_heads = k_pool.shape[2]
    group = q_heads // kv_heads
    out, lse = np.zeros(q.shape), np.full((tokens, q_heads), -np.inf)
    weight, reach = np.zeros(q.shape), np.zeros((tokens, q_heads))
    done = 0
    for h, n, table in zip(hit, app, tables):
        h, n = int(h), int(n)
        first, last = {"all": (0, h + n), "hit": (0, h), "append": (h, h + n)}[keys]
        for i in range(n):
            p = h + i
            t = np.array([t for t in range(first, min(last, p + 1)) if not window or p - t < window or t < sinks], dtype=np.int64)
            if not t.size:
                continue
            blocks = np.asarray(table)[t // block_tokens]
            k, v = k_pool[blocks, t % block_tokens], v_pool[blocks, t % block_tokens]
            for head in range(q_heads):
                kh, vh, x = k[:, head // group], v[:, head // group], q[done + i, head]
                s = scale * (kh @ x)
                top = s.max()
                e = np.exp(s - top)
                out[done + i, head] = (e @ vh) / e.sum()
                weight[done + i, head] = (e @ np.abs(vh)) / e.sum()
                reach[done + i, head] = scale * (np.abs(kh) @ np.abs(x)).max()
                lse[done + i, head] = top + np.log(e.sum())
        done += n
    return out, lse, weight, reach
