"""The serving step's operators from their definitions, request by request in NumPy with 64 bits, for the tests."""
import numpy as np


def step(ctx, new, table, ring, state, page, n_token):
    """(cu, kv_len, next_len, pos, slot, table, ring, state, refused) after a step; lengths must be possible ones."""
    table, ring = table.copy(), ring.copy()
    N, (first, count) = ring.size, (int(x) for x in state)
    start = ring.copy()
    asked = taken = given = 0
    cu, kv, nxt, pos, slot, refused = [0], [], [], [], [], []
    for b, (c, n) in enumerate(zip(ctx.tolist(), new.tolist())):
        have = -(-c // page)
        if n == -1:
            for i in range(have):
                ring[(first + count + given) % N] = table[b, i]
                given += 1
            kv.append(0); nxt.append(0); cu.append(cu[-1]); refused.append(False)
            continue
        long = c + n > table.shape[1] * page
        need = 0 if long else -(-(c + n) // page) - have
        ok = not long and (need == 0 or asked + need <= count)
        if ok:
            for i in range(need):
                table[b, have + i] = start[(first + asked + i) % N]
            taken += need
        asked += need
        for x in range(c, c + n):
            pos.append(x if ok else -1)
            e = int(table[b, x // page]) if ok else -1
            slot.append(e * page + x % page if 0 <= e < N else -1)
        kv.append(c + n if ok else 0); nxt.append(c + n if ok else c); cu.append(cu[-1] + n); refused.append(not ok)
    i = lambda a: np.asarray(a, np.int32)  # noqa: E731
    assert len(pos) == n_token
    return i(cu), i(kv), i(nxt), i(pos), i(slot), table, ring, i([(first + taken) % N, count - taken + given]), refused


def rotate(x, pos, inv_freq, interleaved, amplitude):
    """x [T][H][D] in float64."""
    x, r = np.array(x, np.float64), 2 * len(inv_freq)
    turns = np.asarray(pos, np.longdouble)[:, None] * np.asarray(inv_freq, np.longdouble)
    c, s = (f(turns).astype(np.float64)[:, None] * amplitude for f in (np.cos, np.sin))
    lo, hi = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    a, b = x[..., lo].copy(), x[..., hi].copy()
    x[..., lo], x[..., hi] = a * c - b * s, b * c + a * s
    return x


def attention(q, k_cache, v_cache, table, cu, kv_len, scale, window=0, sinks=0, k_scale=None, v_scale=None):
    """(out, |v| under the weights, bound of the scores' sizes per row) in float64; q [T][H][D], caches [N][G][P][D]."""
    T, H, D = q.shape
    N, G, P, _ = k_cache.shape
    out, size, score = np.zeros((T, H, D)), np.zeros((T, H, D)), np.zeros((T, H))
    for b in range(len(kv_len)):
        n, L = int(cu[b + 1] - cu[b]), int(kv_len[b])
        if not n or not L:
            continue
        pages = table[b, :-(-L // P)]
        for g in range(G):
            k = k_cache[pages, g].reshape(-1, D)[:L].astype(np.float64) * (1.0 if k_scale is None else float(k_scale[g]))
            v = v_cache[pages, g].reshape(-1, D)[:L].astype(np.float64) * (1.0 if v_scale is None else float(v_scale[g]))
            for i in range(n):
                p = L - n + i
                if p < 0:
                    continue
                j = np.arange(p + 1)
                if window:
                    j = j[(j > p - window) | (j < sinks)]
                for h in range(g * (H // G), (g + 1) * (H // G)):
                    x = q[cu[b] + i, h].astype(np.float64)
                    with np.errstate(invalid="ignore"):
                        s = scale * (k[j] @ x)
                        w = np.exp(s - s.max())
                        w /= w.sum()
                        out[cu[b] + i, h] = (w[:, None] * v[j]).sum(0)
                        size[cu[b] + i, h] = (w[:, None] * np.abs(v[j])).sum(0)
                        score[cu[b] + i, h] = (abs(scale) * (np.abs(k[j]) @ np.abs(x))).max()
    return out, size, score
