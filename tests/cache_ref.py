"""The 4-bit paged KV cache in plain numpy and 64 bits: layout, codes, tables
and attention, written from the definitions in include/rotate_attn.h."""
import numpy as np

MAG = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])


def hadamard(D):
    """Sylvester-Hadamard matrix of +-1."""
    H = np.ones((1, 1))
    while H.shape[0] < D:
        H = np.block([[H, H], [H, -H]])
    return H


def rope_table(rows, D, theta=1e4):
    ang = np.arange(rows)[:, None] * theta ** (-2.0 * np.arange(D // 2) / D)
    return np.stack((np.cos(ang), np.sin(ang)), 2).astype(np.float32)


def turn(x, cs):
    """Adjacent channel pairs of [T, H, D] by [T, D/2, 2]."""
    c, s = cs[:, None, :, 0].astype(np.float64), cs[:, None, :, 1].astype(np.float64)
    y = np.empty_like(x)
    y[..., 0::2] = x[..., 0::2] * c - x[..., 1::2] * s
    y[..., 1::2] = x[..., 0::2] * s + x[..., 1::2] * c
    return y


def codes(y):
    """4-bit codes and a of rows y: nearest E2M1 of 6 y / a, ties to the even code."""
    with np.errstate(invalid="ignore", over="ignore"):
        a = np.abs(y).max(-1)
        a = np.where(np.isnan(y).any(-1), np.nan, a)
    dead = ~np.isfinite(a) | (a < 2.0 ** -100)
    t = np.where(dead[..., None], 0.0, y) * 6.0 / np.where(dead, 1.0, a)[..., None]
    u = np.abs(t)
    c = np.zeros(y.shape, np.int64)
    for i in range(7):
        mid = (MAG[i] + MAG[i + 1]) / 2
        c += (u >= mid) if (i + 1) % 2 == 0 else (u > mid)
    a = np.where(np.isfinite(a), np.where(dead, 0.0, a), np.nan)
    return c | ((t < 0) & (c > 0)).astype(np.int64) << 3, a


def value(c):
    return np.where(c & 8, -1.0, 1.0) * MAG[c & 7]


def k_byte(D, t, d):
    return (t // 16) * 8 * D + (d // (D // 4)) * 2 * D + (t % 16) * (D // 8) + (d % (D // 4)) // 2


def v_byte(D, page, t, d):
    return page * D // 2 + (t // 4) * 2 * D + (d // (D // 16)) * (D // 8) + (t % 4) * (D // 32) + (d % (D // 16)) // 2


def rows(cache, slots, page, Hkv, D):
    """Codes [n, Hkv, D] and scales [n, Hkv] of K and V of these slots, from the page bytes."""
    cache = cache.reshape(cache.shape[0], Hkv, page * (D + 8))
    d = np.arange(D)
    out = []
    for which in (0, 1):
        c = np.zeros((len(slots), Hkv, D), np.int64)
        s = np.zeros((len(slots), Hkv), np.float32)
        for n, slot in enumerate(slots):
            p, t = slot // page, slot % page
            b = cache[p][:, k_byte(D, t, d) if which == 0 else v_byte(D, page, t, d)]
            c[n] = np.where(d % 2, b >> 4, b & 15)
            at = page * D + 4 * page * which + 4 * t
            s[n] = np.ascontiguousarray(cache[p][:, at:at + 4]).view(np.float32)[:, 0]
        out += [c, s]
    return out


def plan(page, max_blocks, num_pages, T, seq, new, table, free, count, release=None):
    """(status, table, free, count, seq, q_start, positions, slots) after the step."""
    table, free, seq = table.copy(), list(free), list(seq)
    R = len(seq)
    old = [0 if release is not None and release[r] else seq[r] for r in range(R)]
    flags = 0
    need = tokens = longest = freed = 0
    up = lambda n: -(-n // page)
    for r in range(R):
        if seq[r] < 0 or seq[r] > max_blocks * page or new[r] < 0 or old[r] + new[r] > max_blocks * page:
            flags |= 1
            continue
        need += up(old[r] + new[r]) - up(old[r])
        tokens += new[r]
        longest = max(longest, old[r] + new[r])
        freed += up(seq[r]) - up(old[r])
    if count < 0 or count + freed > num_pages:
        flags |= 8
    if tokens > T:
        flags |= 2
    if not flags & 8 and need > count + freed:
        flags |= 4
    status = [flags, need, tokens, longest]
    pos, slot = [-1] * T, [-1] * T
    if flags:
        return status, table, free, count, seq, [0] * (R + 1), pos, slot
    for r in range(R):
        if release is not None and release[r]:
            for j in range(up(seq[r])):
                free[count] = int(table[r, j])
                table[r, j] = -1
                count += 1
    start, t = [0], 0
    for r in range(R):
        for j in range(up(old[r]), up(old[r] + new[r])):
            count -= 1
            table[r, j] = free[count]
        for i in range(new[r]):
            pos[t] = old[r] + i
            slot[t] = int(table[r, pos[t] // page]) * page + pos[t] % page
            t += 1
        start.append(t)
        seq[r] = old[r] + new[r]
    return status, table, free, count, seq, start, pos, slot


def attn(q, k, v, causal, window, scale):
    """One request and one head: q [m, D], k, v [n, D] in 64 bits.  Returns o, lse, and for the error bound
    sum_j p_j |v_j| and max over seen j of scale * sum_d |q_d k_jd|."""
    m, n = q.shape[0], k.shape[0]
    pos = n - m + np.arange(m)[:, None]
    key = np.arange(n)[None, :]
    seen = (key <= pos) if causal else np.ones((m, n), bool)
    if window:
        seen &= key > pos - window
    s = np.where(seen, scale * (q @ k.T), -np.inf)
    top = s.max(1, initial=-np.inf)
    p = np.where(seen, np.exp(s - np.where(np.isfinite(top), top, 0.0)[:, None]), 0.0)
    l = p.sum(1)
    with np.errstate(divide="ignore"):
        lse = np.where(l > 0, top + np.log(l), -np.inf)
    p /= np.where(l > 0, l, 1.0)[:, None]
    size = np.where(seen, scale * (np.abs(q) @ np.abs(k).T), 0.0).max(1, initial=0.0)
    return p @ v, lse, p @ np.abs(v), size
