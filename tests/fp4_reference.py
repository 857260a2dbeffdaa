"""Plain statements, in 64 bits, of a cache in 4 bits, of the attention weight that tokens get, and of eviction."""
import numpy as np

MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
MIDS = [(a + b) / 2 for a, b in zip(MAGNITUDES, MAGNITUDES[1:])]


def page_bytes(N, d):
    return -(-N * 17 * d // 32 // 16) * 16


def pack(x):
    """x float16 [..][d] -> codes uint8 [..][d/2], exponent bytes uint8 [..][d/32]."""
    shape = x.shape
    x = x.astype(np.float64).reshape(-1, 32)
    codes, exps = np.zeros(x.shape, np.uint8), np.zeros(len(x), np.uint8)
    for i, g in enumerate(x):
        if not np.isfinite(g).all():
            exps[i] = 255
            continue
        a = np.abs(g).max()
        e = -127
        if a > 0:
            e = -40
            while a > 7 * 2.0 ** e and e < 13:
                e += 1
        exps[i] = e + 127
        y = np.abs(g) / 2.0 ** e if a > 0 else np.zeros(32)
        code = np.zeros(32, np.uint8)
        for k, mid in enumerate(MIDS):  # halfway: to the even code
            code += (y >= mid) if k % 2 else (y > mid)
        codes[i] = code + 8 * np.signbit(g)
    codes = codes.reshape(shape)
    return codes[..., 0::2] | codes[..., 1::2] << 4, exps.reshape(*shape[:-1], shape[-1] // 32)


def values(codes, exps):
    """float64 [..][d] of codes [..][d/2] and exponents [..][d/32]."""
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    x = MAGNITUDES[c & 7] * np.where(c & 8, -1.0, 1.0)
    scale = np.where(exps == 255, np.nan, 2.0 ** (exps.astype(np.float64) - 127))
    return x * np.repeat(scale, 32, -1)


def parts(cache, N, d, ppb):
    """Views of a cache's bytes [blocks][block bytes]: codes [block][page][token][d/2] and exponents [block][page][token][d/32]."""
    p = cache.reshape(len(cache), ppb, page_bytes(N, d))
    codes = p[:, :, :N * d // 2].reshape(len(cache), ppb, N, d // 2)
    exps = p[:, :, N * d // 2:N * d // 2 + N * d // 32].reshape(len(cache), ppb, d // 32, N).transpose(0, 1, 3, 2)
    assert np.shares_memory(codes, cache) and np.shares_memory(exps, cache)
    return codes, exps


def append(cache, ppb, first, N, table, lens, new):
    """Writes the new rows [s][i][h][d] in place, to pages first.. of a cache's bytes."""
    S, n, H, d = new.shape
    codes, exps = parts(cache, N, d, ppb)
    c, e = pack(new)
    for s in range(S):
        for i in range(n):
            t = int(lens[s]) - n + i
            if t < 0 or t // N >= table.shape[1] or not 0 <= table[s, t // N] < len(cache):
                continue
            codes[table[s, t // N], first:first + H, t % N] = c[s, i]
            exps[table[s, t // N], first:first + H, t % N] = e[s, i]


def weigh(weights, positions, seen, q, pages, n_kv, N, table, lens, lse, scale):
    """-> weights, positions, bound: float64 copies, and by how much a weight in 32 bits may be off.  pages: K and further pages [block][page][token][d].

    The bound, term by term, u = 2^-24: a score is a sum of d products in 32 bits, scaled (d * u * scale * sum |q_c k_c| and 2 u of it); -lse goes to powers of two in 32 bits (2 u |lse|);
    their sum is rounded (u of it); in powers of two and back, 2^x is another 2^-21 of the weight; n weights are added with n roundings, and one to what was there.  A weight below the
    smallest normal number becomes zero (2^-126)."""
    S, nq, H, d = q.shape
    u = 2.0 ** -24
    group = H // n_kv
    out, bound, positions = weights.astype(np.float64), np.zeros(weights.shape), positions.copy()
    for s in range(S):
        n = min(int(lens[s]), table.shape[1] * N, weights.shape[2])
        for h in range(n_kv):
            for t in range(n):
                new = t >= int(lens[s]) - nq
                total = 0.0 if new else float(weights[s, h, t])
                off = 0.0
                if new:
                    positions[s, h, t] = int(seen[s]) - (int(lens[s]) - t)
                b = table[s, t // N]
                if 0 <= b < len(pages):
                    k = pages[b, h, t % N].astype(np.float64)
                    for i in range(nq):
                        if t >= int(lens[s]) - (nq - 1 - i):
                            continue
                        for head in range(h * group, (h + 1) * group):
                            if lse[s, i, head] == -np.inf:
                                continue
                            qq = q[s, i, head].astype(np.float64)
                            x = (k @ qq) * scale
                            with np.errstate(invalid="ignore", over="ignore"):
                                w = np.exp(x - float(lse[s, i, head]))
                                total += w
                                off += w * (d * u * abs(scale) * (np.abs(k) @ np.abs(qq)) + 4 * u * np.abs(x) + 4 * u * abs(float(lse[s, i, head])) + 2.0 ** -21) + 2.0 ** -126
                out[s, h, t] = total
                bound[s, h, t] = off + (nq * group + 2) * u * abs(total)
    return out, positions, bound


def stays(weights, positions, seen, length, keep, recent):
    """Slots of a head that stay, in order."""
    keep = max(0, int(keep))
    if length <= keep:
        return list(range(length))
    safe = int(seen) - min(recent, keep)

    def order(t):
        w = float(weights[t])
        return (2, 0.0) if int(positions[t]) >= safe else (1, 0.0) if np.isnan(w) else (0, w)

    gone = sorted(range(length), key=lambda t: (*order(t), t))[:length - keep]
    return sorted(set(range(length)) - set(gone))


def evict(rows, N, table, lens, keep, recent, weights, positions, seen):
    """rows: list of arrays [block][head][token][..] of bytes or values, written in place, as weights and positions are.  -> new lengths, status bits."""
    S, H, width = weights.shape
    new_lens, status = lens.copy(), 0
    for s in range(S):
        n = int(lens[s])
        if n > width or n > table.shape[1] * N or any(not 0 <= table[s, b] < len(rows[0]) for b in range(-(-n // N))):
            status = 4
            continue
        n = max(n, 0)
        k = max(0, int(keep[s]))
        new_lens[s] = min(n, k)
        for h in range(H):
            kept = stays(weights[s, h], positions[s, h], seen[s], n, k, recent)
            holes = sorted(set(range(min(k, n))) - set(kept))
            fillers = [t for t in kept if t >= k]
            assert len(holes) == len(fillers)
            for to, at in zip(holes, fillers):
                for r in rows:
                    r[table[s, to // N], h, to % N] = r[table[s, at // N], h, at % N]
                weights[s, h, to], positions[s, h, to] = weights[s, h, at], positions[s, h, at]
    return new_lens, status
