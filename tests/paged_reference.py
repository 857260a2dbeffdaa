"""Plain statements, in 64 bits and one token at a time, of what the decode-step operators compute."""
import numpy as np


def pages_view(cache, N, d, ppb, token_major):
    """A dense cache array as [block][page][token][channel]."""
    return cache.reshape(-1, N, ppb, d).transpose(0, 2, 1, 3) if token_major else cache.reshape(-1, ppb, N, d)


def tokens_of(row, length, k_pages, v_pages, h, vh, N):
    """K and V rows (float64) of the tokens below `length` that have a block, and their positions."""
    at = [t for t in range(min(length, len(row) * N)) if 0 <= row[t // N] < len(k_pages)]
    b, r = np.array([row[t // N] for t in at], np.int64), np.array([t % N for t in at], np.int64)
    return np.array(at, np.int64), k_pages[b, h, r].astype(np.float64), v_pages[b, vh, r].astype(np.float64)


def attend(q, k_pages, v_pages, v_first, n_kv, N, table, lens, scale, prefix_table=None, prefix_lens=None, prefix_first=None):
    """-> out, lse, bound: float64 [n_seq][n_q][n_heads][d], [..][n_heads], and by how much FP16 output may be off.

    The bound, term by term, with w_t the softmax weights and u = 2^-24: a score is a sum of d products in 32 bits (d * u * sum |q_c k_c|
    at most, times scale) that is scaled and raised in 32 bits (another 2^-20 of weight); a weight is rounded to 11 bits (2^-11) and
    never by more than 2^-35 of the largest; the sums over n tokens take n roundings, and two parts are joined (2 n u and
    2^-20); the output is rounded to FP16 (2^-11 of it, at least 2^-25)."""
    S, nq, H, d = q.shape
    group = H // n_kv
    out, lse, bound = np.zeros((S, nq, H, d)), np.full((S, nq, H), -np.inf), np.zeros((S, nq, H, d))
    lse_bound = np.zeros((S, nq, H))
    u = 2.0 ** -24
    for s in range(S):
        g = next((g for g in range(len(prefix_lens)) if prefix_first[g] <= s < prefix_first[g + 1]), None) if prefix_lens is not None else None
        for h in range(n_kv):
            t, k, v = tokens_of(table[s], int(lens[s]), k_pages, v_pages, h, v_first + h, N)
            t = t - int(lens[s])  # relative to the end
            if g is not None:
                _, pk, pv = tokens_of(prefix_table[g], int(prefix_lens[g]), k_pages, v_pages, h, v_first + h, N)
                t, k, v = np.concatenate([np.full(len(pk), -10**9), t]), np.concatenate([pk, k]), np.concatenate([pv, v])
            for i in range(nq):
                seen = t < -(nq - 1 - i)
                if not seen.any():
                    continue
                kk, vv = k[seen], v[seen]
                for head in range(h * group, (h + 1) * group):
                    qq = q[s, i, head].astype(np.float64)
                    x = (kk @ qq) * scale
                    m = x.max()
                    w = np.exp(x - m)
                    lse[s, i, head] = m + np.log(w.sum())
                    w /= w.sum()
                    out[s, i, head] = w @ vv
                    off = d * u * abs(scale) * (np.abs(kk) @ np.abs(qq)) + 4 * u * np.abs(x) + 2.0 ** -20
                    mean = float(w @ off)
                    n = int(seen.sum())
                    mag = w @ np.abs(vv)
                    bound[s, i, head] = (w * (off + mean)) @ np.abs(vv) + (2.0 ** -11 + 2 * n * u + 2.0 ** -20) * mag + \
                        n * 2.0 ** -35 * w.max() * np.abs(vv).max(0) + 2.0 ** -11 * np.abs(out[s, i, head]) + 2.0 ** -25
                    lse_bound[s, i, head] = float(off.max()) + n * u + 2.0 ** -20 * (1 + abs(lse[s, i, head]))
    return out, lse, bound, lse_bound


def append(k_pages, v_pages, v_first, N, table, lens, k_new, v_new):
    """Writes the new rows in place."""
    S, n, H, _ = k_new.shape
    for s in range(S):
        for i in range(n):
            t = int(lens[s]) - n + i
            if t < 0 or t // N >= table.shape[1] or not 0 <= table[s, t // N] < len(k_pages):
                continue
            b = table[s, t // N]
            k_pages[b, :H, t % N] = k_new[s, i]
            v_pages[b, v_first:v_first + H, t % N] = v_new[s, i]


INVALID = 0xFF


def compact(desc, pool, out_bytes):
    """desc: records of the table; pool: bytes.  -> (records, bytes used, the moved bytes, status bits): every live 16-byte unit
    goes to its rank among the live ones."""
    units = pool.size // 16
    held = np.zeros(units, bool)
    status, ok = 0, np.zeros(len(desc), bool)
    for i, e in enumerate(desc):
        if e["mode"] == INVALID:
            continue
        off, n = int(e["off"]), int(e["n16"])
        if e["mode"] > 5 or off % 16 or off // 16 + n > units:
            status |= 2
            continue
        ok[i] = True
        held[off // 16:off // 16 + n] = True
    rank = np.cumsum(held) - held
    total = int(held.sum())
    room = out_bytes // 16
    new = desc.copy()
    for i, e in enumerate(desc):
        at = int(rank[int(e["off"]) // 16]) if ok[i] and e["n16"] else 0
        if not ok[i] or at + int(e["n16"]) > room:
            status |= 1 if ok[i] else 0
            new[i] = (0, 0.0, 0, INVALID, 0)
        else:
            new[i]["off"] = 16 * at
    moved = pool.reshape(-1, 16)[held].reshape(-1)[:16 * room]
    return new, 16 * min(total, room), moved, status
