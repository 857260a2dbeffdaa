"""Plain statements in 64 bits, of whole sequences at a time on the GPU, for calls that are too large for paged_reference and fp4_reference.  The formulas and the bounds are theirs, term by term."""
import numpy as np
import torch

import fp4_reference as ref
from gpu_util import DEV

U = 2.0 ** -24


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def tables(rng, lens, N, width, spare=3):
    """Blocks of sequences anywhere in a cache -> table [n_seq][width], blocks of the cache."""
    each = [-(-int(n) // N) for n in lens]
    perm = rng.permutation(sum(each) + spare).astype(np.int32)
    table, at = np.full((len(lens), width), -1, np.int32), 0
    for s, n in enumerate(each):
        table[s, :n] = perm[at:at + n]
        at += n
    return table, sum(each) + spare


def owned(table, lens, N, blocks):
    """[block][row]: whether a token is there."""
    out = np.zeros((blocks, N), bool)
    for s, n in enumerate(lens):
        t = np.arange(n)
        out[table[s, t // N], t % N] = True
    return out


def cache_fp4(rng, table, lens, N, d, ppb, blocks, low=121, high=126):
    """A cache in 4 bits of random codes; exponents of a few binades where a token is, NaN's everywhere else."""
    cache = rng.integers(0, 256, (blocks, ppb * ref.page_bytes(N, d)), dtype=np.uint8)
    exps = ref.parts(cache, N, d, ppb)[1]
    exps[:] = np.where(owned(table, lens, N, blocks)[:, None, :, None], rng.integers(low, high, exps.shape), 255)
    return cache


def cache_fp16(rng, table, lens, N, d, ppb, blocks):
    """FP16 pages [block][page][token][d], NaN where no token is."""
    some = rng.standard_normal(256).astype(np.float16)  # (drawn from these: quick)
    x = some[rng.integers(0, 256, (blocks, ppb, N, d), dtype=np.uint8)]
    x[np.broadcast_to(~owned(table, lens, N, blocks)[:, None, :], x.shape[:3])] = np.nan
    return x


class Pages:
    """Rows of tokens out of a cache of either kind, in 64 bits."""

    def __init__(self, cache, N, d, ppb):
        self.N, self.fp4, self.blocks = N, cache.dtype == np.uint8, len(cache)
        if self.fp4:
            codes, exps = ref.parts(cache, N, d, ppb)
            self.codes, self.exps = dev(codes), dev(exps)
            every = np.arange(16, dtype=np.uint8).repeat(16).reshape(1, 1, 256) + np.zeros((256, 1, 1), np.uint8)  # (each code 16 times: 32 channels share an exponent)
            packed = every[..., 0::2] | every[..., 1::2] << 4
            with np.errstate(invalid="ignore"):
                self.value = dev(ref.values(packed, np.arange(256, dtype=np.uint8).reshape(256, 1, 1).repeat(8, 2))[:, 0, ::16])  # [exponent][code]
        else:
            self.pages = dev(cache)

    def tokens(self, row, length):
        """Positions below `length` that have a block."""
        t = np.arange(min(max(int(length), 0), len(row) * self.N))
        b = row[t // self.N]
        return t[(b >= 0) & (b < self.blocks)]

    def rows(self, row, t, first, kv):
        """[head][token][d]"""
        b, r = dev(row[t // self.N].astype(np.int64)), dev(t % self.N)
        if not self.fp4:
            return self.pages[b, first:first + kv, r].double().transpose(0, 1).contiguous()
        c, e = self.codes[b, first:first + kv, r].long(), self.exps[b, first:first + kv, r].long()
        c = torch.stack([c & 15, c >> 4], -1).flatten(-2)
        return self.value[e.repeat_interleave(32, -1), c].transpose(0, 1).contiguous()


def _scores(q, k, scale, t, length, nq):
    """q [n_q][heads][d], k [KV head][token][d] -> scaled scores and sums of magnitudes [KV head][head of the group][query][token], and which are seen [query][token]."""
    kv, T, d = k.shape
    rows = q.double().view(nq, kv, -1, d).permute(1, 2, 0, 3).reshape(kv, -1, d).contiguous()
    kt = k.transpose(1, 2).contiguous()
    x, mag = torch.bmm(rows, kt) * scale, torch.bmm(rows.abs(), kt.abs())
    seen = dev(t)[None] < length - (nq - 1 - torch.arange(nq, device=DEV))[:, None]
    return x.view(kv, -1, nq, T), mag.view(kv, -1, nq, T), seen


def attend(q, k_pages, v_pages, first, kv, table, lens, scale):
    """q: device tensor [n_seq][n_q][n_heads][d] -> out, lse, bound, lse_bound, as paged_reference.attend."""
    S, nq, H, d = q.shape
    out, bound = torch.zeros((S, nq, H, d), dtype=torch.float64, device=DEV), torch.zeros((S, nq, H, d), dtype=torch.float64, device=DEV)
    lse, lse_bound = torch.full((S, nq, H), -torch.inf, dtype=torch.float64, device=DEV), torch.zeros((S, nq, H), dtype=torch.float64, device=DEV)

    def back(x):  # [KV head][head of the group][query].. -> [query][head]..
        return x.movedim(2, 0).flatten(1, 2)

    for s in range(S):
        t = k_pages.tokens(table[s], lens[s])
        if not len(t):
            continue
        k, v = k_pages.rows(table[s], t, 0, kv), v_pages.rows(table[s], t, first, kv)
        x, mag, seen = _scores(q[s], k, scale, t, int(lens[s]), nq)
        off = d * U * abs(scale) * mag + 4 * U * x.abs() + 2.0 ** -20
        x = x.masked_fill(~seen, -torch.inf)
        any_seen = seen.any(-1)
        m = x.amax(-1, keepdim=True)
        w = torch.exp(x - torch.where(any_seen[:, None], m, 0.0))
        total = w.sum(-1, keepdim=True)
        w = w / torch.where(total > 0, total, 1.0)
        n = seen.sum(-1)

        def times(a, b):
            return torch.bmm(a.flatten(1, 2).contiguous(), b).view(*a.shape[:3], d)

        o, weighted = times(w, v), times(w, v.abs())
        mean = (w * off).sum(-1, keepdim=True)
        b = times(w * (off + mean), v.abs()) + (2.0 ** -11 + 2 * U * n[:, None] + 2.0 ** -20) * weighted + 2.0 ** -11 * o.abs() + 2.0 ** -25
        largest = torch.stack([v[:, dev(t) < int(lens[s]) - (nq - 1 - i)].abs().amax(1) if bool(any_seen[i]) else torch.zeros_like(v[:, 0]) for i in range(nq)], 1)  # [KV head][query][d]
        b = b + n[:, None] * 2.0 ** -35 * w.amax(-1, keepdim=True) * largest[:, None]
        l = (m + torch.log(total))[..., 0]
        lb = off.masked_fill(~seen, 0.0).amax(-1) + n * U + 2.0 ** -20 * (1 + l.abs())
        at = any_seen.nonzero()[:, 0]
        out[s, at], bound[s, at], lse[s, at], lse_bound[s, at] = back(o)[at], back(b)[at], back(l)[at], back(lb)[at]
    return out, lse, bound, lse_bound


def weigh(weights, positions, seen, q, pages, kv, table, lens, lse, scale):
    """weights, positions, seen: numpy; q, lse: device tensors -> weights, positions, bound, as fp4_reference.weigh, as numpy."""
    S, nq, H, d = q.shape
    out, bound, positions = weights.astype(np.float64), np.zeros(weights.shape), positions.copy()
    for s in range(S):
        n, length = min(int(lens[s]), table.shape[1] * pages.N, weights.shape[2]), int(lens[s])
        fresh = min(n, max(0, length - nq))
        out[s, :, fresh:n] = 0
        positions[s, :, fresh:n] = int(seen[s]) - (length - np.arange(fresh, n))
        t = pages.tokens(table[s], n)
        if not len(t):
            continue
        x, mag, sees = _scores(q[s], pages.rows(table[s], t, 0, kv), scale, t, length, nq)
        sums = lse[s].double().view(nq, kv, -1).permute(1, 2, 0)[..., None]
        there = sees & (sums != -torch.inf)
        w = torch.where(there, torch.exp(x - sums), 0.0)
        off = torch.where(there, w * (d * U * abs(scale) * mag + 4 * U * x.abs() + 4 * U * sums.abs() + 2.0 ** -21) + 2.0 ** -126, 0.0)
        out[s][:, t] += w.sum((1, 2)).cpu().numpy()
        bound[s][:, t] += off.sum((1, 2)).cpu().numpy()
    return out, positions, bound + (nq * (H // kv) + 2) * U * np.abs(out)


def evict(rows, N, table, lens, keep, recent, weights, positions, seen):
    """As fp4_reference.evict, head by head, for sequences that can all be evicted."""
    S, H, _ = weights.shape
    new_lens = lens.copy()
    for s in range(S):
        n, k = max(int(lens[s]), 0), max(int(keep[s]), 0)
        new_lens[s] = min(n, k)
        if n <= k:
            continue
        t = np.arange(n)
        for h in range(H):
            w = weights[s, h, :n].astype(np.float64)
            kind = np.where(positions[s, h, :n].astype(np.int64) >= int(seen[s]) - min(recent, k), 2, np.isnan(w))
            gone = np.lexsort((t, np.where(kind == 0, w, 0.0), kind))[:n - k]
            stays = np.ones(n, bool)
            stays[gone] = False
            to, at = t[:k][~stays[:k]], t[k:][stays[k:]]
            assert len(to) == len(at)
            for r in rows:
                r[table[s, to // N], h, to % N] = r[table[s, at // N], h, at % N]
            for x in (weights, positions):
                x[s, h, to] = x[s, h, at]
    return new_lens
