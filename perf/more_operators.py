"""Operators that keep a paged cache small while it is attended over, for performance measurement.

Four kinds of pass:

append4  append_fp4 and unpack_fp4: K and V rows of new tokens go to their places in a cache that is held in 4 bits, and
         blocks of it become FP16 again, as they do when they leave for the compressed pool.
attend4  attend_fp4: attention of every sequence's last tokens over a cache held in 4 bits.
weigh    weigh: the attention weight that each token of the cache got from the last tokens' queries is added to what it
         had, for every K/V head; the cache is FP16 or held in 4 bits.
evict    evict: the tokens with the least weight leave, but for the last ones, and those that stay move together.

In 4 bits, 32 neighbouring channels of a token share a power of two 2^e, and each is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 of
it, with a sign.  e is the smallest whole number for which the largest magnitude is at most 7 * 2^e, and at most 13; a
magnitude becomes the nearest of the eight, halfway the one of even number.  A group with a value that is not finite
is NaN.  A page of N tokens of a head is N * d/2 bytes of codes (channel 2i of a token in the low half of its byte i), N
bytes of e + 127 for each 32 channels, and as many more as make a multiple of 16.

Inputs have the distribution of LLaMA-shaped K/V caches: per (K|V, head, channel) a scale exp(N(0, 0.5)), for keys
2 % of the channels ten times larger.  Blocks of a sequence lie anywhere in the cache.  Lengths are spread evenly over a
case's range and dealt to the sequences by the seed."""
import math

import numpy as np
import torch

own = False  # False: the plain forms below; True: the framework's operators

DEV = "cuda:0"
VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
MIDS = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)


def listed():
    append = {"op": "append4", "N": 16, "separate": False, "strided": False, "holes": False}
    attend = {"op": "attend4", "N": 16, "q": 1, "separate": False, "holes": False, "idle": 0}
    weigh = {"op": "weigh", "N": 16, "q": 1, "fp4": False, "separate": False, "strided": False, "holes": False, "idle": 0}
    evict = {"op": "evict", "N": 16, "fp4": False, "separate": False, "strided": False}
    return [
        # the Tiny configuration (4 heads x 64): one new token, and the 16 blocks of its sequence leave
        dict(append, name="append4_tiny", d=64, kv=4, seqs=1, new=1, len_lo=256, len_hi=256),
        # the first and second chunks of 16 prompts, 70B shape, which are offloaded to wait for their turn
        dict(append, name="append4_chunks_70b", d=128, kv=8, seqs=16, new=512, len_lo=512, len_hi=1024),
        # three verified tokens of 45 sequences, 24 x 96 pages, K and V caches apart, blocks that are not there
        dict(append, name="append4_24x96", N=24, d=96, kv=6, seqs=45, new=3, len_lo=7, len_hi=901, separate=True, strided=True, holes=True),
        # the Tiny configuration: one sequence of 256 tokens answers
        dict(attend, name="attend4_tiny", d=64, kv=4, group=1, seqs=1, len_lo=256, len_hi=256),
        # the 7B single-layer configuration (32 heads x 128, batch 8, up to 2048 tokens), K and V caches apart
        dict(attend, name="attend4_7b_layer", d=128, kv=32, group=1, seqs=8, len_lo=1024, len_hi=2048, separate=True),
        # one layer of a decode step of the 70B shape: 64 sequences of 512 to 8192 tokens, 8 query heads to a K/V head
        dict(attend, name="attend4_step_70b", d=128, kv=8, group=8, seqs=64, len_lo=512, len_hi=8192),
        # four tokens to verify in each of 45 sequences, 24 x 96 pages, blocks that are not there, two idle slots of the batch
        dict(attend, name="attend4_24x96", N=24, d=96, kv=6, group=3, q=4, seqs=45, len_lo=7, len_hi=901, holes=True, idle=2),
        # the Tiny configuration: what one token looked at
        dict(weigh, name="weigh_tiny", d=64, kv=4, group=1, seqs=1, len_lo=256, len_hi=256),
        # one layer of a decode step of the 70B shape
        dict(weigh, name="weigh_step_70b", d=128, kv=8, group=8, seqs=64, len_lo=512, len_hi=8192),
        # the last 256 tokens of four prompts look at all of it, in 4 bits
        dict(weigh, name="weigh_chunks_fp4", d=128, kv=8, group=8, q=256, seqs=4, len_lo=1024, len_hi=2048, fp4=True),
        # a decode step of 64 sequences that are at their budget of 4096 tokens: one token of each head leaves
        dict(evict, name="evict_step_70b", d=128, kv=8, seqs=64, len_lo=4097, len_hi=4097, keep=4096, recent=512),
        # 64 sequences of 8192 tokens are cut to half
        dict(evict, name="evict_half_70b", d=128, kv=8, seqs=64, len_lo=8192, len_hi=8192, keep=4096, recent=512),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over their logarithms."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Another call of the same ranges: any page shape, one sequence to 256, one token to 16384."""
    op = rng.choice(["append4", "attend4", "attend4", "weigh", "evict"])
    d = rng.choice([32, 64, 64, 96, 128, 128, 128, 160, 192, 224, 256])
    most = 4096 // d
    case = {"op": op, "N": rng.choice([16, 16, 16, min(32, most), 8, rng.randint(1, most)]), "d": d, "kv": rng.choice([1, 2, 4, 5, 8, 8]), "separate": rng.random() < 0.3,
            "seqs": _spread(rng, 1, 256)}
    hi = _spread(rng, 1, 16384)
    case.update(len_lo=_spread(rng, 1, hi), len_hi=hi)
    if op != "attend4":
        case["strided"] = rng.random() < 0.3
    if op != "evict":
        case["holes"] = rng.random() < 0.2
    if op in ("weigh", "evict"):
        case["fp4"] = rng.random() < 0.5
    if op in ("attend4", "weigh"):
        case.update(group=rng.choice([1, 5, 7] if d % 96 == 0 else [1, 2, 5, 7, 8, 8]), idle=rng.choice([0, 0, 1]) if case["seqs"] > 1 else 0)
        case["q"] = rng.choice([1, 1, 1, 2, 3, 4, rng.randint(1, 8)] if op == "attend4" else [1, 1, 1, 2, 4, rng.randint(1, 8), _spread(rng, 8, 256)])
    if op == "append4":
        case["new"] = min(case["len_lo"], rng.choice([1, 1, 2, 4, _spread(rng, 1, 512)]))
    if op == "evict":
        case["keep"] = rng.choice([max(1, case["len_lo"] - 1), _spread(rng, 1, hi), _spread(rng, 1, hi)])
        case["recent"] = rng.choice([0, _spread(rng, 1, case["keep"]), case["keep"]])
    name = {"append4": "append4_chunks_70b", "attend4": "attend4_step_70b", "weigh": "weigh_step_70b", "evict": "evict_half_70b"}[op]
    size = {"append4": 1, "attend4": 4, "weigh": 4, "evict": 1}[op]
    top, chunk = work(next(c for c in listed() if c["name"] == name)), work(next(c for c in listed() if c["name"] == "weigh_chunks_fp4"))
    # (the flops of the chunks in 4 bits are the most, the bytes those of each operator's largest case; and the cache is no larger than 2 GB)
    while work(case)["bytes"] > top["bytes"] or work(case)["flops"] > chunk["flops"] or case["seqs"] * case["len_hi"] * case["kv"] * d * 4 > 2e9 * size:
        if case["seqs"] > 1:
            case["seqs"] = (case["seqs"] + 1) // 2
            if "idle" in case:
                case["idle"] = min(case["idle"], case["seqs"] - 1)
        else:
            case["len_hi"] = max(1, case["len_hi"] // 2)
            case["len_lo"] = min(case["len_lo"], case["len_hi"])
            if "new" in case:
                case["new"] = min(case["new"], case["len_lo"])
            if "q" in case:
                case["q"] = max(1, case["q"] // 2)
    return case


# ------------------------------------------------------------------------------------------------ sizes


def _even(lo, hi, n):
    """n whole numbers spread evenly over lo..hi."""
    return np.array([round(lo + (hi - lo) * (i + 0.5) / n) if n > 1 else hi for i in range(n)], np.int64)


def _lens(case):
    """Tokens of each sequence before the seed deals them out; idle slots of the batch have none."""
    idle = case.get("idle", 0)
    return np.concatenate([_even(case["len_lo"], case["len_hi"], case["seqs"] - idle), np.zeros(idle, np.int64)])


def _row(case, fp4):
    """Bytes of a token's row of one head, of keys or of values."""
    return 17 * case["d"] // 32 if fp4 else 2 * case["d"]


def work(case):
    N, d, kv = case["N"], case["d"], case["kv"]
    lens = _lens(case)
    tokens, blocks = float(lens.sum()), float((-(-lens // N)).sum())
    there = 0.95 if case.get("holes") else 1.0
    rows = case["seqs"] * kv * case.get("group", 1) * case.get("q", 1)
    if case["op"] == "append4":  # rows in FP16 read, in 4 bits written; blocks in 4 bits read, in FP16 written
        new = 2.0 * case["seqs"] * case["new"] * kv
        return {"bytes": there * new * (_row(case, False) + _row(case, True)) + 2 * blocks * kv * N * (_row(case, False) + _row(case, True)), "flops": 0.0}
    if case["op"] == "attend4":
        return {"bytes": there * 2 * tokens * kv * _row(case, True) + 4.0 * rows * d + 4 * blocks, "flops": there * 4.0 * d * rows / case["seqs"] * tokens}
    if case["op"] == "weigh":  # keys, queries, their sums of weights; weights before and after; positions of new tokens
        return {"bytes": there * tokens * kv * _row(case, case["fp4"]) + rows * (2.0 * d + 4) + 8.0 * tokens * kv + 4.0 * case["seqs"] * case["q"] * kv + 4 * blocks,
                "flops": there * 2.0 * d * rows / case["seqs"] * tokens}
    # weights and positions of all tokens read and of those that stay written; rows behind the budget that stay are moved, a share of them that goes by how many leave
    keep = np.minimum(lens, case["keep"]).astype(float)
    moved = float((keep * (lens - keep) / lens).sum())
    least = {"bytes": kv * (8.0 * tokens + 8.0 * keep.sum() + moved * 4 * _row(case, case["fp4"])) + 4 * blocks, "flops": 0.0}
    if case["fp4"]:  # (and the blocks in FP16, to be looked at)
        least["bytes"] += 2 * blocks * kv * N * (_row(case, False) + _row(case, True))
    return least


# ------------------------------------------------------------------------------------------------ 4 bits


def _page_bytes(case):
    return -(-case["N"] * 17 * case["d"] // 32 // 16) * 16


def _pack(x):
    """x [..., d] -> codes [..., d/2] and exponent bytes [..., d/32], both uint8."""
    g = x.float().unflatten(-1, (-1, 32))
    a = g.abs().amax(-1)
    m, e = torch.frexp(a)  # a = m * 2^e, m from 0.5 to 1
    e = torch.where(m <= 0.875, e - 3, e - 2).clamp_max(13)
    finite = torch.isfinite(g).all(-1)
    y = torch.ldexp(g.abs(), -e[..., None])
    code = torch.zeros_like(y, dtype=torch.uint8)
    for i, mid in enumerate(MIDS):
        code += (y >= mid if i % 2 else y > mid).to(torch.uint8)
    code = torch.where(finite[..., None], code + 8 * torch.signbit(g).to(torch.uint8), 0).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), torch.where(finite, torch.where(a == 0, 0, e + 127), 255).to(torch.uint8)


def _unpack(codes, exps, dtype=torch.float32):
    """The values that codes [..., d/2] and exponent bytes [..., d/32] stand for."""
    values = torch.tensor(VALUES + tuple(-v for v in VALUES), dtype=dtype, device=DEV)
    x = torch.stack([values[(codes & 15).long()], values[(codes >> 4).long()]], -1).flatten(-2).unflatten(-1, (-1, 32))
    scale = torch.where(exps == 255, math.nan, torch.ldexp(torch.ones_like(exps, dtype=dtype), exps.int() - 127))
    return (x * scale[..., None]).flatten(-2)


def _parts(case, cache):
    """Codes [block][page][token][d/2] and exponents [block][page][token][d/32] of a cache in 4 bits, as views."""
    N, d = case["N"], case["d"]
    pages = cache.view(len(cache), -1, _page_bytes(case))
    return pages[:, :, :N * d // 2].unflatten(-1, (N, d // 2)), pages[:, :, N * d // 2:N * d // 2 + N * d // 32].unflatten(-1, (d // 32, N)).transpose(-1, -2)


# ------------------------------------------------------------------------------------------------ inputs


def _gen(seed, *idx):
    g = torch.Generator(device=DEV)
    s = int(seed)
    for i in idx:
        s = s * 1000003 + int(i) + 1
    g.manual_seed(s % (1 << 62))
    return g


def _scales(gen, heads, d, keys):
    c = torch.exp(0.5 * torch.randn((heads, 1, d), generator=gen, device=DEV))
    return torch.where(torch.rand((heads, 1, d), generator=gen, device=DEV) < 0.02, 10.0 * c, c) if keys else c


def _cache(case, gen, n, key_pages, value_pages, fp4):
    """n blocks of pages, keys first: FP16 [n][pages][N][d] (of memory [n][N][pages][d] where the case is strided), or [n][bytes] in 4 bits."""
    N, d, pages = case["N"], case["d"], key_pages + value_pages
    c = torch.cat([_scales(gen, key_pages, d, True), _scales(gen, value_pages, d, False)])
    strided = not fp4 and case.get("strided")
    if fp4:
        out = torch.zeros((n, pages * _page_bytes(case)), dtype=torch.uint8, device=DEV)
        codes, exps = _parts(case, out)
    else:
        out = torch.empty((n, N, pages, d) if strided else (n, pages, N, d), dtype=torch.float16, device=DEV)
        view = out.transpose(1, 2) if strided else out
    step = max(1, (1 << 25 if fp4 else 1 << 27) // (pages * N * d))
    for b in range(0, n, step):
        x = torch.randn((min(step, n - b), pages, N, d), generator=gen, device=DEV, dtype=torch.float16) * c.half()
        if fp4:
            codes[b:b + step], exps[b:b + step] = _pack(x)
        else:
            view[b:b + step] = x
    return out


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def _codec(case, strided):
    from paper_2512_11920_amd import kvc

    ppb = case["kv"] * (1 if case["separate"] else 2)
    c = kvc.Codec(case["N"], case["d"], ppb)
    if strided:
        c.set_cache_layout(case["N"] * ppb * case["d"], case["d"], ppb * case["d"])
    return c


def prepare(case, seed):
    """What a program has in hand: the cache, block tables, lengths, the tokens' projections, and what earlier steps left of weights."""
    N, d, kv, op = case["N"], case["d"], case["kv"], case["op"]
    fp4 = case.get("fp4", True)
    rng, gen = np.random.default_rng([int(seed), 21]), _gen(seed, 1)
    lens = rng.permutation(_lens(case))
    each = -(-lens // N)
    width = -(-case["len_hi"] // N) + 1  # (room in the table for the longest sequence that the case may have, and for the next block)
    n_blocks = int(each.sum()) + 3
    perm = rng.permutation(n_blocks).astype(np.int32)
    table, at = np.full((len(lens), width), -1, np.int32), 0
    for s, n in enumerate(each):
        table[s, :n] = perm[at:at + n]
        at += n
    if case.get("holes"):
        table[rng.random(table.shape) < 0.05] = -1
    if case["separate"]:
        k_cache, v_cache = _cache(case, gen, n_blocks, kv, 0, fp4), _cache(case, gen, n_blocks, 0, kv, fp4)
    else:
        k_cache, v_cache = _cache(case, gen, n_blocks, kv, kv, fp4), None
    st = {"case": case, "k_cache": k_cache, "v_cache": v_cache, "table": _dev(table), "lens": _dev(lens.astype(np.int32)), "longest": int(lens.max())}
    if own:
        from paper_2512_11920_amd import kvc

        st["codec"] = _codec(case, case.get("strided"))
    if op == "append4" or (op == "evict" and fp4):
        # blocks that leave, in any order, and where they go
        st["ids"] = _dev(rng.permutation(n_blocks)[:int(each.sum())].astype(np.int32))
        pages = kv if case["separate"] else 2 * kv
        st["fp16"] = [torch.zeros((len(st["ids"]), N, pages, d) if case["strided"] else (len(st["ids"]), pages, N, d), dtype=torch.float16, device=DEV) for _ in range(2 * kv // pages)]
    if op == "evict":
        heads, room = kv, width * N
        z = torch.randn((len(lens), heads, room), generator=gen, device=DEV)
        gone = torch.rand((len(lens), heads, room), generator=gen, device=DEV) < 0.1  # tokens that nobody has looked at yet
        st["weights"] = torch.where(gone, 0.0, torch.exp(2.0 * z))
        # tokens that stayed after earlier steps lie in any order, the newest behind them
        st["seen"] = _dev((lens + rng.integers(0, 1000, len(lens))).astype(np.int32))
        order = torch.rand((len(lens), heads, room), generator=gen, device=DEV)
        slot = torch.arange(room, device=DEV)
        old = (st["lens"] * 7 // 8)[:, None, None]
        order = torch.where(slot < old, order, 2.0 + slot)
        rank = order.argsort(-1).argsort(-1).int()
        first = (st["seen"] - st["lens"])[:, None, None]  # (positions of tokens that left are missing, here the first ones)
        st["positions"] = (rank + first).int().contiguous()
        st["keep"] = torch.full((len(lens),), case["keep"], dtype=torch.int32, device=DEV)
        st["weights_out"], st["positions_out"] = torch.zeros_like(st["weights"]), torch.zeros_like(st["positions"])
        st["new_lens"] = torch.zeros_like(st["lens"])
        if own:
            st["work"] = torch.empty(kvc.evict_workspace(len(lens), kv, room), dtype=torch.uint8, device=DEV)
        return st
    n, heads = case.get("q", case.get("new")), kv * case.get("group", 1)
    # queries, keys and values of the new tokens as one projection gives them
    st["qkv"] = torch.randn((len(lens), n, heads + 2 * kv, d), generator=gen, device=DEV, dtype=torch.float16)
    if op == "attend4" and own:
        st["work"] = torch.empty(kvc.attend_fp4_workspace(len(lens), n, heads, kv, d), dtype=torch.uint8, device=DEV)
        st["out"] = torch.empty((len(lens), n, heads, d), dtype=torch.float16, device=DEV)
    if op == "weigh":
        room = width * N
        st["weights"] = 0.05 * torch.exp(2.0 * torch.randn((len(lens), kv, room), generator=gen, device=DEV))  # (of some hundred steps)
        st["seen"] = _dev((lens + rng.integers(0, 1000, len(lens))).astype(np.int32))
        st["positions"] = torch.zeros((len(lens), kv, room), dtype=torch.int32, device=DEV)
        st["weights_out"] = torch.zeros_like(st["weights"])
        st["lse"] = _sums(st)  # as attention over this cache gives it
    return st


# ------------------------------------------------------------------------------------------------ passes


def run(state):
    op = state["case"]["op"]
    return globals()[f"_own_{op}" if own else f"_plain_{op}"](state)


def _bits(cache):
    """What was moved, to be equal bit for bit."""
    return None if cache is None else cache.view(torch.int16)


def _own_append4(st):
    kv = st["case"]["kv"]
    st["codec"].append_fp4(st["k_cache"], st["table"], st["lens"], st["qkv"][:, :, -2 * kv:-kv], st["qkv"][:, :, -kv:], v_cache=st["v_cache"])
    for out, cache in zip(st["fp16"], (st["k_cache"], st["v_cache"])):
        st["codec"].unpack_fp4(out, cache, st["ids"])
    return st["fp16"]


def _own_attend4(st):
    st["codec"].attend_fp4(st["out"], st["qkv"][:, :, :-2 * st["case"]["kv"]], st["k_cache"], st["table"], st["lens"], st["work"], v_cache=st["v_cache"])
    return st["out"]


def _own_weigh(st):
    st["codec"].weigh(st["weights"], st["positions"], st["seen"], st["qkv"][:, :, :-2 * st["case"]["kv"]], st["k_cache"], st["table"], st["lens"], st["lse"], weights_out=st["weights_out"])
    return st["weights_out"], st["positions"]


def _own_evict(st):
    st["codec"].evict(st["k_cache"], st["table"], st["lens"], st["keep"], st["case"]["recent"], st["weights"], st["positions"], st["seen"], st["new_lens"], st["work"], v_cache=st["v_cache"],
                      weights_out=st["weights_out"], positions_out=st["positions_out"])
    if st["case"]["fp4"]:
        for out, cache in zip(st["fp16"], (st["k_cache"], st["v_cache"])):
            st["codec"].unpack_fp4(out, cache, st["ids"])
    return (st["fp16"] if st["case"]["fp4"] else (_bits(st["k_cache"]), _bits(st["v_cache"]))), st["weights_out"], st["positions_out"], st["new_lens"]


def _pages(st, cache):
    """An FP16 cache as [block][page][token][channel]."""
    return cache.transpose(1, 2) if st["case"].get("strided") else cache


def _plain_fp16(st):
    """Blocks st["ids"] in FP16."""
    for out, cache in zip(st["fp16"], (st["k_cache"], st["v_cache"])):
        codes, exps = _parts(st["case"], cache)
        _pages(st, out)[:] = _unpack(codes[st["ids"].long()], exps[st["ids"].long()]).half()
    return st["fp16"]


def _plain_append4(st):
    case = st["case"]
    N, kv, n = case["N"], case["kv"], case["new"]
    at = st["lens"].long()[:, None] - n + torch.arange(n, device=DEV)
    block, row = st["table"].long().gather(1, at // N), at % N
    # (a place for rows without a block: behind the others)
    seq, i = (block >= 0).nonzero(as_tuple=True)
    block, row = block[seq, i], row[seq, i]
    for cache, first, x in ((st["k_cache"], 0, st["qkv"][:, :, -2 * kv:-kv]), (st["k_cache"], kv, st["qkv"][:, :, -kv:]) if st["v_cache"] is None else (st["v_cache"], 0, st["qkv"][:, :, -kv:])):
        for part, new in zip(_parts(case, cache), _pack(x[seq, i])):
            part.transpose(1, 2)[:, :, first:first + kv][block, row] = new
    return _plain_fp16(st)


def _plain_tokens(st, table, keys):
    """K or V of the tokens of a table's rows, 32 bits: [rows][head][tokens][d]."""
    case = st["case"]
    N, d, kv = case["N"], case["d"], case["kv"]
    ids = table.long().clamp_min(0)
    cache = st["k_cache"] if keys or st["v_cache"] is None else st["v_cache"]
    first = 0 if keys or st["v_cache"] is not None else kv
    if case.get("fp4", True):
        x = _unpack(*[p[:, first:first + kv][ids] for p in _parts(case, cache)])
    else:
        x = _pages(st, cache)[:, first:first + kv][ids].float()
    return x.permute(0, 2, 1, 3, 4).reshape(len(ids), kv, -1, d)


def _plain_pieces(st):
    """Sequences by the piece, so that scores and tokens in 32 bits stay below a few GB: their rows, scaled scores [rows][head][query of the group][tokens] with
    -infinity where a query does not see a token, and which tokens there are."""
    case = st["case"]
    N, d, kv, group, n, S = case["N"], case["d"], case["kv"], case["group"], case["q"], case["seqs"]
    q = st["qkv"][:, :, :-2 * kv].reshape(S, n, kv, group, d).permute(0, 2, 3, 1, 4).reshape(S, kv, group * n, d).float()
    table = st["table"]
    piece = max(1, (1 << 29) // (table.shape[1] * N * kv * max(d, group * n)))
    for a in range(0, S, piece):
        keys = _plain_tokens(st, table[a:a + piece], True)
        t = torch.arange(keys.shape[2], device=DEV)
        there = (table[a:a + piece] >= 0).repeat_interleave(N, 1) & (t < st["lens"][a:a + piece, None])
        last = st["lens"][a:a + piece, None].long() - (n - 1 - torch.arange(n, device=DEV))  # tokens that query i sees
        seen = (t < last[:, :, None]) & there[:, None, :]
        x = torch.matmul(q[a:a + piece], keys.transpose(-1, -2).contiguous()) * d ** -0.5
        yield slice(a, a + piece), x.masked_fill_(~seen.repeat(1, group, 1)[:, None], -math.inf), there


def _rows_back(st, x):
    """[sequence][head][query of the group].. as [sequence][query][head].."""
    case = st["case"]
    x = x.unflatten(2, (case["group"], case["q"]))
    return x.permute(0, 3, 1, 2, *range(4, x.dim())).flatten(2, 3)


def _sums(st):
    """ln of the sum of e^score of every query: [sequence][query][head], 32 bits."""
    return _rows_back(st, torch.cat([torch.logsumexp(x, -1) for _, x, _ in _plain_pieces(st)])).contiguous()


def _plain_attend4(st):
    out = []
    for rows, x, there in _plain_pieces(st):
        values = torch.where(there[:, None, :, None], _plain_tokens(st, st["table"][rows], False), 0.0)
        m = x.amax(-1, keepdim=True)
        p = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
        total = p.sum(-1, keepdim=True)
        out.append(torch.where(total > 0, torch.matmul(p, values) / total, 0.0))
    return _rows_back(st, torch.cat(out)).half()


def _plain_weigh(st):
    case = st["case"]
    kv, group, n, S = case["kv"], case["group"], case["q"], case["seqs"]
    lse = st["lse"].view(S, n, kv, group).permute(0, 2, 3, 1).reshape(S, kv, group * n, 1)
    lse = torch.where(lse == -math.inf, 0.0, lse)
    t = torch.arange(st["weights"].shape[2], device=DEV)
    lens = st["lens"][:, None, None]
    old = torch.where(t < lens - n, st["weights"], 0.0)  # new tokens have none yet
    for rows, x, _ in _plain_pieces(st):
        got = torch.exp(x - lse[rows]).sum(2)
        old[rows] += got
    st["weights_out"][:] = torch.where(t < lens, old, st["weights_out"])
    new = (t >= lens - n) & (t < lens)
    st["positions"][:] = torch.where(new, st["seen"][:, None, None] - lens + t, st["positions"])
    return st["weights_out"], st["positions"]


def _plain_evict(st):
    case = st["case"]
    N, kv = case["N"], case["kv"]
    lens, t = st["lens"][:, None, None], torch.arange(st["weights"].shape[2], device=DEV)
    keep = torch.minimum(st["keep"], st["lens"])[:, None, None]
    safe = st["positions"] >= (st["seen"] - torch.minimum(st["keep"], torch.full_like(st["keep"], case["recent"])))[:, None, None]
    key = torch.where(t < lens, torch.where(safe, math.inf, st["weights"]), math.nan)  # (slots behind the last token are behind all others)
    rank = torch.empty_like(st["positions"])
    rank.scatter_(2, torch.sort(key, dim=2, stable=True).indices, t.int().expand_as(rank))
    stays = (rank >= lens - keep) & (t < lens)
    # evicted slots below the budget, and tokens behind it that stay: as many of each in every head, in the same order
    s, h, hole = (~stays & (t < keep)).nonzero(as_tuple=True)
    filler = (stays & (t >= keep)).nonzero(as_tuple=True)[2]
    caches = [(st["k_cache"], 0), (st["k_cache"], kv) if st["v_cache"] is None else (st["v_cache"], 0)]
    to, at = st["table"][s, hole // N].long(), st["table"][s, filler // N].long()
    for cache, first in caches:
        for part in _parts(case, cache) if case["fp4"] else [_pages(st, cache)]:
            part[to, first + h, hole % N] = part[at, first + h, filler % N]
    for old, new in ((st["weights"], st["weights_out"]), (st["positions"], st["positions_out"])):
        new[:] = torch.where(t < keep, old, new)
        new[s, h, hole] = old[s, h, filler]
    st["new_lens"][:] = keep[:, 0, 0]
    return (_plain_fp16(st) if case["fp4"] else (_bits(st["k_cache"]), _bits(st["v_cache"]))), st["weights_out"], st["positions_out"], st["new_lens"]


# ------------------------------------------------------------------------------------------------ in 64 bits


def _exact_value(code, exp):
    """What one code (0 to 15) and exponent byte stand for; arrays of them."""
    two, half = (code & 6) >> 1, (code & 1).astype(np.float64)
    x = np.where(two == 0, 0.5 * half, (1 + 0.5 * half) * 2.0 ** (two - 1.0))
    with np.errstate(invalid="ignore"):
        return np.where(exp == 255, np.nan, np.where(code & 8, -x, x) * 2.0 ** (exp.astype(np.float64) - 127))


def _exact_blocks(case, cache):
    """All blocks [block][page][token][channel], in 64 bits, on the host; page by page from the bytes."""
    N, d = case["N"], case["d"]
    raw = cache.cpu().numpy().reshape(len(cache), -1, _page_bytes(case))
    code = raw[:, :, :N * d // 2].reshape(len(raw), -1, N, d // 2)
    exp = raw[:, :, N * d // 2:N * d // 2 + N * d // 32].reshape(len(raw), -1, d // 32, N)
    table = _exact_value(np.arange(16)[None, :], np.arange(256)[:, None])
    out = np.empty((*code.shape[:3], d))
    for c in range(d):
        out[..., c] = table[exp[:, :, c // 32], code[..., c // 2] >> (4 * (c & 1)) & 15]
    return out


def _exact_nearest(x):
    """Rows x [..][d] as the cache holds them: of the eight magnitudes the nearest, of two as near the one of even number."""
    grid = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    g = x.reshape(-1, 32)
    a = np.abs(g).max(1)
    e = np.where(a > 0, np.minimum(13, np.ceil(np.log2(np.where(a > 0, a, 1) / 7))), 0)
    y = np.abs(g) / 2.0 ** e[:, None]
    off = np.abs(y[:, :, None] - grid) - 1e-9 * (np.arange(8) % 2 == 0)
    return (np.copysign(grid[off.argmin(2)], g) * 2.0 ** e[:, None]).reshape(x.shape)


def exact(case, seed):
    """append4: the values by the definition of the cache.  attend4: softmax attention, and weigh: the weights themselves, one sequence at a time in 64 bits.
    evict moves what is there and has no computed numbers."""
    if case["op"] == "evict" or case["op"] != "append4" and case["seqs"] * case["q"] > 10000:
        return None
    st = prepare(case, seed)
    N, d, kv = case["N"], case["d"], case["kv"]
    lens, table = st["lens"].tolist(), st["table"].cpu().numpy()
    if case["op"] == "append4":
        out = []
        new = st["qkv"][:, :, -2 * kv:].double().cpu().numpy()
        for which, cache in enumerate([st["k_cache"]] if st["v_cache"] is None else [st["k_cache"], st["v_cache"]]):
            blocks = _exact_blocks(case, cache)
            rows = _exact_nearest(new if st["v_cache"] is None else new[:, :, which * kv:(which + 1) * kv])
            for s, length in enumerate(lens):
                for i in range(case["new"]):
                    t = length - case["new"] + i
                    if table[s, t // N] >= 0:
                        blocks[table[s, t // N], :, t % N] = rows[s, i]
            blocks = blocks[st["ids"].cpu().numpy()]
            out.append(torch.from_numpy(np.ascontiguousarray(blocks.transpose(0, 2, 1, 3) if case["strided"] else blocks)))
        return out
    group, n = case["group"], case["q"]
    fp4 = case.get("fp4", True)
    value = torch.from_numpy(_exact_value(np.arange(16)[None, :], np.arange(256)[:, None])).to(DEV)

    def tokens(cache, first, s):
        """Positions of the tokens that have a block, and their rows [head][token][channel]."""
        t = torch.arange(lens[s], device=DEV)
        b = st["table"][s].long()[t // N]
        t, b = t[b >= 0], b[b >= 0]
        if not fp4:
            return t, (cache.transpose(1, 2) if case["strided"] else cache)[b, first:first + kv, t % N].double().transpose(0, 1)
        codes, exps = (p[b, first:first + kv, t % N].long() for p in _parts(case, cache))
        x = torch.empty((len(t), kv, d), dtype=torch.float64, device=DEV)
        for half in (0, 1):
            x[..., half::2] = value[exps.repeat_interleave(16, 2), codes >> (4 * half) & 15]
        return t, x.transpose(0, 1)

    if case["op"] == "attend4":
        out = torch.zeros((case["seqs"], n, kv, group, d), dtype=torch.float64, device=DEV)
    else:
        out, positions = st["weights_out"].double(), st["positions"].clone()
    for s in range(case["seqs"]):
        if not lens[s]:
            continue
        t, k = tokens(st["k_cache"], 0, s)
        if case["op"] == "attend4":
            _, v = tokens(st["k_cache"] if st["v_cache"] is None else st["v_cache"], kv if st["v_cache"] is None else 0, s)
        else:
            fresh = max(0, lens[s] - n)
            out[s, :, :lens[s]] = 0
            out[s, :, :fresh] = st["weights"][s, :, :fresh].double()
            positions[s, :, fresh:lens[s]] = torch.arange(fresh, lens[s], device=DEV).int() + (st["seen"][s] - lens[s])
        for i in range(n):
            here = (t < lens[s] - (n - 1 - i)).nonzero()[:, 0]
            if not len(here):
                continue
            whole = len(here) == k.shape[1]
            x = torch.bmm(st["qkv"][s, i, :kv * group].double().view(kv, group, d), (k if whole else k[:, here]).transpose(1, 2).contiguous()) * d ** -0.5
            if case["op"] == "attend4":
                out[s, i] = torch.bmm(torch.softmax(x, -1), v if whole else v[:, here])
            else:
                out[s, :, t[here]] += torch.exp(x - st["lse"][s, i].double().view(kv, group, 1)).sum(1)
    return out.view(case["seqs"], n, kv * group, d) if case["op"] == "attend4" else (out, positions)
