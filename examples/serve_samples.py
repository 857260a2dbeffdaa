"""Samples of several prompts behind one system prompt, decoded together: what a serving program does with the paged cache
and the compressed pool.

    python examples/serve_samples.py

  * the system prompt and the prompts are prefilled in chunks: append, then attention of the chunk's queries;
  * every prompt is forked into samples: whole blocks are shared, the last one, which is not full, is copied;
  * decode steps run from a HIP graph: append and attention over the samples' own blocks and the shared system prompt;
  * the samples of one prompt make room: their blocks go to the pool, blocks that they share once, under several names;
  * one of them ends: its names are given up, the pool is compacted and the rest moves on with the smaller one;
  * the others come back to cache blocks that are free by then, and all go on.

The model is a stack of random projections.  Attention is checked against the formula, in 32 bits over the tokens in the cache, and the
blocks that came back against what they held.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2512_11920_amd import kvc  # noqa: E402

N, D, KV, HEADS, LAYERS = 16, 128, 2, 8, 2
BLOCKS, POOL_BLOCKS, WIDTH = 128, 64, 16  # cache and pool blocks of a layer; blocks of a sequence
SYSTEM, PROMPTS, SAMPLES, CHUNK = 150, (37, 90), 3, 64


class Server:
    def __init__(self, dev="cuda:0", seed=0):
        self.dev, self.gen = dev, torch.Generator(device=dev).manual_seed(seed)
        self.codec = kvc.Codec(N, D, 2 * KV, kvc.MODE_RLE)
        self.codec.alloc_pool(LAYERS * POOL_BLOCKS, LAYERS * POOL_BLOCKS * 2 * KV * N * D * 2, dev)
        self.cache = torch.full((LAYERS * BLOCKS, 2 * KV, N, D), float("nan"), dtype=torch.float16, device=dev)  # (nothing is read that was not written)
        self.free = list(range(BLOCKS))
        self.w_in = [self.random(HEADS * D, (HEADS + 2 * KV) * D) * (HEADS * D) ** -0.5 for _ in range(LAYERS)]
        self.prefix = torch.full((1, WIDTH), -1, dtype=torch.int32, device=dev)
        self.prefix_lens = torch.zeros(1, dtype=torch.int32, device=dev)

    def random(self, *shape):
        return torch.randn(shape, generator=self.gen, device=self.dev, dtype=torch.float32).half()

    def ids(self, rows):
        return torch.tensor(rows, dtype=torch.int32, device=self.dev)

    def layer(self, l):
        return self.cache[l * BLOCKS:(l + 1) * BLOCKS]

    def blocks_for(self, row, tokens):
        """The row's missing blocks up to so many tokens."""
        return row + [self.free.pop() for _ in range(-(-tokens // N) - len(row))]

    def table(self, rows):
        return self.ids([r + [-1] * (WIDTH - len(r)) for r in rows])

    def run_layers(self, x, table, lens, work, prefix):
        """x [n_seq][n_q][HEADS*D], the hidden states of the sequences' last n_q tokens, through all layers."""
        s, n, _ = x.shape
        seen = []
        for l in range(LAYERS):
            qkv = (x @ self.w_in[l]).view(s, n, HEADS + 2 * KV, D)
            q, k, v = qkv[:, :, :HEADS], qkv[:, :, HEADS:HEADS + KV], qkv[:, :, HEADS + KV:]
            out = torch.empty((s, n, HEADS, D), dtype=torch.float16, device=self.dev)
            self.codec.append(self.layer(l), table, lens, k, v)
            self.codec.attend(out, q, self.layer(l), table, lens, work, **prefix)
            seen.append((q, out))
            x = (x + out.view(s, n, -1)) * 0.7071
        return x, seen

    def shared(self, n_seq):
        return dict(prefix_table=self.prefix, prefix_lens=self.prefix_lens, prefix_first=self.ids([0, n_seq]))

    def prefill(self, n, prefix):
        """-> the blocks of a new sequence of n tokens, and how far attention was off."""
        row, worst = self.blocks_for([], n), 0.0
        table = self.table([row])
        for at in range(0, n, CHUNK):
            m = min(CHUNK, n - at)
            lens = self.ids([at + m])
            work = torch.empty(kvc.attend_workspace(1, m, HEADS, KV, D, 1 if prefix else 0), dtype=torch.uint8, device=self.dev)
            _, seen = self.run_layers(self.random(1, m, HEADS * D), table, lens, work, prefix)
            worst = max(worst, self.off(seen, [row], [at + m], bool(prefix)))
        return row, worst

    def tokens(self, l, row, n):
        """K and V of a sequence's n tokens, [n][KV][D] each, in 32 bits."""
        t = torch.arange(n, device=self.dev)
        pages = self.layer(l)[self.ids(row).long()[t // N], :, t % N].float()
        return pages[:, :KV], pages[:, KV:]

    def off(self, seen, rows, lens, prefix):
        """How far the layers' attention is from the formula, as a share of the largest value."""
        worst = 0.0
        for l, (q, out) in enumerate(seen):
            n = q.shape[1]
            for s, row in enumerate(rows):
                k, v = self.tokens(l, row, lens[s])
                before = 0
                if prefix:
                    before = SYSTEM
                    pk, pv = self.tokens(l, [int(b) for b in self.prefix[0] if b >= 0], SYSTEM)
                    k, v = torch.cat([pk, k]), torch.cat([pv, v])
                ends = before + lens[s] - n + 1 + torch.arange(n, device=self.dev)
                hidden = torch.arange(len(k), device=self.dev)[None] >= ends[:, None]
                for h in range(HEADS):
                    x = (q[s, :, h].float() @ k[:, h * KV // HEADS].t().contiguous()) * D ** -0.5
                    want = torch.softmax(x.masked_fill(hidden, float("-inf")), dim=1) @ v[:, h * KV // HEADS].contiguous()
                    worst = max(worst, float((out[s, :, h].float() - want).abs().max() / want.abs().max()))
        return worst


class Decoder:
    """Decode steps of a batch, replayed from a graph; the block tables have room for `steps` of them."""

    def __init__(self, server, rows, lens, steps):
        self.server, self.lens = server, list(lens)
        for i, n in enumerate(lens):
            rows[i] = server.blocks_for(rows[i], n + steps)
        self.rows, s = rows, len(rows)
        self.table, self.dev_lens = server.table(rows), server.ids(lens)
        self.x = server.random(s, 1, HEADS * D)
        self.work = torch.empty(kvc.attend_workspace(s, 1, HEADS, KV, D, 1), dtype=torch.uint8, device=server.dev)
        self.shared = server.shared(s)  # (kept, as everything that the graph uses)
        start, first = self.dev_lens.clone(), self.x.clone()

        def step():
            self.dev_lens.add_(1)
            x, self.seen = server.run_layers(self.x, self.table, self.dev_lens, self.work, self.shared)
            self.x.copy_(x)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            step()  # (what torch sets up on first use; its token is written again by the first replay)
            self.dev_lens.copy_(start)
            self.x.copy_(first)
            side.synchronize()
            with torch.cuda.graph(self.graph, stream=side):
                step()
        torch.cuda.current_stream().wait_stream(side)

    def run(self, steps):
        worst = 0.0
        for _ in range(steps):
            self.graph.replay()
            self.lens = [n + 1 for n in self.lens]
            worst = max(worst, self.server.off(self.seen, self.rows, self.lens, True))
        return worst


def all_layers(server, ids, per_layer):
    return server.ids([l * per_layer + i for l in range(LAYERS) for i in ids])


def main(dev="cuda:0"):
    server = Server(dev)
    codec, worst = server.codec, []

    row, off = server.prefill(SYSTEM, {})
    worst.append(off)
    server.prefix = server.table([row])
    server.prefix_lens.fill_(SYSTEM)

    rows, lens = [], []
    for n in PROMPTS:
        row, off = server.prefill(n, server.shared(1))
        worst.append(off)
        forks = [row]
        for _ in range(SAMPLES - 1):
            forks.append(row[:n // N] + ([server.free.pop()] if n % N else []))
        if n % N:
            codec.copy_blocks(server.cache, server.ids([row[-1]] * (SAMPLES - 1)), server.ids([r[-1] for r in forks[1:]]), LAYERS, BLOCKS)
        rows += forks
        lens += [n] * SAMPLES
    batch = Decoder(server, rows, lens, 20)
    worst.append(batch.run(20))
    rows, lens = batch.rows, batch.lens
    print(f"{len(rows)} samples of {lens} tokens behind {SYSTEM}: attention within {max(worst):.1e}")

    # the second prompt's samples make room
    parked, whole = rows[SAMPLES:], PROMPTS[1] // N
    kept = [[server.tokens(l, r, n) for l in range(LAYERS)] for r, n in zip(parked, lens[SAMPLES:])]
    names, pool_id = [], 0
    for s, r in enumerate(parked):
        names.append(list(range(pool_id, pool_id + len(r))))
        pool_id += len(r)
        new = range(len(r)) if s == 0 else range(whole, len(r))
        src, dst = all_layers(server, [r[i] for i in new], BLOCKS), all_layers(server, [names[s][i] for i in new], POOL_BLOCKS)
        codec.compress_blocks(server.cache, src.numel(), src, dst)
        if s:
            codec.fork_blocks(server.ids(names[0][:whole]), server.ids(names[s][:whole]), LAYERS, POOL_BLOCKS)
    server.free += sorted({b for r in parked for b in r})
    before = codec.stats(check=True)
    rest = Decoder(server, rows[:SAMPLES], lens[:SAMPLES], 12)  # (takes some of the blocks given up)
    worst.append(rest.run(12))

    # the first of them ends
    codec.free_blocks(server.ids(names[0]), LAYERS, POOL_BLOCKS)
    pool, desc, used = torch.empty_like(codec.pool), torch.empty_like(codec.desc), torch.empty(1, dtype=torch.int64, device=dev)
    codec.compact_pool(pool, desc, used, torch.empty(kvc.compact_workspace(pool.numel()), dtype=torch.uint8, device=dev))
    codec.adopt_pool(pool, desc, used)
    after = codec.stats(check=True)
    print(f"pool: {before['pool_bytes_used']:,} bytes used, {after['pool_bytes_used']:,} after one sample ended and compaction")

    # the others come back, with the blocks that they share decoded once
    back = [server.blocks_for([], N * len(names[1]))]
    back += [back[0][:whole] + server.blocks_for([], N * (len(r) - whole)) for r in names[2:]]
    for s, r in enumerate(back):
        take = range(len(r)) if s == 0 else range(whole, len(r))
        src, dst = all_layers(server, [names[1 + s][i] for i in take], POOL_BLOCKS), all_layers(server, [r[i] for i in take], BLOCKS)
        codec.decompress_blocks(server.cache, src.numel(), src, dst)
    codec.free_blocks(server.ids(sum(names[1:], [])), LAYERS, POOL_BLOCKS)
    loss = 0.0
    for s, r in enumerate(back):
        for l in range(LAYERS):
            for was, now in zip(kept[1 + s][l], server.tokens(l, r, lens[SAMPLES + 1 + s])):
                loss = max(loss, float((was - now).abs().max() / was.abs().max()))
    final = Decoder(server, rest.rows + back, rest.lens + lens[SAMPLES + 1:], 20)
    worst.append(final.run(20))
    print(f"{len(final.rows)} samples of {final.lens} tokens: attention within {max(worst):.1e}, tokens that came back within {loss:.1e} (INT8)")
    empty = codec.stats(check=True)
    return dict(worst=max(worst), loss=loss, used_before=before["pool_bytes_used"], used_after=after["pool_bytes_used"], live=after["payload_bytes"],
                live_before=before["payload_bytes"], live_at_end=empty["payload_bytes"])


if __name__ == "__main__":
    main()
