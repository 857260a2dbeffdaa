"""The operators that keep a cache small, run together as a serving program runs them: a prompt in chunks, decode steps from a graph, evictions in place, blocks that leave for the compressed pool."""
import numpy as np
import pytest
import torch

import fp4_reference as ref
from gpu_util import DEV
from paper_2512_11920_amd import kvc

pytestmark = pytest.mark.gpu

N, D, KV, HEADS, S, BUDGET, RECENT, SLACK = 16, 64, 2, 6, 3, 40, 8, 5


class Server:
    """One layer.  Sequences grow to BUDGET + SLACK tokens, then go back to BUDGET."""

    def __init__(self, fp4, prompts):
        self.fp4 = fp4
        self.codec = kvc.Codec(N, D, 2 * KV)
        width = -(-max(max(prompts), BUDGET + SLACK) // N)
        gen = torch.Generator(device=DEV).manual_seed(5)
        blocks = S * width + 2
        self.table = torch.randperm(blocks, generator=gen, device=DEV)[:S * width].view(S, width).int().contiguous()
        if fp4:
            self.cache = torch.full((blocks, self.codec.fp4_block_bytes), 255, dtype=torch.uint8, device=DEV)
        else:
            self.cache = torch.full((blocks, 2 * KV, N, D), float("nan"), dtype=torch.float16, device=DEV)
        room = width * N
        self.weights, self.positions = torch.full((S, KV, room), float("nan"), device=DEV), torch.full((S, KV, room), -1, dtype=torch.int32, device=DEV)
        self.lens, self.seen = torch.zeros(S, dtype=torch.int32, device=DEV), torch.zeros(S, dtype=torch.int32, device=DEV)
        self.keep = torch.full((S,), BUDGET, dtype=torch.int32, device=DEV)
        self.evict_work = torch.empty(kvc.evict_workspace(S, KV, room), dtype=torch.uint8, device=DEV)

    def buffers(self, n):
        size = kvc.attend_fp4_workspace(S, n, HEADS, KV, D) if self.fp4 else kvc.attend_workspace(S, n, HEADS, KV, D)
        return (torch.zeros((S, n, HEADS + 2 * KV, D), dtype=torch.float16, device=DEV), torch.zeros((S, n, HEADS, D), dtype=torch.float16, device=DEV),
                torch.zeros((S, n, HEADS), device=DEV), torch.empty(size, dtype=torch.uint8, device=DEV))

    def step(self, b):
        """n new tokens of every sequence."""
        qkv, out, lse, work = b
        n, c = qkv.shape[1], self.codec
        self.lens += n
        self.seen += n
        (c.append_fp4 if self.fp4 else c.append)(self.cache, self.table, self.lens, qkv[:, :, HEADS:HEADS + KV], qkv[:, :, HEADS + KV:])
        (c.attend_fp4 if self.fp4 else c.attend)(out, qkv[:, :, :HEADS], self.cache, self.table, self.lens, work, lse=lse)
        c.weigh(self.weights, self.positions, self.seen, qkv[:, :, :HEADS], self.cache, self.table, self.lens, lse)

    def evict(self):
        self.codec.evict(self.cache, self.table, self.lens, self.keep, RECENT, self.weights, self.positions, self.seen, self.lens, self.evict_work)

    def state(self):
        return {k: getattr(self, k).cpu().numpy().copy() for k in ("cache", "weights", "positions", "lens", "seen")}


def _tokens(gen, n):
    return torch.randn((S, n, HEADS + 2 * KV, D), generator=gen, device=DEV, dtype=torch.float16)


def _history_check(server, history, out, lse, q):
    """Attention's output from the tokens that positions say are there, in 64 bits."""
    st = server.state()
    rows = [ref.values(*ref.pack(h.cpu().numpy())) if server.fp4 else h.cpu().numpy().astype(np.float64) for h in history]  # [S][1][2 KV][D] of each position
    u = 2.0 ** -24
    for s in range(S):
        n = int(st["lens"][s])
        for head in range(HEADS):
            h = head // (HEADS // KV)
            at = st["positions"][s, h, :n]
            assert len(set(at.tolist())) == n and at.min() >= 0 and at.max() == int(st["seen"][s]) - 1
            k, v = np.stack([rows[p][s, 0, h] for p in at]), np.stack([rows[p][s, 0, KV + h] for p in at])
            qq = q[s, 0, head].astype(np.float64)
            x = (k @ qq) * D ** -0.5
            w = np.exp(x - x.max())
            w /= w.sum()
            want = w @ v
            # as tests/paged_reference.py derives it
            off = D * u * D ** -0.5 * (np.abs(k) @ np.abs(qq)) + 4 * u * np.abs(x) + 2.0 ** -20
            bound = (w * (off + w @ off)) @ np.abs(v) + (2.0 ** -11 + 2 * n * u + 2.0 ** -20) * (w @ np.abs(v)) + n * 2.0 ** -35 * np.abs(v).max(0) + 2.0 ** -11 * np.abs(want) + 2.0 ** -25
            assert (np.abs(out[s, 0, head] - want) <= bound).all()


@pytest.mark.parametrize("fp4", [False, True])
def test_serving_with_a_budget(fp4):
    """Prompts in chunks, then steps with evictions: what attention gives is what the tokens of the recorded positions give, and the recent ones are always there."""
    server = Server(fp4, [BUDGET + SLACK])
    gen = torch.Generator(device=DEV).manual_seed(1)
    history = []  # K and V rows of every position
    for n in (17, 1, 20):
        b = server.buffers(n)
        b[0].copy_(_tokens(gen, n))
        server.step(b)
        history += [b[0][:, i:i + 1, HEADS:].clone() for i in range(n)]
    b = server.buffers(1)
    for step in range(30):
        b[0].copy_(_tokens(gen, 1))
        server.step(b)
        history.append(b[0][:, :, HEADS:].clone())
        _history_check(server, history, b[1].cpu().numpy().astype(np.float64), b[2], b[0].cpu().numpy())
        before = server.state()
        if int(before["lens"][0]) == BUDGET + SLACK:
            server.evict()
            after = server.state()
            assert (after["lens"] == BUDGET).all()
            for s in range(S):
                for h in range(KV):
                    n = int(before["lens"][s])
                    kept = ref.stays(before["weights"][s, h], before["positions"][s, h], before["seen"][s], n, BUDGET, RECENT)
                    assert set(after["positions"][s, h, :BUDGET].tolist()) == {int(before["positions"][s, h, t]) for t in kept}
                    assert set(range(int(before["seen"][s]) - RECENT, int(before["seen"][s]))) <= set(after["positions"][s, h, :BUDGET].tolist())
    assert server.codec is not None and step == 29


@pytest.mark.parametrize("fp4", [False, True])
def test_steps_and_evictions_from_graphs(fp4):
    """A decode step and an eviction, captured once and replayed with other tokens, with eager work in between, give what the eager calls give, bit for bit."""
    eager, replayed = Server(fp4, [BUDGET + SLACK]), Server(fp4, [BUDGET + SLACK])
    gen = torch.Generator(device=DEV).manual_seed(2)
    prompt = _tokens(gen, BUDGET - 1)
    for server in (eager, replayed):
        b = server.buffers(BUDGET - 1)
        b[0].copy_(prompt)
        server.step(b)
    be, br = eager.buffers(1), replayed.buffers(1)
    saved = {k: v.clone() for k, v in vars(replayed).items() if torch.is_tensor(v)}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # (once without a graph, so that everything is loaded; then the state is put back)
        replayed.step(br)
        replayed.evict()
    torch.cuda.current_stream().wait_stream(side)
    for k, v in saved.items():
        getattr(replayed, k).copy_(v)
    step, evict = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(step):
        replayed.step(br)
    with torch.cuda.graph(evict):
        replayed.evict()
    for i in range(20):
        tokens = _tokens(gen, 1)
        be[0].copy_(tokens)
        br[0].copy_(tokens)
        eager.step(be)
        step.replay()
        if i % SLACK == SLACK - 1:
            eager.evict()
            evict.replay()
        torch.cuda.synchronize()
        a, b = eager.state(), replayed.state()
        for k in a:
            assert np.array_equal(a[k].view(np.uint8), b[k].view(np.uint8)), (i, k)
        assert torch.equal(be[1], br[1]) and torch.equal(be[2], br[2])
        assert torch.ones(1000, device=DEV).sum().item() == 1000  # (eager work between the replays)


def test_blocks_leave_for_the_pool_and_come_back():
    """4 bits -> FP16 -> the compressed pool -> FP16: what attend sees of a block that came back is what attend_fp4 saw, rounded as the pool's scheme rounds; raw pages exactly."""
    server = Server(True, [BUDGET + SLACK])
    gen = torch.Generator(device=DEV).manual_seed(3)
    b = server.buffers(BUDGET)
    b[0].copy_(_tokens(gen, BUDGET))
    server.step(b)
    ids = server.table.reshape(-1).contiguous()
    fp16 = torch.empty((len(ids), 2 * KV, N, D), dtype=torch.float16, device=DEV)
    server.codec.unpack_fp4(fp16, server.cache, ids)
    fp16.nan_to_num_(0.0)  # (rows that nobody wrote)
    pool = kvc.Codec(N, D, 2 * KV, kvc.MODE_RAW)
    pool.alloc_pool(len(ids), fp16.numel() * 2 + 64, DEV)
    pool.compress_blocks(fp16)
    back = torch.zeros_like(fp16)
    pool.decompress_blocks(back)
    assert torch.equal(back.view(torch.int16), fp16.view(torch.int16))
    out, lse = torch.empty_like(b[1]), torch.empty_like(b[2])
    table = torch.arange(len(ids), dtype=torch.int32, device=DEV).view(S, -1)
    pool.attend(out, b[0][:, :, :HEADS], back, table, server.lens, torch.empty(kvc.attend_workspace(S, BUDGET, HEADS, KV, D), dtype=torch.uint8, device=DEV), lse=lse)
    # both are within a bound of the same numbers (tests/paged_reference.py): 2^-11 for the weights, 2^-11 for the output, and 2^-17 for all that happens in 32 bits
    scale = torch.full_like(lse, 1.0)[..., None] * fp16.abs().max().float()
    assert ((out.float() - b[1].float()).abs() <= 2 * (2.0 ** -11 + 2.0 ** -11 + 2.0 ** -17) * scale).all()
    assert (lse - b[2]).abs().max() <= 2.0 ** -15


def test_two_calls_at_once():
    """Two streams, a workspace each, one cache that both read: the results are those of the calls one after the other."""
    server = Server(True, [BUDGET + SLACK])
    gen = torch.Generator(device=DEV).manual_seed(4)
    b = server.buffers(BUDGET)
    b[0].copy_(_tokens(gen, BUDGET))
    server.step(b)
    queries = [_tokens(gen, 1) for _ in range(2)]
    want = []
    for q in queries:
        bufs = server.buffers(1)
        server.codec.attend_fp4(bufs[1], q[:, :, :HEADS], server.cache, server.table, server.lens, bufs[3], lse=bufs[2])
        want.append((bufs[1].clone(), bufs[2].clone()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    bufs = [server.buffers(1) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for q, s, x in zip(queries, streams, bufs):
            server.codec.attend_fp4(x[1], q[:, :, :HEADS], server.cache, server.table, server.lens, x[3], lse=x[2], stream=s)
    torch.cuda.synchronize()
    for (o, l), x in zip(want, bufs):
        assert torch.equal(o, x[1]) and torch.equal(l, x[2])
