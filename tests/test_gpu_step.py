"""A step's operators together, as a serving loop runs them: tables, norm and rotation (and matrix), write, attention; prompts, decode steps, rejected drafts and new
sequences in place of ended ones; in a replayed graph against the same steps eagerly, on another stream, in two threads."""
import threading

import numpy as np
import pytest
import torch

from cache_util import D, Batch
from oracle import cache_oracle as co
from oracle import step_oracle as so
from paper_2410_09426_amd import binding as fq
from test_gpu_scored import expect

pytestmark = pytest.mark.gpu


class Layer:
    """One layer's cache, ring and batch of B places, and the buffers of a step of T rows."""

    def __init__(self, seed, B, T, H=2, G=4, page=16, pages=120, width=20, bits=(4, 3), cap=20.0, matrix=True):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.B, self.T, self.H, self.Hq, self.page, self.pages, self.width, self.bits, self.cap = B, T, H, H * G, page, pages, width, bits, cap
        i32 = dict(dtype=torch.int32, device="cuda")
        self.kc, self.vc = (torch.full((pages, H, page, 16 * b), 0xA5, dtype=torch.uint8, device="cuda") for b in bits)
        self.kp, self.vp = (torch.full((pages, H, page), -0x5A5A5A5B, **i32) for _ in bits)
        self.starts, self.lengths, self.table = torch.zeros(B + 1, **i32), torch.zeros(B, **i32), torch.full((B, width), -1, **i32)
        self.held, self.keep, self.rows = (torch.zeros(B, **i32) for _ in range(3))
        self.ring, self.state = torch.randperm(pages, generator=gen, device="cuda").int(), torch.tensor([0, pages, 0], device="cuda")
        self.positions, self.slots = torch.zeros(T, **i32), torch.zeros(T, dtype=torch.int64, device="cuda")
        self.f = np.array([10000.0 ** (-2 * i / D) for i in range(D // 2)])
        self.turns = torch.from_numpy(fq.fq_rope_turns(self.f).view(np.int64)).cuda()
        self.qkv = torch.zeros((T, self.Hq + 2 * H, D), dtype=torch.float16, device="cuda")
        self.wq, self.wk = ((1 + 0.2 * torch.randn(D, generator=gen, device="cuda")).half() for _ in range(2))
        P = torch.eye(D) + 0.05 * torch.randn((D, D), generator=gen, device="cuda").cpu()
        self.Pk = P.half().cuda() if matrix else None
        self.Pq = torch.linalg.inv(P.half().double()).t().contiguous().half().cuda() if matrix else None
        self.q, self.k = (torch.zeros((T, h, D), dtype=torch.float16, device="cuda") for h in (self.Hq, H))
        self.out = torch.full((T, self.Hq, D), -7.25, dtype=torch.float16, device="cuda")
        self.slopes = torch.from_numpy(so.slopes(self.Hq)).cuda()
        self.cache = fq.KvCache(self.kc, self.kp, self.vc, self.vp, pages, page, H, *bits)
        self.batch = fq.KvBatch(self.starts, self.lengths, self.table, B, T, width, width, T, width * page)
        self.pool = fq.PagePool(self.ring, self.state, self.state, pages)
        self.work = torch.empty(fq.fq_cache_attention_workspace(self.cache, self.batch, self.Hq) + 16, dtype=torch.uint8, device="cuda")

    def give(self, keep, rows, qkv):
        self.held.copy_(self.lengths)
        self.keep.copy_(torch.tensor(keep, dtype=torch.int32))
        self.rows.copy_(torch.tensor(rows, dtype=torch.int32))
        self.qkv.copy_(qkv)

    def step(self, stream=None):
        st = stream or torch.cuda.current_stream()
        wide = (self.Hq + 2 * self.H) * D
        q, k, v = self.qkv[:, :self.Hq], self.qkv[:, self.Hq:self.Hq + self.H], self.qkv[:, self.Hq + self.H:]
        fq.flatquant_cache_advance(self.batch, self.pool, self.page, self.pages, self.held, self.keep, self.rows, self.positions, self.slots, stream=st)
        fq.flatquant_head_rope(q, wide, self.Hq, k, wide, self.H, self.T, self.positions, self.turns, D, 0, self.wq, self.wk, 1e-6, self.Pq, None, 0, self.q,
                               self.Hq * D, self.k, self.H * D, stream=st)
        fq.flatquant_cache_write(self.cache, self.batch, self.k, self.H * D, v, wide, self.Pk, None, 1, 0.95, 0.95, stream=st)
        fq.flatquant_cache_scored_attention(self.cache, self.batch, self.q, self.Hq * D, self.Hq, 0.09, self.cap, self.slopes, None, 0, 0, None, self.out, self.Hq * D,
                                            self.work, self.work.numel(), stream=st)

    def all(self):
        return {n: getattr(self, n) for n in ("kc", "kp", "vc", "vp", "starts", "lengths", "table", "ring", "state", "positions", "slots", "q", "k", "out")}


def _plan(seed, B, T, steps, width=320):
    """Kept and new tokens of the steps, as a host scheduler has them: prompts, then decoding with drafts, ends and new prompts."""
    r = np.random.Generator(np.random.PCG64(seed))
    held, plan = [0] * B, []
    for s in range(steps):
        keep, rows, left = list(held), [], T
        for b in range(B):
            what = r.random()
            n = int(r.integers(1, 60)) if held[b] == 0 else 1
            if held[b] and what < 0.15:
                keep[b] = 0
                n = int(r.integers(0, 30))
            elif held[b] and what < 0.35:
                keep[b] -= min(held[b] - 1, int(r.integers(1, 5)))
                n = int(r.integers(1, 6))
            n = min(n, left, width - keep[b])
            left -= n
            rows.append(n)
            held[b] = keep[b] + n
        plan.append((keep, rows))
    return plan


def _inputs(gen, layer):
    return (torch.randn(layer.qkv.shape, generator=gen, device="cuda") * 1.5).half()


def _check(layer, held, keep, rows, table, ring, state, qkv, out_before):
    """Every output of a step against the oracles; returns what the next step starts from."""
    starts, lengths, nxt, positions, slots = so.advance(held, keep, rows, table, layer.width, layer.page, layer.pages, ring, *state, layer.T)
    for name, want in (("starts", starts), ("lengths", lengths), ("table", table), ("ring", ring), ("state", list(nxt)), ("positions", positions), ("slots", slots)):
        assert getattr(layer, name).tolist() == want, name
    n = starts[-1]
    x = qkv.cpu().view(torch.int16).numpy().view(np.float16)
    pos = np.array(positions[:n])
    half = lambda t: t.cpu().view(torch.int16).numpy().view(np.float16)       # noqa: E731
    for got, rows_, w, P in ((layer.q, x[:n, :layer.Hq], layer.wq, layer.Pq), (layer.k, x[:n, layer.Hq:layer.Hq + layer.H], layer.wk, None)):
        want, tol = so.rope64(rows_, half(w), 1e-6, pos, layer.f, False, None if P is None else half(P)[None])
        assert np.all(np.abs(half(got)[:n] - want) <= tol)
    # attention over what the pages hold
    c = Batch.__new__(Batch)
    c.rows, c.lengths, c.H, c.page, c.B, c.bits = [b - a for a, b in zip(starts, starts[1:])], lengths, layer.H, layer.page, layer.B, layer.bits
    c.starts, c.T, c.width, c.pages, c.table = np.array(starts), layer.T, layer.width, layer.pages, np.array(table)
    c.host = [co.Pages(layer.pages, layer.H, layer.page, b) for b in layer.bits]
    for x, codes, params in zip(c.host, (layer.kc, layer.vc), (layer.kp, layer.vp)):
        x.codes, x.params = codes.cpu().numpy(), params.cpu().numpy().view(np.uint32)
    want, tol = expect(c, half(layer.q), layer.Hq // layer.H, 0.09, cap=layer.cap, slopes=layer.slopes.tolist(), heads=[0, layer.Hq - 1])
    looked = ~np.isnan(want)
    assert (np.abs(half(layer.out).astype(np.float64) - want)[looked] <= tol[looked]).all()
    assert torch.equal(layer.out[n:], out_before[n:])                          # rows behind the last sequence
    # and the pages hold the rows: values without a matrix bit by bit
    v = qkv.cpu().view(torch.int16).numpy().view(np.float16)[:n, layer.Hq + layer.H:]
    qv, sv, zv = co.grid32(v, 0.95, layer.bits[1])
    for t, slot in enumerate(slots[:n]):
        p, s = divmod(slot, layer.page)
        assert np.array_equal(c.host[1].codes[p, :, s], co.pack(qv[t], layer.bits[1])) and np.array_equal(c.host[1].params[p, :, s], co.parameters(sv[t], zv[t]))
    return lengths, nxt[:2]


@pytest.mark.parametrize("matrix", [False, True])
def test_steps_of_a_serving_loop(matrix):
    print(f"[case] loop matrix={matrix}", flush=True)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    layer = Layer(1, 6, 200, matrix=matrix)
    table, ring, state, held = layer.table.tolist(), layer.ring.tolist(), (0, layer.pages), [0] * layer.B
    for keep, rows in _plan(2, layer.B, layer.T, 8):
        x = _inputs(gen, layer)
        layer.give(keep, rows, x)
        before = layer.out.clone()
        layer.step()
        torch.cuda.synchronize()
        held, state = _check(layer, held, keep, rows, table, ring, state, x, before)


def test_a_captured_step_is_the_eager_one():
    """Replayed with other inputs every time, the program's own work and synchronizations between: every byte that the eager step leaves."""
    print("[case] captured", flush=True)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    eager, graphed = Layer(3, 8, 64), Layer(3, 8, 64)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graphed.step(side)                                                     # (no rows: nothing is held)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step()
    eager.step()
    for keep, rows in _plan(4, 8, 64, 12):
        x = _inputs(gen, eager)
        for layer in (eager, graphed):
            layer.give(keep, rows, x)
        eager.step()
        graph.replay()
        torch.cuda.synchronize()
        a, b = eager.all(), graphed.all()
        for name in a:
            assert torch.equal(a[name], b[name]), name


def test_two_graphs_and_two_streams_keep_to_their_own():
    """Two layers' captured steps, replayed side by side on streams of their own."""
    print("[case] two graphs", flush=True)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    alone, together = [Layer(s, 5, 40, cap=c) for s, c in ((8, 20.0), (9, 0.0))], [Layer(s, 5, 40, cap=c) for s, c in ((8, 20.0), (9, 0.0))]
    streams, graphs = [torch.cuda.Stream() for _ in together], []
    for layer, st in zip(together, streams):
        with torch.cuda.stream(st):
            layer.step(st)
        st.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            layer.step(st)
        graphs.append(g)
    for layer in alone:
        layer.step()
    for keep, rows in _plan(10, 5, 40, 6):
        x = _inputs(gen, alone[0])
        for layer in alone + together:
            layer.give(keep, rows, x)
        torch.cuda.synchronize()
        for layer in alone:
            layer.step()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for a, b in zip(alone, together):
            x, y = a.all(), b.all()
            for name in x:
                assert torch.equal(x[name], y[name]), name


def test_two_threads_at_once():
    print("[case] threads", flush=True)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)
    plan = _plan(12, 5, 40, 6)
    inputs = [_inputs(gen, Layer(0, 1, 40)) for _ in plan]
    alone, wrong = Layer(13, 5, 40), []

    def loop(layer, st):
        try:
            with torch.cuda.stream(st):
                for (keep, rows), x in zip(plan, inputs):
                    layer.give(keep, rows, x)
                    layer.step(st)
            st.synchronize()
        except Exception as e:                                                 # noqa: BLE001
            wrong.append(e)
    torch.cuda.synchronize()
    loop(alone, torch.cuda.current_stream())
    layers = [Layer(13, 5, 40) for _ in range(3)]
    torch.cuda.synchronize()
    threads = [threading.Thread(target=loop, args=(layer, torch.cuda.Stream())) for layer in layers]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong, wrong
    for layer in layers:
        a, b = alone.all(), layer.all()
        assert all(torch.equal(a[n], b[n]) for n in a)


def test_a_draft_and_its_verification():
    """A tree of drafted tokens, scored with a cap; of them some are kept: the table gives the others' pages back and the next step goes on."""
    print("[case] draft", flush=True)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(14)
    layer = Layer(15, 3, 120, matrix=False)
    x = _inputs(gen, layer)
    layer.give([0] * 3, [40, 17, 33], x)
    layer.step()
    layer.give([40, 17, 33], [20, 20, 20], x)
    layer.step()
    r = np.random.default_rng(16)
    masks = torch.from_numpy(r.integers(0, 2 ** 20, layer.T).astype(np.int64) | 1).cuda()
    tree = fq.KvBatch(layer.starts, layer.lengths, layer.table, 3, layer.T, layer.width, layer.width, 20, layer.width * layer.page)
    work = torch.empty(fq.fq_cache_attention_workspace(layer.cache, tree, layer.Hq) + 16, dtype=torch.uint8, device="cuda")
    fq.flatquant_cache_scored_attention(layer.cache, tree, layer.q, layer.Hq * D, layer.Hq, 0.09, 20.0, None, None, 0, 0, masks, layer.out, layer.Hq * D, work, work.numel(),
                                        stream=torch.cuda.current_stream())
    free = int(layer.state[1] - layer.state[0])
    layer.give([43, 17, 52], [1, 1, 1], x)
    layer.step()
    torch.cuda.synchronize()
    assert layer.lengths.tolist() == [44, 18, 53] and layer.positions[:3].tolist() == [43, 17, 52]
    held = [-(-n // 16) for n in (60, 37, 53)]
    assert int(layer.state[1] - layer.state[0]) == free + sum(held) - sum(-(-n // 16) for n in (44, 18, 53))
    assert torch.isfinite(layer.out[:3].float()).all()
