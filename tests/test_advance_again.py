"""A step whose ring ran short is made again (flatquant_cache_advance): whatever the steps before did, every page is in one place, the ring's free part or one row of a table."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as so
from paper_2410_09426_amd import binding as fq

PAGE, WIDTH = 16, 12


class Pool:
    """Two batches on one ring: B sequences of a step that lacks `missing` pages, and one more that has as many."""

    def __init__(self, B, missing, seed=0):
        r = np.random.Generator(np.random.PCG64(seed))
        # the last ones shrink, end, or end with a chunk of a new sequence in their place; the others need two or three pages more
        self.held, self.keep, self.rows = [100] * B, [100] * (B - 3) + [0, 20, 0], [40 - b % 9 for b in range(B - 3)] + [0, 3, 9]
        self.length = [k + n for k, n in zip(self.keep, self.rows)]
        have, need = ([-(-x // PAGE) for x in y] for y in (self.held, self.length))
        wanted = sum(max(0, n - h) for n, h in zip(need, have))
        self.pages = sum(have) + wanted
        order = [int(p) for p in r.permutation(self.pages)]
        take = lambda n: [order.pop() for _ in range(n)]                       # noqa: E731
        self.table = [take(n) + [-7] * (WIDTH - n) for n in have]
        self.other = take(missing) + [-7] * (WIDTH - missing)
        self.table[-1][2] = -1                                                 # an entry that is no page (the one that was there is nowhere)
        self.ring = take(wanted - missing) + [-3] * (self.pages - wanted + missing)
        self.taken, self.given = 3 * self.pages, 3 * self.pages + wanted - missing
        self.T = sum(self.rows) + 5
        self.missing, self.B = missing, B

    def places(self, table, lengths, other, ring, state):
        """Pages in the ring's free part and in the rows of the tables, as far as their sequences go."""
        free = [ring[i % len(ring)] for i in range(state[0], state[1])]
        return free + [p for row, n in zip(table, lengths) for p in row[:-(-n // PAGE)] if p >= 0] + other


@pytest.mark.parametrize("B,missing", [(4, 1), (4, 2), (30, 5), (1100, 1), (1100, 11)])
def test_the_rule_itself(B, missing):
    p = Pool(B, missing)
    before = sorted(p.places(p.table, p.held, p.other[:missing], p.ring, (p.taken, p.given)))
    assert len(set(before)) == len(before) == p.pages - 1
    table, ring = [list(x) for x in p.table], list(p.ring)
    step = lambda taken, given: so.advance(p.held, p.keep, p.rows, table, WIDTH, PAGE, p.pages, ring, taken, given, p.T)      # noqa: E731
    short = step(p.taken, p.given)
    assert short[2][2] == missing and short[2][0] == p.taken
    again = step(*short[2][:2])                                                # nobody gave anything back, but for the step itself
    assert sorted(p.places(table, again[1] if again[2][2] == 0 else p.held, p.other[:missing], ring, again[2])) == before
    table, ring = [list(x) for x in p.table], list(p.ring)
    short, other = step(p.taken, p.given), [list(p.other)]
    ended = so.advance([missing * PAGE], [0], [0], other, WIDTH, PAGE, p.pages, ring, *short[2][:2], 0)
    again = step(*ended[2][:2])
    assert again[2][2] == 0 and again[:2] == short[:2] and -1 not in again[4][:again[0][-1]]
    assert sorted(p.places(table, again[1], [], ring, again[2])) == before


@pytest.mark.gpu
@pytest.mark.parametrize("replayed", [False, True])
@pytest.mark.parametrize("B,missing", [(4, 1), (4, 2), (30, 5), (1100, 1), (1100, 11)])
def test_the_same_step_again(B, missing, replayed):
    """A short step, pages given back by another batch's call, the same step: eagerly, or the second time as a replay of the first; the state in place."""
    print(f"[case] again B={B} missing={missing} replayed={replayed}", flush=True)
    p = Pool(B, missing, seed=B)
    before = sorted(p.places(p.table, p.held, p.other[:missing], p.ring, (p.taken, p.given)))
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")          # noqa: E731
    i32 = dict(dtype=torch.int32, device="cuda")
    table, other, ring, state = dev(p.table), dev([p.other]), dev(p.ring), torch.tensor([p.taken, p.given, 0], device="cuda")
    held, keep, rows = dev(p.held), dev(p.keep), dev(p.rows)
    starts, lengths, positions, slots = torch.zeros(B + 1, **i32), torch.zeros(B, **i32), torch.zeros(p.T, **i32), torch.zeros(p.T, dtype=torch.int64, device="cuda")
    pool = fq.PagePool(ring, state, state, p.pages)
    batch = fq.KvBatch(starts, lengths, table, B, p.T, WIDTH, WIDTH, max(p.rows), max(p.length))
    call = lambda: fq.flatquant_cache_advance(batch, pool, PAGE, p.pages, held, keep, rows, positions, slots, stream=torch.cuda.current_stream())      # noqa: E731
    if replayed:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        call = graph.replay
    want = [list(x) for x in p.table], [list(p.other)], list(p.ring)
    step = lambda s: so.advance(p.held, p.keep, p.rows, want[0], WIDTH, PAGE, p.pages, want[2], *s[:2], p.T)      # noqa: E731
    same = lambda s: ((state.tolist(), table.tolist(), ring.tolist(), starts.tolist(), lengths.tolist(), positions.tolist(), slots.tolist()) ==      # noqa: E731
                      (list(s[2]), want[0], want[2], *s[:2], *s[3:]))
    call()
    torch.cuda.synchronize()
    short = step((p.taken, p.given))
    assert short[2][2] == missing and same(short)
    one, none = [torch.zeros(n, **i32) for n in (2, 1)], torch.zeros(1, **i32)
    fq.flatquant_cache_advance(fq.KvBatch(*one, other, 1, 0, WIDTH, WIDTH, 0, 0), pool, PAGE, p.pages, dev([missing * PAGE]), none, none, None, None,
                               stream=torch.cuda.current_stream())
    ended = so.advance([missing * PAGE], [0], [0], want[1], WIDTH, PAGE, p.pages, want[2], *short[2][:2], 0)
    call()
    torch.cuda.synchronize()
    again = step(ended[2])
    assert again[2][2] == 0 and same(again) and int((slots < 0).sum()) == 5
    assert sorted(p.places(table.tolist(), lengths.tolist(), [], ring.tolist(), state.tolist())) == before
