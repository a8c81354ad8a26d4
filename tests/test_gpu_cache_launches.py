"""Attention over the paged key/value cache on many (sequence, head) pairs, where the choice of the launch changes: some pairs against fp64, all rows written."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2410_09426_amd import binding as fq
from cache_util import D, Batch, run_attention
from test_cache_plan import plan

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,rows,length,H,G,waves,spread,window", [
    (8, 40, 1400, 32, 1, 4, True, 0),             # 33 to 64 rows of more than 256 pairs: four waves that share their tokens, two stretches
    (33, 13, 3100, 8, 4, 4, True, 0),
    (8, 90, 1500, 32, 1, 8, False, 0),            # a workgroup of eight waves for each CU
    (8, 150, 3200, 32, 1, 8, False, 0),
    (8, 280, 3200, 32, 1, 4, False, 0),           # a tile of eight waves would be mostly idle
    (9, 20, 8000, 32, 1, 4, True, 0),             # 17 to 32 rows, balanced, more than one pair a CU
    (16, 5, 4200, 8, 4, 4, True, 0),
    (16, 5, 4200, 8, 4, 4, True, 2500),
    (20, 1, 4000, 32, 1, 8, False, 0),            # more than 512 pairs, eight waves
    (70, 1, 4000, 8, 2, 8, False, 3700),
])
def test_launches_of_many_pairs(B, rows, length, H, G, waves, spread, window):
    """`spread`: with a workspace, the balanced launch or splits."""
    p = plan(B, rows, length, H, G)
    assert p.waves == waves and (p.workspace > 0) == spread
    print(f"[case] {B} x {rows} rows of {length} tokens, {H} x {G} heads, window {window}", flush=True)
    r = np.random.Generator(np.random.PCG64(B + rows))
    lengths = [length] + [int(n) for n in r.integers(length // 3, length, B - 1)]
    c = Batch(85, lengths, lengths, H, 64, 4, 3, filled=False).upload()
    gen = torch.Generator("cuda").manual_seed(rows)
    k, v = (torch.randn((c.T, H * D), device="cuda", generator=gen).half() for _ in range(2))
    fq.flatquant_cache_write(c.cache(), c.batch(), k, H * D, v, H * D, None, None, 1, 0.95, 0.95, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    for name, x in zip("kv", c.host):
        x.codes[:], x.params[:] = c.d[name + "c"].cpu().numpy(), c.d[name + "p"].cpu().numpy().view(np.uint32)
    c.rows = [rows] * B
    c.starts = np.arange(B + 1, dtype=np.int32) * rows
    c.T = B * rows
    c.d["starts"] = torch.from_numpy(c.starts).cuda()
    q = c.row_tensor(H * G)
    got = run_attention(c, q, G, 0.09, window, 2 if window else 0).astype(np.float64)
    assert np.isfinite(got).all() and not np.all(got == -7.25, axis=-1).any()
    for b, h in ((0, 0), (0, H - 1), (B - 1, H // 2), (B // 2, 1)):
        L = lengths[b]
        seen = c.visible(b, window, 2 if window else 0)
        head = [co.Pages(c.pages, 1, 64, x.bits) for x in c.host]
        for one, x in zip(head, c.host):
            one.codes[:], one.params[:] = x.codes[:, h:h + 1], x.params[:, h:h + 1]
        table = c.table[b, :c.width]
        kk, vv = (x.values(table, np.arange(L))[0] for x in head)
        ks, vs = (x.steps(table, np.arange(L))[0] for x in head)
        t = slice(c.starts[b], c.starts[b + 1])
        for g in range(G):
            y = q[t, (h * G + g) * D:(h * G + g + 1) * D]
            o, *size = co.attention64(y, kk, vv, seen, 0.09, ks, vs, 4)
            assert np.all(np.abs(got[t, h * G + g] - o) <= co.attention_bound(o, *size, L, 3)), (b, h, g)
