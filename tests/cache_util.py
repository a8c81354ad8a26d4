"""Batches on a paged cache for the tests: built on the host by the oracle, copied to the device, and their calls."""
import numpy as np
import torch

from oracle import cache_oracle as co
from paper_2410_09426_amd import binding as fq

D = 128


class Batch:
    """rows, lengths: per sequence.  Pages in a shuffled order among spare ones; whatever no token was written to holds NaN steps."""

    def __init__(self, seed, rows, lengths, H, page=16, k_bits=4, v_bits=4, pad=0, extra_width=1, stride_pad=3, filled=True, k_gain=1.0, v_gain=1.0,
                 no_page=()):
        r = self.r = np.random.Generator(np.random.PCG64(seed))
        self.rows, self.lengths, self.H, self.page = list(rows), list(lengths), H, page
        self.B, self.bits = len(rows), (k_bits, v_bits)
        self.starts = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.T = int(self.starts[-1]) + pad
        need = [max(0, -(-n // page)) for n in lengths]
        self.width = max(need + [0]) + extra_width
        self.pages = sum(need) + 2
        order = r.permutation(self.pages)
        self.table = np.full((self.B, self.width + stride_pad), -1, dtype=np.int32)
        self.table[:, self.width:] = 0x7FFFFFF                     # behind the width: not to be read
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        for b, j in no_page:                                       # pages that are none
            self.table[b, j] = (-1, self.pages, -2 ** 31, 2 ** 31 - 1)[(b + j) % 4]
        self.host = [co.Pages(self.pages, H, page, bits) for bits in self.bits]
        if filled:
            for x, gain in zip(self.host, (k_gain, v_gain)):
                for b, n in enumerate(lengths):
                    for j in range(need[b]):
                        p = int(self.table[b, j])
                        if not 0 <= p < self.pages:
                            continue
                        m = min(page, n - j * page)
                        y = (r.standard_normal((H, m, D)) * gain).astype(np.float16)
                        q, s, z = co.grid32(y, 0.95, x.bits)
                        x.codes[p, :, :m] = co.pack(q, x.bits)
                        x.params[p, :, :m] = co.parameters(s, z)

    def upload(self):
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()      # noqa: E731
        self.d = {"starts": dev(self.starts), "lengths": dev(np.asarray(self.lengths, dtype=np.int32)), "table": dev(self.table)}
        for name, x in zip("kv", self.host):
            self.d[name + "c"], self.d[name + "p"] = dev(x.codes), dev(x.params.view(np.int32))
        return self

    def cache(self):
        d = self.d
        return fq.KvCache(d["kc"], d["kp"], d["vc"], d["vp"], self.pages, self.page, self.H, *self.bits)

    def batch(self, max_rows=None, max_length=None):
        d = self.d
        return fq.KvBatch(d["starts"], d["lengths"], d["table"], self.B, self.T, self.width, self.table.shape[1],
                          max(self.rows + [0]) if max_rows is None else max_rows, max([0] + self.lengths) if max_length is None else max_length)

    def row_tensor(self, heads, pad=0, gain=1.0):
        """[T, heads, 128] fp16 in rows of heads * 128 + pad halves."""
        x = (self.r.standard_normal((self.T, heads * D + pad)) * gain).astype(np.float16)
        return x

    def visible(self, b, window=0, sinks=0, masks=None):
        """[rows, tokens] of sequence b."""
        n, L = self.rows[b], max(0, self.lengths[b])
        j = np.arange(L)
        pos = self.lengths[b] - n + np.arange(n)
        if masks is None:
            seen = j[None] <= pos[:, None]
            if window:
                seen &= (j[None] > pos[:, None] - window) | (j[None] < sinks)
        else:
            bit = j - (self.lengths[b] - n)
            m = np.asarray(masks[self.starts[b]:self.starts[b] + n], dtype=np.uint64)
            seen = (bit[None] < 0) | ((bit[None] >= 0) & (bit[None] < 64) & ((m[:, None] >> np.clip(bit, 0, 63).astype(np.uint64)) & np.uint64(1)).astype(bool))
        held = np.array([self.host[0].place(self.table[b, :self.width], int(t)) is not None for t in j], dtype=bool)
        return seen & held[None]

    def attention(self, q, G, scale, window=0, sinks=0, masks=None):
        """(out, bound) fp64 [T, H G, 128] of q [T, H G, 128]; NaN for the rows of no sequence."""
        out = np.full((self.T, self.H * G, D), np.nan)
        tol = np.zeros_like(out)
        for b in range(self.B):
            if self.rows[b] == 0:
                continue
            L = max(0, self.lengths[b])
            k, v = (np.nan_to_num(x.values(self.table[b, :self.width], np.arange(L))) for x in self.host)
            ks, vs = (np.nan_to_num(x.steps(self.table[b, :self.width], np.arange(L))) for x in self.host)
            seen = self.visible(b, window, sinks, masks)
            t = slice(self.starts[b], self.starts[b + 1])
            for h in range(self.H * G):
                o, *size = co.attention64(q[t, h], k[h // G], v[h // G], seen, scale, ks[h // G], vs[h // G], self.bits[0])
                out[t, h], tol[t, h] = o, co.attention_bound(o, *size, L, self.bits[1])
        return out, tol


def run_attention(c, q, G, scale, window=0, sinks=0, masks=None, pad=0, batch=None, workspace=None, stream=None):
    """q: numpy [T, H G 128 + pad]; returns fp16 [T, H G, 128].  The output's padding and the rows of no sequence keep what they held."""
    st = stream or torch.cuda.current_stream()
    cache, batch = c.cache(), batch or c.batch()
    Hq = c.H * G
    dq = torch.from_numpy(q.view(np.uint16).copy()).view(torch.float16).cuda()
    out = torch.full((c.T, Hq * D + pad), -7.25, dtype=torch.float16, device="cuda")
    size = fq.fq_cache_attention_workspace(cache, batch, Hq)
    guard = 256
    work = torch.full((size + guard,), 0xFF, dtype=torch.uint8, device="cuda") if workspace is None else workspace      # NaNs
    if masks is None:
        fq.flatquant_cache_attention(cache, batch, dq, q.shape[1], Hq, scale, window, sinks, out, Hq * D + pad, work, size, stream=st)
    else:
        dm = torch.from_numpy(np.asarray(masks, dtype=np.uint64).view(np.int64)).cuda()
        fq.flatquant_cache_tree_attention(cache, batch, dq, q.shape[1], Hq, scale, dm, out, Hq * D + pad, work, size, stream=st)
    torch.cuda.synchronize()
    if workspace is None:
        assert bool((work[size:] == 0xFF).all()), "written behind the workspace"
    got = out.cpu().view(torch.int16).numpy().view(np.float16)
    assert np.all(got[:, Hq * D:] == np.float16(-7.25)), "padding of the rows overwritten"
    assert np.all(got[c.starts[-1]:] == np.float16(-7.25)), "rows behind the last sequence overwritten"
    return got[:, :Hq * D].reshape(c.T, Hq, D)


def check_attention(c, q, G, scale, got, **how):
    pad = q.shape[1] - c.H * G * D
    want, tol = c.attention(q[:, :q.shape[1] - pad].reshape(c.T, c.H * G, D), G, scale, **how)
    n = c.starts[-1]
    err = np.abs(got[:n].astype(np.float64) - want[:n])
    assert np.all(np.isfinite(got[:n])), "not finite"
    worst = float((err / tol[:n]).max()) if n else 0.0
    print(f"[case] worst error {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0, np.unravel_index(int((err / tol[:n]).argmax()), err.shape)
    return want, tol
