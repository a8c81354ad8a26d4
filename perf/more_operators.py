"""What a step of a served model needs between the products and the cached attention, and what is measured of it.

Three operators that run one after the other, on the batch of the paged, quantized key/value cache:
  advance   the tables of the step: from how many tokens every sequence holds, keeps and gets, its pages (taken from and given back to a ring of
            free ones), row starts and lengths, and for every row its position and its place in the pages
  rope      queries and keys, head by head: norm over the 128 channels, rotation by the row's position, for a transformed key cache the
            matrix of the head; one rounding at the end
  score     attention over the cache whose scores are capped by a tanh, lowered by a distance times the head's slope, or seen through a prefix mask

`run` has every operator twice: in plain torch operations, and (own) as calls of the library.  The pages of a layer: codes
u8 [pages, H, page, 128 bits / 8], code d of a group at bits [bits d, bits d + bits) of its bytes read as one little-endian
integer; parameters one 32-bit word per (page, head, token), the fp16 step in the low half and the zero point in the high one;
value = step (code - zero point).
"""
import math
import random

import torch

own = False

D = 128                   # channels of a head, and of a group
CLIP = 0.95               # clipping threshold of the benchmark's cache configuration
EPS = 1e-6


def listed():
    advance = dict(kind="advance")
    rope = dict(kind="rope", rotary=128, interleaved=False, norm=False, matrix=0, packed=False, pad=0)
    score = dict(kind="score", page=64, rows=1, window=0, sinks=0, cap=0.0, slopes=False, prefix=False, tree=False)
    return [
        # a decode step of 64 sequences, a token each: a page for one sequence in 64; nothing but latency
        dict(advance, name="advance_64x1", B=64, page=64, length=4096, chunk=1, change=0.0),
        # continuous batching: 512 places, most of them decode, others have ended, had drafted tokens rejected or start a prompt; small pages
        dict(advance, name="advance_512_mixed", B=512, page=16, length=8192, chunk=512, change=0.3),
        # long prompts enter an empty cache at once: tens of thousands of pages, hundreds of thousands of rows
        dict(advance, name="advance_16x65536", B=16, page=16, length=0, chunk=65536, change=1.0),
        # a decode step of 64 sequences, norms and rotation, four query heads to a key/value head
        dict(rope, name="rope_64", T=64, Hq=32, H=8, norm=True, far=8192),
        # a long prefill, queries and keys where the fused product left them, rotation alone
        dict(rope, name="rope_16384", T=16384, Hq=32, H=8, packed=True, far=2048),
        # a quarter of the channels rotated, as neighbours, a ragged batch far into long documents, key/value heads not shared
        dict(rope, name="rope_777_quarter", T=777, Hq=32, H=32, rotary=32, interleaved=True, far=1000000, pad=7),
        # queries that go to a transformed key cache: norm, rotation and the inverse transposed matrix of the keys
        dict(rope, name="rope_8192_matrix", T=8192, Hq=32, H=8, norm=True, matrix=1, packed=True, far=4096),
        # 64 ragged sequences decode a token each, capped scores
        dict(score, name="score_64x4096_cap", B=64, length=4096, H=8, G=4, k_bits=4, v_bits=4, cap=50.0),
        # key/value heads not shared, a slope for each head, a wider key than value grid, small pages
        dict(score, name="score_16x6000_slopes", B=16, length=6000, H=32, G=1, k_bits=4, v_bits=2, page=16, slopes=True),
        # verification of small trees of drafted tokens, capped scores
        dict(score, name="score_tree_16x13_cap", B=16, rows=13, length=3000, H=8, G=4, k_bits=4, v_bits=4, cap=30.0, tree=True),
        # a chunk of a long prompt, capped scores, the earlier chunks already in the cache
        dict(score, name="score_2048_of_8192_cap", B=1, rows=2048, length=8192, H=8, G=8, k_bits=4, v_bits=4, cap=50.0),
        # several ragged prompts from their first token, whose first part is seen by all of their rows
        dict(score, name="score_6x777_prefix", B=6, rows=777, length=777, H=32, G=1, k_bits=4, v_bits=4, page=16, prefix=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("advance", "rope", "rope", "score", "score", "score"))
    if kind == "advance":
        c = dict(kind=kind, B=_log_uniform(rng, 1, 2048), page=rng.choice((16, 32, 64, 256)), change=rng.choice((0.0, 0.3, 1.0)))
        c["length"] = rng.choice((0, _log_uniform(rng, 1, 2000000 // c["B"])))
        c["chunk"] = _log_uniform(rng, 1, 1000000 // c["B"])
        return c
    if kind == "rope":
        c = dict(kind=kind, norm=rng.random() < 0.5, matrix=rng.choice((0, 0, 1, 2)), packed=rng.random() < 0.5, interleaved=rng.random() < 0.3)
        c["Hq"], c["H"] = rng.choice(((32, 8), (64, 8), (32, 32), (28, 4), (5, 1), (1, 1)))
        c["T"] = _log_uniform(rng, 1, 600000 // (c["Hq"] + c["H"]))
        return dict(c, rotary=rng.choice((32, 64, 96, 128, 128)), far=_log_uniform(rng, c["T"], 4000000), pad=rng.choice((0, 0, rng.randint(0, c["T"] - 1))))
    c = dict(kind=kind, page=rng.choice((16, 32, 64, 128)), k_bits=rng.choice((4, 4, 4, 3, 2)), v_bits=rng.choice((4, 4, 3, 2)))
    c["H"], c["G"] = rng.choice(((8, 4), (8, 8), (32, 1), (4, 7), (8, 5), (2, 16), (1, 1), (16, 2)))
    c["B"] = _log_uniform(rng, 1, 64)
    c["length"] = _log_uniform(rng, 1, 1048576 // (c["B"] * c["H"]))
    c["cap"] = rng.choice((0.0, 20.0, 50.0, rng.uniform(5.0, 100.0)))
    c.update(window=0, sinks=0, slopes=False, prefix=False, tree=rng.random() < 0.25)
    if c["tree"]:
        c["rows"] = min(c["length"], rng.randint(1, 64))
        return c
    most = min(c["length"], 4096, max(1, 500000000 // (c["B"] * c["H"] * c["G"] * c["length"])))     # rows that the chunk case's scores allow
    c["rows"] = 1 if rng.random() < 0.5 else _log_uniform(rng, 1, most)
    c["window"], c["sinks"] = rng.choice(((0, 0), (0, 0), (rng.randint(1, 4096), rng.randint(0, 8))))
    c["slopes"], c["prefix"] = rng.random() < 0.4, rng.random() < 0.4
    return c


def _sizes(case):
    """New tokens and tokens in all of every sequence: ragged, up to what the case says (the first sequence has that)."""
    r = random.Random(case["B"] * 1009 + case["length"])
    rows = [max(1, round(case["rows"] * (1.0 if b == 0 else r.uniform(0.4, 1.0)))) for b in range(case["B"])]
    lengths = [max(n, round(case["length"] * (1.0 if b == 0 else r.uniform(0.4, 1.0)))) for b, n in enumerate(rows)]
    return (rows, rows) if case["rows"] == case["length"] else (rows, lengths)


def _steps(case):
    """Tokens held, kept and new of every sequence of a step (advance)."""
    r = random.Random(case["B"] * 1013 + case["length"] + case["chunk"])
    held, keep, rows = [], [], []
    for b in range(case["B"]):
        h = round(case["length"] * (1.0 if b == 0 else r.uniform(0.1, 1.0)))
        k, n = h, 1
        if b == 0 or r.random() < case["change"]:
            what = 0 if case["length"] == 0 or b == 0 else r.randint(0, 2)
            if what == 0:                                        # a prompt, or its next part
                n = round(case["chunk"] * (1.0 if b == 0 else r.uniform(0.3, 1.0)))
            elif what == 1:                                      # has ended
                k, n = 0, 0
            else:                                                # some of its drafted tokens are kept
                k, n = h - min(h, r.randint(0, 40)), 1
        held.append(h)
        keep.append(k)
        rows.append(n)
    return held, keep, rows


# ---- codes and values

def _quotient(a, b):
    """fp32 a / b, rounded once (a quotient of 32-bit numbers in 64 bits rounds to 32 as the exact one does)."""
    return (a.double() / b).float()


def _quantize(y, bits):
    """Rows [..., 128] to codes (whole numbers), steps (fp16) and zero points, with the operations that define them in 32 bits."""
    top = 2 ** bits - 1
    y = y.float()
    mx, mn = y.amax(-1).clamp(min=0) * CLIP, y.amin(-1).clamp(max=0) * CLIP
    step = _quotient(mx - mn, top).half()
    by = torch.where(step > 0, step, torch.ones_like(step))
    zero = torch.where(step > 0, _quotient(-mn, by.double()).round().clamp(0, top), torch.zeros_like(mn))
    code = (_quotient(y, by.double()[..., None]).round() + zero[..., None]).clamp(0, top)
    return torch.where(step[..., None] > 0, code, torch.zeros_like(code)), step, zero


def _pack(code, bits):
    """Eight codes to `bits` bytes."""
    eight = code.long().unflatten(-1, (D // 8, 8)) << (bits * torch.arange(8, device=code.device))
    return ((eight.sum(-1)[..., None] >> (8 * torch.arange(bits, device=code.device))) & 255).byte().flatten(-2)


def _parameters(step, zero):
    return (step.view(torch.int16).int() & 0xFFFF) | (zero.int() << 16)


def _values(codes, params, bits):
    """Codes and parameters to fp32 values."""
    at = bits * torch.arange(D, device=codes.device)
    lo = at // 8
    hi = (lo + 1).clamp(max=D * bits // 8 - 1)
    two = codes[..., lo].int() | (codes[..., hi].int() << 8)
    code = (two >> (at % 8).int()) & (2 ** bits - 1)
    step = (params & 0xFFFF).to(torch.int16).view(torch.float16).float()
    return step[..., None] * (code - (params >> 16)[..., None]).float()


# ---- inputs

def _heads(gen, n, H):
    """[n, H, 128] fp16 ~ N(0, 1), two channels of every head x 3."""
    gain = torch.ones((H, D), device="cuda")
    gain.scatter_(1, torch.rand((H, D), generator=gen, device="cuda").argsort(1)[:, :2], 3.0)
    x = torch.empty((n, H, D), dtype=torch.float16, device="cuda")
    for r in range(0, n, 8192):
        x[r:r + 8192] = (torch.randn((min(8192, n - r), H, D), generator=gen, device="cuda") * gain).half()
    return x


def _pages(gen, s, case, lengths):
    """Pages in an order of their own, as they come when sequences grow and end.  With a window a sequence has the pages of its first
    tokens, of its prefix and of the window only; what the table says of the others is no page."""
    page, width = s["page"], -(-case["length"] // s["page"])
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)
    held = []
    for b, n in enumerate(lengths):
        first = max(0, n - s["rows_of"][b] - case["window"] + 1) if case["window"] else 0
        for p in range(-(-n // page)):
            if (p + 1) * page > first or p * page < max(case["sinks"], s["prefix_of"][b]):
                held.append((b, p))
    pages = len(held) + 3
    order = torch.randperm(pages, generator=gen, device="cuda")[:len(held)].int().cpu()
    at = torch.tensor(held)
    table[at[:, 0], at[:, 1]] = order
    s["pages"], s["width"], s["table"] = pages, width, table.cuda()
    for x in ("k", "v"):
        bits = s[x + "_bits"]
        s[x + "_codes"] = torch.zeros((pages, s["H"], page, D * bits // 8), dtype=torch.uint8, device="cuda")
        s[x + "_params"] = torch.zeros((pages, s["H"], page), dtype=torch.int32, device="cuda")
        for p in range(0, pages, max(1, 8192 // page)):
            n = min(pages - p, max(1, 8192 // page))
            y = _heads(gen, n * page, s["H"]).unflatten(0, (n, page)).transpose(1, 2)
            code, step, zero = _quantize(y, bits)
            s[x + "_codes"][p:p + n] = _pack(code, bits)
            s[x + "_params"][p:p + n] = _parameters(step, zero)


def _prepare_advance(gen, case, seed):
    held, keep, rows = _steps(case)
    page = case["page"]
    have = [-(-h // page) for h in held]
    need = [-(-(k + n) // page) for k, n in zip(keep, rows)]
    width = max(max(have), max(need)) + 1
    pages = sum(have) + sum(max(0, n - h) for n, h in zip(need, have)) + 5
    order = torch.randperm(pages, generator=gen, device="cuda").int()
    inside = torch.arange(width, device="cuda") < torch.tensor(have, device="cuda")[:, None]
    rank = inside.flatten().cumsum(0).sub(1).clamp(min=0).view_as(inside)
    table = torch.where(inside, order[rank], torch.full_like(rank, -1, dtype=torch.int32))
    taken = random.Random(seed).randint(0, 10 * pages)           # pages that have gone through the ring so far
    ring = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
    free = order[sum(have):]
    ring[(taken + torch.arange(len(free), device="cuda")) % pages] = free
    i32 = dict(dtype=torch.int32, device="cuda")
    T = sum(rows) + 3                                            # three rows of padding
    return dict(kind="advance", page=page, B=case["B"], T=T, width=width, pages=pages, table=table.contiguous(), ring=ring,
                state=torch.tensor([taken, taken + len(free), 0], device="cuda"), next=torch.zeros(3, dtype=torch.int64, device="cuda"),
                held=torch.tensor(held, **i32), keep=torch.tensor(keep, **i32), rows=torch.tensor(rows, **i32), max_rows=max(rows),
                max_length=max(k + n for k, n in zip(keep, rows)), starts=torch.zeros(case["B"] + 1, **i32), lengths=torch.zeros(case["B"], **i32),
                positions=torch.zeros(T, **i32), slots=torch.zeros(T, dtype=torch.int64, device="cuda"))


def _prepare_rope(gen, case, seed):
    T, Hq, H = case["T"], case["Hq"], case["H"]
    s = {k: v for k, v in case.items() if k != "name"}
    r = random.Random(seed)
    pos, left = [], T - case["pad"]
    while left > 0:                                              # sequences one behind the other, each from a position of its own
        n = min(left, r.randint(1, max(1, left)))
        first = r.randint(0, case["far"] - n) if case["far"] > n else 0
        pos += range(first, first + n)
        left -= n
    s["positions"] = torch.tensor(pos + [-1] * case["pad"], dtype=torch.int32, device="cuda")
    s["freq"] = torch.tensor([500000.0 ** (-2 * i / case["rotary"]) for i in range(case["rotary"] // 2)], dtype=torch.float64, device="cuda")
    if case["packed"]:
        rows = _heads(gen, T, Hq + 2 * H)
        s["q"], s["k"], s["q_stride"], s["k_stride"] = rows[:, :Hq], rows[:, Hq:Hq + H], (Hq + 2 * H) * D, (Hq + 2 * H) * D
    else:
        s["q"], s["k"], s["q_stride"], s["k_stride"] = _heads(gen, T, Hq), _heads(gen, T, H), Hq * D, H * D
    for x, heads in (("q", Hq), ("k", H)):
        s["w_" + x] = (1 + 0.2 * torch.randn(D, generator=gen, device="cuda")).half() if case["norm"] else None
        s["P_" + x] = None
        s[x + "_out"] = torch.zeros((T, heads, D), dtype=torch.float16, device="cuda")
    if case["matrix"]:                                           # one for all heads, or one each (and then for the keys too)
        P = torch.eye(D) + 0.05 * torch.randn((Hq + H if case["matrix"] == 2 else 1, D, D), generator=gen, device="cuda").cpu()
        s["P_q"] = torch.linalg.inv(P[:Hq].double()).transpose(1, 2).contiguous().half().cuda()
        s["P_k"] = P[Hq:].half().cuda() if case["matrix"] == 2 else None
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["kind"] == "advance":
        return _prepare_advance(gen, case, seed)
    if case["kind"] == "rope":
        return _prepare_rope(gen, case, seed)
    rows, lengths = _sizes(case)
    r = random.Random(seed)
    s = dict({k: v for k, v in case.items() if k not in ("rows", "length", "name")}, T=sum(rows), max_rows=max(rows), max_length=max(lengths), rows_of=rows)
    s["prefix_of"] = [r.randint(0, n) if case["prefix"] else 0 for n in lengths]
    _pages(gen, s, case, lengths)
    starts = [0]
    for n in rows:
        starts.append(starts[-1] + n)
    s["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    s["prefix"] = torch.tensor(s["prefix_of"], dtype=torch.int32, device="cuda") if case["prefix"] else None
    Hq = s["H"] * s["G"]
    s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / Hq) for h in range(Hq)], device="cuda") if case["slopes"] else None
    s["scale"] = D ** -0.5
    # capped scores come from queries whose products reach the cap
    s["q"] = (torch.randn((s["T"], Hq, D), generator=gen, device="cuda") * (8.0 if case["cap"] else 1.0)).half()
    s["out"] = torch.empty_like(s["q"])
    s["visible"] = None
    if case["tree"]:                       # the tree of a sequence: every drafted token behind the root continues an earlier one
        masks = []
        for n in rows:
            first = len(masks)
            for i in range(n):
                masks.append((masks[first + r.randint(max(0, i - 8), i - 1)] if i else 0) | 1 << i)
        s["visible"] = torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], dtype=torch.int64, device="cuda")
    return s


# ---- the tables of a step

def _advance(s):
    page, pages, T = s["page"], s["pages"], s["T"]
    held = s["held"].long().clamp(min=0)
    keep = torch.minimum(s["keep"].long().clamp(min=0), held)
    starts = torch.cat([held.new_zeros(1), s["rows"].long().clamp(min=0).cumsum(0)]).clamp(max=T)
    n = starts[1:] - starts[:-1]
    length = keep + n
    have, need = (((x + page - 1) // page).clamp(max=s["width"])[:, None] for x in (held, length))
    j = torch.arange(s["width"], device="cuda")
    new = (j >= have) & (j < need)
    gone = (j >= need) & (j < have) & (s["table"] >= 0) & (s["table"] < pages)
    wanted, released = new.sum(), gone.sum()
    taken, given = s["state"][0], s["state"][1]
    enough = wanted <= given - taken
    got = s["ring"][(taken + new.flatten().cumsum(0) - 1).clamp(min=0) % pages].view_as(s["table"])
    back = torch.where(gone.flatten(), (given + gone.flatten().cumsum(0) - 1) % pages, torch.full_like(wanted, pages))
    ring = torch.cat([s["ring"], s["ring"][:1]]).scatter(0, back, s["table"].flatten())
    s["ring"].copy_(ring[:pages])
    s["table"].copy_(torch.where(new, torch.where(enough, got, torch.full_like(got, -1)), s["table"]))
    s["next"].copy_(torch.stack([torch.where(enough, taken + wanted, taken), given + released, torch.where(enough, 0, wanted - (given - taken))]))
    s["starts"].copy_(starts)
    s["lengths"].copy_(length)
    t = torch.arange(T, device="cuda")
    b = torch.bucketize(t, starts[1:], right=True).clamp(max=s["B"] - 1)
    pos = keep[b] + t - starts[b]
    at = s["table"][b, (pos // page).clamp(0, s["width"] - 1)].long()
    row = t < starts[-1]
    s["positions"].copy_(torch.where(row, pos, -1))
    s["slots"].copy_(torch.where(row & (pos // page < s["width"]) & (at >= 0) & (at < pages), at * page + pos % page, -1))


# ---- norm, rotation, matrix

def _rotated(s, x, w):
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()
    r = s["rotary"]
    angle = s["positions"].double()[:, None] * s["freq"]
    c, sn = angle.cos().float()[:, None], angle.sin().float()[:, None]
    z = y.clone()
    if s["interleaved"]:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        z[..., 0:r:2], z[..., 1:r:2] = a * c - b * sn, a * sn + b * c
    else:
        a, b = y[..., :r // 2], y[..., r // 2:r]
        z[..., :r // 2], z[..., r // 2:r] = a * c - b * sn, a * sn + b * c
    return z


def _rope(s):
    token = (s["positions"] >= 0)[:, None, None]
    q, k = _rotated(s, s["q"], s["w_q"]), _rotated(s, s["k"], s["w_k"])
    if s["matrix"] == 1:
        q = q @ s["P_q"][0].float()
    elif s["matrix"] == 2:
        q, k = ((x.transpose(0, 1).contiguous() @ P.float()).transpose(0, 1) for x, P in ((q, s["P_q"]), (k, s["P_k"])))
    s["q_out"].copy_(torch.where(token, q.half(), s["q_out"]))
    s["k_out"].copy_(torch.where(token, k.half(), s["k_out"]))


# ---- attention

def _where(s):
    """Sequence and place among its new tokens of every row."""
    t = torch.arange(s["T"], device="cuda")
    b = torch.bucketize(t, s["starts"][1:].long(), right=True)
    return b, t - s["starts"][b]


def _whole(s, x):
    """Every sequence's values of one tensor, fp32 [B, H, length, 128]."""
    j = torch.arange(s["max_length"], device="cuda")
    p = s["table"][:, j // s["page"]].long().clamp(min=0)                      # [B, length]
    at = (p, slice(None), (j % s["page"]).expand_as(p))
    return _values(s[x + "_codes"][at], s[x + "_params"][at], s[x + "_bits"]).transpose(1, 2).contiguous()


def _attend(s):
    B, H, G, n = s["B"], s["H"], s["G"], s["max_rows"]
    b_of, i_of = _where(s)
    i = torch.arange(n, device="cuda")
    at = (s["starts"][:-1, None] + i).clamp(max=s["T"] - 1).long()             # [B, n]
    q = s["q"][at].float().unflatten(2, (H, G)).permute(0, 2, 1, 3, 4).flatten(2, 3)          # [B, H, n G, 128]
    scores = (q @ _whole(s, "k").transpose(2, 3).contiguous()).unflatten(2, (n, G)) * s["scale"]
    if s["cap"]:
        scores = (scores / s["cap"]).tanh() * s["cap"]
    j = torch.arange(s["max_length"], device="cuda")
    rows = s["starts"][1:] - s["starts"][:-1]
    if s["tree"]:
        before = (s["lengths"] - rows)[:, None, None]
        seen = (j < before) | ((j - before < 64) & (((s["visible"][at][..., None] >> (j - before).clamp(0, 63)) & 1) != 0))
    else:
        pos = ((s["lengths"] - rows)[:, None] + i)[..., None]                  # [B, n, 1]
        if s["slopes"] is not None:
            scores = scores - s["slopes"].view(1, H, 1, G, 1) * (pos - j).abs().float()[:, None, :, None, :]
        seen = j <= pos
        if s["window"]:
            seen = seen & ((j > pos - s["window"]) | (j < s["sinks"]))
        if s["prefix"] is not None:
            seen = seen | (j < s["prefix"][:, None, None])
    seen = (seen & (j < s["lengths"][:, None, None]))[:, None, :, None, :]     # [B, 1, n, 1, length]
    scores = scores.masked_fill(~seen, -math.inf)
    e = (scores - scores.amax(-1, keepdim=True).clamp(min=-3e38)).exp()
    out = (e.flatten(2, 3) @ _whole(s, "v")) / e.sum(-1).flatten(2, 3)[..., None].clamp(min=1e-30)
    out = out.unflatten(2, (n, G)).permute(0, 2, 1, 3, 4).flatten(2, 3).half()                # [B, n, H G, 128]
    s["out"].copy_(out[b_of, i_of])


# ---- a pass

def _outputs(s):
    names = {"advance": ("starts", "lengths", "table", "ring", "next", "positions", "slots"), "rope": ("q_out", "k_out"), "score": ("out",)}
    return {x: s[x] for x in names[s["kind"]]}


def _kept(s):
    """What a program makes once of the library's structs, constants and workspace."""
    from paper_2410_09426_amd import binding as fq
    if s["kind"] == "advance":
        batch = fq.KvBatch(s["starts"], s["lengths"], s["table"], s["B"], s["T"], s["width"], s["width"], s["max_rows"], s["max_length"])
        return fq, batch, fq.PagePool(s["ring"], s["state"], s["next"], s["pages"])
    if s["kind"] == "rope":
        return fq, torch.from_numpy(fq.fq_rope_turns(s["freq"].cpu().numpy()).view("int64")).cuda()
    cache = fq.KvCache(s["k_codes"], s["k_params"], s["v_codes"], s["v_params"], s["pages"], s["page"], s["H"], s["k_bits"], s["v_bits"])
    batch = fq.KvBatch(s["starts"], s["lengths"], s["table"], s["B"], s["T"], s["width"], s["width"], s["max_rows"], s["max_length"])
    return fq, cache, batch, torch.empty(fq.fq_cache_attention_workspace(cache, batch, s["H"] * s["G"]), dtype=torch.uint8, device="cuda")


def run(s):
    kind = s["kind"]
    if own:
        if "kept" not in s:
            s["kept"] = _kept(s)
        stream = torch.cuda.current_stream()
        if kind == "advance":
            fq, batch, pool = s["kept"]
            fq.flatquant_cache_advance(batch, pool, s["page"], s["pages"], s["held"], s["keep"], s["rows"], s["positions"], s["slots"], stream=stream)
        elif kind == "rope":
            fq, turns = s["kept"]
            fq.flatquant_head_rope(s["q"], s["q_stride"], s["Hq"], s["k"], s["k_stride"], s["H"], s["T"], s["positions"], turns, s["rotary"], s["interleaved"],
                                   s["w_q"], s["w_k"], EPS, s["P_q"], s["P_k"], s["matrix"] == 2, s["q_out"], s["Hq"] * D, s["k_out"], s["H"] * D, stream=stream)
        else:
            fq, cache, batch, work = s["kept"]
            row = s["H"] * s["G"] * D
            fq.flatquant_cache_scored_attention(cache, batch, s["q"], row, s["H"] * s["G"], s["scale"], s["cap"], s["slopes"], s["prefix"], s["window"],
                                                s["sinks"], s["visible"], s["out"], row, work, work.numel(), stream=stream)
        return _outputs(s)
    if kind == "advance":
        _advance(s)
    elif kind == "rope":
        _rope(s)
    else:
        _attend(s)
    return _outputs(s)


def _visible_pairs(case, rows, lengths):
    """Pairs of a row and a token that it sees; in a tree every drafted token counts as seeing the earlier half of the others, and a prefix as half of its sequence."""
    pairs = 0
    for n, length in zip(rows, lengths):
        if case["tree"]:
            pairs += n * (length - n) + n * (n + 1) // 2
            continue
        for pos in range(length - n, length):
            w, first = case["window"], max(0, pos - case["window"] + 1) if case["window"] else 0
            seen = pos + 1 - first + (min(case["sinks"], first) if w else 0)
            pairs += max(seen, length // 2) if case["prefix"] else seen
    return pairs


def _tokens_read(case, rows, lengths):
    """Tokens that any row of their sequence sees."""
    total = 0
    for n, length in zip(rows, lengths):
        first = max(0, length - n - case["window"] + 1) if case["window"] else 0
        total += length - first + min(max(case["sinks"], length // 2 if case["prefix"] else 0), first)
    return total


def work(case):
    if case["kind"] == "advance":
        held, keep, rows = _steps(case)
        pages = sum(abs(-(-(k + n) // case["page"]) + -h // case["page"]) for h, k, n in zip(held, keep, rows))
        return {"bytes": 20 * case["B"] + 52 + 8 * pages + 12 * (sum(rows) + 3), "flops": 0}
    if case["kind"] == "rope":
        T, heads = case["T"], case["Hq"] + case["H"]
        matrices, through = ((0, 0), (1, case["Hq"]), (heads, heads))[case["matrix"]]
        live = T - case["pad"]
        return {"bytes": live * heads * 4 * D + 4 * T + matrices * 2 * D * D,
                "flops": live * heads * (3 * case["rotary"] + (4 * D if case["norm"] else 0)) + live * through * 2 * D * D}
    rows, lengths = _sizes(case)
    T, H = sum(rows), case["H"]
    group = D * (case["k_bits"] + case["v_bits"]) // 8 + 8                     # codes and parameters of a token's key and value
    pairs = _visible_pairs(case, rows, lengths)
    return {"bytes": _tokens_read(case, rows, lengths) * H * group + 4 * T * H * case["G"] * D, "flops": 4 * D * H * case["G"] * pairs}


# ---- the definitions in 64 bits

def _rows64(s, x, b, first, last):
    """Tokens first .. last - 1 of sequence b: fp64 [H, tokens, 128], bit by bit."""
    bits, page = s[x + "_bits"], s["page"]
    at = torch.tensor([max(int(n), 0) for n in s["table_host"][b][first // page:-(-last // page)]], device="cuda")
    c, w = s[x + "_codes"][at].transpose(0, 1).flatten(1, 2), s[x + "_params"][at].transpose(0, 1).flatten(1, 2)
    c, w = (a[:, first % page:first % page + last - first] for a in (c, w))
    q = torch.zeros(c.shape[:2] + (D,), dtype=torch.float64, device="cuda")
    for d in range(D):
        for k in range(bits):
            q[..., d] += ((c[..., (bits * d + k) // 8] >> ((bits * d + k) % 8)) & 1).double() * 2.0 ** k
    step = (w % 65536).to(torch.int32).to(torch.int16).view(torch.float16).double()
    return step[..., None] * (q - (w // 65536).double()[..., None])


def _rope64(s, x, heads):
    """Every pair as a complex number, turned."""
    r, out = s["rotary"], torch.zeros((s["T"], heads, D), dtype=torch.float64, device="cuda")
    live = s["T"] - s["pad"]
    for t in range(0, live, 2048):
        u = min(live, t + 2048)
        y = s[x][t:u].double()
        if s["w_" + x] is not None:
            y = y / (y.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt() * s["w_" + x].double()
        pairs = y[..., :r].unflatten(-1, (r // 2, 2)) if s["interleaved"] else y[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2)
        turn = torch.polar(torch.ones((u - t, r // 2), dtype=torch.float64, device="cuda"), s["positions"][t:u].double()[:, None] * s["freq"])
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None])
        y = torch.cat([(z if s["interleaved"] else z.transpose(-1, -2)).flatten(-2), y[..., r:]], -1)
        if s["P_" + x] is not None:
            P = s["P_" + x].double()
            y = torch.stack([y[:, h] @ P[h % len(P)] for h in range(heads)], 1)
        out[t:u] = y
    return out


def exact(case, seed):
    if case["kind"] == "advance":
        return None
    s = prepare(case, seed)
    if case["kind"] == "rope":
        return {"q_out": _rope64(s, "q", s["Hq"]), "k_out": _rope64(s, "k", s["H"])}
    starts, lengths, s["table_host"] = s["starts"].tolist(), s["lengths"].tolist(), s["table"].tolist()
    H, G = s["H"], s["G"]
    out = torch.zeros((s["T"], H * G, D), dtype=torch.float64, device="cuda")
    for b in range(case["B"]):
        r0, r1, L = starts[b], starts[b + 1], lengths[b]
        n = r1 - r0
        j = torch.arange(L, device="cuda")
        pos = torch.arange(L - n, L, device="cuda")[:, None]
        if case["tree"]:
            m = s["visible"][r0:r1, None]
            ok = torch.cat([torch.ones((n, L - n), dtype=torch.bool, device="cuda"), (m >> torch.arange(n, device="cuda")) & 1 == 1], 1)
        else:
            ok = j <= pos
            if case["window"]:
                ok &= (pos - j < case["window"]) | (j < case["sinks"])
            ok |= j < s["prefix_of"][b]
        k, v = _rows64(s, "k", b, 0, L), _rows64(s, "v", b, 0, L)
        for h in range(H):
            for g in range(G):
                x = (s["q"][r0:r1, h * G + g].double() @ k[h].t().contiguous()) * s["scale"]
                if case["cap"]:
                    x = case["cap"] * torch.tanh(x / case["cap"])
                if case["slopes"]:
                    x = x - float(s["slopes"][h * G + g]) * (pos - j).abs()
                out[r0:r1, h * G + g] = torch.where(ok, x, -math.inf).softmax(-1) @ v[h]
    return {"out": out}
