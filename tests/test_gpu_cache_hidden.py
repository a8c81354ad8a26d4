"""What lies in places of the paged key/value cache that no row sees, whatever it is, does not change attention: infinities and NaN of both signs
as steps, zero points that are none."""
import numpy as np
import pytest

from cache_util import Batch, check_attention, run_attention

STEPS = (0x7C00, 0xFC00, 0x7E00, 0xFFFF)      # +infinity, -infinity, NaN of both signs


def poisoned(seed, rows, lengths, H, page, bits, window=0, sinks=0, masks_of=None):
    """A batch with STEPS wherever no row sees a token: pages of nobody, what lies behind the lengths, tokens before all windows, drafted tokens that
    nobody sees, and all of page 0, which is read in the place of pages that are none (the sequence that had it has none there)."""
    c = Batch(seed, rows, lengths, H, page, *bits)
    c.table[:, :c.width][c.table[:, :c.width] == 0] = -1
    masks = None if masks_of is None else masks_of(c)
    seen = np.zeros((c.pages, page), dtype=bool)
    for b in range(c.B):
        for j in np.flatnonzero(c.visible(b, window, sinks, masks).any(0)):
            seen[c.host[0].place(c.table[b, :c.width], int(j))] = True
    p, s = np.nonzero(~seen)
    for x in c.host:
        x.codes[p, :, s] = 0xFF
        x.params[p, :, s] = (0xFFFF0000 | np.resize(np.array(STEPS, dtype=np.uint32), len(p)))[:, None]
    return c, masks


def few_see(c):
    """Bits of the row itself and of the first; nobody but the first rows sees drafted token 2."""
    masks = np.zeros(c.T, dtype=np.uint64)
    for b in range(c.B):
        for i in range(c.rows[b]):
            masks[c.starts[b] + i] = 1 | (1 << i if i != 2 else 0)
    return masks


def test_the_hidden_steps_are_no_numbers():
    bits = np.array(STEPS, dtype=np.uint16).view(np.float16)
    assert not np.isfinite(bits).any() and np.isposinf(bits[0]) and np.isneginf(bits[1]) and np.isnan(bits[2:]).all()
    c, _ = poisoned(1, (1, 3), (20, 70), 2, 16, (4, 3), window=30)
    for x in c.host:
        steps = (x.params & 0xFFFF).astype(np.uint16).view(np.float16)
        assert not np.isfinite(steps[0]).any() and np.isneginf(steps).any()
        at = x.place(c.table[1, :c.width], 3)                 # before every window
        assert at is None or not np.isfinite(steps[at[0], :, at[1]]).any()


CASES = [  # rows, lengths, H, G
    ((1, 1), (45, 300), 2, 4),
    ((5, 3), (45, 300), 2, 5),
    ((60, 7), (77, 300), 2, 2),
    ((300, 64), (300, 500), 1, 4),
]
LAUNCHES = {"chosen": {}, "balanced": {"FLATQUANT_ATT_WAVES": 0, "FLATQUANT_ATT_CHUNK": 128}, "4 waves": {"FLATQUANT_ATT_WAVES": 4},
            "8 waves": {"FLATQUANT_ATT_WAVES": 8}, "16 waves": {"FLATQUANT_ATT_WAVES": 16}}


@pytest.mark.gpu
@pytest.mark.parametrize("launch", LAUNCHES)
@pytest.mark.parametrize("bits", [(4, 4), (3, 2), (2, 3)])
@pytest.mark.parametrize("rows,lengths,H,G", CASES)
def test_hidden_places_change_nothing(rows, lengths, H, G, bits, launch, tuning):
    for name, value in LAUNCHES[launch].items():
        tuning(name, value)
    print(f"[case] hidden places, {rows} of {lengths}, {H} x {G} heads, {bits} bits, {launch}", flush=True)
    for how in ({}, {"window": 20, "sinks": 3}):
        c, _ = poisoned(sum(lengths), rows, lengths, H, 16, bits, **how)
        c.upload()
        q = c.row_tensor(H * G)
        check_attention(c, q, G, 0.09, run_attention(c, q, G, 0.09, **how), **how)
    if max(rows) <= 64:
        c, masks = poisoned(sum(lengths), rows, lengths, H, 16, bits, masks_of=few_see)
        c.upload()
        q = c.row_tensor(H * G)
        check_attention(c, q, G, 0.09, run_attention(c, q, G, 0.09, masks=masks), masks=masks)
