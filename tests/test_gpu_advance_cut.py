"""Rows of a step that are many more than the batch holds (flatquant_cache_advance): cut to T, whatever they add up to."""
import numpy as np
import pytest
import torch

from paper_2410_09426_amd import binding as fq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", ["T", "2^31 - 1"])
@pytest.mark.parametrize("B,T", [(4, 2 ** 29), (3, 2 ** 29), (64, 2 ** 25), (64, 2 ** 26), (64, 2 ** 26 + 12345), (1024, 2 ** 21), (1024, 2 ** 29), (1025, 2 ** 21),
                                 (5000, 2 ** 19 + 1), (40000, 2 ** 29), (5000, 100)])
def test_counts_that_add_up_to_any_number(B, T, rows):
    """Every sequence wants all of the batch, or the largest number: the first one gets it, also where the sums pass 2^31; pages for that one alone."""
    print(f"[case] B={B} T={T} rows={rows}", flush=True)
    i32 = dict(dtype=torch.int32, device="cuda")
    width, held = 3, 5
    starts, lengths = torch.full((B + 1,), -9, **i32), torch.full((B,), -9, **i32)
    table, ring, state = torch.full((B, width), -1, **i32), torch.arange(7, **i32), torch.tensor([0, 7, 0], device="cuda")
    table[:, 0] = torch.arange(B, device="cuda") + 7
    want = torch.full((B,), T if rows == "T" else 2 ** 31 - 1, **i32)
    want[::3] = 0
    have = torch.full((B,), held, **i32)
    batch = fq.KvBatch(starts, lengths, table, B, T, width, width, 1, 1)
    fq.flatquant_cache_advance(batch, fq.PagePool(ring, state, state, 7), 16, B + 7, have, have, want, None, None, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    n = np.minimum(want.cpu().numpy().astype(np.int64), 2 ** 31 - 1 - held)
    first = np.minimum(np.concatenate([[0], np.cumsum(n)]), T)
    assert np.array_equal(starts.cpu().numpy(), first)
    assert np.array_equal(lengths.cpu().numpy(), held + np.diff(first))
    need = np.minimum(-(-(held + np.diff(first)) // 16), width)
    pages = np.full((B, width), -1, dtype=np.int64)
    pages[:, 0] = np.arange(B) + 7
    pages[1, 1:need[1]] = np.arange(need[1] - 1)
    assert np.array_equal(table.cpu().numpy(), pages) and state.tolist() == [need[1] - 1, 7, 0]
