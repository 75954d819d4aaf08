"""Appends to the paged window whose row pointers say something odd.  References and tolerances are those of test_gpu_window."""
import numpy as np
import pytest
import torch

import paper_2502_02617_b200 as pq
from test_gpu_window import BF16, DEV, check_append, f64, half_step, make_window
from window_reference import rotate, rows_of

pytestmark = pytest.mark.gpu


def falling_case(ends, n, d, rotary, before, most, seed=4):
    B, hq, hkv = len(ends) - 1, 2, 1
    w = make_window(B, hq, hkv, d, 16, most, frequencies=pq.pq_rotary_frequencies(rotary), seed=seed)
    w.lens.copy_(torch.tensor(before, dtype=torch.int32))
    g = torch.Generator(DEV).manual_seed(7)
    q, k, v = (torch.randn((n, h, d), generator=g, device=DEV).to(BF16) for h in (hq, hkv, hkv))
    return w, q, k, v, torch.tensor(ends, dtype=torch.int32, device=DEV)


def visible(w, lens):
    """Every row that an attention reads, and the pages that belong to no sequence."""
    pool, table = f64(w.pool), w.page_table.cpu().numpy()
    rows = [np.concatenate(rows_of(pool, table, w.page_tokens, b, n)) for b, n in enumerate(lens)]
    free = sorted(set(range(w.n_pages)) - set(table.flatten().tolist()))
    return rows + [pool[free]]


@pytest.mark.parametrize("d,rotary", [(64, 64), (16, 6)])   # rows as 16-byte pieces, and pair by pair
@pytest.mark.parametrize("ends,n", [([0, 60, 30, 5, 60], 60), ([0, 60, -7, 60, 60], 60), ([0, 40, 20, 200, 60], 60), ([-7, 20, 40, 50, 60], 60),
                                    ([0, 3, 1, 4, 4], 4), ([0, 1, 2, 3, 2], 3), ([0, 0, 0, -1, 5], 5)])
def test_no_window_grows_where_the_ends_fall(ends, n, d, rotary):
    """Which rows are a sequence's is then no question with one answer: nothing that an attention could read changes, and the status says so."""
    before = [3, 16, 0, 7]
    w, q, k, v, cu = falling_case(ends, n, d, rotary, before, 128)
    seen = visible(w, before)
    w.append(q, k, v, cu)
    torch.cuda.synchronize()
    assert w.lens.cpu().tolist() == before
    assert w.status.cpu().tolist()[0] != pq.OK
    assert all(np.array_equal(a, b) for a, b in zip(visible(w, before), seen))


@pytest.mark.parametrize("d,rotary", [(64, 64), (16, 6)])
@pytest.mark.parametrize("where", [1, 250, 256, 300, 599])
def test_one_fall_among_many_sequences(where, d, rotary):
    """Seen by every block, whichever sequences its own rows belong to."""
    B = 600
    ends = np.minimum(2 * np.arange(B + 1), 1100)
    ends[where] = ends[where - 1] - 1 if where > 1 else -1
    before = (np.arange(B) % 20).tolist()
    w, q, k, v, cu = falling_case(ends.tolist(), 1100, d, rotary, before, 40)
    seen = visible(w, before)
    w.append(q, k, v, cu)
    torch.cuda.synchronize()
    assert w.lens.cpu().tolist() == before
    assert w.status.cpu().tolist()[0] != pq.OK
    assert all(np.array_equal(a, b) for a, b in zip(visible(w, before), seen))


@pytest.mark.parametrize("d,rotary", [(64, 64), (16, 6)])
def test_rows_before_the_first_sequence_belong_to_none(d, rotary):
    """cu_seqlens that start behind row 0: those rows are reported, the sequences' own rows are written as ever."""
    before, counts = [3, 16, 0, 7], [10, 0, 20, 25]
    ends = (5 + np.concatenate(([0], np.cumsum(counts)))).tolist()
    w, q, k, v, cu = falling_case(ends, 60, d, rotary, before, 128)
    pool = f64(w.pool)
    w.append(q, k, v, cu)
    torch.cuda.synchronize()
    assert w.status.cpu().tolist()[0] == pq.ERR_INVALID_ARG
    check_append(w, counts, None, k[5:], v[5:], cu, None, pool, before)


@pytest.mark.parametrize("d,rotary", [(64, 64), (16, 6)])
def test_an_end_behind_the_rows_refuses_its_sequence_alone(d, rotary):
    before = [3, 16, 0, 7]
    w, q, k, v, cu = falling_case([0, 40, 90, 90, 90], 60, d, rotary, before, 128)
    seen = visible(w, before)
    got = w.append(q, k, v, cu)
    torch.cuda.synchronize()
    assert w.lens.cpu().tolist() == [43, 16, 0, 7] and w.status.cpu().tolist()[0] == pq.ERR_INVALID_ARG
    assert all(np.array_equal(a, b) for a, b in zip(visible(w, before), seen))
    want = rotate(f64(q)[:40], 3 + np.arange(40), f64(w.frequencies), False)
    assert np.all(np.abs(f64(got)[:40] - want) <= 2.0 ** -18 * 5 + half_step(BF16) * np.abs(want))
