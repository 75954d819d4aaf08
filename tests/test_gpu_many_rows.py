"""Calls of as many (query, head) rows as the entry points take.  References and tolerances are those of test_gpu_window and test_gpu_shared_prefix."""
import numpy as np
import pytest
import torch

import paper_2502_02617_b200 as pq
from paper_2502_02617_b200 import synthetic
from parity_utils import to_f64
from test_gpu_shared_prefix import check, decoded, make_cache, reference
from test_gpu_window import BF16, DEV, F32, check_append, f64, fill_windows, half_step, make_window
from window_reference import attention, rows_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,hq,hkv,n_q,dtype", [(64, 64, 8, 16384, BF16), (16, 64, 8, 8300, F32), (16, 8, 8, 66000, BF16)])
def test_more_row_blocks_than_a_grid_has_in_its_second_dimension(d, hq, hkv, n_q, dtype):
    """Row blocks times kv heads beyond 65535; only the last 100 positions see anything."""
    n = 100
    w = make_window(1, hq, hkv, d, 16, 128, dtype, seed=3, fill=float("nan"))
    fill_windows(w, [n])
    q = torch.randn((1, n_q, hq, d), generator=torch.Generator(DEV).manual_seed(5), device=DEV).to(dtype)
    lse = torch.empty((1, n_q, hq), device=DEV)
    out = w.attend(q, lse=lse)
    torch.cuda.synchronize()
    assert w.check_status()[0] == 0
    assert bool((out[0, :-n] == 0).all()) and bool((lse[0, :-n] == -float("inf")).all())
    K, V = rows_of(f64(w.pool), w.page_table.cpu().numpy(), 16, 0, n)
    want, want_lse = attention(f64(q[0, -n:]), K, V, d ** -0.5)
    assert np.all(np.abs(f64(out[0, -n:]) - want) <= 2e-5 + half_step(dtype) * np.abs(want))
    assert np.all(np.abs(f64(lse[0, -n:]) - want_lse) <= 2e-5)


@pytest.mark.parametrize("d,hq,hkv,n_queries", [(16, 64, 8, 65535), (64, 64, 8, 65535)])
def test_as_many_queries_as_are_allowed(d, hq, hkv, n_queries):
    """65535 queries, 64 rows a block: row blocks times kv heads beyond 65535."""
    n, some = 70, 40
    cache = make_cache([n], hq, hkv, d, capacity=128)
    K, V = decoded(cache, 0, n)
    few = synthetic.queries(2, some, hq, d, BF16, DEV)
    q = few.repeat(-(-n_queries // some), 1, 1)[:n_queries].contiguous()
    out = cache.attend_prefix(q)
    torch.cuda.synchronize()
    assert cache.check_status()[0] == 0
    want, _ = reference(to_f64(few), K, V, d ** -0.5)
    check(cache, few, out[:some], want)
    assert torch.equal(out, out[:some].repeat(-(-n_queries // some), 1, 1)[:n_queries])


@pytest.mark.parametrize("kind", ["one", "ragged"])
@pytest.mark.parametrize("hq,hkv,d,dtype", [(64, 8, 128, F32), (96, 24, 128, BF16), (300, 1, 64, BF16)])
def test_appended_rows_of_more_pieces_than_a_block_takes(hq, hkv, d, dtype, kind):
    """A row's 16-byte pieces go to several blocks."""
    assert (hq + 2 * hkv) * d * (4 if dtype == F32 else 2) // 32 > 768
    before, counts = [0, 5, 31], [1, 1, 1] if kind == "one" else [20, 0, 7]
    w = make_window(3, hq, hkv, d, 16, 40, dtype, seed=2, frequencies=pq.pq_rotary_frequencies(d))
    w.lens.copy_(torch.tensor(before, dtype=torch.int32))
    g = torch.Generator(DEV).manual_seed(3)
    q, k, v = (torch.randn((sum(counts), h, d), generator=g, device=DEV).to(dtype) for h in (hq, hkv, hkv))
    cu = None if kind == "one" else torch.tensor(np.concatenate(([0], np.cumsum(counts))), dtype=torch.int32, device=DEV)
    pool = f64(w.pool)
    got = w.append(q, k, v, cu)
    torch.cuda.synchronize()
    assert w.check_status()[0] == 0
    want = check_append(w, counts, q, k, v, cu, None, pool, before)
    assert np.all(np.abs(f64(got) - want) <= 2.0 ** -18 * 5 + half_step(dtype) * np.abs(want))
