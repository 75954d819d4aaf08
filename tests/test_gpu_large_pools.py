"""Pools and caches beyond 2^32 bytes and elements, and outputs that take their queries' place.  References and tolerances are those of test_gpu_window and
test_gpu_shared_prefix."""
import numpy as np
import pytest
import torch

import paper_2502_02617_b200 as pq
from paper_2502_02617_b200 import synthetic
from parity_utils import to_f64
from test_gpu_shared_prefix import check, decoded, fill_window, make_cache, reference
from test_gpu_window import BF16, DEV, F32, f64, half_step
from window_reference import attention, rotate

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,hq,hkv,P,dtype,n_q,rotary", [(128, 16, 8, 256, BF16, 1, 128), (128, 16, 8, 256, BF16, 9, 6), (64, 8, 8, 512, F32, 3, 64)])
def test_a_window_whose_pages_lie_beyond_32_bits(d, hq, hkv, P, dtype, n_q, rotary):
    """Two sequences on the last pages of a pool of more than 2^32 elements: appended (16-byte pieces, and pair by pair) and attended."""
    pages = (1 << 32) // (hkv * 2 * P * d) + 8
    table = torch.tensor([[pages - 1, pages - 4], [pages - 2, pages - 3]])
    freq = pq.pq_rotary_frequencies(rotary)
    w = pq.PagedWindow(2, hq, hkv, d, P, pages, table, dtype=dtype, frequencies=freq, device=DEV)
    counts = [P + 70, 33]
    g = torch.Generator(DEV).manual_seed(1)
    k, v = (torch.randn((sum(counts), hkv, d), generator=g, device=DEV).to(dtype) for _ in range(2))
    w.append(None, k, v, torch.tensor([0, counts[0], sum(counts)], dtype=torch.int32, device=DEV))
    q = torch.randn((2, n_q, hq, d), generator=g, device=DEV).to(dtype)
    lse = torch.empty((2, n_q, hq), device=DEV)
    out = w.attend(q, lse=lse)
    torch.cuda.synchronize()
    assert w.check_status()[0] == 0 and w.lens.tolist() == counts
    at = 0
    for b, n in enumerate(counts):
        page = w.pool[table[b, torch.arange(n) // P].to(DEV), :, :, (torch.arange(n) % P).to(DEV)]   # [n, hkv, 2, d]
        want = rotate(f64(k[at:at + n]), np.arange(n), freq.numpy(), False)
        assert np.all(np.abs(f64(page[:, :, 0]) - want) <= 2.0 ** -18 * 5 + half_step(dtype) * np.abs(want))
        assert torch.equal(page[:, :, 1], v[at:at + n])
        want, want_lse = attention(f64(q[b]), f64(page[:, :, 0]), f64(page[:, :, 1]), d ** -0.5)
        assert np.all(np.abs(f64(out[b]) - want) <= 2e-5 + half_step(dtype) * np.abs(want))
        assert np.all(np.abs(f64(lse[b]) - want_lse) <= 2e-5)
        at += n


@pytest.mark.parametrize("d,R", [(128, 3), (128, 8), (128, 64), (64, 20)])
def test_a_prefix_beyond_32_bits_of_a_paged_cache(d, R):
    hq, hkv, P, n = 8, 2, 256, 600
    pages = (1 << 32) // pq.pq_paged_cache_bytes(d, hkv, P, 1) + 8
    table = torch.tensor([[0, 1, 2], [pages - 1, pages - 3, pages - 2]])
    cache = pq.PagedPolarQuantCache(2, hq, hkv, d, P, pages, table, seed=6, device=DEV)
    K, V = synthetic.kv_like(21, n + 5, hkv, d, BF16, DEV, n_outliers=4)
    cache.encode(K, V, torch.tensor([0, 5, n + 5], dtype=torch.int32, device=DEV))
    small = pq.PolarQuantCache(1, hq, hkv, d, capacity=n, seed=6, device=DEV)
    small.encode(K[5:].contiguous(), V[5:].contiguous(), torch.tensor([0, n], dtype=torch.int32, device=DEV))
    q = synthetic.queries(2, R, hq, d, F32, DEV)
    out = cache.attend_prefix(q, seq=1)
    torch.cuda.synchronize()
    assert cache.check_status()[0] == 0
    Kh, Vh = decoded(small, 0, n)
    want, _ = reference(to_f64(q), Kh, Vh, d ** -0.5)
    check(cache, q, out, want)


@pytest.mark.parametrize("d,R", [(128, 1), (128, 3), (128, 8), (128, 64), (64, 20)])
def test_outputs_in_the_place_of_the_queries(d, R):
    cache = make_cache([3000], 8, 2, d)
    w = pq.PagedWindow(R, 8, 2, d, 16, R * 4, torch.arange(R * 4).view(R, 4), device=DEV)
    fill_window(w, [(17 * b) % 50 + 1 for b in range(R)], 3)
    q = synthetic.queries(1, R, 8, d, BF16, DEV)
    for call in (lambda x, out: cache.attend_prefix(x, out=out), lambda x, out: cache.attend_shared(x, w, out=out), lambda x, out: w.attend(x, out=out)):
        want = call(q, None)
        same = q.clone()
        assert call(same, same) is same and torch.equal(same, want)
