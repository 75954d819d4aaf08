"""A shared prefix long enough that its kernel goes round its rings, and beside windows long enough for parts beyond a cluster.  Tolerances
are those of test_gpu_shared_prefix."""
import numpy as np
import pytest
import torch

import paper_2502_02617_b200 as pq
from paper_2502_02617_b200 import synthetic
from parity_utils import TOL_ATTENTION_F32_IO, rel_l2, to_f64
from test_gpu_shared_prefix import BF16, DEV, F32, check, decoded, fill_window, make_cache, reference
from window_reference import rows_of

pytestmark = pytest.mark.gpu
CLUSTER, PERSISTENT, ROWS, TENSOR = 6, 7, 8, 9   # the head_dim-128 kernels, named for the next call


def named(kernel, call):
    if kernel is not None:
        pq.pq_debug_fail_next_wait(kernel)
    out = call()
    pq.pq_debug_fail_next_wait(0)
    return out


def softmax_rows(q, K, V, scale):
    """reference() without windows, all rows of a head at once."""
    out, lse = np.zeros_like(q), np.zeros(q.shape[:2])
    for h in range(q.shape[1]):
        e = q[:, h] @ K[h * K.shape[0] // q.shape[1]].T * scale
        m = e.max(1, keepdims=True)
        w = np.exp(e - m)
        out[:, h] = w @ V[h * K.shape[0] // q.shape[1]] / w.sum(1, keepdims=True)
        lse[:, h] = (m + np.log(w.sum(1, keepdims=True)))[:, 0]
    return out, lse


@pytest.mark.parametrize("R,hq,hkv,n,paged", [(1024, 8, 1, 2900, False), (700, 8, 2, 6001, True), (300, 8, 1, 20000, False), (2100, 2, 1, 2500, True)])
def test_ranges_of_many_blocks_on_tcgen05(R, hq, hkv, n, paged):
    """Ranges of 10 to 45 blocks of 64 tokens: the stages, the packed buffers and the score accumulators, four of each, are all used again."""
    d = 128
    cache = make_cache([9, n], hq, hkv, d, paged, capacity=n + 70)
    K, V = decoded(cache, 1, n)
    for io in (F32, BF16):
        q = synthetic.queries(R, R, hq, d, io, DEV)
        lse = torch.empty((R, hq), device=DEV)
        out = named(TENSOR, lambda: cache.attend_prefix(q, seq=1, lse=lse))
        torch.cuda.synchronize()
        assert cache.check_status()[0] == 0
        want, want_lse = softmax_rows(to_f64(q), K, V, d ** -0.5)
        check(cache, q, out, want)
        assert np.max(np.abs(to_f64(lse) - want_lse)) < 2e-3


@pytest.mark.parametrize("n", [700, 0])
@pytest.mark.parametrize("kernel,d,dtype,lens,bound", [
    (CLUSTER, 128, BF16, [9000, 0, 4097], 20000), (PERSISTENT, 128, BF16, [9000, 0, 4097], 20000), (ROWS, 128, BF16, [9000, 0, 4097], 20000),
    (TENSOR, 128, BF16, [9000, 0, 4097], 20000), (CLUSTER, 128, F32, [2600, 3], 4000), (PERSISTENT, 128, F32, [2600, 3], 4000),
    (ROWS, 128, F32, [2600, 3], 4000), (TENSOR, 128, F32, [2600, 3], 4000), (None, 64, BF16, [8000, 1, 90], 20000), (None, 16, F32, [7000, 5], 20000)])
def test_shared_attention_with_windows_in_parts(kernel, d, dtype, lens, bound, n):
    """Windows cut beyond a cluster, whose parts a kernel of their own merges between the window's and the prefix's kernels: each order of
    launches, back to back and replayed."""
    B, hq, hkv, n_q, P = len(lens), 8, 2, 2, 64
    assert pq.pq_window_workspace_bytes(d, B, n_q, hq, hkv, bound) > 16   # parts
    cache = make_cache([30, n], hq, hkv, d, capacity=max(n, 30) + 40)
    K, V = decoded(cache, 1, n)
    pages = -(-max(lens) // P)
    table = torch.from_numpy(np.random.default_rng(2).permutation(B * pages).reshape(B, pages).astype(np.int32))
    w = pq.PagedWindow(B, hq, hkv, d, P, B * pages, table, dtype=dtype, device=DEV)
    fill_window(w, lens, 4)
    pool, windows = to_f64(w.pool), []
    for b in range(B):
        k, v = rows_of(pool, table.numpy(), P, b, lens[b])
        windows += [(k[:max(0, lens[b] - (n_q - 1 - j))], v[:max(0, lens[b] - (n_q - 1 - j))]) for j in range(n_q)]
    q = synthetic.queries(2, B * n_q, hq, d, F32, DEV).view(B, n_q, hq, d)
    call = lambda: named(kernel, lambda: cache.attend_shared(q, w, seq=1, max_window=bound))  # noqa: E731
    first = call()
    torch.cuda.synchronize()
    want, _ = reference(to_f64(q).reshape(-1, hq, d), K, V, d ** -0.5, windows)
    assert rel_l2(to_f64(first).reshape(want.shape), want) < TOL_ATTENTION_F32_IO
    nothing = n == 0 and any(len(x[0]) == 0 for x in windows)
    assert cache.status.cpu().tolist()[0] == (pq.ERR_EMPTY if nothing else 0)
    again = [call() for _ in range(8)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = [call() for _ in range(3)]
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(first, x) for x in again + held)
