"""Parts of an attention that are no numbers: merged with others they make the whole none."""
import pytest
import torch

import paper_2502_02617_b200 as pq
from paper_2502_02617_b200 import synthetic
from test_gpu_shared_prefix import BF16, DEV, fill_window, make_cache

pytestmark = pytest.mark.gpu
CLUSTER, PERSISTENT, ROWS, TENSOR = 6, 7, 8, 9   # the head_dim-128 kernels, named for the next call


def named(kernel, call):
    pq.pq_debug_fail_next_wait(kernel)
    out = call()
    pq.pq_debug_fail_next_wait(0)
    return out


def spoil(head, n):
    """NaN in all key radii of the first n tokens of a kv head's part of a packed cache: pairs of blocks, keys and values, of 64 tokens, in
    each 46 bytes of codes a token before the radii."""
    blocks = head.view(-1, 2, 64 * 62)[:, 0, 64 * 46:].view(-1, 64, 16)
    for j in range(-(-n // 64)):
        blocks[j, :n - 64 * j] = 255


@pytest.mark.parametrize("kernel", [CLUSTER, PERSISTENT, ROWS, TENSOR])
@pytest.mark.parametrize("R", [1, 5, 40])
@pytest.mark.parametrize("every", [False, True])
def test_a_prefix_that_is_no_number_is_not_lost_beside_a_window(kernel, R, every):
    """Each head_dim-128 kernel: the heads that read a radius of NaN (of one token or of all) are NaN, their log-sum-exps too, and the
    attention over prefix and window does not take the window alone for them."""
    n, hq, hkv, d = 333, 8, 2, 128
    cache = make_cache([n], hq, hkv, d, capacity=384)
    q = synthetic.queries(1, R, hq, d, BF16, DEV)
    w = pq.PagedWindow(R, hq, hkv, d, 16, R, torch.arange(R).view(R, 1), device=DEV)
    fill_window(w, [5] * R, 3)
    lse = torch.empty((R, hq), device=DEV)
    good, good_lse = named(kernel, lambda: cache.attend_prefix(q, lse=lse)).clone(), lse.clone()
    good_shared = named(kernel, lambda: cache.attend_shared(q, w)).clone()
    spoil(cache.cache.view(hkv, -1)[1], n if every else 1)
    out = named(kernel, lambda: cache.attend_prefix(q, lse=lse))
    shared = named(kernel, lambda: cache.attend_shared(q, w))
    torch.cuda.synchronize()
    for a, b in ((out, good), (shared, good_shared)):
        assert torch.equal(a[:, :hq // 2], b[:, :hq // 2]) and bool(torch.isnan(a[:, hq // 2:]).all())
    assert torch.equal(lse[:, :hq // 2], good_lse[:, :hq // 2]) and bool(torch.isnan(lse[:, hq // 2:]).all())


@pytest.mark.parametrize("kernel", [CLUSTER, PERSISTENT, ROWS, TENSOR])
@pytest.mark.parametrize("R", [1, 5, 40])
def test_a_query_that_is_no_number_is_not_an_empty_one(kernel, R):
    """Behind it an empty window, whose part says nothing: its row is NaN, and the others are as they were."""
    n, hq, hkv, d = 333, 8, 2, 128
    cache = make_cache([n], hq, hkv, d, capacity=384)
    q = synthetic.queries(1, R, hq, d, BF16, DEV)
    w = pq.PagedWindow(R, hq, hkv, d, 16, R, torch.arange(R).view(R, 1), device=DEV)
    fill_window(w, [0] * R, 3)
    good = named(kernel, lambda: cache.attend_shared(q, w)).clone()
    bad = torch.zeros((R, hq), dtype=torch.bool, device=DEV)
    bad[R - 1, 3] = True
    q[R - 1, 3, 7] = float("nan")
    lse = torch.empty((R, hq), device=DEV)
    out = named(kernel, lambda: cache.attend_prefix(q, lse=lse))
    shared = named(kernel, lambda: cache.attend_shared(q, w))
    torch.cuda.synchronize()
    assert cache.check_status()[0] == 0
    assert torch.equal(torch.isnan(lse), bad) and torch.equal(torch.isnan(out), bad[..., None].expand(out.shape))
    assert torch.equal(torch.isnan(shared), bad[..., None].expand(out.shape)) and torch.equal(shared[~bad], good[~bad])


@pytest.mark.parametrize("kernel", [CLUSTER, PERSISTENT, ROWS])
@pytest.mark.parametrize("every", [False, True])
def test_a_partial_attention_that_is_no_number_says_so(kernel, every):
    """The same of the attention that gives its log-sum-exp to be merged with others."""
    n, hq, hkv, d = 333, 8, 2, 128
    cache = make_cache([n, 100], hq, hkv, d, capacity=384)
    q = synthetic.queries(1, 2, hq, d, BF16, DEV)
    spoil(cache.cache.view(2, hkv, -1)[0, 0], n if every else 1)
    out, lse = named(kernel, lambda: cache.attend_lse(q))
    torch.cuda.synchronize()
    bad = torch.zeros((2, hq), dtype=torch.bool, device=DEV)
    bad[0, :hq // 2] = True
    assert torch.equal(torch.isnan(lse), bad) and torch.equal(torch.isnan(out).all(-1), bad) and torch.equal(torch.isnan(out).any(-1), bad)
