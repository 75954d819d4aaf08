"""What the extension module refuses before anything is launched: a refused call reads none of its tensors."""
import pytest
import torch

import paper_2502_02617_b200 as pq
from paper_2502_02617_b200 import api

D, HQ, HKV, P, PAGES = 128, 8, 2, 128, 4


def prefix_args(table):
    return [torch.eye(D), torch.zeros(16, dtype=torch.uint8), torch.zeros((3, HQ, D)), torch.zeros(pq.pq_paged_cache_bytes(D, HKV, P, PAGES), dtype=torch.uint8),
            torch.zeros(2, dtype=torch.int32), 0, HKV, 0, 100, 0.1, torch.zeros((3, HQ, D)), torch.zeros(1 << 22, dtype=torch.uint8),
            torch.zeros(api.STATUS_WORDS, dtype=torch.int32), (table, P, PAGES), None]


def shared_args(table):
    pool = torch.zeros((4, HKV, 2, 16, D))
    return prefix_args(table) + [pool, torch.zeros(3, dtype=torch.int32), 16, (torch.zeros((3, 1), dtype=torch.int32), 16, 4)]


@pytest.mark.parametrize("entry,args", [("prefix_attend", lambda t: prefix_args(t) + [None]), ("shared_attend", shared_args)])
def test_a_page_table_on_another_device_than_the_cache_is_refused(entry, args):
    """A kernel would follow its address."""
    with pytest.raises(AssertionError, match="page table.*device"):
        getattr(api.native(), entry)(*args(torch.zeros((2, 2), dtype=torch.int32, device="meta")))


@pytest.mark.gpu
def test_a_page_table_left_on_the_host_is_refused():
    cache = pq.PagedPolarQuantCache(2, HQ, HKV, D, P, PAGES, torch.arange(4, dtype=torch.int32).view(2, 2), device="cuda:0")
    q = torch.zeros((3, HQ, D), dtype=torch.bfloat16, device="cuda:0")
    window = pq.PagedWindow(3, HQ, HKV, D, 16, 3, torch.arange(3).view(3, 1), device="cuda:0")
    cache.attend_prefix(q)
    cache.page_table = cache.page_table.cpu()
    with pytest.raises(AssertionError, match="page table.*device"):
        cache.attend_prefix(q)
    with pytest.raises(AssertionError, match="page table.*device"):
        cache.attend_shared(q, window)
