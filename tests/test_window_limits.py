"""Windows at the limit of 32-bit positions, refused before anything is launched."""
import pytest

import paper_2502_02617_b200 as pq
from test_window_host import append, attend, paging, shared


@pytest.mark.parametrize("page_tokens,pages", [(16, (1 << 27) - 1), (16, (1 << 27) - 15), (1 << 16, 1 << 15), (2147483392 // 16 * 16 + 16, 1)])
def test_a_window_whose_last_step_would_pass_32_bits_is_refused(page_tokens, pages):
    """A warp steps up to 64 tokens beyond the end of its range: past 2^31 that is a negative position, and the loop would go on."""
    bad = paging(page_tokens=page_tokens, pages_per_seq=pages)
    assert append(pg=bad) == attend(pg=bad) == shared(window_paging=bad) == pq.ERR_UNSUPPORTED
