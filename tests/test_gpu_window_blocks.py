"""Blocks of 64 rows of the window attention, which larger windows than the other tests have take.  References and tolerances are those of test_gpu_window."""
import numpy as np
import pytest
import torch

from test_gpu_window import BF16, DEV, F32, check_attention, fill_windows, make_window

pytestmark = pytest.mark.gpu


# Windows that together exceed L2 by their bound, with more than 48 (query, head) rows a kv head, are read once for 64 rows.
def read_once(B, hkv, d, max_len):
    return 4 * d * B * hkv * max_len > 126e6


@pytest.mark.parametrize("io", [BF16, F32])
@pytest.mark.parametrize("n_q,hq,hkv,d", [(7, 16, 2, 128), (64, 8, 2, 128), (33, 6, 2, 64), (5, 32, 2, 64), (49, 1, 1, 128), (16, 8, 2, 64)])
def test_blocks_of_64_rows(n_q, hq, hkv, d, io):
    """Windows around the tile and the chunk, parts beyond a cluster; then with a last token whose key is infinite and whose value is NaN:
    the queries that must not see it are as they were."""
    lens = [0, 1, n_q - 1, n_q, n_q + 1, 16, 40, 333, 1200, 2500]
    B, max_len = len(lens), 70000
    assert read_once(B, hkv, d, max_len) and n_q * hq // hkv > 48
    w = make_window(B, hq, hkv, d, 16, max(lens) + 3, seed=n_q, fill=float("nan"))
    fill_windows(w, lens)
    q = torch.randn((B, n_q, hq, d), generator=torch.Generator(DEV).manual_seed(n_q), device=DEV).to(io)
    lse = torch.empty((B, n_q, hq), device=DEV)
    out = w.attend(q, lse=lse, max_len=max_len)
    torch.cuda.synchronize()
    assert w.check_status()[0] == 0
    with np.errstate(invalid="ignore"):
        check_attention(w, lens, q, out, lse, d ** -0.5)
    for b, n in enumerate(lens):   # only the last query sees the last token
        if n:
            w.pool[int(w.page_table[b, (n - 1) // 16]), :, 0, (n - 1) % 16] = float("inf")
            w.pool[int(w.page_table[b, (n - 1) // 16]), :, 1, (n - 1) % 16] = float("nan")
    hidden = w.attend(q, lse=lse, max_len=max_len)
    torch.cuda.synchronize()
    assert torch.allclose(hidden[:, :-1].float(), out[:, :-1].float(), atol=4e-5, rtol=2.0 ** -7 if io == BF16 else 0.0)   # two ways to sum, each within 2e-5
    assert all(bool(torch.isnan(hidden[b, -1]).all()) for b, n in enumerate(lens) if n)


@pytest.mark.parametrize("B,d,max_len", [(64, 128, 2000), (130, 64, 3900), (300, 128, 500)])
def test_blocks_of_64_rows_in_clusters_of_every_size(B, d, max_len):
    n_q, hq, hkv = 13, 8, 2
    assert read_once(B, hkv, d, max_len)
    lens = [(37 * b) % 410 for b in range(B)]
    w = make_window(B, hq, hkv, d, 64, max(lens), seed=B, fill=float("nan"))
    fill_windows(w, lens)
    q = torch.randn((B, n_q, hq, d), generator=torch.Generator(DEV).manual_seed(B), device=DEV).to(BF16)
    lse = torch.empty((B, n_q, hq), device=DEV)
    out = w.attend(q, lse=lse, max_len=max_len)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        check_attention(w, lens, q, out, lse, d ** -0.5)
