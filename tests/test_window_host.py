"""The paged window's entry points without a GPU: sizes, frequencies, and the calls that are refused before anything is launched."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2502_02617_b200 as pq
from paper_2502_02617_b200 import api

L = pq.lib()
GOOD = 1 << 20   # a 16-byte aligned address that no refused call reads


def paging(table=GOOD, page_tokens=16, pages_per_seq=4, n_pages=8):
    return api.Paging(table, page_tokens, pages_per_seq, n_pages)


def append(pg=None, **kw):
    a = dict(d=64, hq=4, hkv=2, q=GOOD, k=GOOD, v=GOOD, dtype=pq.DTYPE_BF16, qts=256, qhs=64, kts=128, khs=64, cu=None, batch=2, total=2, freq=GOOD,
             rotary=64, interleaved=0, offsets=None, q_out=GOOD, pool=GOOD, lens=GOOD, status=GOOD)
    a.update(kw)
    pg = paging() if pg is None else pg
    return L.pq_append_window(a["d"], a["hq"], a["hkv"], a["q"], a["k"], a["v"], a["dtype"], a["qts"], a["qhs"], a["kts"], a["khs"], a["cu"], a["batch"],
                              a["total"], a["freq"], a["rotary"], a["interleaved"], a["offsets"], a["q_out"], a["pool"], a["lens"],
                              ctypes.addressof(pg) if pg else None, a["status"], None)


def attend(pg=None, **kw):
    a = dict(d=64, hq=4, hkv=2, q=GOOD, io=pq.DTYPE_BF16, pool=GOOD, kv=pq.DTYPE_BF16, lens=GOOD, batch=2, n_q=1, most=64, out=GOOD, lse=None, ws=GOOD,
             status=GOOD)
    a.update(kw)
    pg = paging() if pg is None else pg
    return L.pq_window_attention(a["d"], a["hq"], a["hkv"], a["q"], a["io"], a["pool"], a["kv"], a["lens"], a["batch"], a["n_q"],
                                 ctypes.addressof(pg) if pg else None, a["most"], 0.1, a["out"], a["lse"], a["ws"], a["status"], None)


BAD_PAGING = [(paging(table=None), pq.ERR_INVALID_ARG), (paging(page_tokens=24), pq.ERR_INVALID_ARG), (paging(page_tokens=0), pq.ERR_INVALID_ARG),
              (paging(pages_per_seq=0), pq.ERR_INVALID_ARG), (paging(n_pages=0), pq.ERR_INVALID_ARG), (paging(table=GOOD + 2), pq.ERR_ALIGNMENT),
              (paging(page_tokens=1 << 16, pages_per_seq=1 << 15), pq.ERR_UNSUPPORTED)]


@pytest.mark.parametrize("change,status", [
    (dict(d=48), "UNSUPPORTED"), (dict(d=256), "UNSUPPORTED"), (dict(dtype=7), "UNSUPPORTED"),
    (dict(k=None), "INVALID_ARG"), (dict(v=None), "INVALID_ARG"), (dict(pool=None), "INVALID_ARG"), (dict(lens=None), "INVALID_ARG"),
    (dict(status=None), "INVALID_ARG"), (dict(q=None), "INVALID_ARG"), (dict(q_out=None), "INVALID_ARG"), (dict(hq=0), "INVALID_ARG"),
    (dict(hkv=0), "INVALID_ARG"), (dict(batch=0), "INVALID_ARG"), (dict(total=-1), "INVALID_ARG"), (dict(total=3), "INVALID_ARG"),
    (dict(rotary=63), "INVALID_ARG"), (dict(rotary=66), "INVALID_ARG"), (dict(rotary=-2), "INVALID_ARG"), (dict(rotary=0), "INVALID_ARG"),
    (dict(freq=None), "INVALID_ARG"), (dict(qts=-1), "INVALID_ARG"), (dict(khs=-1), "INVALID_ARG"),
    (dict(pool=GOOD + 8), "ALIGNMENT"), (dict(freq=GOOD + 4), "ALIGNMENT"), (dict(lens=GOOD + 2), "ALIGNMENT"), (dict(k=GOOD + 1), "ALIGNMENT"),
    (dict(dtype=pq.DTYPE_F32, q=GOOD + 2), "ALIGNMENT"), (dict(offsets=GOOD + 1), "ALIGNMENT"),
    (dict(cu=GOOD, total=(1 << 31) - 1, hq=64, d=128, rotary=128), "UNSUPPORTED")])
def test_append_refuses(change, status):
    assert append(**change) == getattr(pq, "ERR_" + status)


@pytest.mark.parametrize("change,status", [
    (dict(d=48), "UNSUPPORTED"), (dict(d=256), "UNSUPPORTED"), (dict(io=3), "UNSUPPORTED"), (dict(kv=3), "UNSUPPORTED"),
    (dict(q=None), "INVALID_ARG"), (dict(pool=None), "INVALID_ARG"), (dict(lens=None), "INVALID_ARG"), (dict(out=None), "INVALID_ARG"),
    (dict(ws=None), "INVALID_ARG"), (dict(status=None), "INVALID_ARG"), (dict(batch=0), "INVALID_ARG"), (dict(n_q=0), "INVALID_ARG"),
    (dict(hq=3), "INVALID_ARG"), (dict(hkv=0), "INVALID_ARG"), (dict(most=0), "INVALID_ARG"),
    (dict(q=GOOD + 8), "ALIGNMENT"), (dict(pool=GOOD + 8), "ALIGNMENT"), (dict(out=GOOD + 4), "ALIGNMENT"), (dict(ws=GOOD + 8), "ALIGNMENT"),
    (dict(lens=GOOD + 2), "ALIGNMENT"), (dict(lse=GOOD + 2), "ALIGNMENT"),
    (dict(batch=70000), "UNSUPPORTED"), (dict(n_q=1 << 20, hq=64, hkv=2), "UNSUPPORTED")])
def test_attention_refuses(change, status):
    assert attend(**change) == getattr(pq, "ERR_" + status)


@pytest.mark.parametrize("pg,status", BAD_PAGING)
def test_bad_paging_is_refused(pg, status):
    assert append(pg=pg) == status and attend(pg=pg) == status


def test_an_append_of_no_rows_does_nothing():
    assert append(total=0, cu=GOOD, q=None, k=None, v=None, q_out=None) == pq.OK
    assert append(total=0, cu=GOOD) == pq.OK
    assert append(total=0, cu=GOOD, lens=None) == pq.ERR_INVALID_ARG and append(total=0) == pq.ERR_INVALID_ARG


def test_missing_paging_is_refused():
    args = [64, 4, 2, GOOD, pq.DTYPE_BF16, GOOD, pq.DTYPE_BF16, GOOD, 2, 1, None, 64, 0.1, GOOD, None, GOOD, GOOD, None]
    assert L.pq_window_attention(*args) == pq.ERR_INVALID_ARG


def test_sizes():
    assert pq.pq_window_bytes(128, 8, 64, 10) == 10 * 8 * 2 * 64 * 128 * 2
    assert pq.pq_window_bytes(64, 2, 16, 3, torch.float32) == 3 * 2 * 2 * 16 * 64 * 4
    for bad in [(48, 8, 64, 10), (128, 0, 64, 10), (128, 8, 60, 10), (128, 8, 64, 0)]:
        with pytest.raises(pq.PolarQuantError):
            pq.pq_window_bytes(*bad)
    # parts beyond a cluster only where few units would leave the device idle; nothing shrinks with the length
    sizes = [pq.pq_window_workspace_bytes(128, 1, 1, 32, 8, n) for n in (1, 300, 4096, 65536, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[0] == 16 and sizes[-1] > 16
    assert pq.pq_window_workspace_bytes(128, 256, 1, 32, 8, 1 << 20) == 16
    with pytest.raises(pq.PolarQuantError):
        pq.pq_window_workspace_bytes(128, 1, 1, 30, 8, 64)


@pytest.mark.parametrize("rotary,theta", [(2, 10000.0), (64, 10000.0), (128, 500000.0)])
def test_frequencies(rotary, theta):
    want = np.array([theta ** (-2 * i / rotary) for i in range(rotary // 2)])
    assert np.allclose(pq.pq_rotary_frequencies(rotary, theta).numpy(), want, rtol=4e-16 * 8, atol=0)


@pytest.mark.parametrize("rotary,theta", [(0, 1e4), (-2, 1e4), (3, 1e4), (64, 0.0), (64, -1.0), (64, float("inf")), (64, float("nan"))])
def test_bad_frequencies_are_refused(rotary, theta):
    with pytest.raises(pq.PolarQuantError):
        pq.pq_rotary_frequencies(rotary, theta)


def prefix(**kw):
    a = dict(d=128, hq=8, hkv=2, S=GOOD, tables=GOOD, q=GOOD, io=pq.DTYPE_BF16, n=4, cache=GOOD, lens=GOOD, cache_batch=2, seq=1, capacity=256, pg=None,
             most=200, out=GOOD, lse=None, ws=GOOD, status=GOOD)
    a.update(kw)
    return L.pq_prefix_attention(a["d"], a["hq"], a["hkv"], a["S"], a["tables"], a["q"], a["io"], a["n"], a["cache"], a["lens"], a["cache_batch"], a["seq"],
                                 a["capacity"], ctypes.addressof(a["pg"]) if a["pg"] else None, a["most"], 0.1, a["out"], a["lse"], a["ws"], a["status"], None)


PREFIX_REFUSALS = [
    (dict(d=48), "UNSUPPORTED"), (dict(d=256), "UNSUPPORTED"), (dict(io=5), "UNSUPPORTED"), (dict(hq=36, hkv=2), "UNSUPPORTED"),
    (dict(q=None), "INVALID_ARG"), (dict(S=None), "INVALID_ARG"), (dict(tables=None), "INVALID_ARG"), (dict(cache=None), "INVALID_ARG"),
    (dict(lens=None), "INVALID_ARG"), (dict(out=None), "INVALID_ARG"), (dict(ws=None), "INVALID_ARG"), (dict(status=None), "INVALID_ARG"),
    (dict(seq=-1), "INVALID_ARG"), (dict(seq=2), "INVALID_ARG"), (dict(cache_batch=0), "INVALID_ARG"), (dict(n=0), "INVALID_ARG"), (dict(hq=7), "INVALID_ARG"),
    (dict(capacity=0), "INVALID_ARG"), (dict(most=0), "INVALID_ARG"), (dict(lens=GOOD + 2), "ALIGNMENT"), (dict(q=GOOD + 8), "ALIGNMENT"),
    (dict(cache=GOOD + 8), "ALIGNMENT"), (dict(n=65536), "UNSUPPORTED"), (dict(pg=paging(page_tokens=64)), "INVALID_ARG"),
    (dict(pg=paging(table=GOOD + 1, page_tokens=128)), "ALIGNMENT")]


@pytest.mark.parametrize("change,status", PREFIX_REFUSALS)
def test_prefix_attention_refuses(change, status):
    assert prefix(**change) == getattr(pq, "ERR_" + status)


def shared(window_paging=None, **kw):
    a = dict(d=128, hq=8, hkv=2, S=GOOD, tables=GOOD, q=GOOD, io=pq.DTYPE_BF16, batch=4, n_q=1, cache=GOOD, lens=GOOD, cache_batch=2, seq=1, capacity=256, pg=None,
             most=200, pool=GOOD, kv=pq.DTYPE_BF16, wlens=GOOD, most_window=64, out=GOOD, ws=GOOD, status=GOOD)
    a.update(kw)
    wpg = paging() if window_paging is None else window_paging
    return L.pq_shared_attention(a["d"], a["hq"], a["hkv"], a["S"], a["tables"], a["q"], a["io"], a["batch"], a["n_q"], a["cache"], a["lens"], a["cache_batch"],
                                 a["seq"], a["capacity"], ctypes.addressof(a["pg"]) if a["pg"] else None, a["most"], a["pool"], a["kv"], a["wlens"],
                                 ctypes.addressof(wpg), a["most_window"], 0.1, a["out"], a["ws"], a["status"], None)


@pytest.mark.parametrize("change,status", [(c, s) for c, s in PREFIX_REFUSALS if "n" not in c and "lse" not in c] + [
    (dict(pool=None), "INVALID_ARG"), (dict(wlens=None), "INVALID_ARG"), (dict(kv=4), "UNSUPPORTED"), (dict(most_window=0), "INVALID_ARG"),
    (dict(pool=GOOD + 8), "ALIGNMENT"), (dict(wlens=GOOD + 1), "ALIGNMENT"), (dict(batch=0), "INVALID_ARG"), (dict(n_q=0), "INVALID_ARG"),
    (dict(batch=300, n_q=300), "UNSUPPORTED")])
def test_shared_attention_refuses(change, status):
    assert shared(**change) == getattr(pq, "ERR_" + status)


@pytest.mark.parametrize("pg,status", BAD_PAGING)
def test_shared_attention_refuses_a_bad_window(pg, status):
    assert shared(window_paging=pg) == status
