"""Several host threads on one stream: the launches of their calls may interleave, what a call leaves between its kernels is its own."""
import threading

import pytest
import torch

import paper_2502_02617_b200 as pq
from paper_2502_02617_b200 import synthetic
from test_gpu_shared_prefix import BF16, DEV, fill_window, make_cache

pytestmark = pytest.mark.gpu


def together(calls, rounds):
    """Each call on a thread of its own, `rounds` times: the outputs by call."""
    start, got, errors = threading.Barrier(len(calls)), [[] for _ in calls], []

    def work(i):
        try:
            start.wait()
            for _ in range(rounds):
                got[i].append(calls[i]())
        except Exception as e:   # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    return got


@pytest.mark.parametrize("named_stream", [False, True])
@pytest.mark.parametrize("what", ["prefix of many queries", "prefix of smaller heads", "prefix and window", "window in parts"])
def test_calls_of_several_threads(what, named_stream):
    d = 64 if what == "prefix of smaller heads" else 128
    R = 64 if what == "prefix of many queries" else 2
    cache = make_cache([700], 8, 2, d)
    w = pq.PagedWindow(R, 8, 2, d, 64, 320 * R, torch.arange(320 * R).view(R, 320), device=DEV)
    fill_window(w, [20000 if what == "window in parts" else 50] * R, 3)
    stream = torch.cuda.Stream() if named_stream else None
    qs = [synthetic.queries(i, R, 8, d, BF16, DEV) for i in range(4)]
    one = {"prefix and window": lambda q: cache.attend_shared(q, w, stream=stream), "window in parts": lambda q: w.attend(q, stream=stream)}.get(
        what, lambda q: cache.attend_prefix(q, stream=stream))
    torch.cuda.synchronize()
    want = [one(q) for q in qs]
    torch.cuda.synchronize()
    got = together([lambda q=q: one(q) for q in qs], 300)
    for outs, wanted in zip(got, want):
        assert all(torch.equal(x, wanted) for x in outs)
