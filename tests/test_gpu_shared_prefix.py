"""Attention over a compressed prefix that many queries share, alone and followed by each sequence's paged window, on the GPU
against the oracle's DeQuant of the same codes.  Tolerances are those of the packed cache's other attentions (parity_utils)."""
import numpy as np
import pytest
import torch

import paper_2502_02617_b200 as pq
from oracle import polarquant_oracle as orc
from paper_2502_02617_b200 import synthetic
from parity_utils import TOL_ATTENTION, TOL_ATTENTION_F32_IO, oracle_codebooks, rel_l2, to_f64
from window_reference import rotate, rows_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def make_cache(lens, hq, hkv, d, paged=False, capacity=None, seed=6):
    capacity = max(max(lens), 1) if capacity is None else capacity
    if paged:
        pages = -(-capacity // 128)
        table = torch.from_numpy(np.random.default_rng(1).permutation(len(lens) * pages + 1)[1:].reshape(len(lens), pages).astype(np.int32))
        cache = pq.PagedPolarQuantCache(len(lens), hq, hkv, d, 128, len(lens) * pages + 1, table, seed=seed, device=DEV)
    else:
        cache = pq.PolarQuantCache(len(lens), hq, hkv, d, capacity=capacity, seed=seed, device=DEV)
    cache.cache.fill_(255)   # what lies behind a sequence's end is not read: radii of NaN
    if sum(lens):
        K, V = synthetic.kv_like(21, sum(lens), hkv, d, BF16, DEV, n_outliers=4 if d >= 64 else 0)
        cache.encode(K, V, torch.tensor(np.concatenate(([0], np.cumsum(lens))), dtype=torch.int32, device=DEV))
    return cache


def decoded(cache, seq, n):
    """(K_hat, V_hat) [Hkv, n, d] float64 of the first n tokens of a sequence, in the original basis."""
    codes, radii = cache.unpack(max(n, 1))
    cb, S = oracle_codebooks(cache), cache.S_host.double().numpy()
    codes, radii = codes[seq].cpu().numpy(), radii[seq].cpu().numpy()
    return [np.stack([orc.dequant(codes[h, i, :n], radii[h, i, :n], cb, S) for h in range(cache.n_kv_heads)]) for i in (0, 1)]


def reference(q, K, V, scale, windows=None, n_q=1):
    """q [R, Hq, d] over K, V [Hkv, n, d] and, for row r, the first windows[r] = (K, V) [n, Hkv, d] rows: (out, lse)."""
    R, hq, d = q.shape
    g = hq // K.shape[0]
    out, lse = np.zeros_like(q), np.full((R, hq), -np.inf)
    for h in range(hq):
        e_all = q[:, h] @ K[h // g].T * scale
        for r in range(R):
            e, v = e_all[r], V[h // g]
            if windows is not None and len(windows[r][0]):
                e = np.concatenate([e, windows[r][0][:, h // g] @ q[r, h] * scale])
                v = np.concatenate([v, windows[r][1][:, h // g]])
            if len(e):
                w = np.exp(e - e.max())
                out[r, h] = w @ v / w.sum()
                lse[r, h] = e.max() + np.log(w.sum())
    return out, lse


def check(cache, q, out, want):
    if q.dtype == F32:
        assert rel_l2(to_f64(out), want) < TOL_ATTENTION_F32_IO
    elif out.numel() >= 1024:   # fewer values: the rounding alone can exceed the bound
        assert rel_l2(to_f64(out), want) < TOL_ATTENTION


@pytest.mark.parametrize("n", [1, 63, 65, 500, 2900])
@pytest.mark.parametrize("R", [1, 2, 7, 8, 33, 64, 130])
@pytest.mark.parametrize("d,hq,hkv,paged", [(128, 8, 2, False), (128, 8, 2, True), (128, 7, 1, False), (128, 8, 1, False), (128, 2, 2, False)])
def test_prefix_attention(d, hq, hkv, paged, R, n):
    """Every query sees all tokens of the middle one of three sequences; what follows its end is NaN."""
    cache = make_cache([40, n, 17], hq, hkv, d, paged, capacity=max(n, 40) + 70)
    K, V = decoded(cache, 1, n)
    for io in (F32, BF16):
        q = synthetic.queries(R, R, hq, d, io, DEV)
        lse = torch.empty((R, hq), device=DEV)
        out = cache.attend_prefix(q, seq=1, lse=lse)
        plain = cache.attend_prefix(q, seq=1)
        torch.cuda.synchronize()
        assert cache.check_status()[0] == 0 and torch.equal(plain, out)
        want, want_lse = reference(to_f64(q), K, V, d ** -0.5)
        check(cache, q, out, want)
        assert np.max(np.abs(to_f64(lse) - want_lse)) < 2e-3


@pytest.mark.parametrize("d,hq,hkv,R,n", [(64, 16, 8, 16, 700), (64, 4, 1, 5, 65), (32, 4, 2, 33, 130), (16, 2, 1, 3, 300), (16, 1, 1, 1, 1), (64, 8, 1, 70, 1500),
                                          (64, 2, 2, 200, 64), (32, 8, 1, 129, 257), (16, 8, 2, 64, 1000)])
@pytest.mark.parametrize("paged", [False, True])
def test_prefix_attention_of_smaller_heads(d, hq, hkv, R, n, paged):
    cache = make_cache([n, 5], hq, hkv, d, paged, capacity=n + 9)
    K, V = decoded(cache, 0, n)
    for io in (F32, BF16):
        q = synthetic.queries(R, R, hq, d, io, DEV)
        lse = torch.empty((R, hq), device=DEV)
        out = cache.attend_prefix(q, lse=lse)
        torch.cuda.synchronize()
        assert cache.check_status()[0] == 0
        want, want_lse = reference(to_f64(q), K, V, d ** -0.5)
        check(cache, q, out, want)
        assert np.max(np.abs(to_f64(lse) - want_lse)) < 2e-3


@pytest.mark.parametrize("kernel", [6, 7, 8, 9])
@pytest.mark.parametrize("R", [9, 40])
def test_every_kernel_takes_a_prefix(kernel, R):
    """The four head_dim-128 kernels on the same prefix, each with its log-sum-exps."""
    n, hq, hkv, d = 333, 8, 2, 128
    cache = make_cache([n], hq, hkv, d, capacity=400)
    K, V = decoded(cache, 0, n)
    q = synthetic.queries(3, R, hq, d, F32, DEV)
    lse = torch.empty((R, hq), device=DEV)
    pq.pq_debug_fail_next_wait(kernel)
    out = cache.attend_prefix(q, lse=lse)
    pq.pq_debug_fail_next_wait(0)
    torch.cuda.synchronize()
    assert cache.check_status()[0] == 0
    want, want_lse = reference(to_f64(q), K, V, d ** -0.5)
    assert rel_l2(to_f64(out), want) < TOL_ATTENTION_F32_IO and np.max(np.abs(to_f64(lse) - want_lse)) < 2e-3


@pytest.mark.parametrize("d,R", [(128, 3), (128, 6), (128, 90), (64, 5), (16, 40)])
def test_an_empty_prefix(d, R):
    cache = make_cache([0, 3], 8, 2, d, capacity=200)
    q = synthetic.queries(1, R, 8, d, BF16, DEV)
    lse = torch.zeros((R, 8), device=DEV)
    out = cache.attend_prefix(q, lse=lse)
    torch.cuda.synchronize()
    assert bool((out == 0).all()) and bool((lse == -float("inf")).all()) and cache.check_status()[0] == 0
    out = cache.attend_prefix(q)
    torch.cuda.synchronize()
    assert bool((out == 0).all()) and cache.status.cpu().tolist()[0] == pq.ERR_EMPTY


@pytest.mark.parametrize("d,R", [(128, 4), (128, 90), (64, 20)])
def test_a_radius_that_is_no_number_spoils_its_own_head_only(d, R):
    """Stored radii of NaN (an encoder's input that was not finite): the heads that read them are NaN, the others as they were, and
    so it is with a window behind, empty or not."""
    n, hq, hkv = 200, 4, 2
    cache = make_cache([n], hq, hkv, d, capacity=256)
    q = synthetic.queries(1, R, hq, d, BF16, DEV)
    w = pq.PagedWindow(R, hq, hkv, d, 16, R, torch.arange(R).view(R, 1), device=DEV)
    fill_window(w, [0, 5] * (R // 2), 3)
    good, good_shared = cache.attend_prefix(q).clone(), cache.attend_shared(q, w).clone()
    half = cache.cache.numel() // hkv                    # the second kv head's part of the cache
    radii = 64 * (62 * d // 128) - 64 * (d // 8)         # the last plane of a block of 64 tokens
    cache.cache[half + radii:half + radii + d // 8] = 255   # token 0's radii: NaN
    out, shared = cache.attend_prefix(q), cache.attend_shared(q, w)
    torch.cuda.synchronize()
    for a, b in ((out, good), (shared, good_shared)):
        assert torch.equal(a[:, :hq // 2], b[:, :hq // 2]) and bool(torch.isnan(a[:, hq // 2:]).all())


def test_queries_of_several_positions_are_just_more_queries():
    cache = make_cache([700], 8, 2, 128)
    q = synthetic.queries(5, 12, 8, 128, BF16, DEV)
    assert torch.equal(cache.attend_prefix(q.view(4, 3, 8, 128)).view(12, 8, 128), cache.attend_prefix(q))


def fill_window(w, lens, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    w.pool.fill_(float("nan"))
    for b, n in enumerate(lens):
        t = torch.arange(n, device=DEV)
        w.pool[w.page_table[b].long()[t // w.page_tokens], :, :, t % w.page_tokens] = torch.randn((n, w.n_kv_heads, 2, w.d), generator=g, device=DEV).to(w.pool.dtype)
    w.lens.copy_(torch.tensor(lens, dtype=torch.int32))


@pytest.mark.parametrize("n_q", [1, 3])
@pytest.mark.parametrize("d,hq,hkv,n,lens,dtype,paged", [
    (128, 8, 2, 700, [0, 1, 16, 90, 300], BF16, False), (128, 8, 2, 1, [2, 5], BF16, True), (128, 7, 1, 2000, [40] * 40, BF16, False),
    (128, 4, 4, 130, [33, 0, 7], F32, True), (64, 16, 8, 300, [5, 70], BF16, False), (16, 2, 1, 100, [0, 9], F32, False), (128, 8, 2, 0, [4, 0, 200], BF16, False)])
def test_shared_attention(d, hq, hkv, n, lens, dtype, paged, n_q):
    B = len(lens)
    cache = make_cache([30, n], hq, hkv, d, paged, capacity=max(n, 30) + 40)
    K, V = decoded(cache, 1, n)
    pages = -(-(max(lens) + 1) // 16)
    table = torch.from_numpy(np.random.default_rng(2).permutation(B * pages).reshape(B, pages).astype(np.int32))
    w = pq.PagedWindow(B, hq, hkv, d, 16, B * pages, table, dtype=dtype, device=DEV)
    fill_window(w, lens, 4)
    pool = to_f64(w.pool)
    for io in (F32, BF16):
        q = synthetic.queries(2, B * n_q, hq, d, io, DEV)
        windows = []
        for b in range(B):
            k, v = rows_of(pool, table.numpy(), 16, b, lens[b])
            windows += [(k[:max(0, lens[b] - (n_q - 1 - j))], v[:max(0, lens[b] - (n_q - 1 - j))]) for j in range(n_q)]
        out = cache.attend_shared(q if n_q == 1 else q.view(B, n_q, hq, d), w, seq=1)
        torch.cuda.synchronize()
        nothing = n == 0 and any(len(x[0]) == 0 for x in windows)
        assert cache.status.cpu().tolist()[0] == (pq.ERR_EMPTY if nothing else 0)
        cache.status.zero_()
        want, _ = reference(to_f64(q), K, V, d ** -0.5, windows)
        check(cache, q, out.view(q.shape), want)
        assert not nothing or bool((out.view(q.shape)[[len(x[0]) == 0 for x in windows]] == 0).all())


def test_a_serving_run_from_prompt_to_generated_tokens():
    """A prompt is rotated, compressed once and shared; four sequences then generate six tokens each, the first step with two drafted
    positions, every step's rows rotated on their way into the window: against exact arithmetic on the decoded prompt.  The last
    steps run from a captured graph."""
    B, hq, hkv, d, n = 4, 8, 2, 128, 300
    freq = pq.pq_rotary_frequencies(d, 500000.0)
    g = torch.Generator(DEV).manual_seed(11)
    rows = lambda count, heads: torch.randn((count, heads, d), generator=g, device=DEV).to(BF16)  # noqa: E731
    # the prompt's keys take their positions through a window of one sequence, whose pages are then read as they are
    prompt = pq.PagedWindow(1, hq, hkv, d, 64, 5, torch.arange(5).view(1, 5), frequencies=freq, device=DEV)
    prompt.append(None, rows(n, hkv), rows(n, hkv), torch.tensor([0, n], dtype=torch.int32, device=DEV))
    K, V = (prompt.pool[:, :, i].transpose(1, 2).reshape(-1, hkv, d)[:n].contiguous() for i in (0, 1))
    cache = pq.PolarQuantCache(1, hq, hkv, d, capacity=n, seed=3, device=DEV)
    cache.encode(K, V, torch.tensor([0, n], dtype=torch.int32, device=DEV))
    Kh, Vh = decoded(cache, 0, n)
    table = torch.from_numpy(np.random.default_rng(5).permutation(B * 2).reshape(B, 2).astype(np.int32))
    w = pq.PagedWindow(B, hq, hkv, d, 16, B * 2, table, frequencies=freq, device=DEV)
    offsets = cache.lens.repeat(B)
    kept = [[np.zeros((0, hkv, d))] * 2 for _ in range(B)]

    def check_step(q, k, v, out, n_q, start):
        pos = np.tile(n + start + np.arange(n_q), B)
        qr = rotate(to_f64(q), pos, freq.numpy(), False)
        kr = torch.from_numpy(rotate(to_f64(k), pos, freq.numpy(), False)).to(BF16)
        windows = []
        for b in range(B):
            kept[b] = [np.concatenate([kept[b][0], to_f64(kr[b * n_q:(b + 1) * n_q])]), np.concatenate([kept[b][1], to_f64(v[b * n_q:(b + 1) * n_q])])]
            m = len(kept[b][0])
            windows += [(kept[b][0][:m - (n_q - 1 - j)], kept[b][1][:m - (n_q - 1 - j)]) for j in range(n_q)]
        want, _ = reference(to_f64(torch.from_numpy(qr).to(BF16)), Kh, Vh, d ** -0.5, windows)
        # the rotated rows may be rounded the other way in a few places (float32 against float64): one bf16 step of those
        assert rel_l2(to_f64(out).reshape(want.shape), want) < TOL_ATTENTION + 2e-4

    q, k, v = rows(B * 2, hq), rows(B * 2, hkv), rows(B * 2, hkv)
    cu = torch.arange(0, 2 * B + 1, 2, dtype=torch.int32, device=DEV)
    out = cache.attend_shared(w.append(q, k, v, cu, offsets=offsets).view(B, 2, hq, d), w)
    torch.cuda.synchronize()
    check_step(q, k, v, out, 2, 0)
    q, k, v = rows(B, hq), rows(B, hkv), rows(B, hkv)
    out = cache.attend_shared(w.append(q, k, v, offsets=offsets), w)
    torch.cuda.synchronize()
    check_step(q, k, v, out, 1, 2)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        out = cache.attend_shared(w.append(q, k, v, offsets=offsets), w)
    for step in range(3, 6):
        q.copy_(rows(B, hq)), k.copy_(rows(B, hkv)), v.copy_(rows(B, hkv))
        graph.replay()
        torch.cuda.synchronize()
        check_step(q, k, v, out, 1, step)
    assert w.lens.cpu().tolist() == [6] * B and w.check_status()[0] == 0 and cache.check_status()[0] == 0


def test_shared_attention_on_two_streams():
    cache = make_cache([3000], 8, 2, 128)
    w = pq.PagedWindow(8, 8, 2, 128, 16, 32, torch.arange(32).view(8, 4), device=DEV)
    fill_window(w, [50] * 8, 3)
    qs = [synthetic.queries(i, 8, 8, 128, BF16, DEV) for i in range(2)]
    want = [cache.attend_shared(q, w) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            got[i].append(cache.attend_shared(qs[i], w, stream=s))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want[i]) for i in range(2) for x in got[i])


def test_two_captured_graphs_do_not_share_what_they_write_between():
    """Two graphs of the same calls, captured one after the other and replayed at once on two streams."""
    cache = make_cache([5000], 8, 2, 128)
    w = pq.PagedWindow(4, 8, 2, 128, 64, 128, torch.arange(128).view(4, 32), device=DEV)
    fill_window(w, [2000] * 4, 3)
    qs = [synthetic.queries(i, 4, 8, 128, BF16, DEV) for i in range(2)]
    want = [(cache.attend_shared(q, w), cache.attend_prefix(q), w.attend(q)) for q in qs]
    graphs, outs, streams = [], [], [torch.cuda.Stream() for _ in qs]
    for q in qs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append((cache.attend_shared(q, w), cache.attend_prefix(q), w.attend(q)))
    torch.cuda.synchronize()
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for got, wanted in zip(outs, want) for a, b in zip(got, wanted))


def test_a_serving_step_under_a_stream_of_its_own():
    """Everything on a side stream while the current one is busy with something else."""
    B, hq, hkv, d = 3, 8, 2, 128
    cache = make_cache([700], hq, hkv, d)
    offsets = cache.lens.repeat(B)
    side = torch.cuda.Stream()
    results = []
    for stream in (None, side):
        w = pq.PagedWindow(B, hq, hkv, d, 16, 6, torch.arange(6).view(B, 2), frequencies=pq.pq_rotary_frequencies(d), device=DEV)
        w.pool.zero_()
        g = torch.Generator(DEV).manual_seed(1)
        q, k, v = (torch.randn((B, h, d), generator=g, device=DEV).to(BF16) for h in (hq, hkv, hkv))
        torch.cuda.synchronize()
        if stream is not None:
            torch.empty(1 << 26, device=DEV).normal_()
        out = cache.attend_shared(w.append(q, k, v, offsets=offsets, stream=stream), w, stream=stream)
        torch.cuda.synchronize()
        results.append((out.clone(), w.pool.clone(), w.lens.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_refusals():
    cache = make_cache([100], 8, 2, 128)
    w = pq.PagedWindow(4, 8, 2, 128, 16, 16, torch.arange(16).view(4, 4), device=DEV)
    q = synthetic.queries(1, 4, 8, 128, BF16, DEV)
    for bad in (-1, 1):
        with pytest.raises(pq.PolarQuantError):
            cache.attend_prefix(q, seq=bad)
    with pytest.raises(pq.PolarQuantError):
        cache.attend_prefix(q[:, :7].contiguous())
    for args in [dict(q=q.cpu()), dict(q=q[:, :, :64].contiguous()), dict(q=q.transpose(0, 1)), dict(q=q, lse=torch.empty((4, 7), device=DEV)),
                 dict(q=q, out=torch.empty((4, 8, 128), device=DEV))]:
        with pytest.raises((AssertionError, pq.PolarQuantError)):
            cache.attend_prefix(**args)
    with pytest.raises((AssertionError, pq.PolarQuantError)):
        cache.attend_shared(q[:3].contiguous(), w)   # a window of another batch
    other = pq.PagedWindow(4, 8, 1, 128, 16, 16, torch.arange(16).view(4, 4), device=DEV)
    with pytest.raises((AssertionError, pq.PolarQuantError)):
        cache.attend_shared(q, other)
