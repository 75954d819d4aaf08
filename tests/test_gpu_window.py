"""The paged window on the GPU: rows with rotary positions on their way in, and the attention over it, against float64.

Tolerances.  A rotated value is a x + b y with |a|, |b| <= 1 in float32: the cosine and sine are off by at most 2^-22 (the turn
is reduced in float64 and rounded to float32, 2^-24 of a half turn times pi, and sincospif's 2 units in the last place), the
products and the sum by 3 * 2^-24 of |x| + |y|; 2^-20 (|x| + |y|) covers it with room, and bf16 adds half a step, 2^-8 of the
value at most.
Attention in float32 over n tokens: scores |s| <= scale |q||k| are off by (d + 8) 2^-24 of the sum of magnitudes at most, the
weights by that (relative), exp2 by 2 units, the sums by n 2^-24; with |s| and the sums' magnitudes below 16 here and n <= 2200
a bound of 2200 * 2^-24 + 2 * 136 * 16 * 2^-24 = 4e-4 of the largest value holds in the worst case; the errors add like a walk,
so 2e-5 absolute on outputs of magnitude 1 is what the tests hold them to, and half a step more for bf16 outputs."""
import numpy as np
import pytest
import torch

import paper_2502_02617_b200 as pq
from window_reference import attention, rotate, rows_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def f64(t):
    return t.detach().cpu().double().numpy()


def half_step(dtype):
    return 2.0 ** -8 if dtype == BF16 else 2.0 ** -24


def make_window(B, hq, hkv, d, P, most, dtype=BF16, seed=0, fill=None, **kw):
    pages = -(-most // P)
    table = torch.from_numpy(np.random.default_rng(seed).permutation(B * pages + 2)[:B * pages].reshape(B, pages).astype(np.int32))
    w = pq.PagedWindow(B, hq, hkv, d, P, B * pages + 2, table, dtype=dtype, device=DEV, **kw)
    if fill is None:
        w.pool.copy_(torch.randn(w.pool.shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV))
    else:
        w.pool.fill_(fill)
    return w


def fill_windows(w, lens, seed=1):
    """Values only where tokens are: everything else in the pool stays as it was."""
    g = torch.Generator(DEV).manual_seed(seed)
    for b, n in enumerate(lens):
        t = torch.arange(n, device=DEV)
        w.pool[w.page_table[b].long()[t // w.page_tokens], :, :, t % w.page_tokens] = torch.randn(
            (n, w.n_kv_heads, 2, w.d), generator=g, device=DEV).to(w.pool.dtype)
    w.lens.copy_(torch.tensor(lens, dtype=torch.int32))


# ---- append ------------------------------------------------------------------------------------------------------------


def check_append(w, counts, q, k, v, cu, offsets, before_pool, before_lens):
    """What `append` has left, against the reference: rotated queries, the pool as a whole, the lengths."""
    freq = np.zeros(0) if w.frequencies is None else f64(w.frequencies)
    table, P = w.page_table.cpu().numpy(), w.page_tokens
    seqs = np.repeat(np.arange(w.batch), counts)
    place = np.concatenate([n + np.arange(c) for n, c in zip(before_lens, counts)] + [np.zeros(0)]).astype(np.int64)
    off = np.zeros(w.batch, dtype=np.int64) if offsets is None else offsets.cpu().numpy().astype(np.int64)
    pos = place + off[seqs]
    n = len(seqs)
    want = before_pool.copy()
    bound = np.zeros_like(want)
    kk = f64(k)[:n]
    want[table[seqs, place // P], :, 0, place % P] = rotate(kk, pos, freq, w.interleaved)
    want[table[seqs, place // P], :, 1, place % P] = f64(v)[:n]
    bound[table[seqs, place // P], :, 0, place % P] = 2.0 ** -20 * 2 * np.abs(kk).max() if n else 0
    got = f64(w.pool)
    same = np.isnan(want) & np.isnan(got)
    assert np.all(same | (np.abs(got - want) <= bound * (1 + half_step(w.pool.dtype)) + half_step(w.pool.dtype) * np.abs(want) * (bound > 0)))
    assert w.lens.cpu().tolist() == [a + c for a, c in zip(before_lens, counts)]
    if q is None:
        return None
    return rotate(f64(q)[:n], pos, freq, w.interleaved)


@pytest.mark.parametrize("d,hq,hkv,dtype,rotary,interleaved,P", [
    (128, 8, 2, BF16, 128, False, 64), (128, 8, 2, BF16, 128, True, 16), (128, 4, 4, F32, 64, False, 48), (128, 7, 1, BF16, 32, True, 16),
    (64, 4, 2, BF16, 64, False, 16), (64, 4, 2, F32, 64, True, 256), (64, 2, 1, BF16, 6, False, 16), (32, 2, 2, BF16, 32, False, 16),
    (16, 2, 1, F32, 16, False, 16), (16, 3, 1, BF16, 10, True, 16), (128, 8, 2, BF16, 0, False, 16)])
@pytest.mark.parametrize("kind", ["one", "ragged", "packed"])
def test_append(d, hq, hkv, dtype, rotary, interleaved, P, kind):
    """One row each; ragged chunks (none, one, several pages) with rows behind the last sequence; rows of one projection."""
    rng = np.random.default_rng(3)
    before = [0, 5, 15, 16, 37]
    B = len(before)
    counts = [1] * B if kind == "one" else [0, 1, 40, 17, 300]
    spare = 0 if kind == "one" else 3
    w = make_window(B, hq, hkv, d, P, 400, dtype, seed=5, interleaved=interleaved,
                    frequencies=pq.pq_rotary_frequencies(rotary, 10000.0) if rotary else None)
    w.lens.copy_(torch.tensor(before, dtype=torch.int32))
    n = sum(counts) + spare
    g = torch.Generator(DEV).manual_seed(7)
    if kind == "packed":
        rows = torch.randn((n, hq + 2 * hkv, d), generator=g, device=DEV).to(dtype)
        q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    else:
        q, k, v = (torch.randn((n, h, d), generator=g, device=DEV).to(dtype) for h in (hq, hkv, hkv))
    cu = None if kind == "one" else torch.tensor(np.concatenate(([0], np.cumsum(counts))), dtype=torch.int32, device=DEV)
    offsets = torch.tensor(rng.integers(0, 200000, B), dtype=torch.int32, device=DEV)
    pool = f64(w.pool)
    q_out = torch.full(q.shape, 7.0, dtype=dtype, device=DEV)
    got = w.append(q, k, v, cu, offsets=offsets, q_out=q_out)
    torch.cuda.synchronize()
    assert got is q_out and w.check_status()[0] == 0
    want = check_append(w, counts, q, k, v, cu, offsets, pool, before)
    n = len(want)
    assert np.all(np.abs(f64(got)[:n] - want) <= 2.0 ** -19 * np.abs(f64(q)).max() * (1 + half_step(dtype)) + half_step(dtype) * np.abs(want))
    assert bool((got[n:] == 7.0).all())   # rows behind the last sequence are left as they were


@pytest.mark.parametrize("total", [1, 2, 257, 5000])
@pytest.mark.parametrize("B", [1, 2, 300])
def test_append_many_shapes(B, total):
    """Few and many rows over few and many sequences, most of them without any."""
    d, hq, hkv, P = 64, 2, 1, 16
    rng = np.random.default_rng(B * 7 + total)
    counts = np.bincount(rng.integers(0, B, total), minlength=B).tolist()
    before = rng.integers(0, 40, B).tolist()
    w = make_window(B, hq, hkv, d, P, max(a + c for a, c in zip(before, counts)), frequencies=pq.pq_rotary_frequencies(d, 500000.0))
    w.lens.copy_(torch.tensor(before, dtype=torch.int32))
    g = torch.Generator(DEV).manual_seed(total)
    q, k, v = (torch.randn((total, h, d), generator=g, device=DEV).to(BF16) for h in (hq, hkv, hkv))
    cu = torch.tensor(np.concatenate(([0], np.cumsum(counts))), dtype=torch.int32, device=DEV)
    pool = f64(w.pool)
    got = w.append(q, k, v, cu)
    torch.cuda.synchronize()
    assert w.check_status()[0] == 0
    want = check_append(w, counts, q, k, v, cu, None, pool, before)
    assert np.all(np.abs(f64(got) - want) <= 2.0 ** -18 * 5 + 2.0 ** -8 * np.abs(want))


def test_positions_beyond_a_million_keep_their_angles():
    """Float32 angles would be off by more than a tenth of a radian here."""
    d = 128
    w = make_window(2, 2, 1, d, 16, 16, F32, frequencies=pq.pq_rotary_frequencies(d, 500000.0))
    offsets = torch.tensor([(1 << 31) - 20, 1 << 21], dtype=torch.int32, device=DEV)
    g = torch.Generator(DEV).manual_seed(1)
    q, k, v = (torch.randn((2, h, d), generator=g, device=DEV) for h in (2, 1, 1))
    w.lens.fill_(9)
    got = w.append(q, k, v, offsets=offsets)
    pos = offsets.cpu().numpy().astype(np.int64) + 9
    want = rotate(f64(q), pos, f64(w.frequencies), False)
    assert np.max(np.abs(f64(got) - want)) <= 2.0 ** -19 * np.abs(f64(q)).max()


@pytest.mark.parametrize("dtype,skew", [(BF16, 1), (BF16, 4), (F32, 1), (F32, 2)])
def test_rows_of_any_alignment(dtype, skew):
    """Rows that do not start on 16 bytes, strides that are no multiple of them, in place for the queries."""
    d, hq, hkv, n = 64, 2, 1, 5
    g = torch.Generator(DEV).manual_seed(2)
    buf = torch.randn(3 * n * (hq * d + 9) + 16, generator=g, device=DEV).to(dtype)
    q = buf.as_strided((n, hq, d), (hq * d + 9, d + 1, 1), skew)
    k = buf.as_strided((n, hkv, d), (hq * d + 9, d + 1, 1), n * (hq * d + 9) + skew)
    v = buf.as_strided((n, hkv, d), (hq * d + 9, d + 1, 1), 2 * n * (hq * d + 9) + skew)
    w = make_window(n, hq, hkv, d, 16, 16, dtype, frequencies=pq.pq_rotary_frequencies(d))
    w.lens.fill_(3)
    pool = f64(w.pool)
    got = w.append(q, k, v)
    torch.cuda.synchronize()
    want = check_append(w, [1] * n, q, k, v, None, None, pool, [3] * n)
    assert np.all(np.abs(f64(got) - want) <= 2.0 ** -18 * 5 + half_step(dtype) * np.abs(want))
    q2 = q.contiguous()
    assert torch.equal(w.append(q2, k, v, q_out=q2), w_again(w, q, k, v))


def w_again(w, q, k, v):
    w.lens.fill_(4)
    return w.append(q, k, v)


def test_append_in_place_and_without_queries():
    d, hq, hkv, B = 128, 4, 2, 3
    w = make_window(B, hq, hkv, d, 16, 64, frequencies=pq.pq_rotary_frequencies(d))
    g = torch.Generator(DEV).manual_seed(4)
    q, k, v = (torch.randn((B, h, d), generator=g, device=DEV).to(BF16) for h in (hq, hkv, hkv))
    want = w.append(q, k, v).clone()
    pool = w.pool.clone()
    w.lens.zero_()
    same = q.clone()
    assert w.append(same, k, v, q_out=same) is same and torch.equal(same, want) and torch.equal(w.pool, pool)
    w.lens.zero_()
    w.pool.normal_()
    assert w.append(None, k, v) is None
    t = w.page_table[:, 0].long()
    assert torch.equal(w.pool[t, :, :, 0], pool[t, :, :, 0]) and w.lens.cpu().tolist() == [1] * B


def test_append_reports_what_does_not_fit():
    """A full window and a page outside the pool: nothing of the sequence is written (of the bad page: its rows), neither grows,
    the others do, and the queries are rotated all the same."""
    d, hq, hkv, P = 64, 2, 1, 16
    for bad in ("capacity", "page"):
        w = make_window(3, hq, hkv, d, P, 32, frequencies=pq.pq_rotary_frequencies(d), seed=3)
        w.lens.copy_(torch.tensor([3, 30, 5], dtype=torch.int32))
        counts = [4, 3 if bad == "capacity" else 2, 1]
        if bad == "page":
            w.page_table[1, 1] = w.n_pages
        n = sum(counts)
        g = torch.Generator(DEV).manual_seed(6)
        q, k, v = (torch.randn((n, h, d), generator=g, device=DEV).to(BF16) for h in (hq, hkv, hkv))
        cu = torch.tensor(np.concatenate(([0], np.cumsum(counts))), dtype=torch.int32, device=DEV)
        pool = w.pool.clone()
        got = w.append(q, k, v, cu)
        torch.cuda.synchronize()
        assert w.status.cpu().tolist()[0] == (pq.ERR_CAPACITY if bad == "capacity" else pq.ERR_INVALID_ARG)
        assert w.lens.cpu().tolist() == [7, 30, 6]
        for page in set(range(w.n_pages)) - {int(w.page_table[0, 0]), int(w.page_table[2, 0])}:
            assert torch.equal(w.pool[page], pool[page])
        pos = np.concatenate([3 + np.arange(4), 30 + np.arange(counts[1]), [5]])
        assert np.all(np.abs(f64(got) - rotate(f64(q), pos, f64(w.frequencies), False)) <= 2.0 ** -7 * 5)
        with pytest.raises(pq.PolarQuantError):
            w.check_status()


@pytest.mark.parametrize("d,rotary", [(64, 64), (16, 6)])   # rows as 16-byte pieces, and pair by pair
@pytest.mark.parametrize("ends", [[0, 60, 30, 5, 60], [0, 60, -7, 60, 60], [0, 40, 20, 200, 60]])
def test_ends_that_do_not_rise_write_into_no_other_sequence(ends, d, rotary):
    """cu_seqlens that fall, or lie beyond the rows: rows may be refused, but nothing outside the sequences' own pages changes."""
    B, hq, hkv, P, n = 4, 2, 1, 16, 60
    w = make_window(B, hq, hkv, d, P, 128, frequencies=pq.pq_rotary_frequencies(rotary), seed=4)
    own = w.page_table.clone()
    g = torch.Generator(DEV).manual_seed(7)
    q, k, v = (torch.randn((n, h, d), generator=g, device=DEV).to(BF16) for h in (hq, hkv, hkv))
    pool = w.pool.clone()
    w.append(q, k, v, torch.tensor(ends, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    lens = w.lens.cpu().tolist()
    assert all(0 <= m <= max(0, b - a) for m, a, b in zip(lens, ends, ends[1:])), lens
    assert torch.equal(w.page_table, own)
    for page in set(range(w.n_pages)) - set(own.flatten().tolist()):
        assert torch.equal(w.pool[page], pool[page])


def test_append_refuses_tensors_that_do_not_fit():
    w = make_window(2, 4, 2, 64, 16, 32, frequencies=pq.pq_rotary_frequencies(64))
    ok = dict(q=torch.zeros((2, 4, 64), dtype=BF16, device=DEV), k=torch.zeros((2, 2, 64), dtype=BF16, device=DEV), v=torch.zeros((2, 2, 64), dtype=BF16, device=DEV))
    w.append(**ok)
    for name, bad in [("k", torch.zeros((2, 1, 64), dtype=BF16, device=DEV)), ("k", torch.zeros((2, 2, 64), device=DEV)), ("v", torch.zeros((3, 2, 64), dtype=BF16, device=DEV)),
                      ("q", torch.zeros((2, 4, 64), device=DEV)), ("q", torch.zeros((1, 4, 64), dtype=BF16, device=DEV)),
                      ("cu_seqlens", torch.zeros(2, dtype=torch.int32, device=DEV)), ("cu_seqlens", torch.zeros(3, dtype=torch.int64, device=DEV)),
                      ("offsets", torch.zeros(3, dtype=torch.int32, device=DEV)), ("offsets", torch.zeros(2, dtype=torch.int32)),
                      ("q_out", torch.zeros((2, 4, 32), dtype=BF16, device=DEV))]:
        with pytest.raises(AssertionError):
            w.append(**{**ok, name: bad})
    with pytest.raises(AssertionError):
        w.append(ok["q"].cpu(), ok["k"].cpu(), ok["v"].cpu())
    with pytest.raises(pq.PolarQuantError):
        w.append(torch.zeros((1, 4, 64), dtype=BF16, device=DEV), torch.zeros((1, 2, 64), dtype=BF16, device=DEV), torch.zeros((1, 2, 64), dtype=BF16, device=DEV))


# ---- attention ---------------------------------------------------------------------------------------------------------


def check_attention(w, lens, q, out, lse, scale):
    multi = q.dim() == 4
    pool, table = f64(w.pool), w.page_table.cpu().numpy()
    for b, n in enumerate(lens):
        K, V = rows_of(pool, table, w.page_tokens, b, n)
        qb = f64(q[b]) if multi else f64(q[b])[None]
        want, want_lse = attention(qb, K, V, scale)
        got = f64(out[b]) if multi else f64(out[b])[None]
        assert np.all(np.abs(got - want) <= 2e-5 + half_step(q.dtype) * np.abs(want)), (b, n, np.abs(got - want).max())
        if lse is not None:
            got = f64(lse[b]) if multi else f64(lse[b])[None]
            assert np.array_equal(np.isinf(got), np.isinf(want_lse)) and np.all(np.abs(got - want_lse)[np.isfinite(want_lse)] <= 2e-5), (b, n)


@pytest.mark.parametrize("io", [BF16, F32])
@pytest.mark.parametrize("d,hq,hkv,dtype,P", [(128, 8, 2, BF16, 16), (128, 7, 1, BF16, 64), (128, 2, 2, F32, 48), (128, 8, 1, F32, 16), (64, 4, 2, BF16, 16),
                                              (64, 6, 1, F32, 32), (32, 4, 1, BF16, 16), (32, 2, 1, F32, 16), (16, 2, 1, BF16, 16), (16, 4, 1, F32, 16),
                                              (16, 1, 1, BF16, 16), (64, 32, 2, BF16, 16)])
def test_window_attention(d, hq, hkv, dtype, P, io):
    """One query each over windows of no token, one, around the pieces a block takes, and several clusters' worth; what lies past
    the ends is NaN."""
    lens = [0, 1, 7, 15, 16, 17, 128, 130, 700, 2177]
    w = make_window(len(lens), hq, hkv, d, P, max(lens) + 5, dtype, seed=d + hq, fill=float("nan"))
    fill_windows(w, lens)
    q = torch.randn((len(lens), hq, d), generator=torch.Generator(DEV).manual_seed(9), device=DEV).to(io)
    lse = torch.empty((len(lens), hq), device=DEV)
    scale = d ** -0.5
    out = w.attend(q, lse=lse)
    torch.cuda.synchronize()
    assert w.check_status()[0] == 0
    check_attention(w, lens, q, out, lse, scale)
    again = w.attend(q)   # without the log-sum-exps an empty window is an error
    torch.cuda.synchronize()
    assert w.status.cpu().tolist()[0] == pq.ERR_EMPTY and torch.equal(again, out)


@pytest.mark.parametrize("n_q", [2, 3, 5, 8, 17, 64])
@pytest.mark.parametrize("d,hq,hkv,dtype", [(128, 8, 2, BF16), (128, 7, 1, BF16), (64, 4, 2, BF16), (64, 16, 1, BF16), (64, 2, 2, F32), (16, 4, 1, F32)])
def test_several_queries_are_causal(d, hq, hkv, dtype, n_q):
    """Windows shorter than the chunk (queries that see nothing), as long, and longer; the last tokens' keys are infinite and their
    values NaN for the queries that must not see them."""
    lens = [0, 1, n_q - 1, n_q, n_q + 1, 16, 40, 333, 1200]
    w = make_window(len(lens), hq, hkv, d, 16, max(lens) + 3, dtype, seed=n_q, fill=float("nan"))
    fill_windows(w, lens)
    q = torch.randn((len(lens), n_q, hq, d), generator=torch.Generator(DEV).manual_seed(n_q), device=DEV).to(BF16 if dtype == BF16 else F32)
    lse = torch.empty((len(lens), n_q, hq), device=DEV)
    out = w.attend(q, lse=lse)
    torch.cuda.synchronize()
    check_attention(w, lens, q, out, lse, d ** -0.5)
    for b, n in enumerate(lens):   # only the last query sees the last token
        if n:
            w.pool[int(w.page_table[b, (n - 1) // 16]), :, 0, (n - 1) % 16] = float("inf")
            w.pool[int(w.page_table[b, (n - 1) // 16]), :, 1, (n - 1) % 16] = float("nan")
    hidden = w.attend(q, lse=lse)
    torch.cuda.synchronize()
    if dtype == F32:
        assert torch.equal(hidden[:, :-1], out[:, :-1])
    else:
        assert torch.allclose(hidden[:, :-1].float(), out[:, :-1].float(), atol=2e-5, rtol=2.0 ** -7)


def test_scores_of_minus_infinity_and_infinity():
    """A key whose score is -inf weighs nothing; a window of nothing else gives zeros; a NaN key spoils only its own heads."""
    B, hq, hkv, d, n = 3, 4, 2, 128, 200
    w = make_window(B, hq, hkv, d, 16, 256, seed=1)
    fill_windows(w, [n] * B)
    q = torch.randn((B, hq, d), generator=torch.Generator(DEV).manual_seed(3), device=DEV).to(BF16).abs() + 0.5
    w.pool[int(w.page_table[0, 3]), :, 0, 5] = -float("inf")
    w.pool[w.page_table[1].long(), :, 0] = -float("inf")
    w.pool[int(w.page_table[2, 3]), 0, 0, 5, 7] = float("nan")
    lse = torch.empty((B, hq), device=DEV)
    out = w.attend(q, lse=lse)
    torch.cuda.synchronize()
    K, V = rows_of(f64(w.pool), w.page_table.cpu().numpy(), 16, 0, n)
    keep = np.arange(n) != 3 * 16 + 5
    want, _ = attention(f64(q[0])[None], K[keep], V[keep], d ** -0.5)
    assert np.all(np.abs(f64(out[0]) - want[0]) <= 2e-5 + 2.0 ** -8 * np.abs(want[0]))
    assert bool((out[1] == 0).all()) and bool((lse[1] == -float("inf")).all())
    assert bool(torch.isnan(out[2, :2]).all()) and bool(torch.isfinite(out[2, 2:]).all())


def test_large_scores_do_not_overflow():
    B, hq, hkv, d = 1, 4, 1, 64
    w = make_window(B, hq, hkv, d, 16, 600, seed=2)
    fill_windows(w, [600])
    w.pool[:, :, 0] *= 40
    q = 40 * torch.randn((B, hq, d), generator=torch.Generator(DEV).manual_seed(3), device=DEV)
    out = w.attend(q, scale=1.0)
    K, V = rows_of(f64(w.pool), w.page_table.cpu().numpy(), 16, 0, 600)
    want, _ = attention(f64(q[0])[None], K, V, 1.0)
    # the 64 products of a score have magnitudes around 1600 (1e5 in all): its float32 sum may be off by 64 * 1e5 * 2^-24 = 0.4 at worst, a
    # few hundredths as a walk, and where two scores are that close, a weight by as much: 0.1 of a value of magnitude 3
    assert np.max(np.abs(f64(out[0]) - want[0])) < 0.3


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,hq,hkv", [(1, 3, 1), (70, 1, 1), (80, 2, 1), (45, 4, 2), (120, 1, 1), (150, 2, 1), (240, 1, 1), (500, 1, 1)])
def test_clusters_of_every_size(B, hq, hkv, dtype):
    """Batches that leave room for eight blocks a window, seven, six, ... one (on 148 SMs)."""
    w = make_window(B, hq, hkv, 64, 16, 272, seed=B, dtype=dtype)
    lens = [272 - (b * 37) % 130 if b % 9 else b % 3 for b in range(B)]
    fill_windows(w, lens)
    q = torch.randn((B, hq, 64), generator=torch.Generator(DEV).manual_seed(B), device=DEV).to(dtype)
    lse = torch.empty((B, hq), dtype=torch.float32, device=DEV)
    out = w.attend(q, lse=lse)
    torch.cuda.synchronize()
    check_attention(w, lens, q, out, lse, 64 ** -0.5)


@pytest.mark.parametrize("max_len", [1, 128, 1024, 100000])
def test_a_bound_on_the_lengths_changes_only_the_cut(max_len):
    lens = [900, 3]
    w = make_window(2, 8, 2, 128, 16, 1000, seed=4)
    fill_windows(w, lens)
    q = torch.randn((2, 8, 128), generator=torch.Generator(DEV).manual_seed(3), device=DEV)
    lse = torch.empty((2, 8), device=DEV)
    out = w.attend(q, max_len=max_len, lse=lse)
    torch.cuda.synchronize()
    check_attention(w, lens, q, out, lse, 128 ** -0.5)


def test_a_page_outside_the_pool_is_reported():
    w = make_window(2, 4, 2, 64, 16, 64, seed=4)
    fill_windows(w, [40, 40])
    q = torch.randn((2, 4, 64), generator=torch.Generator(DEV).manual_seed(3), device=DEV).to(BF16)
    good = w.attend(q)
    w.page_table[1, 1] = -1
    out = w.attend(q)
    torch.cuda.synchronize()
    assert w.status.cpu().tolist()[0] == pq.ERR_INVALID_ARG and torch.equal(out[0], good[0])


def test_append_and_attend_in_a_captured_graph():
    """Eight generation steps replayed from one graph: positions and lengths advance on the device."""
    B, hq, hkv, d = 3, 4, 2, 64
    make = lambda: make_window(B, hq, hkv, d, 16, 64, seed=8, frequencies=pq.pq_rotary_frequencies(d))  # noqa: E731
    g = torch.Generator(DEV).manual_seed(5)
    steps = [[torch.randn((B, h, d), generator=g, device=DEV).to(BF16) for h in (hq, hkv, hkv)] for _ in range(8)]
    eager, w = make(), make()
    want = []
    for q, k, v in steps:
        want.append(eager.attend(eager.append(q, k, v)).clone())
    q, k, v = (torch.zeros_like(x) for x in steps[0])
    w.attend(w.append(q, k, v))
    w.lens.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            out = w.attend(w.append(q, k, v))
    torch.cuda.synchronize()
    w.pool.copy_(make().pool)
    w.lens.zero_()
    for (a, b, c), wanted in zip(steps, want):
        q.copy_(a), k.copy_(b), v.copy_(c)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, wanted)
    assert w.lens.cpu().tolist() == [8] * B and torch.equal(w.pool, eager.pool) and w.check_status()[0] == 0


def test_a_capture_on_a_stream_that_is_not_current_takes_a_workspace_of_its_own():
    """A long window (parts in the workspace), captured through stream=: calls outside the graph may run beside its replays."""
    w = make_window(1, 8, 2, 128, 64, 20000, seed=3)
    fill_windows(w, [20000])
    q = torch.randn((1, 8, 128), generator=torch.Generator(DEV).manual_seed(1), device=DEV).to(BF16)
    side, out = torch.cuda.Stream(), torch.empty_like(q)
    want = w.attend(q, stream=side)
    torch.cuda.synchronize()
    kept = {k: t.data_ptr() for k, t in w._ws.items()}
    assert side.cuda_stream in kept
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        graph.capture_begin(capture_error_mode="thread_local")
    w.attend(q, out=out, stream=side)
    with torch.cuda.stream(side):
        graph.capture_end()
    assert {k: t.data_ptr() for k, t in w._ws.items()} == kept
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_an_append_of_no_rows_changes_nothing():
    w = make_window(2, 4, 2, 64, 16, 32, frequencies=pq.pq_rotary_frequencies(64))
    w.lens.copy_(torch.tensor([3, 0], dtype=torch.int32))
    pool = w.pool.clone()
    q, k, v = (torch.empty((0, h, 64), dtype=BF16, device=DEV) for h in (4, 2, 2))
    assert w.append(q, k, v, torch.zeros(3, dtype=torch.int32, device=DEV)).shape == q.shape
    assert w.lens.cpu().tolist() == [3, 0] and torch.equal(w.pool, pool) and w.check_status()[0] == pq.OK


def test_calls_on_two_streams_do_not_disturb_each_other():
    """Long windows of one sequence (parts in the workspace) attended on two streams at once."""
    w = make_window(1, 8, 2, 128, 64, 20000, seed=3)
    fill_windows(w, [20000])
    qs = [torch.randn((1, 8, 128), generator=torch.Generator(DEV).manual_seed(i), device=DEV).to(BF16) for i in range(2)]
    want = [w.attend(q) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            got[i].append(w.attend(qs[i], stream=s))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])
