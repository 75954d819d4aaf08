"""The operators of a serving step around the compressed KV cache that are timed on their own: the rotary position of new
rows on their way into a paged 16-bit window, the attention over that window, the attention of a whole batch over one
compressed prefix that all its sequences share, and the two attentions as one.

A case is a dict of plain values.  `call` says which operator:

  append   rotate the new rows of queries and keys of every sequence by their positions, put keys and values behind what
           the window's pages hold already, and return the rotated queries
  window   the last `n_q` positions of every sequence attend causally over the sequence's pages
  prefix   every query of the batch attends over the same compressed prefix
  shared   every query attends over the compressed prefix and, causally, over its own sequence's window

Rotary angles are position * frequency; the element pairs are (i, i + rotary / 2), or (2i, 2i + 1) where `interleaved`.
The window is a pool [page][kv head][K | V][token of the page][head_dim] behind a table [sequence][logical page].  The
prefix is the packed cache of one sequence: [kv head][block of 64 tokens][K | V][planes of the codes of levels 1 to 4 and of
the radii], angles of a polar recursion over 16 coordinates in 4, 2, 2 and 2 bits, keys and values in a basis rotated by S.
"""
from __future__ import annotations

import functools
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LEVEL_BITS = (4, 2, 2, 2)
BLOCK = 64          # tokens of a block of the packed cache
THETA = 500000.0    # base of the rotary frequencies


def _case(call, **kw):
    c = {"call": call, "batch": 1, "n_q": 1, "prefix": 0, "window": 0, "spread": 1.0, "q_heads": 32, "kv_heads": 8, "head_dim": 128,
         "dtype": "bf16", "page_tokens": 64, "rotary": 128, "interleaved": False, "packed_qkv": True, "far": 0}
    c.update(kw)
    return c


def listed():
    return [
        # One token of one interactive session goes into the window of a layer: latency is all there is.
        _case("append", name="append_b1", batch=1, window=700, far=131072),
        # A step with drafted tokens of a small model in float32: 1 to 9 new tokens a sequence, half of the head rotated, pairs
        # side by side, separate projections.
        _case("append", name="append_draft_b16_d64_f32", batch=16, n_q=9, spread=9.0, window=500, q_heads=16, head_dim=64, dtype="f32",
              rotary=32, interleaved=True, packed_qkv=False, page_tokens=16, far=32768),
        # Four prompts of uneven length, 32k tokens and fewer, whose rows come out of one projection.
        _case("append", name="append_prompts_32k", batch=4, n_q=16384, spread=4.0, window=40, far=8192, page_tokens=256),
        # The first generated tokens of a session.
        _case("window", name="window_b1_300", batch=1, window=300),
        # Five drafted tokens are verified in eight sequences, seven query heads per kv head.
        _case("window", name="window_draft5_b8_2k", batch=8, n_q=5, window=2048, spread=3.0, q_heads=28, kv_heads=4, page_tokens=16),
        # A small model in float32.
        _case("window", name="window_d64_f32_b4_1k", batch=4, window=1000, spread=2.0, q_heads=16, head_dim=64, rotary=64, dtype="f32"),
        # A loaded server: sixty-four sequences that have generated up to 4k tokens each.
        _case("window", name="window_b64_4k", batch=64, window=4096, spread=4.0),
        # A short system prompt that a few sessions share.
        _case("prefix", name="prefix_b4_2k", batch=4, prefix=2000),
        # One document of 32k tokens, 64 questions about it.
        _case("prefix", name="prefix_b64_32k", batch=64, prefix=32768),
        # A smaller model's heads.
        _case("prefix", name="prefix_d64_b16_4k", batch=16, prefix=4096, q_heads=16, head_dim=64, rotary=64),
        # The attention of a whole step: a shared document of 16k tokens and the tokens generated so far.
        _case("shared", name="shared_b16_16k_w500", batch=16, prefix=16384, window=500, spread=5.0),
        # A large batch over a long document, each sequence with two new positions.
        _case("shared", name="shared_b128_64k_w1000", batch=128, n_q=2, prefix=65536, window=1000, spread=8.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same calls, sizes spread over the whole range of each, odd ones included."""
    most = max(_cost(c) for c in listed())
    while True:
        call = rng.choice(["append", "append", "window", "window", "prefix", "shared", "shared"])
        q_heads, kv_heads, d = rng.choice([(32, 8, 128), (32, 8, 128), (28, 4, 128), (16, 2, 128), (12, 12, 128), (16, 8, 64)])
        c = _case(call, q_heads=q_heads, kv_heads=kv_heads, head_dim=d, rotary=rng.choice([d, d, d // 2]), interleaved=rng.random() < 0.3,
                  packed_qkv=rng.random() < 0.7, page_tokens=rng.choice([16, 64, 256]), spread=rng.choice([1.0, round(rng.uniform(1.5, 16.0), 2)]),
                  far=rng.choice([0, _log_int(rng, 1, 1 << 20)]))
        if call == "append":
            c.update(batch=_log_int(rng, 1, 128), n_q=_log_int(rng, 1, 16384), window=_log_int(rng, 1, 4096), dtype=rng.choice(["bf16", "bf16", "f32"]))
        elif call == "window":
            c.update(batch=_log_int(rng, 1, 64), n_q=rng.choice([1, 1, _log_int(rng, 1, 16)]), window=_log_int(rng, 1, 8192),
                     dtype=rng.choice(["bf16", "bf16", "f32"]))
        elif call == "prefix":
            c.update(batch=_log_int(rng, 1, 256), prefix=_log_int(rng, 1, 65536))
        else:
            c.update(batch=_log_int(rng, 1, 128), n_q=rng.choice([1, 1, _log_int(rng, 1, 4)]), prefix=_log_int(rng, 64, 65536),
                     window=_log_int(rng, 1, 2000))
        if d < 128 and c["prefix"] * c["batch"] * c["n_q"] > 131072:   # the smaller heads belong to smaller models
            continue
        if _cost(c) <= most and sum(_new(c)) <= 65536 and sum(_windows(c)) <= 300000:
            return c


def _uneven(seed, count, top, spread):
    """`count` lengths from top / spread to top, the first of them `top`."""
    low = max(1, int(top / spread))
    r = random.Random(seed)
    return [top] + [r.randint(low, top) for _ in range(count - 1)]


def _new(case):
    """New tokens of each sequence."""
    B, top = case["batch"], case["n_q"]
    return _uneven(B * 1000003 + top, B, top, case["spread"]) if case["call"] == "append" else [top] * B


def _windows(case):
    """Tokens in each sequence's window (of an append: before it)."""
    if case["window"] == 0:
        return [0] * case["batch"]
    lens = _uneven(case["batch"] * 7919 + case["window"], case["batch"], case["window"], case["spread"])
    return lens if case["call"] == "append" else [max(n, case["n_q"]) for n in lens]


def _packed_bytes(d):
    """Bytes of one compressed vector: code planes of whole bytes and an fp16 radius for 16 coordinates."""
    nb = d // 16
    return 4 * nb + nb + max(1, nb // 2) + max(1, nb // 4) + 2 * nb


def work(case):
    d, hq, hkv = case["head_dim"], case["q_heads"], case["kv_heads"]
    size, B, n_q = (4 if case["dtype"] == "f32" else 2), case["batch"], case["n_q"]
    if case["call"] == "append":
        n = sum(_new(case))
        return {"bytes": 2.0 * n * (hq + 2 * hkv) * d * size, "flops": 3.0 * n * (hq + hkv) * case["rotary"]}
    rows = B * n_q
    bytes_, pairs = 2.0 * rows * hq * d * size, 0
    if case["call"] in ("window", "shared"):
        lens = _windows(case)
        bytes_ += 2.0 * sum(lens) * hkv * d * size
        pairs += sum(n_q * n - n_q * (n_q - 1) // 2 for n in lens)
    if case["call"] in ("prefix", "shared"):
        bytes_ += 2.0 * case["prefix"] * hkv * _packed_bytes(d) + 4.0 * d * d
        pairs += rows * case["prefix"]
    return {"bytes": bytes_, "flops": 4.0 * d * hq * pairs}


def _cost(case):
    w = work(case)
    return w["bytes"] / 6e12 + w["flops"] / 1e15


# ---- inputs ------------------------------------------------------------------------------------------------------------


@functools.lru_cache(maxsize=None)
def _codebooks():
    """Per level, the centroids that minimise the mean squared error for angles of Gaussian vectors: uniform on the circle at
    level 1, density proportional to sin(2 psi)^(2^(l-1) - 1) on [0, pi/2] at level l (Lloyd's iteration on a fine grid)."""
    out = []
    for level, bits in enumerate(LEVEL_BITS, 1):
        n, top = 1 << bits, 2 * math.pi if level == 1 else math.pi / 2
        c = (torch.arange(n, dtype=torch.float64) + 0.5) * (top / n)
        if level > 1:
            x = (torch.arange(200000, dtype=torch.float64) + 0.5) * (top / 200000)
            w = torch.sin(2 * x) ** (2 ** (level - 1) - 1)
            for _ in range(400):
                cell = torch.bucketize(x, (c[1:] + c[:-1]) / 2)
                c = torch.zeros(n, dtype=torch.float64).index_add_(0, cell, w * x) / torch.zeros(n, dtype=torch.float64).index_add_(0, cell, w)
        out.append(c)
    return out


def _generator(seed, device):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    return g


def _pack(y):
    """[heads, tokens, d] in the rotated basis -> packed planes, uint8 [heads, blocks, bytes of a block]; tokens past the end are 0xFF."""
    H, N, d = y.shape
    nb, planes, r = d // 16, [], y
    for level, cen in enumerate(_codebooks(), 1):
        a, b = r[..., 0::2].contiguous(), r[..., 1::2].contiguous()
        angle = torch.atan2(b, a)
        if level == 1:
            angle = torch.where(angle < 0, angle + 2 * math.pi, angle)
        code = torch.bucketize(angle, ((cen[1:] + cen[:-1]) / 2).to(angle), out_int32=True)
        r = torch.hypot(a, b)
        per = 8 // LEVEL_BITS[level - 1]                                      # codes of a byte, first one lowest
        code = torch.nn.functional.pad(code, (0, -code.shape[-1] % per)).unflatten(-1, (-1, per))
        planes.append((code << (torch.arange(per, device=y.device, dtype=torch.int32) * LEVEL_BITS[level - 1])).sum(-1).to(torch.uint8))
    planes.append(r.to(torch.float16).contiguous().view(torch.uint8))
    blocks = -(-N // BLOCK)
    full = [torch.nn.functional.pad(p, (0, 0, 0, blocks * BLOCK - N), value=255).view(H, blocks, -1) for p in planes]
    out = torch.cat(full, -1)
    assert out.shape[-1] == BLOCK * _packed_bytes(d) and nb == r.shape[-1]
    return out


def _prefix(case, seed, device):
    """A prompt's keys (four large channels a head) and values, compressed."""
    d, hkv, n = case["head_dim"], case["kv_heads"], case["prefix"]
    g = _generator(seed, device)
    S = torch.linalg.qr(torch.randn((d, d), generator=_generator(seed ^ 0x5A, "cpu"), dtype=torch.float64))[0].float().to(device)
    scale = torch.ones((hkv, 1, d), device=device)
    scale.scatter_(2, torch.rand((hkv, 1, d), generator=g, device=device).argsort(-1)[..., :4], 10.0)
    k = torch.randn((hkv, n, d), generator=g, device=device) * scale
    v = torch.randn((hkv, n, d), generator=g, device=device)
    packed = torch.stack([_pack(k.bfloat16().float() @ S), _pack(v.bfloat16().float() @ S)], 2)   # [head][block][K | V][bytes]
    return S, packed.contiguous()


def prepare(case, seed):
    device = torch.device("cuda")
    d, hq, hkv, B, P = case["head_dim"], case["q_heads"], case["kv_heads"], case["batch"], case["page_tokens"]
    dtype, g = DTYPES[case["dtype"]], _generator(seed, device)
    s = {"case": dict(case), "scale": d ** -0.5}
    lens, new = _windows(case), _new(case)
    if case["call"] != "prefix":
        most = max(n + (m if case["call"] == "append" else 0) for n, m in zip(lens, new))
        pages = -(-most // P)
        used = B * pages
        order = torch.randperm(used + 3, generator=_generator(seed ^ 0x7AB1E, "cpu"))[:used]
        s["table"] = order.view(B, pages).to(torch.int32).to(device)
        s["pool"] = torch.randn((used + 3, hkv, 2, P, d), generator=g, device=device, dtype=dtype)
        s["base"] = torch.tensor(lens, dtype=torch.int32, device=device)
        s["lens"], s["most"] = s["base"].clone(), most
    if case["call"] == "append":
        total = sum(new)
        if case["packed_qkv"]:   # one projection gives queries, keys and values of a token side by side
            rows = torch.randn((total, hq + 2 * hkv, d), generator=g, device=device, dtype=dtype)
            s["q"], s["k"], s["v"] = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
        else:
            s["q"] = torch.randn((total, hq, d), generator=g, device=device, dtype=dtype)
            s["k"], s["v"] = (torch.randn((total, hkv, d), generator=g, device=device, dtype=dtype) for _ in range(2))
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        s["cu"] = torch.tensor(cu, dtype=torch.int32, device=device)
        s["offsets"] = torch.randint(case["far"] // 2, case["far"] + 1, (B,), generator=g, device=device, dtype=torch.int32)
        half = case["rotary"] // 2
        s["frequencies"] = (THETA ** (-torch.arange(half, dtype=torch.float64) / half)).to(device)
    else:
        shape = (B, hq, d) if case["n_q"] == 1 else (B, case["n_q"], hq, d)
        s["q"] = torch.randn(shape, generator=g, device=device, dtype=dtype)
    if case["prefix"]:
        s["S"], s["packed"] = _prefix(case, seed, device)
        s["centroids"] = [c.to(device) for c in _codebooks()]
    if own:
        import paper_2502_02617_b200 as pq
        if "pool" in s:
            s["kept"] = pq.PagedWindow(B, hq, hkv, d, P, s["pool"].shape[0], s["table"], dtype=dtype, frequencies=s.get("frequencies"),
                                       interleaved=case["interleaved"], device=device)
            s["kept"].pool.copy_(s["pool"])
            s["kept"].lens.copy_(s["base"])
            del s["pool"], s["lens"]
        if case["prefix"]:
            bounds = [(c[1:] + c[:-1]) / 2 for c in _codebooks()]
            s["cache"] = pq.PolarQuantCache(1, hq, hkv, d, capacity=case["prefix"], S=s["S"], codebooks=(torch.cat(_codebooks()), torch.cat(bounds)),
                                            device=device)
            s["cache"].cache.copy_(s["packed"].view(-1))
            s["cache"].lens.fill_(case["prefix"])
            del s["packed"]
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------


def run(s):
    case = s["case"]
    if own:
        if case["call"] == "append":
            w = s["kept"]
            w.lens.copy_(s["base"])
            q = w.append(s["q"], s["k"], s["v"], s["cu"], offsets=s["offsets"])
            return {"q": q, "pool": w.pool, "lens": w.lens}
        if case["call"] == "window":
            return s["kept"].attend(s["q"], scale=s["scale"], max_len=s["most"])
        if case["call"] == "prefix":
            return s["cache"].attend_prefix(s["q"], scale=s["scale"])
        return s["cache"].attend_shared(s["q"], s["kept"], scale=s["scale"], max_window=s["most"])
    if case["call"] == "append":
        return _plain_append(s, case)
    out = _plain_attention(s, case)
    return out.to(s["q"].dtype).reshape(s["q"].shape)


def _plain_append(s, case):
    s["lens"].copy_(s["base"])
    n, half, P = s["q"].shape[0], case["rotary"] // 2, case["page_tokens"]
    cu = s["cu"].long()
    index = torch.arange(n, device=cu.device)
    seq = torch.bucketize(index, cu[1:], right=True)
    place = index - cu[seq] + s["lens"].long()[seq]
    angle = (place + s["offsets"].long()[seq]).double()[:, None] * s["frequencies"]       # far positions: the angle in 64 bits
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def rotated(x):
        x32 = x.float()
        pairs = x32[..., :2 * half]
        a, b = (pairs[..., 0::2], pairs[..., 1::2]) if case["interleaved"] else (pairs[..., :half], pairs[..., half:])
        a, b = a * cos - b * sin, b * cos + a * sin
        turned = torch.stack([a, b], -1).flatten(-2) if case["interleaved"] else torch.cat([a, b], -1)
        return torch.cat([turned, x32[..., 2 * half:]], -1).to(x.dtype)

    page = s["table"].long()[seq, place // P]
    s["pool"][page, :, 0, place % P] = rotated(s["k"])
    s["pool"][page, :, 1, place % P] = s["v"]
    s["lens"] += s["cu"][1:] - s["cu"][:-1]
    return {"q": rotated(s["q"]), "pool": s["pool"], "lens": s["lens"]}


def _plain_decode(s, case):
    """The packed prefix as float32 keys and values of the rotated basis [kv head, K | V, token, d]."""
    d, n = case["head_dim"], case["prefix"]
    nb, packed = d // 16, s["packed"]
    widths = (4 * nb, nb, max(1, nb // 2), max(1, nb // 4), 2 * nb)
    planes = packed.split([BLOCK * w for w in widths], -1)
    planes = [p.unflatten(-1, (BLOCK, -1)).permute(0, 2, 1, 3, 4).flatten(2, 3)[:, :, :n] for p in planes]
    r = planes[4].contiguous().view(torch.float16).float()
    for level in (4, 3, 2, 1):
        bits, count = LEVEL_BITS[level - 1], d >> level
        shifts = torch.arange(0, 8, bits, device=packed.device, dtype=torch.uint8)
        code = ((planes[level - 1][..., None] >> shifts) & ((1 << bits) - 1)).flatten(-2)[..., :count].int()
        cen = s["centroids"][level - 1]
        r = torch.stack([r * torch.cos(cen).float()[code], r * torch.sin(cen).float()[code]], -1).flatten(-2)
    return r


def _plain_attention(s, case):
    B, n_q, hq, hkv, d = case["batch"], case["n_q"], case["q_heads"], case["kv_heads"], case["head_dim"]
    q = s["q"].float().view(B, n_q, hkv, hq // hkv, d).transpose(1, 2) * s["scale"]           # [B, kv head, n_q, group, d]
    scores, values = [], []
    if case["call"] != "window":
        keys, vals = _plain_decode(s, case).unbind(1)
        turned = (q @ s["S"]).transpose(0, 1).reshape(hkv, -1, d)
        scores.append((turned @ keys.transpose(1, 2)).view(hkv, B, n_q, -1, case["prefix"]).transpose(0, 1))
    if case["call"] != "prefix":
        n = s["most"]
        at = torch.arange(n, device=q.device)
        rows = s["pool"][s["table"].long()[:, at // case["page_tokens"]], :, :, at % case["page_tokens"]].float()   # [B, n, kv head, K | V, d]
        k, v = rows.permute(3, 0, 2, 1, 4)
        w = (q.reshape(B, hkv, -1, d) @ k.transpose(2, 3)).view(B, hkv, n_q, -1, n)
        seen = s["lens"].long()[:, None] - (n_q - 1 - torch.arange(n_q, device=q.device))                         # tokens each query sees
        hidden = at >= seen[..., None]                                                                           # [B, n_q, n]
        scores.append(w.masked_fill(hidden[:, None, :, None], -math.inf))
        values.append(torch.where((at < s["lens"].long()[:, None])[:, None, :, None], v, torch.zeros((), device=q.device)))
    top = torch.stack([x.amax(-1) for x in scores]).amax(0)[..., None]
    weights = [torch.exp(x - top) for x in scores]
    total = sum(w.sum(-1, keepdim=True) for w in weights)
    out = 0.0
    if case["call"] != "prefix":
        w = weights.pop()
        out = (w.reshape(B, hkv, -1, w.shape[-1]) @ values[0]).view(B, hkv, n_q, -1, d)
    if case["call"] != "window":
        w = weights.pop().transpose(0, 1).reshape(hkv, -1, case["prefix"])
        out = out + (w @ vals).view(hkv, B, n_q, -1, d).transpose(0, 1) @ s["S"].t()
    return (out / total).transpose(1, 2)


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------


def exact(case, seed):
    """Sequence by sequence and kv head by kv head, from the definitions of the operators, in float64."""
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    lens, new, P, d = _windows(case), _new(case), case["page_tokens"], case["head_dim"]
    if case["call"] == "append":
        q, pool = s["q"].double(), s["pool"].double()
        freq, offsets, table = s["frequencies"].cpu(), s["offsets"].tolist(), s["table"]
        half, at = case["rotary"] // 2, 0
        even = (torch.arange(half) * 2 if case["interleaved"] else torch.arange(half)).cuda()
        odd = even + (1 if case["interleaved"] else half)
        for b, (have, count) in enumerate(zip(lens, new)):
            place = torch.arange(have, have + count, device="cuda")
            turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), (place + offsets[b]).double()[:, None] * freq.cuda())[:, None]
            for what, x in (("q", q[at:at + count]), ("k", s["k"][at:at + count].double())):
                z = torch.complex(x[..., even].contiguous(), x[..., odd].contiguous()) * turn
                x[..., even], x[..., odd] = z.real, z.imag
                if what == "k":
                    pool[table[b].long()[place // P], :, 0, place % P] = x
            pool[table[b].long()[place // P], :, 1, place % P] = s["v"][at:at + count].double()
            at += count
        return {"q": q, "pool": pool, "lens": torch.tensor([a + b for a, b in zip(lens, new)], dtype=torch.int32)}
    B, n_q, hq, hkv = case["batch"], case["n_q"], case["q_heads"], case["kv_heads"]
    group, q = hq // hkv, s["q"].double().view(B, n_q, hq, d)
    out = torch.empty((B, n_q, hq, d), dtype=torch.float64, device="cuda")
    for h in range(hkv):
        mine = q[:, :, h * group:(h + 1) * group]
        if case["prefix"]:
            keys, vals = (_decode64(s, case, h, i) @ s["S"].double().t() for i in (0, 1))   # back in the basis of the model
        for b in range(B):
            if case["call"] != "prefix":
                n = lens[b]
                pages = s["pool"][s["table"][b, :-(-n // P)].long(), h].double()                # [page, K | V, token, d]
                wk, wv = pages[:, 0].reshape(-1, d)[:n], pages[:, 1].reshape(-1, d)[:n]
            for j0 in range(0, n_q, 1 if case["call"] != "prefix" else n_q):
                x = mine[b, j0:j0 + (1 if case["call"] != "prefix" else n_q)].reshape(-1, d)
                e, v = [], []
                if case["prefix"]:
                    e.append(x @ keys.t()), v.append(vals)
                if case["call"] != "prefix":
                    see = n - (n_q - 1 - j0)
                    e.append(x @ wk[:see].t()), v.append(wv[:see])
                p = torch.softmax(torch.cat(e, 1) * d ** -0.5, 1)
                y = sum(a @ c for a, c in zip(p.split([t.shape[0] for t in v], 1), v))
                out[b, j0:j0 + max(1, x.shape[0] // group), h * group:(h + 1) * group] = y.view(-1, group, d)
    return out.view(s["q"].shape)


def _decode64(s, case, h, which):
    """Keys (which = 0) or values of kv head h: every coordinate is its block's radius times the cosines or sines down the tree."""
    d, n = case["head_dim"], case["prefix"]
    nb = d // 16
    raw = s["packed"][h, :, which]                                            # [block, bytes]
    token = torch.arange(n, device=raw.device)
    blk, tok = token // BLOCK, token % BLOCK
    out = torch.empty((n, d), dtype=torch.float64, device=raw.device)
    widths = (4 * nb, nb, max(1, nb // 2), max(1, nb // 4))
    start = [0]
    for w in widths:
        start.append(start[-1] + BLOCK * w)
    for i in range(d):
        two = raw[blk[:, None], (start[4] + tok * 2 * nb + 2 * (i // 16))[:, None] + torch.arange(2, device=raw.device)]
        x = two.contiguous().view(torch.float16).double()[:, 0]
        for level in (1, 2, 3, 4):
            node, bits = i >> level, LEVEL_BITS[level - 1]                    # the angle above coordinate i at this level
            byte = raw[blk, start[level - 1] + tok * widths[level - 1] + node * bits // 8].long()
            angle = s["centroids"][level - 1][(byte >> (node * bits % 8)) & ((1 << bits) - 1)]
            x = x * (torch.sin(angle) if (i >> (level - 1)) & 1 else torch.cos(angle))
        out[:, i] = x
    return out
