"""A shared prefix whose weights are small but many.  Tolerances are those of test_gpu_shared_prefix."""
import math

import numpy as np
import pytest
import torch

import paper_2502_02617_b200 as pq
from parity_utils import TOL_ATTENTION_F32_IO, rel_l2, to_f64
from test_gpu_shared_prefix import DEV, decoded

pytestmark = pytest.mark.gpu


def spread(d, R, n, first_value):
    """One token whose score is 25.5 octaves above n - 1 equal others, each of which weighs 2^-25.5 of it: (output, log-sum-exp, what they are,
    the others' part of the output)."""
    hq, hkv = 8, 1
    cache = pq.PolarQuantCache(1, hq, hkv, d, capacity=n, seed=6, device=DEV)
    g = torch.Generator(DEV).manual_seed(3)
    K = torch.zeros((n, hkv, d), device=DEV)
    K[0] = torch.randn((hkv, d), generator=g, device=DEV)
    V = 4 * torch.randn((1, hkv, d), generator=g, device=DEV).expand(n, hkv, d).clone()
    V[0] = first_value * torch.randn((hkv, d), generator=g, device=DEV)
    cache.encode(K, V, torch.tensor([0, n], dtype=torch.int32, device=DEV))
    Kh, Vh = decoded(cache, 0, 2)
    assert not Kh[0, 1].any()
    q = K[0].expand(R, hq, d).contiguous()
    scale = 25.5 * math.log(2.0) / float(to_f64(K[0, 0]) @ Kh[0, 0])
    lse = torch.empty((R, hq), device=DEV)
    out = cache.attend_prefix(q, scale=scale, lse=lse)
    torch.cuda.synchronize()
    assert cache.check_status()[0] == 0
    rest = (n - 1) * 2.0 ** -25.5
    others = rest * Vh[0, 1] / (1 + rest)
    return to_f64(out), to_f64(lse), np.broadcast_to(Vh[0, 0] / (1 + rest) + others, out.shape), 25.5 * math.log(2.0) + math.log1p(rest), others


# Rounding errors, of the whole output: an fp16 weight of 2^-18.5 (the reference has 2^7 of room) is off by 2^-6.5 of itself at most, and so is the others' part;
# keys and values as elsewhere; and a float32 sum of n products, each of which may lose a unit in the last place of what is there already: n 2^-23.  (That is
# the tensor cores' own: one range holds all n tokens here, and equal scores of 2^18 tokens, whose weights are exact, measure 1.4e-3.)
def bound(n, want, others):
    return TOL_ATTENTION_F32_IO + 2.0 ** -6.5 * np.linalg.norm(others) / np.linalg.norm(want[0, 0]) + n * 2.0 ** -23


@pytest.mark.parametrize("d,R", [(128, 2600), (64, 1300)])
def test_many_small_weights_behind_a_large_one(d, R):
    """2^18 tokens: together the small weights are 0.55 % of the sum, and with values four times as large 2 % of the output."""
    n = 1 << 18
    out, lse, want, want_lse, others = spread(d, R, n, 1.0)
    assert rel_l2(out, want) < bound(n, want, others)
    assert np.max(np.abs(lse - want_lse)) < 2e-3


@pytest.mark.parametrize("d,R", [(128, 2600), (64, 1300), (128, 3), (64, 3), (16, 9)])
@pytest.mark.parametrize("n", [300, 4096, 65536])
def test_small_weights_alone_make_the_output(d, R, n):
    """The large weight's value is zero: the output is the small ones' alone."""
    out, lse, want, want_lse, others = spread(d, R, n, 0.0)
    assert rel_l2(out, want) < bound(n, want, others)
    assert np.max(np.abs(lse - want_lse)) < 2e-3
