"""Scores of a few hundred over a shared prefix: an error that a softmax over small scores hides moves the log-sum-exp by its share of them."""
import numpy as np
import pytest
import torch

import paper_2502_02617_b200 as pq
from paper_2502_02617_b200 import synthetic
from parity_utils import to_f64
from test_gpu_shared_prefix import BF16, DEV, F32, decoded, make_cache

pytestmark = pytest.mark.gpu
CLUSTER, PERSISTENT, ROWS, TENSOR = 6, 7, 8, 9   # the head_dim-128 kernels, named for the next call


# The bound of the other attentions over the packed cache: keys and rotated queries are fp16 values with fp16 residuals, 22 bits of each coordinate, 2^-22 of
# sum |q_i||k_i| <= |q||k| for each of the two, and the float32 sums of the rotation and of the score take 2^-21 more: 2^-20.  The smaller heads' keys are
# decoded in float32 from four cosines or sines a coordinate, each rounded to 2^-24, by three products and one with the radius, 2^-24 each: 8 * 2^-24 = 2^-21
# more before they become a value and a residual; and their scores, 3 sums to magnitudes up to 2^7 (in octaves) rounded to 2^-24 of that with |q||k| d^-1/2
# no larger than 2^7, another 2^-22: below 2^-19 in all.
@pytest.mark.parametrize("io", [F32, BF16])
@pytest.mark.parametrize("kernel,d,hq,hkv,R", [(CLUSTER, 128, 8, 2, 5), (PERSISTENT, 128, 8, 2, 5), (ROWS, 128, 8, 2, 5), (TENSOR, 128, 8, 2, 40), (TENSOR, 128, 7, 1, 130),
                                               (None, 64, 8, 2, 3), (None, 64, 16, 2, 70), (None, 32, 4, 2, 33), (None, 16, 8, 1, 9)])
def test_large_scores_keep_the_precision_of_keys_and_queries(kernel, d, hq, hkv, R, io):
    n = 600
    cache = make_cache([33, n], hq, hkv, d, capacity=700)
    K, _ = decoded(cache, 1, n)
    q = (16 * synthetic.queries(5, R, hq, d, F32, DEV)).to(io)
    lse = torch.empty((R, hq), device=DEV)
    if kernel is not None:
        pq.pq_debug_fail_next_wait(kernel)
    cache.attend_prefix(q, seq=1, lse=lse)
    pq.pq_debug_fail_next_wait(0)
    torch.cuda.synchronize()
    assert cache.check_status()[0] == 0
    qs = to_f64(q)
    for h in range(hq):
        k = K[h * hkv // hq]
        e = qs[:, h] @ k.T * d ** -0.5
        m = e.max(1)
        want = m + np.log(np.exp(e - m[:, None]).sum(1))
        bound = 2.0 ** (-20 if d == 128 else -19) * np.linalg.norm(qs[:, h], axis=1) * np.linalg.norm(k, axis=1).max() * d ** -0.5
        assert np.all(np.abs(to_f64(lse[:, h]) - want) < bound), np.max(np.abs(to_f64(lse[:, h]) - want) / bound)
