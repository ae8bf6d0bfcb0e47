"""Attention over the 4-bit cache with any softmax scale above 0, over queries of zeros, of the smallest and of the largest numbers: what a score is worth is the scale times a power
of two that the row of queries was divided by, and that product may leave the numbers of fp32."""
import numpy as np
import pytest

from gpu_util import REL_LARGE, check_attention
from lr_workloads import bf16_round, bf16_to_f32
from oracle import lr_oracle as O
from test_gpu_fp4_attention import PATHS, check, run, stored
from test_gpu_fp8_attention_edges import chain

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q", [1, 3, 40])
@pytest.mark.parametrize("scale", [1e-6, 1e-9, 1e-30, 1e-44])
def test_scales_that_leave_every_key_the_same_weight(scale, q, d, path):
    """Keys that a row does not see among those that it does: pages that end inside, tokens behind a query."""
    w = chain([700, 33, 5], d, hq=8, h=2, q=q, seed=70)
    t = w.tensors
    t.q[0] = 0
    t.q[1, ::2] = 0x8000  # -0
    t.q[1, 1::2] = 0x0001  # the smallest there is
    t.q[-1, :, 3:] = 0
    check(w, path, REL_LARGE, scale=scale)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("q", [1, 40])
def test_a_scale_and_queries_whose_product_is_beyond_fp32(q, path):
    """Scores of 0 all the same: the one channel that the queries have the keys do not."""
    w = chain([300, 33], 128, q=q, seed=71)
    t = w.tensors
    rows, k = np.zeros(t.q.shape, dtype=np.float32), bf16_to_f32(t.k_pool)
    rows[:, :, 5] = 2.0 ** 126
    k[..., 5] = 0.0
    t.q[:], t.k_pool[:] = bf16_round(rows), bf16_round(k)
    pools, k, v = stored(w)
    out, lse = run(w, pools, path, scale=1e6)
    check_attention(out, lse, *O.verify_attention(w.batch, t.q, k, v, 1e6), None, REL_LARGE)
