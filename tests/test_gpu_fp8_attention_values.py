"""What a key's part of an output of the attention over the 8-bit cache may be off by: 2^-11 of itself, or 2^-23 of the largest number of V among the tokens of
its own request and KV head.  The limit of each output is worked out from that request and head alone."""
import numpy as np
import pytest

from fp8_util import as_bf16, store_pools
from gpu_util import LSE_ABS
from lr_workloads import bf16_round, bf16_to_f32, make_random_tree
from oracle import lr_oracle as O
from paper_2506_19830_b200 import runner as R
from test_gpu_fp8_attention import PATHS
from test_gpu_fp8_attention_edges import SIZES, chain, few_rows, run_stored

pytestmark = pytest.mark.gpu


def tokens_of(b, r):
    """(page, place) of the tokens of request r."""
    spans = [(int(b.span_slot[s]), int(b.span_len[s])) for s in range(int(b.req_span_off[r]), int(b.req_span_off[r + 1]))]
    spans += [(int(b.br_own_slot[i]), int(b.br_own_len[i])) for i in range(b.n_branch) if int(b.br_req[i]) == r]
    return np.array([(int(b.page_ids[f + t // 16]), t % 16) for f, n in spans for t in range(n)], dtype=np.int64).reshape(-1, 2)


def limit_of(w, k, v, scale=None):
    """The definition's outputs and log-sums, what an output may be off by, and the weighted sums of |v|.  An output may be off by half a step of bf16; by 2^-9 of
    the weighted sum of |v|, of which the weights' halves are 2^-11 and the scores, which are 2^-10 (as exponents of 2) off at most, 2 x 0.69 x 2^-10; and for each key
    by 2^-23 of the request's and head's largest, but by no more than all of the key's part."""
    b = w.batch
    o_ref, l_ref, weights = O.verify_attention(b, w.tensors.q, k, v, scale, return_weights=True)
    a, step = np.zeros(o_ref.shape), np.zeros(o_ref.shape)
    group = b.model.n_q_heads // b.model.n_kv_heads
    for i in range(b.n_branch):
        at = tokens_of(b, int(b.br_req[i]))
        top = np.abs(bf16_to_f32(v[at[:, 0], :, at[:, 1]])).max(axis=(0, 2)).astype(np.float64)  # of each KV head
        pages, places, _ = O.branch_token_table(b, i)
        mine = np.abs(bf16_to_f32(v[pages, :, places])).astype(np.float64)
        for row in range(int(b.cu_q[i]), int(b.cu_q[i + 1])):
            for h in range(b.model.n_q_heads):
                part = weights[(row, h)][:, None] * mine[:len(weights[(row, h)]), h // group]
                a[row, h], step[row, h] = part.sum(axis=0), np.minimum(part, 2.0 ** -23 * top[h // group]).sum(axis=0)
    return o_ref, l_ref, 2.0 ** -8 * np.abs(o_ref) + 2.0 ** -9 * a + step, a, step


def compare(w, path, sharp):
    """sharp: the part of the outputs where the limit's steps of the smallest halves have to be below 1/32 of the weighted sum of |v|."""
    pools = store_pools(w.tensors.k_pool, w.tensors.v_pool)
    k, v = as_bf16(pools[0], pools[2]), as_bf16(pools[1], pools[3])
    o_ref, l_ref, limit, a, step = limit_of(w, k, v)
    assert np.mean(step < a / 32) >= sharp, "the limit says nothing"
    out, lse = run_stored(w, pools, path)
    got = bf16_to_f32(R.bf16_bits(out)).astype(np.float64)
    assert (np.abs(got - o_ref) <= limit).all(), np.nanmax(np.abs(got - o_ref) / limit)
    assert np.abs(lse.cpu().numpy() - l_ref).max() <= LSE_ABS


MAKE = {
    "few rows": lambda: few_rows(128, 8, 4, 2, 51, n_req=4), "few rows, 64": lambda: few_rows(64, 8, 4, 2, 52, n_req=4),
    "rows": lambda: chain([900, 170, 333], 128, h=4, q=16, seed=53), "rows, 64": lambda: chain([900, 170, 333], 64, h=4, q=70, seed=54),
    "tree": lambda: make_random_tree(9112),
}


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("how", list(SIZES))
@pytest.mark.parametrize("make", list(MAKE))
def test_each_request_and_head_with_sizes_of_its_own(make, how, path):
    w = MAKE[make]()
    b, t, rng = w.batch, w.tensors, np.random.default_rng(55)
    v = bf16_to_f32(t.v_pool)
    with np.errstate(all="ignore"):
        for r in range(b.n_req):
            at = tokens_of(b, r)
            for h in range(b.model.n_kv_heads):
                by = np.round(SIZES[how](len(at), rng))[::1 if (r + h) % 2 else -1] + rng.integers(-30, 31)  # what is large in one is small in the next
                v[at[:, 0], h, at[:, 1]] *= np.exp2(by).astype(np.float32)[:, None]
        t.v_pool[:] = bf16_round(v)
    # (with sizes 2^120 apart a row of a few keys, or whose weights are on small ones, has none but the last term)
    compare(w, path, 0.1 if make == "tree" else 0.5)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("where", [0, 1, 3, 6])
@pytest.mark.parametrize("below", [4, 9])
@pytest.mark.parametrize("make", [m for m in MAKE if m != "tree"])
def test_small_values_where_the_weight_is(make, below, where, path):
    """The weights of every row lie on 64 keys whose values are 2^below smaller than those of the others."""
    w = MAKE[make]()
    b, t = w.batch, w.tensors
    d = b.model.head_dim
    axis = np.random.default_rng(56).choice([-1.0, 1.0], d)
    k, v = bf16_to_f32(t.k_pool), bf16_to_f32(t.v_pool)
    with np.errstate(all="ignore"):
        for r in range(b.n_req):
            at = tokens_of(b, r)
            for h in range(b.model.n_kv_heads):
                first = min(where + h, (len(at) - 1) // 64) * 64
                here = (np.arange(len(at)) // 64 * 64 == first) | (np.arange(len(at)) < 8)  # (a few that every row sees)
                k[at[:, 0], h, at[:, 1]] = (0.25 * k[at[:, 0], h, at[:, 1]] + np.where(here, 1.5, -1.0)[:, None] * axis).astype(np.float32)
                v[at[:, 0], h, at[:, 1]] *= np.where(here, 2.0 ** -below, 1.0).astype(np.float32)[:, None]
        t.k_pool[:], t.v_pool[:] = bf16_round(k), bf16_round(v)
    t.q[:] = bf16_round((axis + 0.1 * np.random.default_rng(57).standard_normal(t.q.shape)).astype(np.float32))
    compare(w, path, 0.9)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("d,prefix,q", [(64, 110, 1), (128, 110, 1), (128, 238, 1), (64, 238, 1), (128, 110, 70)])
@pytest.mark.parametrize("score", [-12, -13, -14, -15, -16, -18])
@pytest.mark.parametrize("lead", [0.0, 0.3125, 0.625])
def test_a_small_weight_on_the_largest_value(lead, score, d, prefix, q, path):
    """Key 1 has the weight and no value, key 0 sets the unit with a number just too large for the next smaller scale, and key 70, in the next half-tile, has the
    largest code of that smaller scale and a weight at the end of what halves hold."""
    w = chain([prefix], d, hq=2, h=1, q=q)
    b, t = w.batch, w.tensors
    at = tokens_of(b, 0)
    k, v = np.zeros((len(at), 1, d), np.float32), np.zeros((len(at), 1, d), np.float32)
    k[:, 0, :64] = -24.0  # a score is a key's sum over 64 channels / 8
    k[1, 0, :64], k[1, 0, 0] = 0.0, 8 * lead
    k[70, 0, :64] = score / 8
    v[0], v[70] = 226.0, 224.0
    for pool, rows in ((t.k_pool, k), (t.v_pool, v)):
        pool[at[:, 0], :, at[:, 1]] = bf16_round(rows)
    x = np.zeros(t.q.shape, np.float32)
    x[:, :, :64] = 1.0
    t.q[:] = bf16_round(x)
    pools = store_pools(t.k_pool, t.v_pool)
    k, v = as_bf16(pools[0], pools[2]), as_bf16(pools[1], pools[3])
    o_ref, l_ref = O.verify_attention(b, t.q, k, v, 0.125)
    part = np.exp(score - l_ref) * 224.0  # key 70's; all that there is, but for e^-190
    assert np.allclose(o_ref, part[:, :, None], rtol=1e-9, atol=1e-60)
    out, lse = run_stored(w, pools, path, scale=0.125)
    got = bf16_to_f32(R.bf16_bits(out)).astype(np.float64)
    assert (np.abs(got - o_ref) <= 2.0 ** -8 * o_ref + np.maximum(2.0 ** -9 * o_ref, 2.0 ** -23 * 224.0)).all(), (got.flat[0], o_ref.flat[0])
    assert np.abs(lse.cpu().numpy() - l_ref).max() <= LSE_ABS
