"""Attention over the 4-bit cache for many short requests with drafts: pieces of one tile each, several to a CTA, every one of which has numbers that halves do not hold."""
import numpy as np
import pytest

from fp4_util import as_bf16, store_pools
from gpu_util import LSE_ABS
from lr_workloads import Model, bf16_round, bf16_to_f32
from lr_workloads.gen import _finish
from oracle import lr_oracle as O
from paper_2506_19830_b200 import binding as B
from paper_2506_19830_b200 import runner as R
from test_gpu_fp4_attention import bound, compare, run_stored

pytestmark = pytest.mark.gpu


def short(d, seed, n_req=400):
    """Two branches of six query tokens each behind a short prefix: 24 rows and 128 keys at the most over a KV head."""
    rng = np.random.default_rng(seed)
    reqs = [{"P": int(n), "segs": [], "branches": [(0, 6, 6, 6), (0, 6, 6, 6)]} for n in rng.integers(0, 91, n_req)]
    w = _finish("short", 11, Model(8, 4, d, 16), reqs, rng, 0.3, 0.6, False, True, "nan")
    ctx = B.Context(w.batch.model, 0)
    plan = B.Plan(ctx, w.batch)
    plan.lr_plan_set_attention_path(B.PATH_TENSOR_CORE)
    info = plan.lr_plan_describe()
    assert info["n_pieces"] == 4 * n_req and info["n_pieces"] >= 10 * info["n_cta"]
    plan.close()
    ctx.close()
    return w


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("which", ["k", "v", "both"])
@pytest.mark.parametrize("byte", [90, 150])
def test_scales_beyond_halves_in_every_request(byte, which, d):
    w = short(d, byte + d)
    t, rng = w.tensors, np.random.default_rng(byte)
    pools = list(store_pools(t.k_pool, t.v_pool))
    for i in (2, 3):
        if which in ("both", "kv"[i - 2]):
            pools[i][:] = np.where(pools[i] == 255, 255, byte + rng.integers(0, 4, pools[i].shape)).astype(np.uint8)
    if which != "v":
        with np.errstate(all="ignore"):
            t.q[:] = bf16_round(np.ldexp(bf16_to_f32(t.q), 126 - byte))
    compare(w, pools, B.PATH_TENSOR_CORE)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("which", ["k", "v", "both"])
def test_rows_that_stand_for_nan_in_a_tail_of_every_request(which, d):
    """A branch's NaN reaches that branch's rows and not those of the branch beside it, of the same piece."""
    w = short(d, 7 + d)
    b, t = w.batch, w.tensors
    pools = store_pools(t.k_pool, t.v_pool)
    k, v = as_bf16(pools[0], pools[2]), as_bf16(pools[1], pools[3])
    o_ref, l_ref = O.verify_attention(b, t.q, k, v)
    limit = bound(w, k, v, o_ref)
    bad = np.zeros(t.q.shape[0], dtype=bool)
    for i in range(0, b.n_branch, 2):
        page, place = b.page_ids[int(b.br_own_slot[i])], i // 2 % 6
        for side in (0, 1):
            if which in ("both", "kv"[side]):
                pools[side][page, :, place] = 0
                pools[2 + side][page, :, place] = 255
        bad[b.cu_q[i] + place:b.cu_q[i + 1]] = True  # (the token itself and those behind it)
    out, lse = run_stored(w, pools, B.PATH_TENSOR_CORE)
    got, l = bf16_to_f32(R.bf16_bits(out)).astype(np.float64), lse.cpu().numpy()
    assert np.isnan(got[bad]).all() and np.isnan(l[bad]).all()
    assert not np.isnan(got[~bad]).any() and not np.isnan(l[~bad]).any()
    assert (np.abs(got - o_ref) <= limit)[~bad].all()
    assert (np.abs(l - l_ref) <= LSE_ABS)[~bad].all()
