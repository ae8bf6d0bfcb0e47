"""Attention over the 8-bit cache for queries with channels of very different sizes: the tolerances of `lr_verify_attention`, whatever the row."""
import numpy as np
import pytest
import torch

from fp8_util import as_bf16, on_device, poison_slack, store_pools
from gpu_util import LSE_ABS, REL_LARGE, check_attention
from lr_workloads import bf16_round, bf16_to_f32, make_random_small, make_random_tree
from oracle import lr_oracle as O
from paper_2506_19830_b200 import binding as B
from paper_2506_19830_b200 import runner as R
from test_gpu_fp8_attention import DEV, PATHS, run, stored
from test_gpu_fp8_attention_edges import bound, chain, few_rows, tokens

pytestmark = pytest.mark.gpu


def with_outliers(w, ratio, seed, every=1, key=0.0):
    """Every `every`-th row of Q has a channel 2^ratio above its others, in which the keys are `key`."""
    b, t, rng = w.batch, w.tensors, np.random.default_rng(seed)
    q = rng.standard_normal(t.q.shape).astype(np.float32)
    hit = np.arange(q.shape[0] * q.shape[1]).reshape(q.shape[:2]) % every == 0
    q[:, :, 5] = np.where(hit, np.float32(2.0 ** ratio) * rng.choice([-1.0, 1.0], hit.shape), q[:, :, 5])
    t.q[:] = bf16_round(q)
    at = tokens(b)
    k = bf16_to_f32(t.k_pool)
    k[at[:, 0], :, at[:, 1], 5] = key
    with np.errstate(all="ignore"):  # (poison)
        t.k_pool[:] = bf16_round(k)
    return w


def compare(w, path, scale=0.0):
    pools, k, v = stored(w)
    o_ref, l_ref = O.verify_attention(w.batch, w.tensors.q, k, v, scale if scale > 0 else None)
    out, lse = run(w, pools, path, scale)
    return check_attention(out, lse, o_ref, l_ref, None, REL_LARGE)


# pieces of one and of two M-tiles, cut among CTAs and whole, rows that share keys and rows that do not, requests of a few keys, trees
SHAPES = {
    "two tiles": lambda: chain([4096], 128, q=40),
    "two tiles, 64": lambda: chain([4096, 700], 64, q=70),
    "one tile": lambda: chain([900, 170, 33], 128, q=16),
    "one tile, 64": lambda: chain([900, 170, 33], 64, q=16),
    "shared keys": lambda: few_rows(128, 8, 4, 2, 41, n_req=6),
    "shared keys, 64": lambda: few_rows(64, 8, 4, 2, 42, n_req=6),
    "few": lambda: chain([7, 0, 60], 128, q=1),
    "long": lambda: chain([20000], 128, hq=2, h=1, q=3),
    "ragged": lambda: make_random_small(9010),
    "tree": lambda: make_random_tree(9110),
}


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("ratio", [9, 11, 13, 20])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_a_channel_far_above_the_others(shape, ratio, path):
    compare(with_outliers(SHAPES[shape](), ratio, ratio), path)


@pytest.mark.parametrize("ratio", [12, 30, 60, 100])
def test_rows_with_such_a_channel_beside_rows_without(ratio):
    compare(with_outliers(chain([2500, 300], 128, q=40, seed=3), ratio, 4, every=5), B.PATH_TENSOR_CORE)
    compare(with_outliers(few_rows(64, 8, 8, 3, 43, n_req=5), ratio, 5, every=3), B.PATH_TENSOR_CORE)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("ratio", [9, 11])
def test_such_a_channel_where_the_keys_agree(ratio, path):
    # (its part of the scores, 2^11 / 11 at the most, is the same for all keys; in fp32 it leaves the others 2^-16)
    compare(with_outliers(chain([4096], 128, q=10), ratio, ratio, key=1.0), path)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("ratio", [16, 34])
def test_two_channels_and_nothing_else(ratio, path):
    """A row of (2^ratio, 1, 0, ..): all that tells its keys apart is in the small one."""
    w = with_outliers(chain([1200, 90], 128, q=20), ratio, 6)
    q = bf16_to_f32(w.tensors.q)
    big = q[:, :, 5].copy()
    q[:] = 0.0
    q[:, :, 5], q[:, :, 77] = big, 9.0
    w.tensors.q[:] = bf16_round(q)
    compare(w, path)


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("make", [lambda: chain([300, 1, 640], q=9), lambda: few_rows(128, 8, 8, 2, 44, n_req=6), lambda: make_random_tree(9111)])
def test_such_rows_and_keys_that_stand_for_nan(make, which):
    w = with_outliers(make(), 18, 7, every=2)
    b, t, rng = w.batch, w.tensors, np.random.default_rng(8)
    pools = store_pools(t.k_pool, t.v_pool)
    at = tokens(b)
    pick = at[rng.choice(len(at), min(len(at), 3), replace=False)]
    heads = rng.integers(0, b.model.n_kv_heads, len(pick))
    k, v = as_bf16(pools[0], pools[2]), as_bf16(pools[1], pools[3])
    mark = np.zeros_like(v)
    mark[pick[:, 0], heads, pick[:, 1]] = 0x3F80
    zero = np.zeros_like(k)
    seen = O.verify_attention(b, t.q, zero, mark)[0][:, :, 0] > 0  # (equal weights: whoever sees one)
    codes, scale = (pools[0], pools[2]) if which == "k" else (pools[1], pools[3])
    codes[pick[:, 0], heads, pick[:, 1]] = 0
    scale[pick[:, 0], heads, pick[:, 1]] = 255
    o_ref, l_ref = O.verify_attention(b, t.q, k, v)
    out, lse = run(w, poison_slack(b, pools, rng), B.PATH_TENSOR_CORE)
    got, l = bf16_to_f32(R.bf16_bits(out)).astype(np.float64), lse.cpu().numpy()
    assert seen.any()
    assert np.array_equal(np.isnan(got), np.repeat(seen[:, :, None], got.shape[2], 2))
    assert np.array_equal(np.isnan(l), seen if which == "k" else np.zeros_like(seen))
    assert (np.abs(got - o_ref) <= bound(w, k, v, o_ref))[~seen].all()
    assert (np.abs(l - l_ref) <= LSE_ABS)[~np.isnan(l)].all()


def test_such_rows_over_a_page_outside_the_pool():
    w = with_outliers(chain([500, 40], q=6), 20, 9)
    b = w.batch
    pools, k, v = stored(w)
    ctx = B.Context(b.model, 0)
    plan = B.Plan(ctx, b)
    plan.lr_plan_set_attention_path(B.PATH_TENSOR_CORE)
    q, cache = R.bf16_tensor(w.tensors.q, DEV), on_device(pools)
    out, lse, slot = torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV), int(b.span_slot[0]) + 7
    plan.lr_plan_debug_set_page(slot, int(b.n_pool_pages) + 3)
    plan.lr_verify_attention_fp8(q, cache, out, lse)
    with pytest.raises(B.LrError) as e:
        plan.lr_poll_status()
    assert e.value.status == -5
    plan.lr_plan_debug_set_page(slot, int(b.page_ids[slot]))
    plan.lr_verify_attention_fp8(q, cache, out, lse)
    assert plan.lr_poll_status() == 0
    check_attention(out, lse, *O.verify_attention(b, w.tensors.q, k, v), None, REL_LARGE)
    plan.close()
    ctx.close()


def test_such_rows_leave_the_same_bits_every_time():
    w = with_outliers(chain([3000, 65], q=40, seed=45), 15, 10, every=3)
    pools, _, _ = stored(w)
    got = [(R.bf16_bits(o), l.cpu().numpy().view(np.uint32)) for o, l in (run(w, pools, B.PATH_TENSOR_CORE) for _ in range(5))]
    assert all(np.array_equal(a, b) for g in got[1:] for a, b in zip(g, got[0]))


def test_waits_for_such_rows_do_not_run_out():
    """Going through the rows of a piece again takes longer than any wait may: who waits for it meanwhile sees that it goes on."""
    w = with_outliers(chain([1024] * 220, 128, hq=4, h=1, q=64, seed=46), 20, 11)
    b = w.batch
    pools, k, v = stored(w)
    ctx = B.Context(b.model, 0)
    plan = B.Plan(ctx, b)
    plan.lr_plan_set_attention_path(B.PATH_TENSOR_CORE)
    assert plan.lr_plan_describe()["n_pieces"] > plan.lr_plan_describe()["n_cta"]  # some CTA has one piece behind another
    q, cache = R.bf16_tensor(w.tensors.q, DEV), on_device(pools)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV)
    plan.lr_plan_debug_set_wait_limit(3000)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    plan.lr_verify_attention_fp8(q, cache, out, lse)
    end.record()
    assert plan.lr_poll_status() == 0
    assert start.elapsed_time(end) > 6.0  # ms: twice the limit
    some = [0, 57, 219]
    rows = np.concatenate([np.arange(b.cu_q[i], b.cu_q[i + 1]) for i in some])
    o_ref, l_ref = O.verify_attention(b, w.tensors.q, k, v, branches=some)
    check_attention(out, lse, o_ref, l_ref, rows, REL_LARGE)
    plan.close()
    ctx.close()
