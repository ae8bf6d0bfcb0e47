"""Attention over the 4-bit cache on both sides of what its kernels choose by: queries and scales that halves hold and that they do not, 16 rows and 17 over a KV head,
more pieces than a CTA keeps the records of."""
import numpy as np
import pytest
import torch

from fp4_util import on_device, store_pools
from gpu_util import REL_LARGE, check_attention
from lr_workloads import Model, bf16_round, bf16_to_f32, make_random_small, make_random_tree
from lr_workloads.gen import _finish
from oracle import lr_oracle as O
from paper_2506_19830_b200 import binding as B
from paper_2506_19830_b200 import runner as R
from test_gpu_fp4_attention import DEV, PATHS, check, compare, run, stored
from test_gpu_fp8_attention_edges import chain, few_rows, tokens
from test_gpu_fp8_attention_queries import with_outliers

pytestmark = pytest.mark.gpu


def compare_rows(w, path):
    """Inputs whose scores are of ordinary sizes: the tolerances of the bf16 call."""
    pools, k, v = stored(w)
    out, lse = run(w, pools, path)
    check_attention(out, lse, *O.verify_attention(w.batch, w.tensors.q, k, v), None, REL_LARGE)


# rows that the few-row kernel takes and rows that it does not, pieces whole and cut among CTAs, trees
SHAPES = {
    "two tiles": lambda: chain([4096], 128, q=40),
    "two tiles, 64": lambda: chain([4096, 700], 64, q=70),
    "one tile": lambda: chain([900, 170, 33], 128, q=16),
    "one tile, 64": lambda: chain([900, 170, 33], 64, q=16),
    "few rows": lambda: few_rows(128, 8, 4, 2, 41, n_req=6),
    "few rows, 64": lambda: few_rows(64, 8, 4, 4, 42, n_req=6),
    "few": lambda: chain([7, 0, 60], 128, q=1),
    "long": lambda: chain([20000], 128, hq=2, h=1, q=3),
    "ragged": lambda: make_random_small(9210),
    "tree": lambda: make_random_tree(9310),
}


# a bf16 number has 8 bits: a half keeps one down to 2^-17, and the largest is brought to 2^14 .. 2^15: others are exact down to 2^-31 of it
@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("ratio", [11, 28, 33, 45])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_a_channel_of_the_queries_far_above_the_others(shape, ratio, path):
    compare_rows(with_outliers(SHAPES[shape](), ratio, ratio), path)


@pytest.mark.parametrize("ratio", [31, 60, 100])
def test_rows_with_such_a_channel_beside_rows_without(ratio):
    compare_rows(with_outliers(chain([2500, 300], 128, q=40, seed=3), ratio, 4, every=5), B.PATH_TENSOR_CORE)
    compare_rows(with_outliers(few_rows(64, 8, 8, 3, 43, n_req=5), ratio, 5, every=3), B.PATH_TENSOR_CORE)
    compare_rows(with_outliers(few_rows(128, 16, 2, 2, 44, n_req=5), ratio, 6, every=7), B.PATH_TENSOR_CORE)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("q", [1, 20])
@pytest.mark.parametrize("ratio", [16, 34])
def test_two_channels_and_nothing_else(ratio, q, path):
    """A row of (2^ratio, 9, 0, ..): all that tells its keys apart is in the small one."""
    w = with_outliers(chain([1200, 90], 128, q=q), ratio, 6)
    rows = bf16_to_f32(w.tensors.q)
    big = rows[:, :, 5].copy()
    rows[:] = 0.0
    rows[:, :, 5], rows[:, :, 77] = big, 9.0
    w.tensors.q[:] = bf16_round(rows)
    compare_rows(w, path)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("q", [1, 40])
def test_queries_of_zeros_and_of_the_smallest_numbers(q, path):
    w = chain([700, 33], 128, q=q, seed=50)
    t = w.tensors
    t.q[0] = 0
    t.q[1, ::2] = 0x8000  # -0
    t.q[1, 1::2] = 0x0001  # the smallest there is
    t.q[-1, :, 3:] = 0
    compare_rows(w, path)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("q", [1, 2, 33])
@pytest.mark.parametrize("which", ["k", "v", "both"])
@pytest.mark.parametrize("byte", [12, 102, 139])
def test_scales_on_both_sides_of_those_that_halves_hold(byte, which, q, path):
    """Groups of scales byte .. byte + 3, in turn; queries that bring scores back to ordinary sizes."""
    w = chain([500, 21, 1300], 128, hq=4, h=2, q=q, seed=byte)
    b, t, rng = w.batch, w.tensors, np.random.default_rng(byte + q)
    pools = list(store_pools(t.k_pool, t.v_pool))
    for i in (2, 3):
        if which != "both" and which != "kv"[i - 2]:
            continue
        pools[i][:] = np.where(pools[i] == 255, 255, byte + rng.integers(0, 4, pools[i].shape)).astype(np.uint8)
    if which != "v":
        with np.errstate(all="ignore"):
            t.q[:] = bf16_round(np.ldexp(bf16_to_f32(t.q), 126 - byte))
    compare(w, pools, path)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("q", [1, 33])
def test_one_group_beyond_halves_among_many(q, path):
    w = chain([2600, 700], 128, hq=8, h=2, q=q, seed=51)
    b, t, rng = w.batch, w.tensors, np.random.default_rng(52)
    pools = store_pools(t.k_pool, t.v_pool)
    at = tokens(b)
    page, place = at[len(at) // 3]
    pools[3][page, 1, place, 2] = 150
    page, place = at[2 * len(at) // 3]
    pools[2][page, 0, place, 1] = 90
    compare(w, pools, path)


@pytest.mark.parametrize("d,hq,h,q", [(128, 16, 1, 1), (128, 1, 1, 17), (128, 4, 4, 16), (128, 4, 4, 17), (64, 8, 1, 2), (64, 9, 1, 2), (64, 4, 4, 16), (64, 4, 4, 17), (128, 8, 1, 1), (128, 9, 1, 1), (64, 3, 3, 8), (64, 3, 3, 9)])
def test_rows_around_those_that_choose_the_kernel(d, hq, h, q):
    """8 and 9, 16 and 17 rows over a KV head."""
    for prefixes in ([0], [1500, 3, 40], [5000]):
        check(chain(prefixes, d, hq=hq, h=h, q=q, seed=q), B.PATH_TENSOR_CORE, REL_LARGE)


@pytest.mark.parametrize("d,q", [(128, 1), (64, 1), (128, 3)])
def test_more_pieces_than_a_cta_keeps_the_records_of(d, q):
    """Several thousand short requests: some 50 pieces to a CTA."""
    rng = np.random.default_rng(d + q)
    reqs = [{"P": int(n), "segs": [], "branches": [(0, q, q, q)]} for n in rng.integers(0, 40, 2000)]
    w = _finish("short", 11, Model(8, 4, d, 16), reqs, rng, 0.3, 0.6, False, True, "nan")
    ctx = B.Context(w.batch.model, 0)
    plan = B.Plan(ctx, w.batch)
    plan.lr_plan_set_attention_path(B.PATH_TENSOR_CORE)
    assert plan.lr_plan_describe()["n_pieces"] > 33 * plan.lr_plan_describe()["n_cta"]
    plan.close()
    ctx.close()
    check(w, B.PATH_TENSOR_CORE, REL_LARGE)


@pytest.mark.parametrize("make", [lambda: chain([3000, 65], q=40, seed=45), lambda: few_rows(128, 8, 2, 2, 46, n_req=5)])
def test_rows_gone_through_again_leave_the_same_bits_every_time(make):
    w = with_outliers(make(), 40, 10, every=3)
    pools, _, _ = stored(w)
    got = [(R.bf16_bits(o), l.cpu().numpy().view(np.uint32)) for o, l in (run(w, pools, B.PATH_TENSOR_CORE) for _ in range(5))]
    assert all(np.array_equal(a, b) for g in got[1:] for a, b in zip(g, got[0]))


def test_rows_gone_through_again_over_a_page_outside_the_pool():
    for w in (with_outliers(chain([500, 40], q=20), 40, 9), with_outliers(chain([500, 40], q=2), 40, 9)):
        b = w.batch
        pools, k, v = stored(w)
        ctx = B.Context(b.model, 0)
        plan = B.Plan(ctx, b)
        plan.lr_plan_set_attention_path(B.PATH_TENSOR_CORE)
        q, cache = R.bf16_tensor(w.tensors.q, DEV), on_device(pools)
        out, lse, slot = torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV), int(b.span_slot[0]) + 7
        plan.lr_plan_debug_set_page(slot, int(b.n_pool_pages) + 3)
        plan.lr_verify_attention_fp4(q, cache, out, lse)
        with pytest.raises(B.LrError) as e:
            plan.lr_poll_status()
        assert e.value.status == -5
        plan.lr_plan_debug_set_page(slot, int(b.page_ids[slot]))
        plan.lr_verify_attention_fp4(q, cache, out, lse)
        assert plan.lr_poll_status() == 0
        check_attention(out, lse, *O.verify_attention(b, w.tensors.q, k, v), None, REL_LARGE)
        plan.close()
        ctx.close()


def test_waits_for_rows_gone_through_again_do_not_run_out():
    """Going through the rows of a piece again takes longer than any wait may: who waits for it meanwhile sees that it goes on."""
    w = with_outliers(chain([1024] * 220, 128, hq=4, h=1, q=64, seed=46), 40, 11)
    b = w.batch
    pools, k, v = stored(w)
    ctx = B.Context(b.model, 0)
    plan = B.Plan(ctx, b)
    plan.lr_plan_set_attention_path(B.PATH_TENSOR_CORE)
    assert plan.lr_plan_describe()["n_pieces"] > plan.lr_plan_describe()["n_cta"]  # some CTA has one piece behind another
    q, cache = R.bf16_tensor(w.tensors.q, DEV), on_device(pools)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV)
    plan.lr_plan_debug_set_wait_limit(1000)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    plan.lr_verify_attention_fp4(q, cache, out, lse)
    end.record()
    assert plan.lr_poll_status() == 0
    assert start.elapsed_time(end) > 2.0  # ms: twice the limit
    some = [0, 57, 219]
    rows = np.concatenate([np.arange(b.cu_q[i], b.cu_q[i + 1]) for i in some])
    o_ref, l_ref = O.verify_attention(b, w.tensors.q, k, v, branches=some)
    check_attention(out, lse, o_ref, l_ref, rows, REL_LARGE)
    plan.close()
    ctx.close()


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("q", [1, 9])
@pytest.mark.parametrize("extra", [1, 200])
def test_rows_behind_the_last_branch_are_neither_read_nor_written(extra, q, path):
    w = chain([300, 77], 128, q=q, seed=60)
    b = w.batch
    pools, k, v = stored(w)
    ctx = B.Context(b.model, 0)
    plan = B.Plan(ctx, b)
    plan.lr_plan_set_attention_path(path)
    n = w.tensors.q.shape[0]
    rows = R.bf16_tensor(w.tensors.q, DEV)
    padded = torch.full((n + extra, *rows.shape[1:]), float("nan"), dtype=torch.bfloat16, device=DEV)
    padded[:n] = rows
    out, lse = torch.full_like(padded, -7.0), torch.full(padded.shape[:2], -7.0, device=DEV)
    plan.lr_verify_attention_fp4(padded, on_device(pools), out, lse)
    assert plan.lr_poll_status() == 0
    assert bool((out[n:] == -7.0).all()) and bool((lse[n:] == -7.0).all())
    check_attention(out[:n], lse[:n], *O.verify_attention(b, w.tensors.q, k, v), None, REL_LARGE)
    plan.close()
    ctx.close()


@pytest.mark.parametrize("q", [1, 20])
def test_a_first_call_that_is_captured(q):
    w = chain([900, 170], 128, q=q, seed=61)
    b = w.batch
    pools, k, v = stored(w)
    ctx = B.Context(b.model, 0)
    plan = B.Plan(ctx, b)
    plan.lr_plan_set_attention_path(B.PATH_TENSOR_CORE)
    rows, cache = R.bf16_tensor(w.tensors.q, DEV), on_device(pools)
    out, lse = torch.zeros_like(rows), torch.zeros(rows.shape[:2], device=DEV)
    torch.cuda.synchronize()
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        plan.lr_verify_attention_fp4(rows, cache, out, lse, 0.0, s)
    for _ in range(2):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert plan.lr_poll_status() == 0
        check_attention(out, lse, *O.verify_attention(b, w.tensors.q, k, v), None, REL_LARGE)
    del g
    plan.close()
    ctx.close()
