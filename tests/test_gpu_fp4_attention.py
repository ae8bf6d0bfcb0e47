"""Attention over the 4-bit cache against the fp64 oracle, which is given the bf16 pools that the stored rows stand for (they stand for
bf16 numbers exactly, so both see the same keys and values): shapes, numbers that are hard, and the ways of calling it."""
import numpy as np
import pytest
import torch

from fp4_util import as_bf16, on_device, poison_slack, store_pools
from gpu_util import LSE_ABS, REL_LARGE, check_attention
from lr_workloads import Model, bf16_round, bf16_to_f32, make_config, make_random_mid, make_random_small, make_random_tree, make_tree
from lr_workloads.gen import _finish
from oracle import lr_oracle as O
from paper_2506_19830_b200 import binding as B
from paper_2506_19830_b200 import runner as R
from test_gpu_fp8_attention_edges import SCORES, SIZES, chain, few_rows, tokens

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PATHS = [B.PATH_GENERIC, B.PATH_TENSOR_CORE]


def stored(w, seed=0):
    """The workload's pools in 4 bits, anything in unused slots, and the bf16 pools they stand for."""
    pools = poison_slack(w.batch, store_pools(w.tensors.k_pool, w.tensors.v_pool), np.random.default_rng(seed))
    return pools, as_bf16(pools[0], pools[2]), as_bf16(pools[1], pools[3])


def run(w, pools, path, scale=0.0, lse=True, stream=None):
    b = w.batch
    ctx = B.Context(b.model, 0)
    plan = B.Plan(ctx, b)
    plan.lr_plan_set_attention_path(path)
    q, cache = R.bf16_tensor(w.tensors.q, DEV), on_device(pools)
    n, guard = q.numel(), 4096
    buf = torch.full((n + 2 * guard,), -7.0, dtype=torch.bfloat16, device=DEV)
    out = buf[guard:guard + n].view(q.shape)
    l = torch.full(q.shape[:2], -7.0, device=DEV) if lse else None
    plan.lr_verify_attention_fp4(q, cache, out, l, scale, stream)
    assert plan.lr_poll_status(stream) == 0
    assert bool((buf[:guard] == -7.0).all()) and bool((buf[guard + n:] == -7.0).all())
    plan.close()
    ctx.close()
    return out, l


def check(w, path, rel_large=0.0, scale=0.0, branches=None):
    pools, k, v = stored(w)
    out, lse = run(w, pools, path, scale)
    o_ref, l_ref = O.verify_attention(w.batch, w.tensors.q, k, v, scale if scale > 0 else None, branches=branches)
    rows = None if branches is None else np.concatenate([np.arange(w.batch.cu_q[i], w.batch.cu_q[i + 1]) for i in branches])
    return check_attention(out, lse, o_ref, l_ref, rows, rel_large)


# ---- shapes ------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("cfg", [1, 2])
def test_configurations(cfg, path):
    check(make_config(cfg, with_logits=False), path)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("seed", range(10))
def test_ragged_small(seed, path):
    check(make_random_small(9200 + seed), path, REL_LARGE)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("seed", range(6))
def test_irregular_trees(seed, path):
    check(make_random_tree(9300 + seed), path, REL_LARGE)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("prefix,q", [(0, 1), (1, 1), (15, 1), (16, 1), (127, 1), (128, 1), (129, 2), (700, 1)])
def test_single_tokens(d, prefix, q, path):
    rng = np.random.default_rng(prefix + d)
    w = _finish("token", 11, Model(10, 2, d, 16), [{"P": prefix, "segs": [], "branches": [(0, q, q, q)]} for _ in range(3)], rng, 0.3, 0.6, False, True, "nan")
    check(w, path, REL_LARGE)


@pytest.mark.parametrize("cfg,branches", [(3, [0, 5, 15]), (4, [0, 5]), (5, [0, 20, 40])])
def test_large_configurations_on_the_tensor_cores(cfg, branches):
    """Two M-tiles a piece, several pieces a CTA, results merged from many."""
    w = make_config(cfg, with_logits=False)
    check(w, B.PATH_TENSOR_CORE, branches=[b for b in branches if b < w.batch.n_branch])


@pytest.mark.parametrize("seed", range(12))
def test_both_sides_of_the_grouping_switch(seed):
    check(make_random_mid(seed), B.PATH_TENSOR_CORE, REL_LARGE)


@pytest.mark.parametrize("W,size", [(2, "tiny"), (3, "tiny"), (2, "layer")])
def test_full_trees(W, size):
    check(make_tree(W, 2, size=size, with_logits=False), B.PATH_TENSOR_CORE, REL_LARGE)


@pytest.mark.parametrize("d,hq,h,q", [(64, 8, 8, 1), (64, 32, 8, 8), (128, 8, 8, 1), (128, 40, 8, 6), (128, 16, 2, 4), (128, 32, 8, 9), (64, 16, 1, 1), (128, 16, 1, 2)])
def test_few_rows_over_many_tiles(d, hq, h, q):
    check(few_rows(d, hq, h, q, d + q), B.PATH_TENSOR_CORE, REL_LARGE)


@pytest.mark.parametrize("d", [64, 128])
def test_single_tokens_of_many_requests_of_all_lengths(d):
    """More pieces than CTAs, several to a CTA, some split among CTAs."""
    rng = np.random.default_rng(d)
    reqs = [{"P": int(n), "segs": [], "branches": [(0, 1, 1, 1)]} for n in np.exp(rng.uniform(0, np.log(6000), 70))]
    w = _finish("lengths", 11, Model(8, 4, d, 16), reqs, rng, 0.3, 0.6, False, True, "nan")
    check(w, B.PATH_TENSOR_CORE, REL_LARGE)


# ---- numbers that are hard -----------------------------------------------------------------------------------------------------
def run_stored(w, pools, path, **kw):
    return run(w, poison_slack(w.batch, pools, np.random.default_rng(5)), path, **kw)


def bound(w, k, v, o_ref):
    """What an output may be off by: half a step of bf16, and of the weighted sum of |v| half a step of a weight in bf16, 2^-8, and as much for
    scores in fp32 of a few hundred at most (2^-8 of a weight is 2^-8 / ln 2 in its exponent, 2^-16 of 400).  On the tensor cores weights are halves, multiples of 2^-24 at
    the least, in a row whose sum is 2^2 or more (its largest weight is when its reference is set, and may rise): a key's part of an output may be off by 2^-27 of its V."""
    a, _ = O.verify_attention(w.batch, w.tensors.q, k, v & 0x7FFF)
    at = tokens(w.batch)
    sizes = np.abs(bf16_to_f32(v[at[:, 0], :, at[:, 1]])).astype(np.float64)
    return 2.0 ** -8 * np.abs(o_ref) + 2.0 ** -7 * a + len(at) * 2.0 ** -27 * sizes[np.isfinite(sizes)].max()


def compare(w, pools, path):
    k, v = as_bf16(pools[0], pools[2]), as_bf16(pools[1], pools[3])
    o_ref, l_ref = O.verify_attention(w.batch, w.tensors.q, k, v)
    limit = bound(w, k, v, o_ref)
    out, lse = run_stored(w, pools, path)
    got = bf16_to_f32(R.bf16_bits(out)).astype(np.float64)
    assert (np.abs(got - o_ref) <= limit).all(), np.nanmax(np.abs(got - o_ref) / limit)
    assert np.abs(lse.cpu().numpy() - l_ref).max() <= LSE_ABS


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("make", [lambda: make_random_small(9201), lambda: make_random_tree(9304), lambda: chain([300, 1, 640]), lambda: chain([129, 2000], 64),
                                  lambda: few_rows(128, 8, 8, 2, 24, n_req=6), lambda: few_rows(64, 8, 8, 2, 25, n_req=6), lambda: make_tree(2, 2, size="tiny", with_logits=False)])
def test_rows_that_stand_for_nan_reach_those_who_see_them(make, which, path):
    w = make()
    b, t = w.batch, w.tensors
    rng = np.random.default_rng(3)
    pools = store_pools(t.k_pool, t.v_pool)
    at = tokens(b)
    pick = at[rng.choice(len(at), min(len(at), 3), replace=False)]
    heads = rng.integers(0, b.model.n_kv_heads, len(pick))
    k, v = as_bf16(pools[0], pools[2]), as_bf16(pools[1], pools[3])
    # who sees one: whoever gets something from a V that is 1 there and 0 elsewhere
    mark = np.zeros_like(v)
    mark[pick[:, 0], heads, pick[:, 1]] = 0x3F80
    seen = O.verify_attention(b, t.q, k, mark)[0][:, :, 0] > 0
    codes, scale = (pools[0], pools[2]) if which == "k" else (pools[1], pools[3])
    codes[pick[:, 0], heads, pick[:, 1]] = 0
    scale[pick[:, 0], heads, pick[:, 1]] = 255
    o_ref, l_ref = O.verify_attention(b, t.q, k, v)  # (those who do not see it have the result of any row in its place)
    out, lse = run_stored(w, pools, path)
    got, l = bf16_to_f32(R.bf16_bits(out)).astype(np.float64), lse.cpu().numpy()
    assert seen.any()
    assert np.array_equal(np.isnan(got), np.repeat(seen[:, :, None], got.shape[2], 2))
    assert np.array_equal(np.isnan(l), seen)
    assert (np.abs(got - o_ref) <= bound(w, k, v, o_ref))[~seen].all()
    assert (np.abs(l - l_ref) <= LSE_ABS)[~seen].all()


@pytest.mark.parametrize("path", PATHS)
def test_queries_that_are_no_numbers_keep_to_themselves(path):
    w = chain([200, 50], q=5)
    bad = np.zeros(w.tensors.q.shape[:2], dtype=bool)
    pools, k, v = stored(w)
    o_ref, l_ref = O.verify_attention(w.batch, w.tensors.q, k, v)
    limit = bound(w, k, v, o_ref)
    for row, head, value in ((0, 1, 0x7FC0), (3, 4, 0x7FFF), (7, 0, 0xFFC0)):
        w.tensors.q[row, head, 17] = value
        bad[row, head] = True
    out, lse = run(w, pools, path)
    got = bf16_to_f32(R.bf16_bits(out)).astype(np.float64)
    assert np.isnan(got[bad]).all() and np.isnan(lse.cpu().numpy()[bad]).all()
    assert (np.abs(got - o_ref)[~bad] <= limit[~bad]).all()


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("d,q", [(64, 1), (128, 3), (128, 40)])
@pytest.mark.parametrize("how", list(SIZES))
def test_values_of_very_different_sizes(how, d, q, path):
    w = chain([900, 170], d, q=q, seed=7)
    b, t, rng = w.batch, w.tensors, np.random.default_rng(8)
    at = tokens(b)
    v = bf16_to_f32(t.v_pool)
    with np.errstate(all="ignore"):
        v[at[:, 0], :, at[:, 1]] *= np.exp2(np.round(SIZES[how](len(at), rng))).astype(np.float32)[:, None, None]
        t.v_pool[:] = bf16_round(v)
    compare(w, store_pools(t.k_pool, t.v_pool), path)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("d", [64, 128])
def test_groups_of_a_row_of_very_different_sizes(d, path):
    """Scales on both sides of those that take one multiplication, within rows and among neighbours; queries that make up for it in the scores."""
    w = chain([900, 170], d, q=5, seed=40)
    b, t, rng = w.batch, w.tensors, np.random.default_rng(41)
    by = np.repeat(rng.choice([-30, -3, 0, 14, 15, 16, 17, 40], d // 32), 32)
    up = rng.choice([0, 30, -30], (b.n_pool_pages, 1, 16, 1))
    with np.errstate(all="ignore"):
        t.k_pool[:] = bf16_round(np.ldexp(bf16_to_f32(t.k_pool), by))
        t.q[:] = bf16_round(np.ldexp(bf16_to_f32(t.q), -by))
        t.v_pool[:] = bf16_round(np.ldexp(bf16_to_f32(t.v_pool), by[::-1] + up))
    compare(w, store_pools(t.k_pool, t.v_pool), path)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("d,q", [(64, 1), (128, 3), (128, 40)])
@pytest.mark.parametrize("how", list(SCORES))
def test_scores_that_grow_fall_and_jump(how, d, q, path):
    w = chain([900, 170], d, q=q, seed=9)
    b, t, rng = w.batch, w.tensors, np.random.default_rng(10)
    at = tokens(b)
    axis = rng.choice([-1.0, 1.0], d)
    k = bf16_to_f32(t.k_pool)
    want = SCORES[how](len(at), rng)
    k[at[:, 0], :, at[:, 1]] = (0.2 * rng.standard_normal((len(at), b.model.n_kv_heads, d)) + (want / np.sqrt(d))[:, None, None] * axis).astype(np.float32)
    t.k_pool[:] = bf16_round(k)
    t.q[:] = bf16_round((axis + 0.2 * rng.standard_normal(t.q.shape)).astype(np.float32))
    compare(w, store_pools(t.k_pool, t.v_pool), path)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("by", [60, -60, 100, -100])
def test_large_queries_over_small_keys_and_the_reverse(by, path):
    w = chain([400, 30], seed=11)
    t = w.tensors
    with np.errstate(all="ignore"):  # (poison)
        t.q[:] = bf16_round(bf16_to_f32(t.q) * np.float32(2.0 ** by))
        t.k_pool[:] = bf16_round(bf16_to_f32(t.k_pool) * np.float32(2.0 ** -by))
    compare(w, store_pools(t.k_pool, t.v_pool), path)


# ---- ways of calling it ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("path", PATHS)
def test_a_softmax_scale_of_the_callers(path):
    check(chain([500, 77], seed=12), path, REL_LARGE, scale=0.031)


@pytest.mark.parametrize("path", PATHS)
def test_without_lse_and_on_a_stream_of_its_own(path):
    w = chain([500, 77], seed=13)
    pools, k, v = stored(w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out, _ = run(w, pools, path, lse=False, stream=s)
    s.synchronize()
    check_attention(out, None, O.verify_attention(w.batch, w.tensors.q, k, v)[0], None, None, REL_LARGE)


def test_two_plans_at_once_and_replayed():
    ws = [chain([2100, 40], seed=14), make_random_tree(9303)]
    ctxs = [B.Context(w.batch.model, 0) for w in ws]
    plans = [B.Plan(c, w.batch) for c, w in zip(ctxs, ws)]
    data = [stored(w) for w in ws]
    ref = [O.verify_attention(w.batch, w.tensors.q, k, v) for w, (_, k, v) in zip(ws, data)]
    qs, caches = [R.bf16_tensor(w.tensors.q, DEV) for w in ws], [on_device(d[0]) for d in data]
    outs, lses = [torch.zeros_like(q) for q in qs], [torch.zeros(q.shape[:2], device=DEV) for q in qs]
    torch.cuda.synchronize()
    streams, graphs = [torch.cuda.Stream() for _ in ws], []
    for p, q, c, o, l, s in zip(plans, qs, caches, outs, lses, streams):
        p.lr_plan_set_attention_path(B.PATH_TENSOR_CORE)
        p.lr_verify_attention_fp4(q, c, o, l, 0.0, s)
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            p.lr_verify_attention_fp4(q, c, o, l, 0.0, s)
        graphs.append(g)
    for o, l in zip(outs, lses):
        o.zero_()
        l.zero_()
    torch.cuda.synchronize()
    for _ in range(6):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for p, o, l, (o_ref, l_ref) in zip(plans, outs, lses, ref):
        assert p.lr_poll_status() == 0
        check_attention(o, l, o_ref, l_ref, None, REL_LARGE)
    del graphs
    for x in plans + ctxs:
        x.close()


def test_more_branches_than_the_tensor_cores_number():
    """A request of 300 branches takes the CUDA cores by itself, and the tensor cores are refused for it."""
    rng = np.random.default_rng(16)
    w = _finish("wide", 11, Model(4, 1, 64, 16), [{"P": 40, "segs": [], "branches": [(0, 1, 1, 1)] * 300}], rng, 0.3, 0.6, False, True, "nan")
    check(w, 0, REL_LARGE)
    ctx = B.Context(w.batch.model, 0)
    plan = B.Plan(ctx, w.batch)
    plan.lr_plan_set_attention_path(B.PATH_TENSOR_CORE)
    q = R.bf16_tensor(w.tensors.q, DEV)
    with pytest.raises(B.LrError) as e:
        plan.lr_verify_attention_fp4(q, B.Fp4Cache.empty(w.batch.model, w.batch.n_pool_pages), torch.zeros_like(q))
    assert e.value.status == -2
    plan.close()
    ctx.close()


def test_refusals():
    w = make_config(2, with_logits=False)
    b = w.batch
    pools, k, v = stored(w)
    ctx = B.Context(b.model, 0)
    plan = B.Plan(ctx, b)
    q, cache = R.bf16_tensor(w.tensors.q, DEV), on_device(pools)
    out = torch.full_like(q, -7.0)
    lse = torch.full(q.shape[:2], -7.0, device=DEV)

    def refused(status, words, **kw):
        a = dict(dict(q=q, cache=cache, out=out, lse=lse, scale=0.0), **kw)
        with pytest.raises(B.LrError) as e:
            plan.lr_verify_attention_fp4(a["q"], a["cache"], a["out"], a["lse"], a["scale"])
        assert e.value.status == status and words in str(e.value), str(e.value)

    n = b.n_pool_pages
    refused(-1, "pages", cache=B.Fp4Cache(*(x[: n - 1] for x in (cache.k, cache.v, cache.k_scale, cache.v_scale))))
    refused(-1, "null", q=None)
    refused(-1, "null", out=None)
    flat = torch.zeros(q.numel() + 8, dtype=torch.bfloat16, device=DEV)
    refused(-1, "aligned", q=flat[1:1 + q.numel()].view(q.shape))
    refused(-1, "aligned", out=flat[1:1 + q.numel()].view(q.shape))
    other = Model(b.model.n_q_heads, b.model.n_kv_heads, 64 if b.model.head_dim == 128 else 128, 16)
    for wrong in (B.Fp4Cache.empty(other, n), B.Fp8Cache.empty(b.model, n)):
        with pytest.raises(ValueError):
            plan.lr_verify_attention_fp4(q, wrong, out)
    with pytest.raises(ValueError):
        plan.lr_verify_attention_fp8(q, cache, out)
    for bad in (q.float(), q[:-1], q.cpu()):
        with pytest.raises(ValueError, match="lr_verify_attention_fp4: q"):
            plan.lr_verify_attention_fp4(bad, cache, out)
    plan.lr_plan_set_attention_path(B.PATH_PAIR)
    refused(-2, "4-bit")
    plan.lr_plan_set_attention_path(0)
    torch.cuda.synchronize()
    assert bool((out == -7.0).all()) and bool((lse == -7.0).all())
    plan.lr_verify_attention_fp4(q, cache, out, lse)
    assert plan.lr_poll_status() == 0
    check_attention(out, lse, *O.verify_attention(b, w.tensors.q, k, v))
    plan.close()
    ctx.close()


@pytest.mark.parametrize("path,slot_of", [
    (B.PATH_GENERIC, lambda b: int(b.span_slot[0]) + 100), (B.PATH_TENSOR_CORE, lambda b: int(b.span_slot[0]) + 100),
    (B.PATH_TENSOR_CORE, lambda b: int(b.span_slot[0])), (B.PATH_TENSOR_CORE, lambda b: int(b.br_own_slot[1])),
])
@pytest.mark.parametrize("bad", [-3, 5])
@pytest.mark.parametrize("q_len", [None, 1])
def test_a_page_outside_the_pool_is_reported_not_read(q_len, bad, path, slot_of):
    if q_len is None:
        w = make_config(2, with_logits=False)
    else:
        w = _finish("token", 11, Model(8, 4, 128, 16), [{"P": 1700, "segs": [9], "branches": [(0, 1, 1, 1), (1, 1, 1, 1)]}], np.random.default_rng(2), 0.3, 0.6, False, True, "nan")
    b = w.batch
    pools, k, v = stored(w)
    ctx = B.Context(b.model, 0)
    plan = B.Plan(ctx, b)
    plan.lr_plan_set_attention_path(path)
    q, cache = R.bf16_tensor(w.tensors.q, DEV), on_device(pools)
    out, slot = torch.zeros_like(q), slot_of(b)
    good = int(b.page_ids[slot])
    plan.lr_plan_debug_set_page(slot, bad if bad < 0 else int(b.n_pool_pages) + bad)
    plan.lr_verify_attention_fp4(q, cache, out)
    with pytest.raises(B.LrError) as e:
        plan.lr_poll_status()
    assert e.value.status == -5, e.value  # LR_EBOUNDS
    assert plan.lr_poll_status() == 0
    plan.lr_plan_debug_set_page(slot, good)
    plan.lr_verify_attention_fp4(q, cache, out)
    assert plan.lr_poll_status() == 0
    check_attention(out, None, O.verify_attention(b, w.tensors.q, k, v)[0], None, None, REL_LARGE)
    plan.close()
    ctx.close()


def test_a_wait_that_runs_out_is_reported_and_the_context_stays_usable():
    w = make_config(2, with_logits=False)
    b = w.batch
    pools, k, v = stored(w)
    ctx = B.Context(b.model, 0)
    plan = B.Plan(ctx, b)
    plan.lr_plan_set_attention_path(B.PATH_TENSOR_CORE)
    q, cache = R.bf16_tensor(w.tensors.q, DEV), on_device(pools)
    out = torch.zeros_like(q)
    plan.lr_plan_debug_set_wait_limit(3000)
    plan.lr_plan_debug_set_phantom_bytes(4096)
    plan.lr_verify_attention_fp4(q, cache, out)
    with pytest.raises(B.LrError) as e:
        plan.lr_poll_status()
    assert e.value.status == -4, e.value  # LR_ETIMEOUT
    plan.lr_plan_debug_set_phantom_bytes(0)
    plan.lr_plan_debug_set_wait_limit(1_000_000)
    for _ in range(2):
        plan.lr_verify_attention_fp4(q, cache, out)
        assert plan.lr_poll_status() == 0
    check_attention(out, None, O.verify_attention(b, w.tensors.q, k, v)[0], None)
    plan.close()
    ctx.close()


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("q_len", [3, 1])
def test_a_cache_whose_bytes_pass_32_bits(q_len, path):
    """The batch's pages lie in the last of 2,200,000: rows written, attended to, compacted and read there."""
    w = chain([200, 37], q=q_len, seed=30)
    b, t = w.batch, w.tensors
    n, used = 2_200_000, int(b.n_pool_pages)
    at = tokens(b)
    k_rows, v_rows = (x[at[:, 0], :, at[:, 1]] for x in (t.k_pool, t.v_pool))
    pools = store_pools(t.k_pool, t.v_pool)
    k, v = as_bf16(pools[0], pools[2]), as_bf16(pools[1], pools[3])
    o_ref, l_ref = O.verify_attention(b, t.q, k, v)
    c = O.commit(b, t.verdict, np.asarray(b.br_n_draft, dtype=np.int32))
    want = O.compact(c["keep_off"], c["keep_pages"], c["keep_valid"], k, v)
    b.page_ids = b.page_ids + (n - used)
    b.n_pool_pages = n
    ctx = B.Context(b.model, 0)
    plan = B.Plan(ctx, b)
    plan.lr_plan_set_attention_path(path)
    cache = B.Fp4Cache.empty(b.model, n, DEV)
    slots = torch.from_numpy((at[:, 0] + (n - used)) * 16 + at[:, 1]).to(DEV)
    ctx.lr_fp4_write(cache, R.bf16_tensor(k_rows, DEV), R.bf16_tensor(v_rows, DEV), slots)
    q = R.bf16_tensor(t.q, DEV)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV)
    plan.lr_verify_attention_fp4(q, cache, out, lse)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)  # noqa: E731
    new_len, kept = (torch.zeros(b.n_req, dtype=torch.int32, device=DEV) for _ in range(2))
    plan.lr_compact_fp4(i32(c["keep_off"]), i32(c["keep_pages"] + (n - used)), i32(c["keep_valid"]), cache, new_len, kept)
    assert plan.lr_poll_status() == 0
    check_attention(out, lse, o_ref, l_ref, None, REL_LARGE)
    assert np.array_equal(new_len.cpu().numpy(), want[0]) and np.array_equal(kept.cpu().numpy(), want[1])
    for r in range(b.n_req):
        pages = c["keep_pages"][c["keep_off"][r]:c["keep_off"][r + 1]]
        place = np.array([int(pages[i // 16]) * 16 + i % 16 for i in range(int(want[0][r]))], dtype=np.int64)
        got = [torch.zeros((len(place), b.model.n_kv_heads, b.model.head_dim), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        ctx.lr_fp4_read(cache, torch.from_numpy(place + (n - used) * 16).to(DEV), *got)
        for x, ref in zip(got, want[2:]):
            assert np.array_equal(R.bf16_bits(x), ref[place // 16, :, place % 16])
    plan.close()
    ctx.close()


@pytest.mark.parametrize("make", [lambda: few_rows(64, 8, 8, 2, 31), lambda: chain([3000, 700, 65], q=40, seed=32), lambda: make_random_tree(9305)])
def test_the_same_bits_every_time(make):
    """Also beside another pass, whose leavings in shared and tensor memory differ."""
    w, other = make(), chain([1200], q=30, seed=33)
    ctx, octx, plans, bufs = B.Context(w.batch.model, 0), B.Context(other.batch.model, 0), [], []
    for c, x in ((ctx, w), (octx, other)):
        p = B.Plan(c, x.batch)
        p.lr_plan_set_attention_path(B.PATH_TENSOR_CORE)
        q = R.bf16_tensor(x.tensors.q, DEV)
        plans.append(p)
        bufs.append((q, on_device(stored(x)[0]), torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV)))
    first = None
    for i in range(12):
        if i % 3 == 2:
            plans[1].lr_verify_attention_fp4(*bufs[1])
        bufs[0][2].fill_(-3.0)
        plans[0].lr_verify_attention_fp4(*bufs[0])
        assert plans[0].lr_poll_status() == 0
        got = (R.bf16_bits(bufs[0][2]).copy(), bufs[0][3].cpu().numpy().view(np.uint32).copy())
        first = first or got
        assert all(np.array_equal(a, b) for a, b in zip(got, first)), i
    for x in plans + [ctx, octx]:
        x.close()
