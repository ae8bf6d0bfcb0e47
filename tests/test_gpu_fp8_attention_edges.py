"""Attention over the 8-bit cache where its numbers are hard: rows that stand for NaN, values and scores of very different sizes; and the ways of
calling it: scales, streams, graphs, bad pages, waits that run out."""
import numpy as np
import pytest
import torch

from fp8_util import as_bf16, on_device, poison_slack, store_pools
from gpu_util import LSE_ABS, REL_LARGE, check_attention
from lr_workloads import Model, bf16_round, bf16_to_f32, make_config, make_random_small, make_random_tree, make_tree
from lr_workloads.gen import _finish
from oracle import lr_oracle as O
from paper_2506_19830_b200 import binding as B
from paper_2506_19830_b200 import runner as R
from test_gpu_fp8_attention import DEV, PATHS, check, run, stored

pytestmark = pytest.mark.gpu


def chain(prefixes, d=128, hq=8, h=2, q=3, seed=0):
    """Requests of one branch with q rows each behind the given prefixes."""
    rng = np.random.default_rng(seed)
    reqs = [{"P": p, "segs": [], "branches": [(0, q, q, q)]} for p in prefixes]
    return _finish("chain", 11, Model(hq, h, d, 16), reqs, rng, 0.3, 0.6, False, True, "nan")


def tokens(b):
    """(page, place) of the tokens of all spans, in the order of the spans."""
    at = []
    for first, n in list(zip(b.span_slot, b.span_len)) + list(zip(b.br_own_slot, b.br_own_len)):
        at += [(int(b.page_ids[int(first) + t // 16]), t % 16) for t in range(int(n))]
    return np.array(at, dtype=np.int64).reshape(-1, 2)


def run_stored(w, pools, path, **kw):
    return run(w, poison_slack(w.batch, pools, np.random.default_rng(5)), path, **kw)


def bound(w, k, v, o_ref):
    """What an output may be off by: half a step of bf16, 2^-9 of the weighted sum of |v| for the rounding of the weights (halves: 2^-11) and of the scores,
    and for each key 2^-23 of the largest number of V, the step of the smallest halves."""
    a, _ = O.verify_attention(w.batch, w.tensors.q, k, v & 0x7FFF)
    at = tokens(w.batch)
    top = np.abs(bf16_to_f32(v[at[:, 0], :, at[:, 1]])).max()
    return 2.0 ** -8 * np.abs(o_ref) + 2.0 ** -9 * a + len(at) * 2.0 ** -23 * top


def compare(w, pools, path):
    k, v = as_bf16(pools[0], pools[2]), as_bf16(pools[1], pools[3])
    o_ref, l_ref = O.verify_attention(w.batch, w.tensors.q, k, v)
    limit = bound(w, k, v, o_ref)
    out, lse = run_stored(w, pools, path)
    got = bf16_to_f32(R.bf16_bits(out)).astype(np.float64)
    assert (np.abs(got - o_ref) <= limit).all(), np.nanmax(np.abs(got - o_ref) / limit)
    assert np.abs(lse.cpu().numpy() - l_ref).max() <= LSE_ABS


# ---- queries that fit the rows of one warp: its four neighbours share the keys -----------------------------------------------
def few_rows(d, hq, h, q, seed, n_req=10):
    """Requests whose pieces have several tiles each, with one, a few and the most rows there may be; some with draft steps of their own."""
    rng = np.random.default_rng(seed)
    reqs = []
    for i in range(n_req):
        p = int(rng.integers(300, 2400))
        reqs.append({"P": p, "segs": [], "branches": [(0, q, q, q)]} if i % 2 else {"P": p, "segs": [21], "branches": [(0, max(q - 1, 1), max(q - 1, 1), 1), (1, 1, 1, 1)]})
    return _finish("few", 11, Model(hq, h, d, 16), reqs, rng, 0.3, 0.6, False, True, "nan")


@pytest.mark.parametrize("d,hq,h,q", [(64, 8, 8, 1), (64, 32, 8, 8), (128, 8, 8, 1), (128, 40, 8, 6), (128, 16, 2, 4), (128, 32, 8, 9)])
def test_few_rows_over_many_tiles(d, hq, h, q):
    check(few_rows(d, hq, h, q, d + q), B.PATH_TENSOR_CORE, REL_LARGE)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("how", ["rising", "falling", "steps", "any", "half zeros"])
def test_few_rows_over_values_of_very_different_sizes(how, d):
    w = few_rows(d, 8, 4, 2, 21, n_req=4)
    t, at = w.tensors, tokens(w.batch)
    v = bf16_to_f32(t.v_pool)
    with np.errstate(all="ignore"):
        v[at[:, 0], :, at[:, 1]] *= np.exp2(np.round(SIZES[how](len(at), np.random.default_rng(1)))).astype(np.float32)[:, None, None]
        t.v_pool[:] = bf16_round(v)
    compare(w, store_pools(t.k_pool, t.v_pool), B.PATH_TENSOR_CORE)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("how", ["rising", "falling", "steps", "any", "late"])
def test_few_rows_over_scores_that_grow_fall_and_jump(how, d):
    w = few_rows(d, 8, 4, 2, 22, n_req=4)
    b, t, rng = w.batch, w.tensors, np.random.default_rng(23)
    at = tokens(b)
    axis, k = rng.choice([-1.0, 1.0], d), bf16_to_f32(t.k_pool)
    want = SCORES[how](len(at), rng)
    k[at[:, 0], :, at[:, 1]] = (0.2 * rng.standard_normal((len(at), b.model.n_kv_heads, d)) + (want / np.sqrt(d))[:, None, None] * axis).astype(np.float32)
    t.k_pool[:] = bf16_round(k)
    t.q[:] = bf16_round((axis + 0.2 * rng.standard_normal(t.q.shape)).astype(np.float32))
    compare(w, store_pools(t.k_pool, t.v_pool), B.PATH_TENSOR_CORE)


# ---- rows that stand for NaN -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("make", [lambda: make_random_small(9001), lambda: make_random_tree(9104), lambda: chain([300, 1, 640]), lambda: chain([129, 2000], 64), lambda: few_rows(128, 8, 8, 2, 24, n_req=6), lambda: few_rows(64, 8, 8, 2, 25, n_req=6),
                                  lambda: make_tree(2, 2, size="tiny", with_logits=False)])
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
    assert np.array_equal(np.isnan(l), seen if which == "k" else np.zeros_like(seen))
    assert (np.abs(got - o_ref) <= bound(w, k, v, o_ref))[~seen].all()
    assert (np.abs(l - l_ref) <= LSE_ABS)[~np.isnan(l)].all()


@pytest.mark.parametrize("path", PATHS)
def test_queries_that_are_no_numbers_keep_to_themselves(path):
    w = chain([200, 50], q=5)
    bad = np.zeros(w.tensors.q.shape[:2], dtype=bool)
    pools, k, v = stored(w)
    o_ref, l_ref = O.verify_attention(w.batch, w.tensors.q, k, v)
    limit = bound(w, k, v, o_ref)
    for row, head, value in ((0, 1, 0x7FC0), (3, 4, 0x7F80), (7, 0, 0xFF80)):
        w.tensors.q[row, head, 17] = value
        bad[row, head] = True
    out, lse = run(w, pools, path)
    got = bf16_to_f32(R.bf16_bits(out)).astype(np.float64)
    assert np.isnan(got[bad]).all() and np.isnan(lse.cpu().numpy()[bad]).all()
    assert (np.abs(got - o_ref)[~bad] <= limit[~bad]).all()


# ---- values of very different sizes ----------------------------------------------------------------------------------------
SIZES = {
    "rising": lambda n, rng: np.linspace(-60, 60, n),
    "falling": lambda n, rng: np.linspace(60, -60, n),
    "steps": lambda n, rng: 25.0 * ((np.arange(n) // 64) % 3 - 1),
    "any": lambda n, rng: rng.uniform(-20, 20, n),
    "one large": lambda n, rng: np.where(np.arange(n) == n // 3, 40.0, 0.0),
    "half zeros": lambda n, rng: np.where(np.arange(n) % 128 < 64, -1000.0, 5.0),
}


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


# ---- scores that grow, fall and jump -----------------------------------------------------------------------------------------
SCORES = {
    "rising": lambda n, rng: np.linspace(-45, 45, n),
    "falling": lambda n, rng: np.linspace(45, -45, n),
    "steps": lambda n, rng: 30.0 * ((np.arange(n) // 64) % 3 - 1),
    "any": lambda n, rng: rng.uniform(-40, 40, n),
    "late": lambda n, rng: np.where(np.arange(n) >= n - 2, 40.0, -40.0),
}


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
@pytest.mark.parametrize("by", [60, -60, 100])
def test_large_queries_over_small_keys_and_the_reverse(by, path):
    w = chain([400, 30], seed=11)
    t = w.tensors
    with np.errstate(all="ignore"):  # (poison)
        t.q[:] = bf16_round(bf16_to_f32(t.q) * np.float32(2.0 ** by))
        t.k_pool[:] = bf16_round(bf16_to_f32(t.k_pool) * np.float32(2.0 ** -by))
    compare(w, store_pools(t.k_pool, t.v_pool), path)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("by", [24, 40, 90])
@pytest.mark.parametrize("how", ["falling", "steps", "one large"])
def test_scores_beyond_what_fp32_tells_apart(how, by, path):
    """Queries 2^by times as large: the weights are 1 for one key, and the output is its V, of whichever size."""
    w = chain([900, 170], seed=18)
    b, t, rng = w.batch, w.tensors, np.random.default_rng(19)
    at = tokens(b)
    v = bf16_to_f32(t.v_pool)
    with np.errstate(all="ignore"):
        v[at[:, 0], :, at[:, 1]] *= np.exp2(np.round(SIZES[how](len(at), rng) / 4)).astype(np.float32)[:, None, None]
        t.v_pool[:] = bf16_round(v)
        t.q[:] = bf16_round(bf16_to_f32(t.q) * np.float32(2.0 ** by))
    pools = store_pools(t.k_pool, t.v_pool)
    k, v = as_bf16(pools[0], pools[2]), as_bf16(pools[1], pools[3])
    o_ref, l_ref, weights = O.verify_attention(b, t.q, k, v, return_weights=True)
    assert min(x.max() for x in weights.values()) > 1 - 2.0 ** -20  # (else the input would have to be another)
    limit = bound(w, k, v, o_ref)
    out, lse = run_stored(w, pools, path)
    got = bf16_to_f32(R.bf16_bits(out)).astype(np.float64)
    assert (np.abs(got - o_ref) <= limit).all()
    # scores: D products and sums in fp32, Q to 2^-19 of its largest
    assert (np.abs(lse.cpu().numpy() - l_ref) <= 2.0 ** -16 * np.abs(l_ref)).all()


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
    ws = [chain([2100, 40], seed=14), make_random_tree(9103)]
    ctxs = [B.Context(w.batch.model, 0) for w in ws]
    plans = [B.Plan(c, w.batch) for c, w in zip(ctxs, ws)]
    data = [stored(w) for w in ws]
    ref = [O.verify_attention(w.batch, w.tensors.q, k, v) for w, (_, k, v) in zip(ws, data)]
    qs, caches = [R.bf16_tensor(w.tensors.q, DEV) for w in ws], [on_device(d[0]) for d in data]
    outs, lses = [torch.zeros_like(q) for q in qs], [torch.zeros(q.shape[:2], device=DEV) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ws]
    graphs = []
    for p, q, c, o, l, s in zip(plans, qs, caches, outs, lses, streams):
        p.lr_plan_set_attention_path(B.PATH_TENSOR_CORE)
        p.lr_verify_attention_fp8(q, c, o, l, 0.0, s)
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            p.lr_verify_attention_fp8(q, c, o, l, 0.0, s)
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


def test_a_cache_that_changes_between_replays():
    """The graph holds addresses, nothing of what was there."""
    w = chain([333], seed=15)
    pools, k, v = stored(w)
    ctx = B.Context(w.batch.model, 0)
    plan = B.Plan(ctx, w.batch)
    plan.lr_plan_set_attention_path(B.PATH_TENSOR_CORE)
    q, cache = R.bf16_tensor(w.tensors.q, DEV), on_device(pools)
    out = torch.zeros_like(q)
    plan.lr_verify_attention_fp8(q, cache, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        plan.lr_verify_attention_fp8(q, cache, out)
    other = chain([333], seed=15)
    rng = np.random.default_rng(1)
    other.tensors.k_pool[:] = bf16_round(rng.standard_normal(k.shape).astype(np.float32))
    other.tensors.v_pool[:] = bf16_round(rng.standard_normal(v.shape).astype(np.float32))
    pools2, k2, v2 = stored(other)
    new = on_device(pools2)
    for a, b in ((cache.k, new.k), (cache.v, new.v), (cache.k_scale, new.k_scale), (cache.v_scale, new.v_scale)):
        a.view(torch.uint8).copy_(b.view(torch.uint8))
    g.replay()
    torch.cuda.synchronize()
    check_attention(out, None, O.verify_attention(w.batch, w.tensors.q, k2, v2)[0], None, None, REL_LARGE)
    del g
    plan.close()
    ctx.close()


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
        plan.lr_verify_attention_fp8(q, B.Fp8Cache.empty(w.batch.model, w.batch.n_pool_pages), torch.zeros_like(q))
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
            plan.lr_verify_attention_fp8(a["q"], a["cache"], a["out"], a["lse"], a["scale"])
        assert e.value.status == status and words in str(e.value), str(e.value)

    n = b.n_pool_pages
    few = B.Fp8Cache(*(x[: n - 1] for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)))
    refused(-1, "pages", cache=few)
    refused(-1, "null", q=None)
    refused(-1, "null", out=None)
    flat = torch.zeros(q.numel() + 8, dtype=torch.bfloat16, device=DEV)
    refused(-1, "aligned", q=flat[1:1 + q.numel()].view(q.shape))
    refused(-1, "aligned", out=flat[1:1 + q.numel()].view(q.shape))
    other = Model(b.model.n_q_heads, b.model.n_kv_heads, 64 if b.model.head_dim == 128 else 128, 16)
    with pytest.raises(ValueError):
        plan.lr_verify_attention_fp8(q, B.Fp8Cache.empty(other, n), out)
    plan.lr_plan_set_attention_path(B.PATH_PAIR)
    refused(-2, "", scale=0.0)
    plan.lr_plan_set_attention_path(0)
    torch.cuda.synchronize()
    assert bool((out == -7.0).all()) and bool((lse == -7.0).all())
    plan.lr_verify_attention_fp8(q, cache, out, lse)
    assert plan.lr_poll_status() == 0
    check_attention(out, lse, *O.verify_attention(b, w.tensors.q, k, v))
    plan.close()
    ctx.close()


@pytest.mark.parametrize("path,slot_of", [
    (B.PATH_GENERIC, lambda b: int(b.span_slot[0]) + 100), (B.PATH_TENSOR_CORE, lambda b: int(b.span_slot[0]) + 100),
    (B.PATH_TENSOR_CORE, lambda b: int(b.span_slot[0])), (B.PATH_TENSOR_CORE, lambda b: int(b.br_own_slot[1])),
])
@pytest.mark.parametrize("bad", [-3, 5])
def test_a_page_outside_the_pool_is_reported_not_read(bad, path, slot_of):
    w = make_config(2, with_logits=False)
    b = w.batch
    pools, k, v = stored(w)
    ctx = B.Context(b.model, 0)
    plan = B.Plan(ctx, b)
    plan.lr_plan_set_attention_path(path)
    q, cache = R.bf16_tensor(w.tensors.q, DEV), on_device(pools)
    out, slot = torch.zeros_like(q), slot_of(b)
    good = int(b.page_ids[slot])
    plan.lr_plan_debug_set_page(slot, bad if bad < 0 else int(b.n_pool_pages) + bad)
    plan.lr_verify_attention_fp8(q, cache, out)
    with pytest.raises(B.LrError) as e:
        plan.lr_poll_status()
    assert e.value.status == -5, e.value  # LR_EBOUNDS
    assert plan.lr_poll_status() == 0
    plan.lr_plan_debug_set_page(slot, good)
    plan.lr_verify_attention_fp8(q, cache, out)
    assert plan.lr_poll_status() == 0
    check_attention(out, None, O.verify_attention(b, w.tensors.q, k, v)[0], None)
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
    plan.lr_verify_attention_fp8(q, cache, out)
    with pytest.raises(B.LrError) as e:
        plan.lr_poll_status()
    assert e.value.status == -4, e.value  # LR_ETIMEOUT
    plan.lr_plan_debug_set_phantom_bytes(0)
    plan.lr_plan_debug_set_wait_limit(1_000_000)
    for _ in range(2):
        plan.lr_verify_attention_fp8(q, cache, out)
        assert plan.lr_poll_status() == 0
    check_attention(out, None, O.verify_attention(b, w.tensors.q, k, v)[0], None)
    plan.close()
    ctx.close()


@pytest.mark.parametrize("path", PATHS)
def test_a_cache_whose_bytes_pass_32_bits(path):
    """The batch's pages lie in the last of 270,000: rows written, attended to, compacted and read there."""
    w = chain([200, 37], seed=30)
    b, t = w.batch, w.tensors
    n, used = 270_000, int(b.n_pool_pages)
    at = tokens(b)
    k_rows, v_rows = (x[at[:, 0], :, at[:, 1]] for x in (t.k_pool, t.v_pool))
    pools = store_pools(t.k_pool, t.v_pool)
    k, v = as_bf16(pools[0], pools[2]), as_bf16(pools[1], pools[3])
    o_ref, l_ref = O.verify_attention(b, t.q, k, v)
    n_accept = np.asarray(b.br_n_draft, dtype=np.int32)
    c = O.commit(b, t.verdict, n_accept)
    want = O.compact(c["keep_off"], c["keep_pages"], c["keep_valid"], k, v)
    b.page_ids = b.page_ids + (n - used)
    b.n_pool_pages = n
    ctx = B.Context(b.model, 0)
    plan = B.Plan(ctx, b)
    plan.lr_plan_set_attention_path(path)
    cache = B.Fp8Cache.empty(b.model, n, DEV)
    slots = torch.from_numpy((at[:, 0] + (n - used)) * 16 + at[:, 1]).to(DEV)
    ctx.lr_fp8_write(cache, R.bf16_tensor(k_rows, DEV), R.bf16_tensor(v_rows, DEV), slots)
    q = R.bf16_tensor(t.q, DEV)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV)
    plan.lr_verify_attention_fp8(q, cache, out, lse)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)  # noqa: E731
    new_len, kept = (torch.zeros(b.n_req, dtype=torch.int32, device=DEV) for _ in range(2))
    plan.lr_compact_fp8(i32(c["keep_off"]), i32(c["keep_pages"] + (n - used)), i32(c["keep_valid"]), cache, new_len, kept)
    assert plan.lr_poll_status() == 0
    check_attention(out, lse, o_ref, l_ref, None, REL_LARGE)
    assert np.array_equal(new_len.cpu().numpy(), want[0]) and np.array_equal(kept.cpu().numpy(), want[1])
    for r in range(b.n_req):
        pages = c["keep_pages"][c["keep_off"][r]:c["keep_off"][r + 1]]
        place = np.array([int(pages[i // 16]) * 16 + i % 16 for i in range(int(want[0][r]))], dtype=np.int64)
        back = [torch.zeros((len(place), b.model.n_kv_heads, b.model.head_dim), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        ctx.lr_fp8_read(cache, torch.from_numpy(place + (n - used) * 16).to(DEV), *back)
        for got, ref in zip(back, want[2:]):
            assert np.array_equal(R.bf16_bits(got), ref[place // 16, :, place % 16])
    plan.close()
    ctx.close()


@pytest.mark.parametrize("make", [lambda: few_rows(64, 8, 8, 2, 31), lambda: chain([3000, 700, 65], q=40, seed=32), lambda: make_random_tree(9105)])
def test_the_same_bits_every_time(make):
    """Also beside another pass, whose leavings in shared and tensor memory differ."""
    w, other = make(), chain([1200], q=30, seed=33)
    ctx, plans, bufs = B.Context(w.batch.model, 0), [], []
    octx = B.Context(other.batch.model, 0)
    for c, x in ((ctx, w), (octx, other)):
        p = B.Plan(c, x.batch)
        p.lr_plan_set_attention_path(B.PATH_TENSOR_CORE)
        q = R.bf16_tensor(x.tensors.q, DEV)
        plans.append(p)
        bufs.append((q, on_device(stored(x)[0]), torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV)))
    first = None
    for i in range(12):
        if i % 3 == 2:
            plans[1].lr_verify_attention_fp8(*bufs[1])
        bufs[0][2].fill_(-3.0)
        plans[0].lr_verify_attention_fp8(*bufs[0])
        assert plans[0].lr_poll_status() == 0
        got = (R.bf16_bits(bufs[0][2]).copy(), bufs[0][3].cpu().numpy().view(np.uint32).copy())
        first = first or got
        assert all(np.array_equal(a, b) for a, b in zip(got, first)), i
    for x in plans + [ctx, octx]:
        x.close()
