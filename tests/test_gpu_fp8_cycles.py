"""The operators of the 8-bit cache in a row, as a serving engine uses them: prompt and drafted steps written, verified, sampled drafts accepted, committed
and compacted, cycle after cycle on one cache, against a model without pages that holds every row as it was stored."""
import numpy as np
import pytest
import torch

from fp8_util import as_bf16
from gpu_util import REL_LARGE, assert_attention_close
from lr_workloads import Model, bf16_round, bf16_to_f32, build_batch, fill_kv, fill_q, fill_verdicts
from oracle import lr_oracle as O
from paper_2506_19830_b200 import binding as B
from paper_2506_19830_b200 import runner as R
from paper_2506_19830_b200.cycle import BranchInput, PagedCycleEngine, RequestInput, SampledDrafts
from test_gpu_cycles import PAGE, _span_tokens

DEV = "cuda:0"


def _stored(bits):
    """What rows read back as."""
    return as_bf16(*O.fp8_store(bits))


def test_a_cache_type_that_there_is_not_is_refused():
    with pytest.raises(ValueError):
        PagedCycleEngine(Model(8, 2, 64, 1000), 4, kv_dtype="fp4")


def _drafts(b, rng, V):
    """Target rows, the drafter's near them, drafts sampled from those, uniform numbers."""
    cu = b.cu_draft
    rows = bf16_round((rng.standard_normal((int(cu[-1]) + b.n_branch, V)) * 3).astype(np.float32))
    at = np.array([i + x for x in range(b.n_branch) for i in range(cu[x], cu[x + 1])], dtype=np.int64)
    near = bf16_round(bf16_to_f32(rows[at]) + 0.5 * rng.standard_normal((len(at), V)).astype(np.float32))
    drafts = np.array([O.sample_inverse_cdf(O.target_probs(r, 1.0), rng.random()) for r in near], dtype=np.int32)
    f32 = lambda n: rng.random(n).astype(np.float32)  # noqa: E731
    return rows, SampledDrafts(near, 0.8, 1.0, f32(len(at)), f32(b.n_branch)), drafts


def _specs(rng, lengths, tree):
    specs = []
    for n in lengths:
        n_seg = int(rng.integers(1, 5))
        spec = {"P": n, "segs": [int(x) for x in rng.integers(3, 45, size=n_seg)], "branches": []}
        for node in range(n_seg + 1):
            L = int(rng.integers(1, 9))
            spec["branches"].append((node, L + int(rng.choice([0, 1, 5])), L, L))
        if tree:
            spec["parents"] = [int(rng.integers(0, c + 1)) for c in range(n_seg)]
        specs.append(spec)
    return specs


def _grown(b, ref, r, k, v):
    """The committed sequence of request r, from the pools before compaction."""
    kept = ref["keep_pages"][ref["keep_off"][r]:ref["keep_off"][r + 1]]
    valid = ref["keep_valid"][ref["keep_off"][r]:ref["keep_off"][r + 1]]
    none = np.zeros((0, b.model.n_kv_heads, b.model.head_dim), dtype=np.uint16)
    return [np.concatenate([x[int(p), :, :int(n), :].transpose(1, 0, 2) for p, n in zip(kept, valid)] or [none]) for x in (k, v)]


@pytest.mark.gpu
@pytest.mark.parametrize("head_dim,tree", [(128, False), (64, False), (128, True)])
@pytest.mark.parametrize("sampled", [False, True])
def test_cycles_keep_the_cache_equal_to_the_logical_sequences(head_dim, tree, sampled):
    rng = np.random.default_rng(head_dim + tree + 2 * sampled)
    V, n_req, n_pool = 500, 3, 600
    model = Model(8, 2, head_dim, V)
    eng = PagedCycleEngine(model, n_pool, kv_dtype="fp8")
    seq = []
    for r in range(n_req):
        n0 = int(rng.choice([0, 16, 37, 130]))
        k0, v0 = (bf16_round(rng.standard_normal((n0, 2, head_dim)).astype(np.float32)) for _ in range(2))
        assert eng.add_request(k0, v0) == r
        seq.append((_stored(k0), _stored(v0)))
    for cycle in range(5):
        specs = _specs(rng, [len(x[0]) for x in seq], tree)
        b = build_batch(model, specs, rng)
        k, v = fill_kv(b, rng, poison="zero")
        new_k, new_v = k.copy(), v.copy()  # as they come; in the cache as they are stored
        k, v = _stored(k), _stored(v)
        for r in range(n_req):
            for t in range(len(seq[r][0])):
                pg = int(b.page_ids[int(b.span_slot[int(b.req_span_off[r])]) + t // PAGE])
                k[pg, :, t % PAGE, :], v[pg, :, t % PAGE, :] = seq[r][0][t], seq[r][1][t]
        q, (rows, how, drafts) = fill_q(b, rng), _drafts(b, rng, V)
        verdict = fill_verdicts(b, rng, 0.6)
        if sampled:
            u = [x.astype(np.float64) for x in (how.u_accept, how.u_final)]
            n_ref, id_ref = O.accept_sample_drafted(rows, how.logits, drafts, b.cu_draft, float(np.float32(how.temperature)), how.draft_temperature, *u)[:2]
        else:
            n_ref, id_ref = O.accept_greedy(rows, drafts, b.cu_draft)[:2]
        o_ref, ref = O.verify_attention(b, q, k, v)[0], O.commit(b, verdict, n_ref)
        inputs = []
        for r in range(n_req):
            s0, s1 = int(b.req_span_off[r]), int(b.req_span_off[r + 1])
            tokens = lambda slot, n: tuple(_span_tokens(b, x, int(slot), int(n)) for x in (new_k, new_v))  # noqa: E731
            segs = [tokens(b.span_slot[s], b.span_len[s]) for s in range(s0 + 1, s1)]
            brs = [BranchInput(int(b.br_depth[i]), *tokens(b.br_own_slot[i], b.br_own_len[i]), int(b.cu_q[i + 1] - b.cu_q[i]), int(b.br_n_draft[i]))
                   for i in range(b.n_branch) if b.br_req[i] == r]
            inputs.append(RequestInput(segs, brs, specs[r].get("parents", ())))
        got = eng.run_cycle(inputs, q, rows, drafts, verdict, how if sampled else None)
        assert np.array_equal(got["n_accept"], n_ref) and np.array_equal(got["bonus_id"], id_ref)
        for key in ("n_steps_accepted", "survivor", "committed_len"):
            assert np.array_equal(got[key], ref[key]), (cycle, key)
        assert_attention_close(np.abs(bf16_to_f32(got["out"]).astype(np.float64) - o_ref), o_ref, REL_LARGE)
        for r in range(n_req):
            seq[r] = _grown(b, ref, r, k, v)
            gk, gv = eng.sequence(r)
            assert eng.length[r] == ref["committed_len"][r] == len(seq[r][0]) and np.array_equal(gk, seq[r][0]) and np.array_equal(gv, seq[r][1]), (cycle, r)
        assert sorted([p for pages in eng.pages for p in pages] + eng.free) == list(range(n_pool))


@pytest.mark.gpu
def test_a_captured_cycle():
    """All five calls in one graph, replayed on other rows: what they leave is what they leave one by one."""
    rng = np.random.default_rng(9)
    V = 700
    model = Model(8, 2, 128, V)
    b = build_batch(model, _specs(rng, [170, 33], False), rng)
    q = fill_q(b, rng)
    rows, how, drafts = _drafts(b, rng, V)
    verdict = fill_verdicts(b, rng, 0.6)
    ctx = B.Context(model, 0)
    plan = B.Plan(ctx, b)
    spans = list(zip(b.span_slot, b.span_len)) + list(zip(b.br_own_slot, b.br_own_len))
    slots = np.array([int(b.page_ids[int(f) + t // PAGE]) * PAGE + t % PAGE for f, n in spans for t in range(int(n))], dtype=np.int64)
    n = len(slots)
    to = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a, dtype=dt)).to(DEV)  # noqa: E731
    slots_d, new = to(slots, np.int64), torch.zeros((n, 4 * 128), dtype=torch.bfloat16, device=DEV)
    k, v = new[:, :256].view(n, 2, 128), new[:, 256:].view(n, 2, 128)
    cache, qd = B.Fp8Cache.empty(model, b.n_pool_pages, DEV), R.bf16_tensor(q, DEV)
    out, y = torch.zeros_like(qd), R.PassOutputs(b, DEV, n_rows=1)
    vocab8 = (V + 7) // 8 * 8
    td, dd = (torch.zeros((x.shape[0], vocab8), dtype=torch.bfloat16, device=DEV)[:, :V] for x in (rows, how.logits))
    td.copy_(R.bf16_tensor(rows, DEV))
    dd.copy_(R.bf16_tensor(how.logits, DEV))
    scratch = ctx.accept_sample_drafted_scratch(rows.shape[0])
    n_acc, ids, new_len, kept = (torch.zeros(m, dtype=torch.int32, device=DEV) for m in (b.n_branch, b.n_branch, b.n_req, b.n_req))
    args = (to(drafts, np.int32), to(b.cu_draft, np.int32), how.temperature, how.draft_temperature, to(how.u_accept, np.float32), to(how.u_final, np.float32))
    verdict_d = to(verdict, np.uint8)

    def calls():
        ctx.lr_fp8_write(cache, k, v, slots_d)
        plan.lr_verify_attention_fp8(qd, cache, out)
        ctx.lr_accept_sample_drafted(td, dd, *args, n_acc, ids, scratch)
        plan.lr_commit(verdict_d, n_acc, y.n_steps_accepted, y.survivor, y.committed_len, y.keep_off, y.keep_pages, y.keep_valid, y.free_off, y.free_pages)
        plan.lr_compact_fp8(y.keep_off, y.keep_pages, y.keep_valid, cache, new_len, kept)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for seed in (1, 2):
        bits = bf16_round(np.random.default_rng(seed).standard_normal((2, n, 2, 128)).astype(np.float32))
        k.copy_(R.bf16_tensor(bits[0], DEV))
        v.copy_(R.bf16_tensor(bits[1], DEV))
        graph.replay()
        assert plan.lr_poll_status() == 0
        pools = [np.zeros((b.n_pool_pages, 2, PAGE, 128), dtype=np.uint16) for _ in range(2)]
        for pool, x in zip(pools, bits):
            pool[slots // PAGE, :, slots % PAGE] = _stored(x)
        o_ref = O.verify_attention(b, q, *pools)[0]
        assert_attention_close(np.abs(bf16_to_f32(R.bf16_bits(out)).astype(np.float64) - o_ref), o_ref, REL_LARGE)
        ref = O.commit(b, verdict, n_acc.cpu().numpy())
        for r in range(b.n_req):
            want, m = _grown(b, ref, r, *pools), int(new_len[r])
            pages = y.keep_pages.cpu().numpy()[ref["keep_off"][r]:]
            at = to([int(pages[t // PAGE]) * PAGE + t % PAGE for t in range(m)], np.int64)
            back = [torch.zeros((m, 2, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
            ctx.lr_fp8_read(cache, at, *back)
            assert m == len(want[0]) and all(np.array_equal(R.bf16_bits(g), w) for g, w in zip(back, want))
    del graph
    plan.close()
    ctx.close()
