"""The operators in a row, as a serving engine uses them: prompt and drafted steps turned to their positions and written, verified, accepted, committed and
compacted, a request forked, cycle after cycle on one cache, against a model without pages that holds every row as it was stored."""
import numpy as np
import pytest
import torch

import fp4_util
from fp8_util import as_bf16 as fp8_as_bf16
from gpu_util import REL_LARGE, assert_attention_close
from lr_workloads import Model, bf16_round, bf16_to_f32, build_batch, fill_kv, fill_logits_and_drafts, fill_q, fill_verdicts
from oracle import lr_oracle as O
from paper_2506_19830_b200 import binding as B
from paper_2506_19830_b200 import runner as R
from paper_2506_19830_b200.cycle import BranchInput, PagedCycleEngine, RequestInput
from test_gpu_cycles import PAGE, _span_tokens
from test_gpu_fp8_cycles import _grown, _specs

DEV = "cuda:0"
STORE = {"bf16": lambda x: x, "fp8": lambda x: fp8_as_bf16(*O.fp8_store(x)), "mxfp4": lambda x: fp4_util.as_bf16(*O.fp4_store(x))}


def _positions(b, specs, r):
    """Per span of request r where its first token stands, then per branch."""
    s0 = int(b.req_span_off[r])
    n_span = int(b.req_span_off[r + 1]) - s0
    parents = specs[r].get("parents", list(range(n_span - 1)))
    first, behind = [0], [int(b.span_len[s0])]
    for c in range(1, n_span):
        first.append(behind[parents[c - 1]])
        behind.append(first[-1] + int(b.span_len[s0 + c]))
    return first, [behind[int(b.br_depth[i])] for i in range(b.n_branch) if b.br_req[i] == r]


@pytest.mark.gpu
@pytest.mark.parametrize("kv_dtype,head_dim,tree,turned", [("mxfp4", 128, False, False), ("mxfp4", 64, True, False), ("mxfp4", 128, True, True), ("fp8", 64, False, True), ("bf16", 128, True, True)])
def test_cycles_keep_the_cache_equal_to_the_logical_sequences(kv_dtype, head_dim, tree, turned):
    """Turned keys are taken from the engine as it stored them (how they are turned is tested elsewhere; that they are, and where, below)."""
    rng = np.random.default_rng(head_dim + tree + 2 * turned)
    V, n_req, n_pool = 500, 3, 700
    model = Model(8, 2, head_dim, V)
    rope = B.Rope(head_dim // 2, base=1e4, interleaved=tree) if turned else None
    freq = O.rope_frequencies(head_dim // 2, 1e4)[0]
    eng = PagedCycleEngine(model, n_pool, kv_dtype=kv_dtype, rope=rope)
    store = STORE[kv_dtype]

    def turn(bits, first):
        """Rows at positions from `first` on as the engine's projection hands them over -> as they come to the cache, through the call itself."""
        if not turned or len(bits) == 0:
            return bits
        x = bf16_to_f32(bits).astype(np.float64)
        want = O.rope(x, np.arange(first, first + len(bits)), freq, interleaved=tree)
        n, h = bits.shape[:2]
        out = torch.zeros(bits.shape, dtype=torch.bfloat16, device=DEV)
        side = B.Context(Model(h, h, head_dim, 8), 0)
        pool = B.Bf16Cache(*torch.zeros((2, n // PAGE + 1, h, PAGE, head_dim), dtype=torch.bfloat16, device=DEV))
        xd = R.bf16_tensor(bits, DEV)
        side.lr_rope_write(rope, torch.arange(first, first + n, dtype=torch.int32, device=DEV), pool, xd, xd, torch.arange(n, device=DEV), xd, out)
        got = R.bf16_bits(out)
        assert (np.abs(bf16_to_f32(got) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -18).all()
        side.close()
        return got

    # Keys of a cache in 8 or 4 bits are rounded once, from what was turned in fp32; the model takes those the engine holds, within a step of the exact ones.
    def stored_keys(bits, first, pages):
        if not turned or kv_dtype == "bf16":
            return store(turn(bits, first))
        n = len(bits)
        back = [torch.zeros((n, 2, head_dim), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        (eng.ctx.lr_fp8_read if kv_dtype == "fp8" else eng.ctx.lr_fp4_read)(eng.cache, eng._slots(pages, n), *back)
        got = R.bf16_bits(back[0])
        want = O.rope(bf16_to_f32(bits).astype(np.float64), np.arange(first, first + n), freq, interleaved=tree)
        top = np.abs(want).max(-1, keepdims=True)
        assert (np.abs(bf16_to_f32(got) - want) <= (2.0 ** -4 if kv_dtype == "fp8" else 0.34) * top).all()  # (half a step of the largest codes, 1 of 3 at the most)
        return got

    seq = []
    for r in range(n_req):
        n0 = int(rng.choice([0, 16, 37, 130]))
        k0, v0 = (bf16_round(rng.standard_normal((n0, 2, head_dim)).astype(np.float32)) for _ in range(2))
        assert eng.add_request(k0, v0) == r
        seq.append((stored_keys(k0, 0, eng.pages[r]), store(v0)))
    for cycle in range(4):
        if cycle == 2:  # another answer to the second request's prompt
            assert eng.fork(1) == n_req
            seq.append(tuple(x.copy() for x in seq[1]))
            n_req += 1
            assert not set(eng.pages[1]) & set(eng.pages[-1])
        specs = _specs(rng, [len(x[0]) for x in seq], tree)
        b = build_batch(model, specs, rng)
        new_k, new_v = fill_kv(b, rng, poison="zero")
        q = fill_q(b, rng)
        rows, drafts, _ = fill_logits_and_drafts(b, rng, 0.3)
        verdict = fill_verdicts(b, rng, 0.6)
        n_ref, id_ref = O.accept_greedy(rows, drafts, b.cu_draft)[:2]
        inputs, q_turned = [], q.copy()
        for r in range(n_req):
            s0, s1 = int(b.req_span_off[r]), int(b.req_span_off[r + 1])
            tokens = lambda slot, n: tuple(_span_tokens(b, x, int(slot), int(n)) for x in (new_k, new_v))  # noqa: E731
            segs = [tokens(b.span_slot[s], b.span_len[s]) for s in range(s0 + 1, s1)]
            mine = [i for i in range(b.n_branch) if b.br_req[i] == r]
            brs = [BranchInput(int(b.br_depth[i]), *tokens(b.br_own_slot[i], b.br_own_len[i]), int(b.cu_q[i + 1] - b.cu_q[i]), int(b.br_n_draft[i])) for i in mine]
            for i, at in zip(mine, _positions(b, specs, r)[1]):
                q0, q1 = int(b.cu_q[i]), int(b.cu_q[i + 1])
                q_turned[q0:q1] = turn(q[q0:q1], at + int(b.br_own_len[i]) - (q1 - q0))
            inputs.append(RequestInput(segs, brs, specs[r].get("parents", ())))
        # the engine's pages of the drafted tokens: the order in which it takes them from its free list
        free, taken = list(eng.free), []
        for x in inputs:
            for n in [len(s[0]) for s in x.segs] + [len(y.k_tail) for y in x.branches]:
                taken.append([free.pop() for _ in range((n + PAGE - 1) // PAGE)])
        caught = {}
        if turned and kv_dtype != "bf16":
            compact = "lr_compact_fp8" if kv_dtype == "fp8" else "lr_compact_fp4"
            original = getattr(B.Plan, compact)

            def look(self, *a, **kw):  # what is stored, before compaction moves it
                caught["at"] = 1
                j = 0
                for r in range(n_req):
                    s0, s1 = int(b.req_span_off[r]), int(b.req_span_off[r + 1])
                    first, tails = _positions(b, specs, r)
                    spans = [(int(b.span_slot[s]), int(b.span_len[s]), first[s - s0]) for s in range(s0 + 1, s1)]
                    spans += [(int(b.br_own_slot[i]), int(b.br_own_len[i]), at) for i, at in zip([i for i in range(b.n_branch) if b.br_req[i] == r], tails)]
                    for slot, n, at in spans:
                        caught[slot] = stored_keys(_span_tokens(b, new_k, slot, n), at, taken[j])
                        j += 1
                return original(self, *a, **kw)

            setattr(B.Plan, compact, look)
        try:
            got = eng.run_cycle(inputs, q, rows, drafts, verdict)
        finally:
            if turned and kv_dtype != "bf16":
                setattr(B.Plan, compact, original)
        k, v = np.zeros_like(new_k), store(new_v)
        for r in range(n_req):
            s0, s1 = int(b.req_span_off[r]), int(b.req_span_off[r + 1])
            first, tails = _positions(b, specs, r)
            spans = [(int(b.span_slot[s]), int(b.span_len[s]), first[s - s0]) for s in range(s0 + 1, s1)]
            spans += [(int(b.br_own_slot[i]), int(b.br_own_len[i]), at) for i, at in zip([i for i in range(b.n_branch) if b.br_req[i] == r], tails)]
            for slot, n, at in spans:
                x = caught[slot] if caught else store(turn(_span_tokens(b, new_k, slot, n), at))
                for t in range(n):
                    k[int(b.page_ids[slot + t // PAGE]), :, t % PAGE] = x[t]
            for t in range(len(seq[r][0])):
                pg = int(b.page_ids[int(b.span_slot[s0]) + t // PAGE])
                k[pg, :, t % PAGE, :], v[pg, :, t % PAGE, :] = seq[r][0][t], seq[r][1][t]
        o_ref, ref = O.verify_attention(b, q_turned, k, v)[0], O.commit(b, verdict, n_ref)
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
def test_a_captured_pass():
    """Rotation with the write, attention, compaction and a fork in one graph, replayed at other positions: what they leave is what they leave one by one."""
    rng = np.random.default_rng(9)
    model = Model(8, 2, 128, 16)
    b = build_batch(model, _specs(rng, [170, 33], False), rng)
    ctx = B.Context(model, 0)
    plan = B.Plan(ctx, b)
    verdict = fill_verdicts(b, rng, 0.6)
    c = O.commit(b, verdict, np.asarray(b.br_n_draft, dtype=np.int32))
    spans = list(zip(b.span_slot, b.span_len)) + list(zip(b.br_own_slot, b.br_own_len))
    slots = np.array([int(b.page_ids[int(f) + t // PAGE]) * PAGE + t % PAGE for f, n in spans for t in range(int(n))], dtype=np.int64)
    n, nq = len(slots), int(b.cu_q[-1])
    to = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a, dtype=dt)).to(DEV)  # noqa: E731
    joint = torch.zeros((n, 12, 128), dtype=torch.bfloat16, device=DEV)
    at, slots_d, rope = torch.zeros(n, dtype=torch.int32, device=DEV), to(slots, np.int64), B.Rope(128)
    used = np.unique(slots // PAGE).astype(np.int32)
    lists = [to(c[x], np.int32) for x in ("keep_off", "keep_pages", "keep_valid")]

    def state():
        return SimpleState(B.Fp4Cache.empty(model, b.n_pool_pages, DEV), B.Fp4Cache.empty(model, len(used), DEV),
                           torch.zeros((n, 8, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((nq, 8, 128), dtype=torch.bfloat16, device=DEV),
                           *(torch.zeros(b.n_req, dtype=torch.int32, device=DEV) for _ in range(2)))

    class SimpleState:
        def __init__(self, cache, fork, turned, out, new_len, kept):
            self.cache, self.fork, self.turned, self.out, self.new_len, self.kept = cache, fork, turned, out, new_len, kept

    def calls(s):
        ctx.lr_rope_write(rope, at, s.cache, joint[:, 8:10], joint[:, 10:], slots_d, joint[:, :8], s.turned)
        plan.lr_verify_attention_fp4(s.turned[:nq], s.cache, s.out)
        plan.lr_compact_fp4(*lists, s.cache, s.new_len, s.kept)
        ctx.lr_copy_pages(s.cache, s.fork, to_used, to_fork)

    to_used, to_fork = to(used, np.int32), torch.arange(len(used), dtype=torch.int32, device=DEV)
    a, one = state(), state()
    calls(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(a)
    for seed in (1, 2):
        joint.copy_(R.bf16_tensor(bf16_round(np.random.default_rng(seed).standard_normal((n, 12, 128)).astype(np.float32)), DEV))
        at.copy_(torch.arange(seed * 1000, seed * 1000 + n, device=DEV))
        graph.replay()
        assert plan.lr_poll_status() == 0
        calls(one)
        assert plan.lr_poll_status() == 0
        assert torch.equal(a.turned, one.turned) and torch.equal(a.out, one.out) and torch.equal(a.new_len, one.new_len)
        for x, y in zip(fp4_util.back(a.cache) + fp4_util.back(a.fork), fp4_util.back(one.cache) + fp4_util.back(one.fork)):
            assert np.array_equal(x, y)
        for x, y in zip(fp4_util.back(a.cache), fp4_util.back(a.fork)):
            assert np.array_equal(x[used], y)
    del graph
    plan.close()
    ctx.close()


def test_a_cache_type_that_there_is_not_is_refused():
    with pytest.raises(ValueError, match="mxfp4"):
        PagedCycleEngine(Model(8, 2, 64, 1000), 4, kv_dtype="int4")
