"""The operators of a verify pass over an 8-bit cache, and of one whose drafts come from a draft model, as cases that can be timed
and compared: every case once in its plain form (elementary torch operations) and once as calls of the package.

The cache.  Pools of e4m3 codes [pages][KV heads][16][head size] and one power-of-two scale byte (e8m0, bias 127) for every token and
KV head.  A row x of K or V is stored with the smallest exponent e >= -124 for which max|x| 2^-e <= 448: the codes are x 2^-e rounded
to the nearest e4m3 value, the byte is e + 127; a row with an infinity or a NaN gets codes 0 and the byte 255, which reads as NaN.

Operators (a case's ``op``):
  write    K/V rows of a projection's output, quantised into the slots they are given
  read     rows of the cache back as bf16
  attend   the nested-prefix attention of a verify pass (chain or tree of draft steps) over such a cache
  compact  the drafted tokens of a cycle written, then the committed ones packed densely into the leading kept pages
  accept   rejection sampling of drafts that a draft model sampled, against both models' logits

``lengths`` seeds the lengths of a case, so its work is fixed; ``prepare``'s seed gives the values and the page table.
"""
from __future__ import annotations

import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

DEV = "cuda:0"
PAGE = 16

BASE = {
    "op": "attend", "q_heads": 40, "kv_heads": 8, "head_dim": 128, "requests": 1, "prefix_min": 4096, "prefix_max": 4096, "steps_min": 3,
    "steps_max": 3, "seg_min": 32, "seg_max": 32, "drafts_min": 16, "drafts_max": 16, "tree_width": 0, "tokens": 0, "vocab": 0,
    "temperature": 0.6, "draft_temperature": 0.6, "lengths": 1,
}
SERVING = {"requests": 16, "prefix_min": 1024, "prefix_max": 16384, "steps_min": 2, "steps_max": 6, "seg_min": 16, "seg_max": 64,
           "drafts_min": 4, "drafts_max": 16, "lengths": 5}


def listed():
    def case(name, op, **kw):
        return dict(BASE, name=name, op=op, **kw)

    return [
        # the drafted tokens of one serving pass go into the cache: once a layer, latency counts
        case("write_drafts", "write", tokens=356),
        # a long prompt goes into the cache
        case("write_prompt", "write", tokens=32768),
        # one accepted step is handed on in bf16
        case("read_step", "read", tokens=61),
        # a prompt shared with a program that keeps its cache in bf16
        case("read_prompt", "read", tokens=16384),
        # the smallest call: one request early in its answer takes one token without drafts
        case("attend_token", "attend", prefix_min=250, prefix_max=250, steps_min=0, steps_max=0, drafts_min=1, drafts_max=1),
        # one request at 32 K tokens with deep speculation: many query rows for one cache
        case("attend_long", "attend", q_heads=32, prefix_min=32768, prefix_max=32768, steps_min=6, steps_max=6, seg_min=40, seg_max=40),
        # a serving batch: ragged lengths everywhere
        case("attend_serving", "attend", **SERVING),
        # multi-branch drafting for a model with heads of 64: two proposals a step, two steps deep, a branch on every node
        case("attend_tree64", "attend", **dict(SERVING, q_heads=32, head_dim=64, requests=8, steps_min=2, steps_max=2, tree_width=2)),
        # the end of a cycle of one request at 4 K tokens
        case("compact_one", "compact"),
        # ... and of a serving batch
        case("compact_serving", "compact", **dict(SERVING, prefix_max=4096)),
        # one request's drafts, sampled by a draft model of the same vocabulary
        case("accept_one", "accept", vocab=152064),
        # a serving batch's drafts
        case("accept_serving", "accept", vocab=152064, **SERVING),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        w, m = work(c), most.setdefault(c["op"], {"bytes": 0.0, "flops": 0.0})
        most[c["op"]] = {k: max(w[k], m[k]) for k in m}
    while True:
        op = rng.choices(["write", "read", "attend", "compact", "accept"], [15, 12, 43, 12, 18])[0]
        hq, hkv, hd = rng.choice([(40, 8, 128)] * 3 + [(32, 8, 128)] * 2 + [(16, 4, 128), (8, 8, 128), (5, 1, 128), (16, 1, 128), (32, 8, 64), (12, 4, 64), (4, 1, 64)])
        pmax, smax, dmax = _log_int(rng, 20, 32768), _log_int(rng, 2, 80), rng.randint(1, 20)
        tree = rng.choice([0, 0, 0, 2, 3, 4]) if op == "attend" else 0
        gmax = rng.randint(1, 2) if tree else rng.randint(0, 6)
        c = dict(BASE, op=op, q_heads=hq, kv_heads=hkv, head_dim=hd, requests=_log_int(rng, 1, 48), prefix_min=int(pmax * rng.uniform(0.1, 1.0)),
                 prefix_max=pmax, steps_min=rng.randint(min(1, gmax), gmax), steps_max=gmax, seg_min=rng.randint(1, smax), seg_max=smax,
                 drafts_min=rng.randint(1, dmax), drafts_max=dmax, tree_width=tree, lengths=rng.randrange(1 << 20))
        if op in ("write", "read"):
            c["tokens"] = _log_int(rng, 1, 32768)
        if op == "accept":
            c.update(vocab=_log_int(rng, 1000, 152064), temperature=round(rng.uniform(0.4, 1.2), 2), draft_temperature=round(rng.uniform(0.4, 1.2), 2))
        w = work(c)
        if all(w[k] <= most[op][k] for k in w):
            return c


# ---- the batch of a case ------------------------------------------------------------------------------------------------
def _requests(case):
    """Per request: prefix length, step lengths, the step each step continues (0: the prefix), branches (node, drafts)."""
    rng = random.Random(case["lengths"])
    between = lambda a: rng.randint(case[a + "_min"], case[a + "_max"])  # noqa: E731
    out = []
    for _ in range(case["requests"]):
        prefix, depth, n_draft, parents = between("prefix"), between("steps"), between("drafts"), []
        if case["tree_width"]:  # a full tree of draft steps, numbered level by level
            level = [0]
            for _ in range(depth):
                parents += [p for p in level for _ in range(case["tree_width"])]
                level = list(range(len(parents) - len(level) * case["tree_width"] + 1, len(parents) + 1))
            nodes = range(len(parents) + 1)
        else:
            parents = list(range(depth))
            nodes = range(1, depth + 1) if depth else [0]
        out.append(SimpleNamespace(prefix=prefix, segs=[between("seg") for _ in parents], parents=parents, branches=[(n, n_draft) for n in nodes]))
    return out


def _path(parents, node):
    """The steps from the prefix to a node."""
    path = []
    while node:
        path.append(node)
        node = parents[node - 1]
    return path[::-1]


def _pages(n):
    return (n + PAGE - 1) // PAGE


def _drafts(case):
    return [n for r in _requests(case) for _, n in r.branches]


def work(case):
    h, d = case["kv_heads"], case["head_dim"]
    if case["op"] in ("write", "read"):
        n = case["tokens"]
        return {"bytes": 2.0 * n * h * (3 * d + 1) + 8.0 * n, "flops": 2.0 * n * h * d}
    reqs = _requests(case)
    if case["op"] == "accept":
        drafts = _drafts(case)
        return {"bytes": 2.0 * case["vocab"] * (2 * sum(drafts) + len(drafts)), "flops": 4.0 * case["vocab"] * (2 * sum(drafts) + len(drafts))}
    if case["op"] == "compact":  # every drafted token written; half of them moved
        n = sum(sum(r.segs) + sum(b[1] for b in r.branches) for r in reqs)
        return {"bytes": 2.0 * n * h * (4 * d + 2), "flops": 2.0 * n * h * d}
    rows = kv = seen = 0
    for r in reqs:
        kv += r.prefix + sum(r.segs)
        for node, n in r.branches:
            rows += n
            kv += n
            seen += n * (r.prefix + sum(r.segs[s - 1] for s in _path(r.parents, node))) + n * (n + 1) // 2
    hq = case["q_heads"]
    return {"bytes": 2.0 * kv * h * (d + 1) + 4.0 * rows * hq * d + 4.0 * rows * hq, "flops": 4.0 * hq * d * seen}


def _batch(case, rng):
    """The integer tables of a batch: page slots in the order prefix, steps, tails of each request; shuffled pages."""
    t = {k: [] for k in ("span_len", "span_slot", "br_req", "br_depth", "br_own_len", "br_own_slot", "br_n_draft", "seg_parent")}
    reqs, slot, off, cu_q = _requests(case), 0, [0], [0]
    for r, q in enumerate(reqs):
        for n, parent in zip([q.prefix] + q.segs, [-1] + q.parents):
            t["span_len"].append(n)
            t["span_slot"].append(slot)
            t["seg_parent"].append(parent)
            slot += _pages(n)
        off.append(len(t["span_len"]))
        for node, n in q.branches:
            for k, v in (("br_req", r), ("br_depth", node), ("br_own_len", n), ("br_own_slot", slot), ("br_n_draft", n)):
                t[k].append(v)
            cu_q.append(cu_q[-1] + n)
            slot += _pages(n)
    n_pool = slot + slot // 4 + 1
    b = SimpleNamespace(**{k: np.asarray(v, dtype=np.int32) for k, v in t.items()}, req_span_off=np.asarray(off, dtype=np.int32), n_pool_pages=n_pool,
                        cu_q=np.asarray(cu_q, dtype=np.int32), page_ids=rng.permutation(n_pool)[:slot].astype(np.int32), reqs=reqs)
    if not case["tree_width"]:
        b.seg_parent = None
    return b


def _slots(b, first, n):
    """The token slots (page x 16 + place) of a span of n tokens."""
    at = np.arange(n)
    return b.page_ids[first + at // PAGE].astype(np.int64) * PAGE + at % PAGE


def _keys_and_rows(b):
    """For every request the keys of its cache and its query rows, padded to the longest: where a key lies, the depth-first numbers of
    the nodes that see it, the branch that owns it (-1: padding), its place in the branch's tail; a row's node, branch and place."""
    keys, rows, br = [], [], 0
    for r, q in enumerate(b.reqs):
        tin, last, count = {}, {}, 0
        todo = [(0, False)]
        children = {n: [i + 1 for i, p in enumerate(q.parents) if p == n] for n in range(len(q.segs) + 1)}
        while todo:
            n, done = todo.pop()
            if done:
                last[n] = count - 1
                continue
            tin[n], count = count, count + 1
            todo += [(n, True)] + [(c, False) for c in children[n][::-1]]
        s0, parts, mine = int(b.req_span_off[r]), [], []
        for c in range(len(q.segs) + 1):
            n = int(b.span_len[s0 + c])
            parts.append(np.stack([_slots(b, int(b.span_slot[s0 + c]), n), *(np.full(n, v) for v in (tin[c], last[c], 0)), np.zeros(n, dtype=np.int64)]))
        for i, (node, n) in enumerate(q.branches):
            parts.append(np.stack([_slots(b, int(b.br_own_slot[br]), n), *(np.full(n, v) for v in (0, 0, i + 1)), np.arange(n)]))
            mine.append(np.stack([np.full(n, tin[node]), np.full(n, i + 1), np.arange(n)]))
            br += 1
        keys.append(np.concatenate(parts, axis=1))
        rows.append(np.concatenate(mine, axis=1))
    n_key, n_row = max(k.shape[1] for k in keys), max(r.shape[1] for r in rows)
    pad = lambda a, n, v: np.concatenate([a, np.tile(v[:, None], n - a.shape[1])], axis=1)  # noqa: E731
    k = np.stack([pad(a, n_key, np.array([a[0, 0], 0, 0, -1, 0])) for a in keys])
    q = np.stack([pad(a, n_row, np.array([-1, -2, 0])) for a in rows])
    return torch.from_numpy(k).to(DEV), torch.from_numpy(q).to(DEV)


# ---- the plain forms of the 8-bit cache --------------------------------------------------------------------------------
def _quantise(x):
    """Codes and scale bytes of rows [..., head size]."""
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    half, exponent = torch.frexp(top)  # top = half 2^exponent, 1/2 <= half < 1
    e = (exponent - 9 + (half > 0.875).to(torch.int32)).clamp(min=-124)
    fine = torch.isfinite(top)
    e = torch.where(fine, e, torch.zeros_like(e))
    codes = torch.where(fine, x * _power(-e), torch.zeros_like(x)).to(torch.float8_e4m3fn)
    return codes, torch.where(fine, e + 127, torch.full_like(e, 255)).to(torch.uint8)[..., 0]


def _power(e):
    """2^e, for whole -126 <= e <= 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _values(codes, scale):
    s = torch.where(scale == 255, torch.full(scale.shape, math.nan, device=scale.device), _power(scale.to(torch.int32) - 127))
    return codes.float() * s[..., None]


def _gather(pool, slots):
    """Rows [..., KV heads, head size] of a pool (or its scales) at token slots."""
    got = pool.view(torch.uint8)[slots // PAGE, :, slots % PAGE]
    return got.view(torch.float8_e4m3fn) if pool.dim() == 4 else got


def _put(pool, slots, rows):
    pool.view(torch.uint8)[slots // PAGE, :, slots % PAGE] = rows.view(torch.uint8)


def _write(s):
    keep = s.slots >= 0
    at = s.slots[keep]
    for rows, pool, scale in ((s.k, s.cache.k, s.cache.k_scale), (s.v, s.cache.v, s.cache.v_scale)):
        codes, byte = _quantise(rows)
        _put(pool, at, codes[keep])
        _put(scale, at, byte[keep])


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _rows(gen, n, heads, d, spread=True):
    """K or V rows as a layer gives them: heads and tokens of different sizes, some channels far above the others."""
    x = torch.empty((n, heads, d), device=DEV).normal_(generator=gen)
    if spread:
        x *= torch.exp(0.5 * torch.empty((n, heads, 1), device=DEV).normal_(generator=gen))
        x[..., 3] *= 8.0
    return x.to(torch.bfloat16)


def _cache(pages, heads, d):
    """An empty cache."""
    pool = lambda: torch.zeros((pages, heads, PAGE, d), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)  # noqa: E731
    scale = lambda: torch.full((pages, heads, PAGE), 127, dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu)  # noqa: E731
    return SimpleNamespace(k=pool(), v=pool(), k_scale=scale(), v_scale=scale())


def _fill(cache, gen, slots, h, d):
    """Rows of a model in some slots of a cache."""
    for pool, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        for at in slots.split(16384):
            codes, byte = _quantise(_rows(gen, len(at), h, d))
            _put(pool, at, codes)
            _put(scale, at, byte)


def _projection(gen, n, hq, h, d):
    """K and V of n tokens as they lie in the output of a joint projection [tokens, (q + 2 KV heads) x head size]."""
    joint = torch.zeros((n, hq + 2 * h, d), dtype=torch.bfloat16, device=DEV)
    joint[:, hq:hq + h] = _rows(gen, n, h, d)
    joint[:, hq + h:] = _rows(gen, n, h, d)
    return joint[:, hq:hq + h], joint[:, hq + h:]


def _logits(s, gen, drafts, vocab, t_draft):
    """Target rows: a broad background, one leading token and a few alternatives; draft rows: the same with another model's errors, and
    drafts sampled from them.  Row stride: the vocabulary rounded up to 8 values, what lies behind it is not a number."""
    stride, n_rows = (vocab + 7) // 8 * 8, sum(drafts) + len(drafts)
    full = torch.full((n_rows, stride), math.nan, dtype=torch.bfloat16, device=DEV)
    rows = torch.empty((n_rows, vocab), device=DEV).normal_(0.0, 1.5, generator=gen)
    lead = 6.0 + 8.0 * torch.rand((n_rows, 1), device=DEV, generator=gen)
    gap = torch.empty((n_rows, 20), device=DEV).exponential_(0.4, generator=gen)
    lead_id = torch.randint(0, vocab, (n_rows, 1), device=DEV, generator=gen)
    rows.scatter_(1, (lead_id + torch.arange(1, 21, device=DEV) * (vocab // 21)) % vocab, lead - gap)
    rows.scatter_(1, lead_id, lead)
    full[:, :vocab] = rows
    s.logits = full[:, :vocab]
    with_draft = torch.ones(n_rows, dtype=torch.bool)
    with_draft[np.cumsum(np.asarray(drafts) + 1) - 1] = False
    s.target_row = with_draft.nonzero()[:, 0].to(DEV)
    other = rows[s.target_row]
    other += torch.empty_like(other).normal_(0.0, 0.5, generator=gen)
    full = torch.full((max(1, sum(drafts)), stride), math.nan, dtype=torch.bfloat16, device=DEV)
    full[:sum(drafts), :vocab] = other
    s.draft_logits = full[:, :vocab]
    noise = -torch.log(torch.empty_like(other).exponential_(generator=gen))
    s.draft_ids = (full[:sum(drafts), :vocab].float() / t_draft + noise).argmax(1).to(torch.int32)
    s.cu_draft = torch.from_numpy(np.concatenate([[0], np.cumsum(drafts)]).astype(np.int32)).to(DEV)
    s.u_accept = torch.rand(sum(drafts), device=DEV, generator=gen)
    s.u_final = torch.rand(len(drafts), device=DEV, generator=gen)


def _keep_lists(b, rng):
    """A commit's outcome: the first steps accepted, the branch behind them kept up to some token.  Per request the kept pages and how many
    tokens of each are valid; and where those tokens go."""
    off, pages, valid, src, dst, lens, br = [0], [], [], [], [], [], 0
    for r, q in enumerate(b.reqs):
        s0, j = int(b.req_span_off[r]), rng.integers(0, len(q.segs) + 1)
        spans = [(int(b.span_slot[s0 + c]), int(b.span_len[s0 + c])) for c in range(j + 1)]
        for node, n in q.branches:
            if node == j:
                spans.append((int(b.br_own_slot[br]), int(rng.integers(0, n + 1))))
            br += 1
        listed_pages, tokens = [], []
        for first, n in spans:
            listed_pages += b.page_ids[first:first + _pages(n)].tolist()
            valid += [min(PAGE, n - PAGE * i) for i in range(_pages(n))]
            tokens.append(_slots(b, first, n))
        pages += listed_pages
        off.append(len(pages))
        tokens = np.concatenate(tokens)
        at = np.arange(len(tokens))
        src.append(tokens)
        dst.append(np.asarray(listed_pages, dtype=np.int64)[at // PAGE] * PAGE + at % PAGE)
        lens.append(len(tokens))
    i32 = lambda a: torch.from_numpy(np.asarray(a, dtype=np.int32)).to(DEV)  # noqa: E731
    return i32(off), i32(pages), i32(valid), [torch.from_numpy(np.concatenate(a)).to(DEV) for a in (src, dst)], i32(lens)


def prepare(case, seed):
    rng = np.random.default_rng([int(seed) & 0x7FFFFFFF, case["lengths"]])
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    hq, h, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    s = SimpleNamespace(case=case)
    if case["op"] == "accept":
        drafts = _drafts(case)
        _logits(s, gen, drafts, case["vocab"], case["draft_temperature"])
        i32 = dict(dtype=torch.int32, device=DEV)
        s.n_accept, s.final_id = torch.zeros(len(drafts), **i32), torch.zeros(len(drafts), **i32)
        s.p_draft, s.q_draft = torch.zeros(sum(drafts), device=DEV), torch.zeros(sum(drafts), device=DEV)
    elif case["op"] in ("write", "read"):
        n = case["tokens"]
        pages = _pages(n) + _pages(n) // 4 + 1
        s.cache = _cache(pages, h, d)
        order = rng.permutation(pages)
        at = np.arange(n)
        slots = order[at // PAGE].astype(np.int64) * PAGE + at % PAGE
        if n > 100:
            slots[-(n // 50):] = -1  # rows behind the last sequence of a padded batch
        s.slots = torch.from_numpy(slots).to(DEV)
        if case["op"] == "write":
            s.k, s.v = _projection(gen, n, hq, h, d)
        else:
            _fill(s.cache, gen, s.slots[s.slots >= 0], h, d)
            s.k, s.v = (torch.zeros((n, h, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    else:
        s.batch = b = _batch(case, rng)
        s.cache = _cache(b.n_pool_pages, h, d)
        s.keys, s.rows = _keys_and_rows(b)
        used = s.keys[:, 0][s.keys[:, 3] >= 0]
        if case["op"] == "attend":
            # what no sequence holds is not a number
            for t in (s.cache.k, s.cache.v):
                t.view(torch.uint8).fill_(0x7F)
            for t in (s.cache.k_scale, s.cache.v_scale):
                t.view(torch.uint8).fill_(255)
            s.q = _rows(gen, int(b.cu_q[-1]), hq, d, False)
            s.out, s.lse = torch.zeros_like(s.q), torch.zeros(s.q.shape[:2], device=DEV)
        _fill(s.cache, gen, used, h, d)
        if case["op"] == "compact":
            new = [_slots(b, int(f), int(n)) for first, length in ((b.span_slot, b.span_len), (b.br_own_slot, b.br_own_len))
                   for i, (f, n) in enumerate(zip(first, length)) if first is b.br_own_slot or i not in b.req_span_off]
            s.slots = torch.from_numpy(np.concatenate(new)).to(DEV)
            s.k, s.v = _projection(gen, len(s.slots), hq, h, d)
            s.keep_off, s.keep_pages, s.keep_valid, s.moves, s.lens = _keep_lists(b, rng)
            s.new_len, s.n_kept = torch.zeros_like(s.lens), torch.zeros_like(s.lens)
    if own:
        from paper_2506_19830_b200 import binding as B

        s.ctx = B.Context(SimpleNamespace(n_q_heads=hq, n_kv_heads=h, head_dim=d, page_size=PAGE, vocab=max(1, case["vocab"])), 0)
        if case["op"] == "accept":
            s.scratch = s.ctx.accept_sample_drafted_scratch(s.logits.shape[0])
        else:
            s.cache = B.Fp8Cache(s.cache.k, s.cache.v, s.cache.k_scale, s.cache.v_scale)
        if case["op"] in ("attend", "compact"):
            s.plan = B.Plan(s.ctx, s.batch)
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------------
def run(s):
    op = s.case["op"]
    if op == "write":
        if own:
            s.ctx.lr_fp8_write(s.cache, s.k, s.v, s.slots)
        else:
            _write(s)
        return _whole(s.cache)
    if op == "read":
        if own:
            s.ctx.lr_fp8_read(s.cache, s.slots, s.k, s.v)
        else:
            _read(s)
        return [s.k, s.v]
    if op == "attend":
        if own:
            s.plan.lr_verify_attention_fp8(s.q, s.cache, s.out, s.lse)
            return [s.out, s.lse]
        return _attend(s)
    if op == "compact":
        if own:
            s.ctx.lr_fp8_write(s.cache, s.k, s.v, s.slots)
            s.plan.lr_compact_fp8(s.keep_off, s.keep_pages, s.keep_valid, s.cache, s.new_len, s.n_kept)
        else:
            _write(s)
            _compact(s)
        return _whole(s.cache) + [s.new_len, s.n_kept]
    if own:
        s.ctx.lr_accept_sample_drafted(s.logits, s.draft_logits, s.draft_ids, s.cu_draft, s.case["temperature"], s.case["draft_temperature"], s.u_accept,
                                       s.u_final, s.n_accept, s.final_id, s.scratch, s.p_draft, s.q_draft)
        return [s.n_accept, s.final_id, s.p_draft, s.q_draft]
    return _accept(s)


def _whole(cache):
    """A cache as the values it stands for: e4m3 codes, powers of two."""
    return [cache.k, cache.v, cache.k_scale, cache.v_scale]


def _read(s):
    keep = s.slots >= 0
    at = s.slots[keep]
    for pool, scale, out in ((s.cache.k, s.cache.k_scale, s.k), (s.cache.v, s.cache.v_scale, s.v)):
        out[keep] = _values(_gather(pool, at), _gather(scale, at)).to(torch.bfloat16)


def _compact(s):
    src, dst = s.moves
    for pool in (s.cache.k, s.cache.v, s.cache.k_scale, s.cache.v_scale):
        _put(pool, dst, _gather(pool, src))
    s.new_len.copy_(s.lens)
    s.n_kept.copy_((s.lens + PAGE - 1) // PAGE)


def _attend(s):
    h, d, group = s.case["kv_heads"], s.case["head_dim"], s.case["q_heads"] // s.case["kv_heads"]
    slots, lo, hi, owner, place = s.keys.unbind(1)  # [requests, keys]
    node, branch, limit = s.rows.unbind(1)  # [requests, rows]
    n_req, n_row = node.shape
    live = node.reshape(-1) >= 0
    q = torch.zeros((n_req * n_row, h, group, d), device=slots.device)
    q[live] = s.q.float().reshape(-1, h, group, d)
    q = q.reshape(n_req, n_row, h, group, d).permute(0, 2, 1, 3, 4).reshape(n_req, h, n_row * group, d)
    k, v = (_values(_gather(pool, slots), _gather(scale, slots)).permute(0, 2, 1, 3)
            for pool, scale in ((s.cache.k, s.cache.k_scale), (s.cache.v, s.cache.v_scale)))  # [requests, KV heads, keys, head size]
    lo, hi, owner, place = (t[:, None, :] for t in (lo, hi, owner, place))
    node, branch, limit = (t[:, :, None] for t in (node, branch, limit))
    seen = ((owner == 0) & (lo <= node) & (node <= hi)) | ((owner == branch) & (place <= limit))
    hidden = ~seen[:, None, :, None, :].expand(-1, -1, -1, group, -1).reshape(n_req, 1, n_row * group, -1)
    score = (q @ k.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).masked_fill_(hidden, -math.inf)
    top = score.amax(-1, keepdim=True)
    score = score.sub_(top).exp_()
    total = score.sum(-1, keepdim=True)
    out, lse = (score @ v) / total, top + total.log()
    back = lambda t: t.reshape(n_req, h, n_row, group, -1).permute(0, 2, 1, 3, 4).reshape(n_req * n_row, h * group, -1)[live]  # noqa: E731
    return [back(out).to(torch.bfloat16), back(lse)[..., 0]]


def _accept(s):
    n_branch, n_rows, dev = s.u_final.numel(), s.logits.shape[0], s.logits.device
    cu = s.cu_draft.long()
    first, n_draft = cu[:-1], cu[1:] - cu[:-1]
    p = torch.softmax(s.logits.double() / s.case["temperature"], 1)
    q = torch.softmax(s.draft_logits.double() / s.case["draft_temperature"], 1)
    ids = s.draft_ids.long()[:, None]
    p_draft, q_draft = p[s.target_row].gather(1, ids)[:, 0], q.gather(1, ids)[:, 0]
    refused = ~(s.u_accept.double() * q_draft < p_draft)
    # a row for every draft and one behind the last of each branch, where the walk ends in any case
    stop = torch.ones(n_rows, dtype=torch.bool, device=dev)
    stop[s.target_row] = refused
    row0 = first + torch.arange(n_branch, device=dev)
    branch = torch.repeat_interleave(torch.arange(n_branch, device=dev), n_draft + 1)
    place = torch.arange(n_rows, device=dev) - row0[branch]
    n = torch.full((n_branch,), n_rows, device=dev).scatter_reduce(0, branch, torch.where(stop, place, n_rows), "amin")
    weight = p[row0 + n]
    rejected = n < n_draft
    weight = torch.where(rejected[:, None], (weight - q[(first + n).clamp(max=q.shape[0] - 1)]).clamp(min=0), weight)
    up = weight.cumsum(1)
    final = torch.searchsorted(up, (s.u_final.double() * up[:, -1])[:, None], right=True)[:, 0]
    return [n.to(torch.int32), final.to(torch.int32), p_draft.float(), q_draft.float()]


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------------
def _near_e4m3(y):
    """The nearest e4m3 value of |y| <= 448, ties to even: three fraction bits above 2^-6, multiples of 2^-9 below."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step  # (rounds half to even)


def _stored(x):
    """What a row in 64 bits is stored as: values of the codes, and the scale."""
    top = x.abs().amax(-1, keepdim=True)
    e = torch.where(top > 0, torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / 448.0)), torch.full_like(top, -124.0)).clamp(min=-124.0)
    e = torch.where(top * torch.exp2(-e) > 448.0, e + 1, e)
    e = torch.where((top * torch.exp2(1 - e) <= 448.0) & (e > -124.0), e - 1, e)
    return _near_e4m3(x * torch.exp2(-e)), torch.exp2(e)[..., 0]


def _exact_cache(s):
    return [t.double() for t in _whole(s.cache)]


def _exact_write(s, cache):
    for i, rows in enumerate((s.k, s.v)):
        value, scale = _stored(rows.double())
        for t in (s.slots >= 0).nonzero()[:, 0].split(4096):
            at = s.slots[t]
            cache[i][at // PAGE, :, at % PAGE] = value[t]
            cache[2 + i][at // PAGE, :, at % PAGE] = scale[t]
    return cache


def _exact_attend(s):
    b, h, d = s.batch, s.case["kv_heads"], s.case["head_dim"]
    group, cache = s.case["q_heads"] // h, _exact_cache(s)
    out, lse, br = torch.zeros(s.q.shape, dtype=torch.float64, device=DEV), torch.zeros(s.lse.shape, dtype=torch.float64, device=DEV), 0
    for r, q in enumerate(b.reqs):
        s0 = int(b.req_span_off[r])
        for node, n in q.branches:
            spans = [(int(b.span_slot[s0 + c]), int(b.span_len[s0 + c])) for c in [0] + _path(q.parents, node)] + [(int(b.br_own_slot[br]), n)]
            at = torch.from_numpy(np.concatenate([_slots(b, f, m) for f, m in spans])).to(DEV)
            k, v = (cache[i][at // PAGE, :, at % PAGE] * cache[2 + i][at // PAGE, :, at % PAGE][..., None] for i in range(2))
            q0 = int(b.cu_q[br])
            x = s.q[q0:q0 + n].double().reshape(n, h, group, d)
            score = torch.einsum("nhgd,khd->nhgk", x, k) / math.sqrt(d)
            ahead = torch.arange(len(at), device=DEV)[None] > (len(at) - n + torch.arange(n, device=DEV))[:, None]
            score = score.masked_fill(ahead[:, None, None], -math.inf)
            out[q0:q0 + n] = torch.einsum("nhgk,khd->nhgd", torch.softmax(score, -1), v).reshape(n, h * group, d)
            lse[q0:q0 + n] = torch.logsumexp(score, -1).reshape(n, h * group)
            br += 1
    return [out, lse]


def _exact_accept(s):
    cu, n_accept, final = s.cu_draft.tolist(), [], []
    p_draft, q_draft = torch.zeros(cu[-1], dtype=torch.float64, device=DEV), torch.zeros(cu[-1], dtype=torch.float64, device=DEV)
    share = lambda row, t: (lambda e: e / e.sum())(torch.exp((row.double() - row.double().max()) / t))  # noqa: E731
    for b in range(len(cu) - 1):
        n = None
        for i in range(cu[b], cu[b + 1]):
            token = int(s.draft_ids[i])
            p, q = share(s.logits[i + b], s.case["temperature"]), share(s.draft_logits[i], s.case["draft_temperature"])
            p_draft[i], q_draft[i] = p[token], q[token]
            if n is None and not float(s.u_accept[i]) < float(p[token]) / float(q[token]):
                n, weight = i - cu[b], (p - q).clamp(min=0)
        if n is None:
            n, weight = cu[b + 1] - cu[b], share(s.logits[cu[b + 1] + b], s.case["temperature"])
        up = torch.cumsum(weight, 0)
        n_accept.append(n)
        final.append(int((up <= float(s.u_final[b]) * float(up[-1])).sum()))
    return [torch.tensor(n_accept, dtype=torch.int32), torch.tensor(final, dtype=torch.int32), p_draft, q_draft]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "accept":
        return _exact_accept(s)
    if case["op"] == "attend":
        return _exact_attend(s)
    if case["op"] == "read":
        out, cache, at = [], _exact_cache(s), s.slots.clamp(min=0)
        for i in range(2):
            got = cache[i][at // PAGE, :, at % PAGE] * cache[2 + i][at // PAGE, :, at % PAGE][..., None]
            out.append(torch.where((s.slots >= 0)[:, None, None], got, torch.zeros_like(got)))
        return out
    cache = _exact_write(s, _exact_cache(s))
    if case["op"] == "write":
        return cache
    # the kept tokens of every request one after another, to the places that its kept pages give
    off, pages, valid = s.keep_off.tolist(), s.keep_pages.tolist(), s.keep_valid.tolist()
    lens, places = [], []
    for r in range(len(off) - 1):
        k = 0
        for i in range(off[r], off[r + 1]):
            for t in range(valid[i]):
                places.append((pages[i], t, pages[off[r] + k // PAGE], k % PAGE))
                k += 1
        lens.append(k)
    page, t, to_page, to = torch.tensor(places, device=DEV).T
    for pool in cache:
        pool[to_page, :, to] = pool[page, :, t].clone()
    return cache + [torch.tensor(lens, dtype=torch.int32), torch.tensor([(n + PAGE - 1) // PAGE for n in lens], dtype=torch.int32)]
