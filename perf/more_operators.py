"""What brings tokens into a cache, keeps them in 4 bits and hands them to another sequence, as cases that can be timed and compared: every case once in its
plain form (elementary torch operations) and once as calls of the package.

Operators (a case's ``op``):
  rope     rotary positions: the queries of a joint projection rotated, its keys rotated and written with its values into the cache's slots (bf16 or 8 bits)
  store    K/V rows of a projection's output into the slots of a 4-bit cache, and what they stand for there handed back as bf16
  attend   the nested-prefix attention of a verify pass (chain or tree of draft steps) over a 4-bit cache
  copy     a sequence forked: its pages copied to others, in every layer's cache

Rotary positions.  Of a head's channels the first ``rot`` are turned in pairs, (i, i + rot/2) with the layout "halves" and (2i, 2i + 1) with "interleaved":
(a, b) -> (a cos - b sin, a sin + b cos) * amplitude, at the angle position * f_i, f_i = base^(-2i / rot).  ``scaling`` stretches the frequencies for contexts longer
than ``original`` by ``factor``: "linear" f / factor; "parts" and "smooth" only those that turn few times over the original length: with w_i going from 0
(kept) to 1 (stretched), f (1 - w) + f / factor w.  "smooth": w falls linearly from 1 at ``lo`` turns to 0 at ``hi``.  "parts": w rises linearly with i between the pairs
that turn ``hi`` and ``lo`` times (rounded outwards to whole numbers, within 0 and rot - 1), and the amplitude is 0.1 ln(factor) + 1.

The 4-bit cache.  Pools of e2m1 codes [pages][KV heads][16][head size / 2 bytes] and one power-of-two scale byte (e8m0, bias 127) for every 32 channels of a row.  Such a
group is stored with the smallest exponent e >= -126 for which max|x| 2^-e <= 6: codes x 2^-e rounded to the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives
(ties to the code with a last bit of 0), byte e + 127.  A row with an infinity or a NaN gets codes 0 and bytes 255, which read as NaN.  The eight
codes of channels 8w .. 8w + 7 are a 32-bit word: bits 4j .. 4j + 3 hold channel 8w + 2j for j < 4, channel 8w + 2 (j - 4) + 1 above.

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
GROUP = 32  # channels of a row that share a scale

BASE = {
    "op": "attend", "q_heads": 40, "kv_heads": 8, "head_dim": 128, "requests": 1, "prefix_min": 4096, "prefix_max": 4096, "steps_min": 3,
    "steps_max": 3, "seg_min": 32, "seg_max": 32, "drafts_min": 16, "drafts_max": 16, "tree_width": 0, "tokens": 0, "kind": "fp4", "layers": 1,
    "rot": 128, "layout": "halves", "base": 1e6, "scaling": "none", "factor": 1.0, "original": 32768, "lo": 1.0, "hi": 32.0, "first_position": 0,
    "lengths": 1,
}
SERVING = {"requests": 16, "prefix_min": 1024, "prefix_max": 16384, "steps_min": 2, "steps_max": 6, "seg_min": 16, "seg_max": 64,
           "drafts_min": 4, "drafts_max": 16, "lengths": 5}


def listed():
    def case(name, op, **kw):
        return dict(BASE, name=name, op=op, **kw)

    return [
        # the tokens of one serving pass, in every layer in front of attention: latency counts
        case("rope_drafts", "rope", kind="bf16", tokens=356, first_position=4096),
        # a prompt, for a model that turns half of each head in neighbouring pairs and stretches its positions for long contexts
        case("rope_prompt", "rope", kind="bf16", tokens=32768, rot=64, layout="interleaved", base=1e4, scaling="parts", factor=16.0, original=4096),
        # a prompt's part at far positions into an 8-bit cache
        case("rope_far8", "rope", kind="fp8", tokens=8192, q_heads=32, base=5e5, scaling="smooth", factor=8.0, original=8192, lo=1.0, hi=4.0,
             first_position=1000000),
        # the drafted tokens of one serving pass into the 4-bit cache
        case("store_drafts", "store", tokens=356),
        # a long prompt
        case("store_prompt", "store", tokens=32768),
        # the smallest call: one request early in its answer takes one token without drafts
        case("attend_token", "attend", prefix_min=250, prefix_max=250, steps_min=0, steps_max=0, drafts_min=1, drafts_max=1),
        # many answers in progress without drafts, over long contexts: single tokens, the cache's bytes are the work
        case("attend_decode", "attend", **dict(SERVING, requests=48, prefix_min=2048, steps_min=0, steps_max=0, drafts_min=1, drafts_max=1)),
        # one request at 32 K tokens with deep speculation: many query rows for one cache
        case("attend_long", "attend", q_heads=32, prefix_min=32768, prefix_max=32768, steps_min=6, steps_max=6, seg_min=40, seg_max=40),
        # a serving batch: ragged lengths everywhere
        case("attend_serving", "attend", **SERVING),
        # multi-branch drafting for a model with heads of 64: two proposals a step, two steps deep, a branch on every node
        case("attend_tree64", "attend", **dict(SERVING, q_heads=32, head_dim=64, requests=8, steps_min=2, steps_max=2, tree_width=2)),
        # one sequence at 4 K tokens forked in one layer's 4-bit cache
        case("copy_one", "copy", prefix_min=4096, prefix_max=4096),
        # a batch of sequences forked in several layers' bf16 caches
        case("copy_layers", "copy", kind="bf16", layers=4, requests=4, prefix_min=4096, prefix_max=16384, lengths=7),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        w, m = work(c), most.setdefault(c["op"], {"bytes": 0.0, "flops": 0.0})
        most[c["op"]] = {k: max(w[k], m[k]) for k in m}
    while True:
        op = rng.choices(["rope", "store", "attend", "copy"], [25, 15, 45, 15])[0]
        hq, hkv, hd = rng.choice([(40, 8, 128)] * 3 + [(32, 8, 128)] * 2 + [(16, 4, 128), (8, 8, 128), (5, 1, 128), (16, 1, 128), (32, 8, 64), (12, 4, 64), (4, 1, 64)])
        pmax, smax, dmax = _log_int(rng, 20, 32768), _log_int(rng, 2, 80), rng.randint(1, 20)
        tree = rng.choice([0, 0, 0, 2, 3, 4]) if op == "attend" else 0
        gmax = rng.randint(1, 2) if tree else rng.randint(0, 6)
        c = dict(BASE, op=op, q_heads=hq, kv_heads=hkv, head_dim=hd, rot=hd, requests=_log_int(rng, 1, 48), prefix_min=int(pmax * rng.uniform(0.1, 1.0)),
                 prefix_max=pmax, steps_min=rng.randint(min(1, gmax), gmax), steps_max=gmax, seg_min=rng.randint(1, smax), seg_max=smax,
                 drafts_min=rng.randint(1, dmax), drafts_max=dmax, tree_width=tree, lengths=rng.randrange(1 << 20))
        if op in ("rope", "store"):
            c["tokens"] = _log_int(rng, 1, 32768)
        if op == "rope":
            scaling = rng.choice(["none", "linear", "parts", "smooth"])
            c.update(kind=rng.choice(["bf16", "bf16", "fp8"]), rot=rng.choice([hd, hd, hd // 2, hd // 4, 2 * rng.randint(1, hd // 2)]),
                     layout=rng.choice(["halves", "interleaved"]), base=rng.choice([1e4, 5e5, 1e6]), scaling=scaling, original=_log_int(rng, 2048, 65536),
                     factor=1.0 if scaling == "none" else round(rng.uniform(1.5, 40.0), 2), hi=rng.choice([4.0, 32.0]), first_position=_log_int(rng, 1, 4000000))
        if op == "copy":
            c.update(kind=rng.choice(["bf16", "fp8", "fp4"]), layers=rng.randint(1, 6))
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


def _row_bytes(case, kind):
    """Bytes of a row of K or V of one head."""
    d = case["head_dim"]
    return {"bf16": 2.0 * d, "fp8": d + 1.0, "fp4": d / 2 + d // GROUP}[kind]


def work(case):
    hq, h, d, n = case["q_heads"], case["kv_heads"], case["head_dim"], case["tokens"]
    if case["op"] == "rope":  # queries, keys and values read and written; three operations for each channel turned
        return {"bytes": n * (4.0 * d * hq + 2 * h * (2.0 * d + _row_bytes(case, case["kind"])) + 12.0), "flops": 3.0 * n * (hq + h) * case["rot"]}
    if case["op"] == "store":  # the rows read, their codes written, and the rows that they stand for
        return {"bytes": 2.0 * n * h * (4.0 * d + _row_bytes(case, "fp4")) + 8.0 * n, "flops": 4.0 * n * h * d}
    reqs = _requests(case)
    if case["op"] == "copy":
        pages = sum(_pages(r.prefix) for r in reqs)
        return {"bytes": 2.0 * case["layers"] * 2 * pages * h * PAGE * _row_bytes(case, case["kind"]) + 8.0 * pages, "flops": 0.0}
    rows = kv = seen = 0
    for r in reqs:
        kv += r.prefix + sum(r.segs)
        for node, m in r.branches:
            rows += m
            kv += m
            seen += m * (r.prefix + sum(r.segs[s - 1] for s in _path(r.parents, node))) + m * (m + 1) // 2
    return {"bytes": 2.0 * kv * h * _row_bytes(case, "fp4") + 4.0 * rows * hq * d + 4.0 * rows * hq, "flops": 4.0 * hq * d * seen}


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


# ---- the plain forms of the caches -----------------------------------------------------------------------------------------
def _power(e):
    """2^e, for whole -126 <= e <= 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _exponent(top, most, half_most, least):
    """The smallest whole e >= least with top 2^-e <= most = half_most 2^k, 1/2 <= half_most < 1."""
    half, exponent = torch.frexp(top)  # top = half 2^exponent, 1/2 <= half < 1
    return (exponent - int(math.log2(most / half_most)) + (half > half_most).to(torch.int32)).clamp(min=least)


def _quantise8(x):
    """Codes and scale bytes of rows [..., head size]: e4m3 with one power of two a row, as the 8-bit cache holds them."""
    top = x.abs().amax(-1, keepdim=True)
    e, fine = _exponent(top, 448.0, 0.875, -124), torch.isfinite(top)
    e = torch.where(fine, e, torch.zeros_like(e))
    codes = torch.where(fine, x * _power(-e), torch.zeros_like(x)).to(torch.float8_e4m3fn)
    return codes, torch.where(fine, e + 127, torch.full_like(e, 255)).to(torch.uint8)[..., 0]


def _quantise4(x):
    """Code bytes [..., head size / 2] and scale bytes [..., head size / 32] of rows [..., head size]."""
    x = x.float()
    fine = torch.isfinite(x).all(-1, keepdim=True)[..., None]
    g = x.reshape(*x.shape[:-1], -1, GROUP)
    e = _exponent(g.abs().amax(-1, keepdim=True), 6.0, 0.75, -126)
    e = torch.where(fine, e, torch.zeros_like(e))
    y = torch.where(fine, g * _power(-e), torch.zeros_like(g)).reshape(x.shape)
    a = y.abs()
    code = sum(((a > at) if odd else (a >= at)).to(torch.int32) for at, odd in ((0.25, 1), (0.75, 0), (1.25, 1), (1.75, 0), (2.5, 1), (3.5, 0), (5.0, 1)))
    code = (code | torch.signbit(y).to(torch.int32) << 3).reshape(*x.shape[:-1], -1, 4, 2)
    word = code.movedim(-1, -2)  # [..., words, odd channel, 4]
    codes = (word[..., 0::2] | word[..., 1::2] << 4).to(torch.uint8).reshape(*x.shape[:-1], -1)
    return codes, torch.where(fine, e + 127, torch.full_like(e, 255)).to(torch.uint8)[..., 0]


def _values4(codes, scale):
    """What a 4-bit row stands for."""
    nibble = torch.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1, 2, 4).movedim(-1, -2).reshape(*codes.shape[:-1], -1)
    value = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)[(nibble & 7).long()]
    value = torch.where(nibble > 7, -value, value)
    s = torch.where(scale == 255, torch.full(scale.shape, math.nan, device=scale.device), _power(scale.to(torch.int32) - 127))
    return (value.reshape(*scale.shape, GROUP) * s[..., None]).reshape(value.shape)


def _gather(pool, slots):
    """Rows [..., KV heads, a row's] of a pool (or its scales) at token slots."""
    return pool[slots // PAGE, :, slots % PAGE]


def _put(pool, slots, rows):
    raw = {1: torch.uint8, 2: torch.int16}[pool.element_size()]
    pool.view(raw)[slots // PAGE, :, slots % PAGE] = rows.view(raw)


def _put_rows(kind, cache, side, slots, rows):
    """Rows of K (side 0) or V (1) in 32 bits into a cache."""
    if kind == "bf16":
        _put(cache[side], slots, rows.to(torch.bfloat16))
    else:
        codes, byte = (_quantise8 if kind == "fp8" else _quantise4)(rows)
        _put(cache[side], slots, codes)
        _put(cache[2 + side], slots, byte)


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _rows(gen, n, heads, d, spread=True):
    """Rows as a layer gives them: heads and tokens of different sizes, some channels far above the others."""
    x = torch.empty((n, heads, d), device=DEV).normal_(generator=gen)
    if spread:
        x *= torch.exp(0.5 * torch.empty((n, heads, 1), device=DEV).normal_(generator=gen))
        x[..., 3] *= 8.0
    return x.to(torch.bfloat16)


def _cache(kind, pages, heads, d):
    """An empty cache: K, V and, in 8 or 4 bits, their scales."""
    if kind == "bf16":
        return [torch.zeros((pages, heads, PAGE, d), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    if kind == "fp8":
        return ([torch.zeros((pages, heads, PAGE, d), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) for _ in range(2)] +
                [torch.full((pages, heads, PAGE), 127, dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu) for _ in range(2)])
    return ([torch.zeros((pages, heads, PAGE, d // 2), dtype=torch.uint8, device=DEV) for _ in range(2)] +
            [torch.full((pages, heads, PAGE, d // GROUP), 127, dtype=torch.uint8, device=DEV) for _ in range(2)])


def _projection(gen, n, hq, h, d):
    """Q, K and V of n tokens as they lie in the output of a joint projection [tokens, (q + 2 KV heads) x head size]."""
    joint = torch.zeros((n, hq + 2 * h, d), dtype=torch.bfloat16, device=DEV)
    joint[:, :hq] = _rows(gen, n, hq, d, False)
    joint[:, hq:hq + h] = _rows(gen, n, h, d)
    joint[:, hq + h:] = _rows(gen, n, h, d)
    return joint[:, :hq], joint[:, hq:hq + h], joint[:, hq + h:]


def _token_slots(rng, n):
    """Slots of n tokens over shuffled pages, those of a padded batch's last rows negative; and how many pages there are."""
    pages = _pages(n) + _pages(n) // 4 + 1
    at = np.arange(n)
    slots = rng.permutation(pages)[at // PAGE].astype(np.int64) * PAGE + at % PAGE
    if n > 100:
        slots[-(n // 50):] = -1
    return torch.from_numpy(slots).to(DEV), pages


def prepare(case, seed):
    rng = np.random.default_rng([int(seed) & 0x7FFFFFFF, case["lengths"]])
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    op, hq, h, d, n = case["op"], case["q_heads"], case["kv_heads"], case["head_dim"], case["tokens"]
    s = SimpleNamespace(case=case)
    if op in ("rope", "store"):
        s.slots, pages = _token_slots(rng, n)
        s.cache = _cache(case["kind"], pages, h, d)
        s.q, s.k, s.v = _projection(gen, n, hq, h, d)
        if op == "rope":  # tokens of several sequences: positions run on, with jumps
            jumps = rng.integers(0, 3, n // 100 + 1).repeat(100)[:n].cumsum()
            s.positions = torch.from_numpy((case["first_position"] + np.arange(n) + jumps).astype(np.int32)).to(DEV)
            s.q_out = torch.zeros((n, hq, d), dtype=torch.bfloat16, device=DEV)
        else:
            s.back = [torch.zeros((n, h, d), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    elif op == "copy":
        lengths = [_pages(r.prefix) for r in _requests(case)]
        pages = 2 * sum(lengths) + 3
        order = torch.from_numpy(rng.permutation(pages).astype(np.int32)).to(DEV)
        s.src, s.dst = order[:sum(lengths)].contiguous(), order[sum(lengths):2 * sum(lengths)].contiguous()
        s.caches = []
        for _ in range(case["layers"]):
            cache = _cache(case["kind"], pages, h, d)
            for side in range(2):
                for at in torch.arange(pages * PAGE, device=DEV).split(16384):
                    _put_rows(case["kind"], cache, side, at, _rows(gen, len(at), h, d).float())
            s.caches.append(cache)
    else:
        s.batch = b = _batch(case, rng)
        s.cache = _cache("fp4", b.n_pool_pages, h, d)
        s.keys, s.rows = _keys_and_rows(b)
        for codes, scale in zip(s.cache[:2], s.cache[2:]):  # what no sequence holds is not a number
            codes.fill_(0x77)
            scale.fill_(255)
        for at in s.keys[:, 0][s.keys[:, 3] >= 0].split(16384):
            for side in range(2):
                _put_rows("fp4", s.cache, side, at, _rows(gen, len(at), h, d).float())
        s.q = _rows(gen, int(b.cu_q[-1]), hq, d, False)
        s.out, s.lse = torch.zeros_like(s.q), torch.zeros(s.q.shape[:2], device=DEV)
    if own:
        from paper_2506_19830_b200 import binding as B

        s.ctx = B.Context(SimpleNamespace(n_q_heads=hq, n_kv_heads=h, head_dim=d, page_size=PAGE, vocab=1), 0)
        kind = {"bf16": B.Bf16Cache, "fp8": B.Fp8Cache, "fp4": B.Fp4Cache}[case["kind"]]
        if op == "copy":
            s.own_caches = [kind(*cache) for cache in s.caches]
        else:
            s.own_cache = kind(*s.cache)
        if op == "rope":
            s.rope = B.Rope(case["rot"], base=case["base"], interleaved=case["layout"] == "interleaved", scaling=case["scaling"], factor=case["factor"],
                            original=case["original"], lo=case["lo"], hi=case["hi"])
        if op == "attend":
            s.plan = B.Plan(s.ctx, s.batch)
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------------
def run(s):
    op = s.case["op"]
    if op == "rope":
        if own:
            s.ctx.lr_rope_write(s.rope, s.positions, s.own_cache, s.k, s.v, s.slots, s.q, s.q_out)
        else:
            _rope(s)
        return [s.q_out] + s.cache
    if op == "store":
        if own:
            s.ctx.lr_fp4_write(s.own_cache, s.k, s.v, s.slots)
            s.ctx.lr_fp4_read(s.own_cache, s.slots, *s.back)
        else:
            _store(s)
        return s.back
    if op == "copy":
        if own:
            s.ctx.lr_copy_pages(s.own_caches, s.own_caches, s.src, s.dst)
        else:
            for cache in s.caches:
                for pool in cache:
                    raw = pool.view({1: torch.uint8, 2: torch.int16}[pool.element_size()])
                    raw[s.dst.long()] = raw[s.src.long()]
        return [pool for cache in s.caches for pool in cache]
    if own:
        s.plan.lr_verify_attention_fp4(s.q, s.own_cache, s.out, s.lse)
        return [s.out, s.lse]
    return _attend(s)


def _frequencies(case):
    """Radians a position of every pair in 64 bits, and the amplitude."""
    rot = case["rot"]
    i = torch.arange(rot // 2, dtype=torch.float64, device=DEV)
    f = case["base"] ** (-2.0 * i / rot)
    if case["scaling"] == "none":
        return f, 1.0
    if case["scaling"] == "linear":
        return f / case["factor"], 1.0
    if case["scaling"] == "smooth":
        turns = case["original"] * f / (2.0 * math.pi)
        w = ((case["hi"] - turns) / (case["hi"] - case["lo"])).clamp(0.0, 1.0)
        amplitude = 1.0
    else:
        place = lambda turns: rot * math.log(case["original"] / (2.0 * math.pi * turns)) / (2.0 * math.log(case["base"]))  # noqa: E731
        first, last = max(math.floor(place(case["hi"])), 0), min(math.ceil(place(case["lo"])), rot - 1)
        w = ((i - first) / max(last - first, 0.001)).clamp(0.0, 1.0)
        amplitude = 0.1 * math.log(case["factor"]) + 1.0
    return f * (1.0 - w) + f / case["factor"] * w, amplitude


def _pairs(case, x):
    """The two channels of every pair, as views of rows [tokens, heads, head size]."""
    rot = case["rot"]
    if case["layout"] == "halves":
        return x[..., :rot // 2], x[..., rot // 2:rot]
    return x[..., 0:rot:2], x[..., 1:rot:2]


def _rope(s):
    f, amplitude = _frequencies(s.case)
    angle = s.positions.double()[:, None, None] * f
    cos, sin = (angle.cos() * amplitude).float(), (angle.sin() * amplitude).float()

    def turned(x):
        y = x.float()
        (a, b), (to_a, to_b) = _pairs(s.case, x.float()), _pairs(s.case, y)
        to_a.copy_(a * cos - b * sin)
        to_b.copy_(a * sin + b * cos)
        return y

    s.q_out.copy_(turned(s.q))
    keep = s.slots >= 0
    for side, rows in enumerate((turned(s.k), s.v.float())):
        _put_rows(s.case["kind"], s.cache, side, s.slots[keep], rows[keep])


def _store(s):
    keep = s.slots >= 0
    at = s.slots[keep]
    for side, rows in enumerate((s.k, s.v)):
        _put_rows("fp4", s.cache, side, at, rows[keep])
        s.back[side][keep] = _values4(_gather(s.cache[side], at), _gather(s.cache[2 + side], at)).to(torch.bfloat16)


def _attend(s):
    h, d, group = s.case["kv_heads"], s.case["head_dim"], s.case["q_heads"] // s.case["kv_heads"]
    slots, lo, hi, owner, place = s.keys.unbind(1)  # [requests, keys]
    node, branch, limit = s.rows.unbind(1)  # [requests, rows]
    n_req, n_row = node.shape
    live = node.reshape(-1) >= 0
    q = torch.zeros((n_req * n_row, h, group, d), device=slots.device)
    q[live] = s.q.float().reshape(-1, h, group, d)
    q = q.reshape(n_req, n_row, h, group, d).permute(0, 2, 1, 3, 4).reshape(n_req, h, n_row * group, d)
    k, v = (_values4(_gather(s.cache[side], slots), _gather(s.cache[2 + side], slots)).permute(0, 2, 1, 3) for side in range(2))  # [requests, KV heads, keys, head size]
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


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------------
def _least_exponent(top, most, least):
    """The smallest whole e >= least with top <= most 2^e, by trying."""
    e = torch.where(top > 0, torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / most)), torch.full_like(top, float(least))).clamp(min=float(least))
    e = torch.where(top * torch.exp2(-e) > most, e + 1, e)
    return torch.where((top * torch.exp2(1 - e) <= most) & (e > least), e - 1, e)


def _near(y, fraction_bits, least_exponent):
    """The nearest binary floating-point number of |y| within the range, ties to even: so many fraction bits, a fixed step below 2^least_exponent."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** least_exponent))) - fraction_bits)
    return torch.round(y / step) * step  # (rounds half to even)


def _exact_rope(s):
    case, rot = s.case, s.case["rot"]
    pair = np.arange(rot // 2)
    f = np.power(np.float64(case["base"]), -pair / (rot / 2.0))
    amplitude, turns = 1.0, f * case["original"] / (2.0 * np.pi)
    if case["scaling"] == "linear":
        f = f / case["factor"]
    elif case["scaling"] == "smooth":
        kept = np.clip((turns - case["lo"]) / (case["hi"] - case["lo"]), 0.0, 1.0)
        f = kept * f + (1.0 - kept) * f / case["factor"]
    elif case["scaling"] == "parts":
        ends = [rot / 2.0 * np.log(case["original"] / (2.0 * np.pi * t)) / np.log(case["base"]) for t in (case["hi"], case["lo"])]
        first, last = max(int(np.floor(ends[0])), 0), min(int(np.ceil(ends[1])), rot - 1)
        kept = 1.0 - np.clip((pair - first) / max(last - first, 0.001), 0.0, 1.0)
        f = kept * f + (1.0 - kept) * f / case["factor"]
        amplitude = 1.0 + np.log(case["factor"]) / 10.0
    order = np.stack([pair, pair + rot // 2] if case["layout"] == "halves" else [2 * pair, 2 * pair + 1], 1).reshape(-1)
    order = torch.from_numpy(order).to(DEV)
    turn = torch.from_numpy(f).to(DEV)

    def turned(x, positions):
        y = x.double()
        z = torch.view_as_complex(y[..., order].reshape(*y.shape[:-1], -1, 2))
        angle = positions.double()[:, None, None] * turn
        z = z * torch.polar(torch.full_like(angle, amplitude), angle)
        y[..., order] = torch.view_as_real(z).reshape(*y.shape[:-1], -1)
        return y

    parts = lambda t: t.split(2048)  # noqa: E731
    q_out = torch.cat([turned(x, p) for x, p in zip(parts(s.q), parts(s.positions))])
    cache = [t.double() for t in s.cache]
    for k, v, p, slots in zip(parts(s.k), parts(s.v), parts(s.positions), parts(s.slots)):
        keep = slots >= 0
        at = slots[keep]
        for side, rows in enumerate((turned(k, p), v.double())):
            value = rows[keep]
            if case["kind"] == "fp8":
                e = _least_exponent(value.abs().amax(-1, keepdim=True), 448.0, -124)
                value = _near(value * torch.exp2(-e), 3, -6)
                cache[2 + side][at // PAGE, :, at % PAGE] = torch.exp2(e)[..., 0]
            cache[side][at // PAGE, :, at % PAGE] = value
    return [q_out] + cache


def _exact_store(s):
    out = []
    for rows in (s.k, s.v):
        x = rows.double().reshape(*rows.shape[:-1], -1, GROUP)
        e = _least_exponent(x.abs().amax(-1, keepdim=True), 6.0, -126)
        x = (_near(x * torch.exp2(-e), 1, 0) * torch.exp2(e)).reshape(rows.shape)
        out.append(torch.where((s.slots >= 0)[:, None, None], x, torch.zeros_like(x)))
    return out


def _exact_row_values(cache, side, at):
    """Rows [tokens, KV heads, head size] in 64 bits, from the bits of their codes."""
    codes, scale = cache[side][at // PAGE, :, at % PAGE].int(), cache[2 + side][at // PAGE, :, at % PAGE].double()
    c = torch.arange(2 * codes.shape[-1], device=codes.device)
    bit = 32 * (c // 8) + 16 * (c % 2) + 4 * (c % 8 // 2)  # of the row: where the channel's code starts
    nibble = (codes[..., bit // 8] >> bit % 8) & 15
    exponent, fraction = ((nibble >> 1) & 3).double(), (nibble & 1).double()
    size = torch.where(exponent > 0, (1.0 + fraction / 2.0) * torch.exp2(exponent - 1.0), fraction / 2.0)
    return torch.where(nibble >= 8, -size, size) * torch.exp2(scale[..., c // GROUP] - 127.0)


def _exact_attend(s):
    b, h, d = s.batch, s.case["kv_heads"], s.case["head_dim"]
    group, out, lse, br = s.case["q_heads"] // h, torch.zeros(s.q.shape, dtype=torch.float64, device=DEV), torch.zeros(s.lse.shape, dtype=torch.float64, device=DEV), 0
    for r, q in enumerate(b.reqs):
        s0 = int(b.req_span_off[r])
        chain = [torch.from_numpy(_slots(b, int(b.span_slot[s0 + c]), int(b.span_len[s0 + c]))).to(DEV) for c in range(len(q.segs) + 1)]
        held = [[_exact_row_values(s.cache, side, at) for at in chain] for side in range(2)]
        for node, n in q.branches:
            tail = torch.from_numpy(_slots(b, int(b.br_own_slot[br]), n)).to(DEV)
            k, v = (torch.cat([held[side][c] for c in [0] + _path(q.parents, node)] + [_exact_row_values(s.cache, side, tail)]) for side in range(2))
            q0 = int(b.cu_q[br])
            x = s.q[q0:q0 + n].double().reshape(n, h, group, d)
            score = torch.einsum("nhgd,khd->nhgk", x, k) / math.sqrt(d)
            ahead = torch.arange(len(k), device=DEV)[None] > (len(k) - n + torch.arange(n, device=DEV))[:, None]
            score = score.masked_fill(ahead[:, None, None], -math.inf)
            out[q0:q0 + n] = torch.einsum("nhgk,khd->nhgd", torch.softmax(score, -1), v).reshape(n, h * group, d)
            lse[q0:q0 + n] = torch.logsumexp(score, -1).reshape(n, h * group)
            br += 1
    return [out, lse]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_rope(s)
    if case["op"] == "store":
        return _exact_store(s)
    if case["op"] == "attend":
        return _exact_attend(s)
    out = []
    for cache in s.caches:
        for pool in cache:
            raw = pool.view(torch.uint8 if pool.element_size() == 1 else torch.int16)
            origin = torch.arange(len(raw), device=DEV)  # of every page
            origin[s.dst.long()] = s.src.long()
            whole = raw.index_select(0, origin).view(pool.dtype)
            out.append(whole if whole.dtype == torch.uint8 else whole.double())
    return out
