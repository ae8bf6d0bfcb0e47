"""What the binding finds out about tensors before the C side takes their addresses: shapes, kinds, strides and devices.  On the CPU, with tensors there and a context
whose device is theirs (-1); the calls themselves are refused in the same way on a GPU, below."""
from types import SimpleNamespace

import pytest
import torch

from lr_workloads import Model, make_config
from paper_2506_19830_b200 import binding as B

V = 100


def drafted(dev="cpu", vocab=V):
    """The tensors of a drafted acceptance: two branches, of three drafts and of none."""
    f32, i32 = (lambda n: torch.zeros(n, device=dev)), (lambda *a: torch.tensor(a, dtype=torch.int32, device=dev))
    width = (vocab + 7) // 8 * 8
    return dict(logits=torch.zeros((5, width), dtype=torch.bfloat16, device=dev)[:, :vocab], draft_logits=torch.zeros((3, width), dtype=torch.bfloat16, device=dev)[:, :vocab],
                draft_ids=i32(1, 2, 3), cu_draft=i32(0, 3, 3), u_accept=f32(3), u_final=f32(2), n_accept=i32(-1, -1), final_id=i32(-1, -1), p_draft=f32(3), q_draft=f32(3),
                scratch=torch.zeros(64, dtype=torch.int64, device=dev))


def wrong_drafted(dev):
    good = drafted(dev)
    wide = torch.zeros((5, 2 * V), dtype=torch.bfloat16, device=dev)
    return [("logits", t) for t in (good["logits"].float(), good["logits"].half(), good["logits"][:, :V - 1], wide[:, ::2], good["logits"].reshape(1, 5, V), good["logits"][:1])] + \
           [("draft_logits", t) for t in (good["draft_logits"][:2], good["draft_logits"].float(), good["draft_logits"][:, :V - 8], wide[:3, ::2], good["draft_logits"][:0])] + \
           [("cu_draft", t) for t in (good["cu_draft"].long(), good["cu_draft"][:0], torch.zeros(6, dtype=torch.int32, device=dev)[::2])] + \
           [(name, t) for name, kind in (("draft_ids", torch.int32), ("u_accept", torch.float32), ("p_draft", torch.float32), ("q_draft", torch.float32),
                                         ("u_final", torch.float32), ("n_accept", torch.int32), ("final_id", torch.int32))
            for t in (good[name][:-1], good[name].to(torch.int64 if kind is torch.int32 else torch.float64), torch.zeros(8, dtype=kind, device=dev)[::2])] + \
           [("scratch", t) for t in (good["scratch"][:8], torch.zeros(128, dtype=torch.int64, device=dev)[::2])]


def test_drafted_acceptance_takes_tensors_for_what_they_are():
    ctx = SimpleNamespace(model=Model(1, 1, 64, V), device=-1)
    assert B._check_drafted(ctx, **drafted(), scratch_bytes=80) == (2, 5)
    assert B._check_drafted(ctx, **dict(drafted(), p_draft=None, q_draft=None), scratch_bytes=512) == (2, 5)
    longer = {k: torch.zeros(9, dtype=t.dtype) for k, t in drafted().items() if k in ("draft_ids", "u_accept", "u_final", "n_accept", "final_id", "p_draft", "q_draft")}
    assert B._check_drafted(ctx, **dict(drafted(), **longer), scratch_bytes=80) == (2, 5)
    none = dict(drafted(), logits=drafted()["logits"][:2], cu_draft=torch.zeros(3, dtype=torch.int32))  # no drafts: the drafter's tensors are not looked at
    empty = {k: torch.zeros(0, dtype=drafted()[k].dtype) for k in ("draft_logits", "draft_ids", "u_accept", "p_draft", "q_draft")}
    assert B._check_drafted(ctx, **dict(none, **empty), scratch_bytes=80) == (2, 2)
    for name, t in wrong_drafted("cpu"):
        with pytest.raises(ValueError, match="lr_accept_sample_drafted: "):
            B._check_drafted(ctx, **dict(drafted(), **{name: t}), scratch_bytes=80)
    elsewhere = SimpleNamespace(model=ctx.model, device=0)
    with pytest.raises(ValueError):
        B._check_drafted(elsewhere, **drafted(), scratch_bytes=80)


@pytest.mark.gpu
def test_drafted_acceptance_refuses_before_it_launches():
    ctx = B.Context(Model(1, 1, 64, V), 0)
    names = ("logits", "draft_logits", "draft_ids", "cu_draft", "u_accept", "u_final", "n_accept", "final_id", "scratch", "p_draft", "q_draft")

    def call(a):
        a = [a[n] for n in names]
        ctx.lr_accept_sample_drafted(*a[:4], 1.0, 1.0, *a[4:])

    for name, t in wrong_drafted("cuda:0"):
        with pytest.raises(ValueError, match="lr_accept_sample_drafted: "):
            call(dict(drafted("cuda:0"), **{name: t}))
    for name in names:
        with pytest.raises(ValueError):
            call(dict(drafted("cuda:0"), **{name: drafted("cpu")[name]}))
    assert ctx.launch_count == 0
    call(drafted("cuda:0"))
    torch.cuda.synchronize()
    assert ctx.launch_count == 2
    ctx.close()


def attention(rows, m, dev="cpu"):
    q = torch.zeros((rows, m.n_q_heads, m.head_dim), dtype=torch.bfloat16, device=dev)
    return dict(q=q, out=torch.zeros_like(q), lse=torch.zeros(q.shape[:2], device=dev))


def wrong_attention(rows, m, dev):
    good, wide = attention(rows, m, dev), torch.zeros((rows, 2 * m.n_q_heads, m.head_dim), dtype=torch.bfloat16, device=dev)
    return [(name, t) for name in ("q", "out") for t in (good[name][:-1], good[name].half(), good[name].float(), wide[:, :m.n_q_heads], good[name][:, :, ::2])] + \
           [("lse", t) for t in (good["lse"][:-1], good["lse"].double(), good["lse"].bfloat16(), torch.zeros((rows, 2 * m.n_q_heads), device=dev)[:, ::2])]


def compaction(n_req, slots, dev="cpu"):
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device=dev)  # noqa: E731
    return dict(keep_off=i32(n_req + 1), keep_pages=i32(slots), keep_valid=i32(slots), new_len=i32(n_req), n_pages_kept=i32(n_req))


def wrong_compaction(n_req, slots, dev):
    good = compaction(n_req, slots, dev)
    return [(name, t) for name in good for t in ((good[name].long(), torch.zeros(2 * slots + 4, dtype=torch.int32, device=dev)[::2]) +
                                                 (() if name == "keep_pages" else (good[name][:-1],)))]


def test_attention_and_compaction_take_tensors_for_what_they_are():
    m = Model(8, 2, 64, V)
    ctx = SimpleNamespace(model=m, device=-1)
    good, keep = attention(5, m), compaction(3, 17)
    B._check_attention(ctx, 5, **good)
    B._check_attention(ctx, 5, good["q"].view(5, -1), good["out"].view(-1), None)
    B._check_attention(ctx, 4, **good)  # rows behind the last are left alone
    B._check_compact(ctx, 3, **keep)
    for name, t in wrong_attention(5, m, "cpu"):
        with pytest.raises(ValueError, match=f"lr_verify_attention_fp8: {name}"):
            B._check_attention(ctx, 5, **dict(good, **{name: t}))
    for name, t in wrong_compaction(3, 17, "cpu"):
        with pytest.raises(ValueError, match=f"lr_compact_fp8: {name}"):
            B._check_compact(ctx, 3, **dict(keep, **{name: t}))
    elsewhere = SimpleNamespace(model=m, device=0)
    for call in (lambda: B._check_attention(elsewhere, 5, **good), lambda: B._check_compact(elsewhere, 3, **keep)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_attention_and_compaction_refuse_before_they_launch():
    w = make_config(2, with_logits=False)
    b, dev = w.batch, "cuda:0"
    ctx = B.Context(b.model, 0)
    plan, cache = B.Plan(ctx, b), B.Fp8Cache.empty(b.model, b.n_pool_pages)
    rows = int(b.cu_q[-1])
    for name, t in wrong_attention(rows, b.model, dev) + [(n, attention(rows, b.model)[n]) for n in ("q", "out", "lse")]:
        a = dict(attention(rows, b.model, dev), **{name: t})
        with pytest.raises(ValueError, match=f"lr_verify_attention_fp8: {name}"):
            plan.lr_verify_attention_fp8(a["q"], cache, a["out"], a["lse"])
    here = compaction(b.n_req, b.n_page_slots)
    for name, t in wrong_compaction(b.n_req, b.n_page_slots, dev) + list(here.items()):
        a = dict(compaction(b.n_req, b.n_page_slots, dev), **{name: t})
        with pytest.raises(ValueError, match="lr_compact_fp8: "):
            plan.lr_compact_fp8(a["keep_off"], a["keep_pages"], a["keep_valid"], cache, a["new_len"], a["n_pages_kept"])
    assert ctx.launch_count == 0
    plan.close()
    ctx.close()
