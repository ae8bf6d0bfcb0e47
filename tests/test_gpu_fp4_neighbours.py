"""The 4-bit cache with another sequence's rows in the same 32 bytes of codes and scales, read on a second stream all the while: what a write, a compaction and a read of one
sequence leave is its own, call after call."""
import numpy as np
import pytest
import torch

from lr_workloads import Model, bf16_round
from lr_workloads.gen import _finish
from oracle import lr_oracle as O
from paper_2506_19830_b200 import binding as B
from paper_2506_19830_b200 import runner as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("d,h", [(64, 1), (64, 3), (128, 1)])
def test_rows_that_are_written_beside_rows_that_are_read(d, h):
    rng = np.random.default_rng(d + h)
    reqs = [{"P": 21, "segs": [33, 7], "branches": [(g, 21, 21, 21) for g in range(3)]} for _ in range(6)]
    w = _finish("neighbours", 3, Model(h, h, d, 16), reqs, rng, 0.3, 0.9, False, True, "nan")
    b = w.batch
    mine = np.asarray(b.page_ids) * 2  # every other page; those between are the neighbour's
    b.page_ids, b.n_pool_pages = mine.astype(np.int32), int(b.n_pool_pages) * 2
    c = O.commit(b, w.tensors.verdict, np.full(b.n_branch, 13, dtype=np.int32))
    spans = list(zip(b.span_slot, b.span_len)) + list(zip(b.br_own_slot, b.br_own_len))
    at = np.array([int(b.page_ids[int(f) + t // 16]) * 16 + t % 16 for f, n in spans for t in range(int(n))], dtype=np.int64)
    theirs = np.array([p * 16 + t for p in mine + 1 for t in range(16)], dtype=np.int64)
    to = lambda a, kind: torch.from_numpy(np.ascontiguousarray(a, dtype=kind)).to(DEV)  # noqa: E731
    ctx = B.Context(b.model, 0)
    plan, cache = B.Plan(ctx, b), B.Fp4Cache.empty(b.model, int(b.n_pool_pages), DEV)
    rounds, rows = 12, []
    for _ in range(rounds):
        x = rng.standard_normal((2, len(at), h, d)) * np.exp2(rng.integers(-12, 13, (2, len(at), h, 1)))
        rows.append([bf16_round(y.astype(np.float32)) for y in x])
    given = [[R.bf16_tensor(y, DEV) for y in pair] for pair in rows]
    other = [bf16_round(rng.standard_normal((len(theirs), h, d)).astype(np.float32)) for _ in range(2)]
    at_d, theirs_d = to(at, np.int64), to(theirs, np.int64)
    ctx.lr_fp4_write(cache, R.bf16_tensor(other[0], DEV), R.bf16_tensor(other[1], DEV), theirs_d)
    # the slots of what is left of each request, in order
    wide = [np.zeros((int(b.n_pool_pages), h, 16, d), dtype=np.uint16) for _ in range(2)]
    new_len = O.compact(c["keep_off"], c["keep_pages"], c["keep_valid"], *wide)[0]
    left = np.array([int(c["keep_pages"][int(c["keep_off"][r]) + i // 16]) * 16 + i % 16 for r in range(b.n_req) for i in range(int(new_len[r]))], dtype=np.int64)
    left_d = to(left, np.int64)
    lists = [to(c[n], np.int32) for n in ("keep_off", "keep_pages", "keep_valid")]
    n_new, n_kept = (torch.zeros(b.n_req, dtype=torch.int32, device=DEV) for _ in range(2))
    got = [[torch.zeros((n, h, d), dtype=torch.bfloat16, device=DEV) for n in (len(at), len(at), len(left), len(left))] for _ in range(rounds)]
    seen = [torch.zeros((len(theirs), h, d), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    side, main = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for (k, v), (k1, v1, k2, v2) in zip(given, got):
        for _ in range(8):
            ctx.lr_fp4_read(cache, theirs_d, *seen, stream=side)
        ctx.lr_fp4_write(cache, k, v, at_d, stream=main)
        ctx.lr_fp4_read(cache, at_d, k1, v1, stream=main)
        plan.lr_compact_fp4(*lists, cache, n_new, n_kept, stream=main)
        ctx.lr_fp4_read(cache, left_d, k2, v2, stream=main)
    torch.cuda.synchronize()
    assert plan.lr_poll_status() == 0 and np.array_equal(n_new.cpu().numpy(), new_len)

    def values(bits):
        codes, scale = O.fp4_store(bits)
        return bf16_round(O.fp4_load(codes, scale).astype(np.float32))

    assert all(np.array_equal(R.bf16_bits(s), values(o)) for s, o in zip(seen, other))
    for pair, tensors in zip(rows, got):
        for bits, first, second in zip(pair, tensors[:2], tensors[2:]):
            want = values(bits)
            assert np.array_equal(R.bf16_bits(first), want)
            pool = np.zeros((int(b.n_pool_pages), h, 16, d), dtype=np.uint16)
            pool[at // 16, :, at % 16] = want
            pool = O.compact(c["keep_off"], c["keep_pages"], c["keep_valid"], pool, pool)[2]
            assert np.array_equal(R.bf16_bits(second), pool[left // 16, :, left % 16])
    plan.close()
    ctx.close()
