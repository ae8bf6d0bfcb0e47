"""The 8-bit cache on the GPU: writing, reading back and compaction are the oracle's bit for bit."""
import numpy as np
import pytest
import torch

from fp8_util import back, on_device, poison_slack, store_pools, u8
from lr_workloads import Model, bf16_round, make_config, make_random_small
from lr_workloads.gen import _finish
from oracle import lr_oracle as O
from paper_2506_19830_b200 import binding as B
from paper_2506_19830_b200 import runner as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _rows(rng, n, h, d):
    """Rows of every kind: ordinary ones, zeros, the smallest and the largest numbers, borders of the scale, infinities and NaN."""
    x = rng.standard_normal((n, h, d)) * np.exp(rng.uniform(-3, 3, (n, h, 1)))
    with np.errstate(over="ignore"):
        wide = rng.standard_normal((n, h, d)) * np.exp2(rng.uniform(-133, 126, (n, h, 1)))
    x = np.where(rng.random((n, h, 1)) < 0.3, wide, x)
    bits = bf16_round(x.astype(np.float32))
    kind = rng.integers(0, 14, (n, h))
    bits[kind == 0] = 0
    bits[kind == 1] = rng.integers(0, 128, (int((kind == 1).sum()), d))  # subnormal numbers
    bits[kind == 2, 5] = 0x7FC0
    bits[kind == 3, d - 1] = 0xFF80
    bits[kind == 4, 0] = 0x7F7F
    for k, top in ((5, 0x43E0), (6, 0x43E1), (7, 0xC3DF)):  # 448, the next number, -446
        small = bf16_round(rng.uniform(-400, 400, (int((kind == k).sum()), d)).astype(np.float32))
        small[:, 11] = top
        bits[kind == k] = small
    return bits


def _t(bits):
    return R.bf16_tensor(bits, DEV)


def _start(rng, pages, h, d):
    shape = (pages, h, 16, d)
    return [rng.integers(0, 256, s, dtype=np.uint8) for s in (shape, shape, shape[:3], shape[:3])]


def _place(pools, slots, kb, vb):
    keep = slots >= 0
    for codes, scale, bits in ((pools[0], pools[2], kb), (pools[1], pools[3], vb)):
        c, s = O.fp8_store(bits[keep])
        codes[slots[keep] // 16, :, slots[keep] % 16] = c
        scale[slots[keep] // 16, :, slots[keep] % 16] = s


GEOMETRY = [(1, 1, 64), (4, 1, 64), (8, 2, 128), (40, 8, 128), (5, 1, 128), (12, 3, 64)]


@pytest.mark.parametrize("hq,h,d", GEOMETRY)
@pytest.mark.parametrize("n", [1, 2, 15, 33, 700])
def test_write_and_read_are_the_oracles(hq, h, d, n):
    rng = np.random.default_rng(n * 100 + hq + d)
    pages = (n + 15) // 16 + 3
    ctx = B.Context(Model(hq, h, d, 8), 0)
    pools = _start(rng, pages, h, d)
    cache = on_device(pools)
    slots = rng.permutation(pages * 16)[:n].astype(np.int64)
    slots[rng.random(n) < 0.1] = -1
    kb, vb = _rows(rng, n, h, d), _rows(rng, n, h, d)
    joint = torch.zeros((n, hq + 2 * h, d), dtype=torch.bfloat16, device=DEV)  # as a projection leaves them
    joint[:, hq:hq + h], joint[:, hq + h:] = _t(kb), _t(vb)
    status, at = torch.zeros(2, dtype=torch.int32, device=DEV), torch.from_numpy(slots).to(DEV)
    ctx.lr_fp8_write(cache, joint[:, hq:hq + h], joint[:, hq + h:], at, status)
    _place(pools, slots, kb, vb)
    for got, want in zip(back(cache), pools):
        assert np.array_equal(got, want)  # the slots and nothing else
    ko, vo = (torch.full((n, h + 1, d), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ctx.lr_fp8_read(cache, at, ko[:, :h], vo[:, 1:], status)
    for out, rest, codes, scale in ((ko[:, :h], ko[:, h:], pools[0], pools[2]), (vo[:, 1:], vo[:, :1], pools[1], pools[3])):
        with np.errstate(over="ignore"):
            want = O.fp8_load(codes[slots // 16, :, slots % 16], scale[slots // 16, :, slots % 16]).astype(np.float32)
        want[slots < 0] = 7.0  # rows without a slot are left as they were
        assert np.array_equal(out.float().cpu().numpy(), want, equal_nan=True)
        assert bool((rest == 7.0).all())
    assert status.tolist() == [0, 0]
    assert ctx.launch_count == 2
    ctx.close()


def test_slots_beyond_the_cache_are_skipped_and_reported():
    rng = np.random.default_rng(1)
    ctx, pages = B.Context(Model(4, 2, 64, 8), 0), 5
    pools = _start(rng, pages + 1, 2, 64)
    whole = on_device(pools)
    cache = B.Fp8Cache(whole.k[:pages], whole.v[:pages], whole.k_scale[:pages], whole.v_scale[:pages])
    kb, vb = _rows(rng, 6, 2, 64), _rows(rng, 6, 2, 64)
    for bad in (pages * 16, pages * 16 + 3, 1 << 40, (1 << 63) - 1):
        slots = np.array([3, 8, bad, 70, -1, -(1 << 62)], dtype=np.int64)
        status, at = torch.zeros(2, dtype=torch.int32, device=DEV), torch.from_numpy(slots).to(DEV)
        ctx.lr_fp8_write(cache, _t(kb), _t(vb), at, status)
        assert status.tolist() == [-5, 2]
        good = np.where(slots < pages * 16, slots, -1)
        _place(pools, good, kb, vb)
        for got, want in zip(back(whole), pools):
            assert np.array_equal(got, want)
        status.zero_()
        out = torch.full((6, 2, 64), 7.0, dtype=torch.bfloat16, device=DEV)
        ctx.lr_fp8_read(cache, at, out, out.clone(), status)
        assert status.tolist() == [-5, 2] and bool((out[[2, 4, 5]] == 7.0).all())
        ctx.lr_fp8_read(cache, at, out, out.clone())  # without a status word as well
    ctx.close()


def test_the_same_slot_read_many_times_and_no_tokens():
    rng = np.random.default_rng(2)
    ctx = B.Context(Model(4, 2, 128, 8), 0)
    cache = on_device(store_pools(_rows(rng, 3 * 16, 2, 128).reshape(3, 2, 16, 128), _rows(rng, 3 * 16, 2, 128).reshape(3, 2, 16, 128)))
    slots = torch.full((301,), 37, dtype=torch.int64, device=DEV)
    k, v = (torch.zeros((301, 2, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ctx.lr_fp8_read(cache, slots, k, v)
    assert bool((k.view(torch.int16) == k[:1].view(torch.int16)).all()) and bool((v.view(torch.int16) == v[:1].view(torch.int16)).all())
    n = ctx.launch_count
    ctx.lr_fp8_write(cache, k[:0], v[:0], slots[:0])
    ctx.lr_fp8_read(cache, slots[:0], k[:0], v[:0])
    assert ctx.launch_count == n
    ctx.close()


def test_rows_that_the_call_does_not_take_are_refused():
    ctx = B.Context(Model(4, 2, 64, 8), 0)
    cache = B.Fp8Cache.empty(ctx.model, 4)
    k = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device=DEV)
    slots = torch.arange(3, device=DEV)
    assert B.lib().lr_fp8_write(ctx.handle, cache.c, k.data_ptr() + 2, 128, k.data_ptr(), 128, slots.data_ptr(), 1, None, None) == -1
    assert B.lib().lr_fp8_write(ctx.handle, cache.c, k.data_ptr(), 120, k.data_ptr(), 128, slots.data_ptr(), 3, None, None) == -1
    assert B.lib().lr_fp8_write(ctx.handle, cache.c, k.data_ptr(), 132, k.data_ptr(), 128, slots.data_ptr(), 1, None, None) == -1
    assert B.lib().lr_fp8_read(ctx.handle, cache.c, None, 1, k.data_ptr(), 128, k.data_ptr(), 128, None, None) == -1
    assert B.lib().lr_fp8_read(ctx.handle, cache.c, slots.data_ptr(), -1, k.data_ptr(), 128, k.data_ptr(), 128, None, None) == -1
    for args in ((k.float(), k, slots), (k[:2], k, slots), (k, k, slots.int()), (k, k.transpose(1, 2).contiguous().transpose(1, 2), slots), (k.cpu(), k, slots)):
        with pytest.raises(ValueError):
            ctx.lr_fp8_write(cache, *args)
    other = B.Fp8Cache.empty(Model(4, 4, 64, 8), 4)
    with pytest.raises(ValueError):
        ctx.lr_fp8_write(other, k, k, slots)
    assert ctx.launch_count == 0
    ctx.close()


def test_on_a_stream_of_its_own_and_replayed():
    rng = np.random.default_rng(3)
    ctx = B.Context(Model(8, 2, 128, 8), 0)
    pools = _start(rng, 9, 2, 128)
    cache, slots = on_device(pools), rng.permutation(9 * 16)[:100].astype(np.int64)
    kb, vb = _rows(rng, 100, 2, 128), _rows(rng, 100, 2, 128)
    k, v, at = _t(kb), _t(vb), torch.from_numpy(slots).to(DEV)
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    ctx.lr_fp8_write(cache, k, v, at, stream=side)
    ctx.lr_fp8_read(cache, at, ko, vo, stream=side)
    side.synchronize()
    _place(pools, slots, kb, vb)
    assert all(np.array_equal(a, b) for a, b in zip(back(cache), pools))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.lr_fp8_write(cache, k, v, at)
        ctx.lr_fp8_read(cache, at, ko, vo)
    for seed in (4, 5):
        kb, vb = _rows(np.random.default_rng(seed), 100, 2, 128), _rows(np.random.default_rng(seed + 10), 100, 2, 128)
        k.copy_(_t(kb))
        v.copy_(_t(vb))
        graph.replay()
        _place(pools, slots, kb, vb)
        assert all(np.array_equal(a, b) for a, b in zip(back(cache), pools))
        with np.errstate(over="ignore"):
            want = O.fp8_load(pools[0][slots // 16, :, slots % 16], pools[2][slots // 16, :, slots % 16]).astype(np.float32)
        assert np.array_equal(ko.float().cpu().numpy(), want, equal_nan=True)
    ctx.close()


# ---- compaction -----------------------------------------------------------------------------------------------------------
def _compact(w, n_accept):
    b, t = w.batch, w.tensors
    rng = np.random.default_rng(w.seed)
    pools = poison_slack(b, store_pools(t.k_pool, t.v_pool), rng)
    ctx = B.Context(b.model, 0)
    plan, cache = B.Plan(ctx, b), on_device(pools)
    c = O.commit(b, t.verdict, n_accept)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)  # noqa: E731
    new_len, n_kept = (torch.full((b.n_req,), -7, dtype=torch.int32, device=DEV) for _ in range(2))
    plan.lr_compact_fp8(i32(c["keep_off"]), i32(c["keep_pages"]), i32(c["keep_valid"]), cache, new_len, n_kept)
    assert plan.lr_poll_status() == 0
    # the oracle moves 16-bit words; bytes do as well
    wide = [p.astype(np.uint16) for p in pools]
    len_ref, kept_ref, k_ref, v_ref = O.compact(c["keep_off"], c["keep_pages"], c["keep_valid"], wide[0], wide[1])
    _, _, ks_ref, vs_ref = O.compact(c["keep_off"], c["keep_pages"], c["keep_valid"], wide[2][..., None], wide[3][..., None])
    assert np.array_equal(new_len.cpu().numpy(), len_ref) and np.array_equal(n_kept.cpu().numpy(), kept_ref)
    refs = (k_ref, v_ref, ks_ref[..., 0], vs_ref[..., 0])
    touched = np.zeros(b.n_pool_pages, dtype=bool)
    touched[c["keep_pages"]] = True
    for got, want, before in zip(back(cache), refs, pools):
        for r in range(b.n_req):
            pages, n = c["keep_pages"][c["keep_off"][r]:c["keep_off"][r + 1]], int(len_ref[r])
            for i in range(int(kept_ref[r])):
                assert np.array_equal(got[pages[i]][:, :min(16, n - 16 * i)], want[pages[i]][:, :min(16, n - 16 * i)])
        assert np.array_equal(got[~touched], before[~touched])
    plan.close()
    ctx.close()


@pytest.mark.parametrize("seed", range(8))
def test_compaction_of_ragged_batches(seed):
    w = make_random_small(8100 + seed)
    rng = np.random.default_rng(seed)
    _compact(w, np.array([rng.integers(0, L + 1) for L in w.batch.br_n_draft], dtype=np.int32))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("prefix,n_req", [(5, 1), (17, 40), (16500, 1)])  # a long list of kept pages takes several steps of the scan
def test_compaction_of_long_and_of_many(d, prefix, n_req):
    rng = np.random.default_rng(prefix + d)
    reqs = [{"P": prefix, "segs": [33, 7, 150], "branches": [(g, 21, 21, 21) for g in range(4)]} for _ in range(n_req)]
    w = _finish("compact", 3, Model(4, 2, d, 16), reqs, rng, 0.3, 0.9, False, True, "nan")
    _compact(w, np.full(w.batch.n_branch, 13, dtype=np.int32))


def test_keep_lists_that_are_none_are_reported():
    w = make_config(1, with_logits=False)
    b, t = w.batch, w.tensors
    ctx = B.Context(b.model, 0)
    plan, pools = B.Plan(ctx, b), store_pools(np.zeros_like(t.k_pool), np.zeros_like(t.v_pool))
    cache = on_device(pools)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    out = [torch.zeros(1, dtype=torch.int32, device=DEV) for _ in range(2)]
    for lists in (([0, 2], [0, b.n_pool_pages], [3, 16]), ([0, 2], [-1, 1], [3, 16]), ([0, 2], [0, 1], [3, 17]), ([0, b.n_page_slots + 1], [0], [1])):
        plan.lr_compact_fp8(*(i32(a) for a in lists), cache, *out)
        with pytest.raises(B.LrError) as e:
            plan.lr_poll_status()
        assert e.value.status == -5
    small = B.Fp8Cache(cache.k[:b.n_pool_pages - 1], cache.v[:b.n_pool_pages - 1], cache.k_scale[:b.n_pool_pages - 1], cache.v_scale[:b.n_pool_pages - 1])
    with pytest.raises(B.LrError) as e:
        plan.lr_compact_fp8(i32([0, 1]), i32([0]), i32([1]), small, *out)
    assert e.value.status == -1
    plan.close()
    ctx.close()
