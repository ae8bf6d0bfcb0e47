"""Rotary positions and the cache writes behind them, against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

import fp4_util
import fp8_util
from lr_workloads import Model, bf16_round, bf16_to_f32
from oracle import lr_oracle as O
from paper_2506_19830_b200 import binding as B
from paper_2506_19830_b200 import runner as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = ["bf16", "fp8", "fp4"]
# What fp32 may put a turned number off by, of the larger channel of its pair: sine and cosine (2^-23 each, of an angle that is within 2^-24 of half
# a turn, pi 2^-24), two products and a sum (2^-24 each); together below 2^-20.
SLACK = 2.0 ** -20


def empty(kind, model, pages):
    if kind == "bf16":
        return B.Bf16Cache(*(torch.full((pages, model.n_kv_heads, 16, model.head_dim), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)))
    return (B.Fp8Cache if kind == "fp8" else B.Fp4Cache).empty(model, pages, DEV)


def raw(cache):
    if isinstance(cache, B.Bf16Cache):
        return [cache.k.view(torch.int16).cpu().numpy(), cache.v.view(torch.int16).cpu().numpy()]
    return (fp8_util if isinstance(cache, B.Fp8Cache) else fp4_util).back(cache)


def rows(rng, n, heads, d):
    return bf16_round((rng.standard_normal((n, heads, d)) * np.exp(rng.uniform(-2, 2, (n, heads, 1)))).astype(np.float32))


def pair_size(x, rot, interleaved):
    """Per channel the larger of its pair's (0 where nothing is turned)."""
    a, s = np.abs(x), np.zeros_like(x)
    if interleaved:
        m = np.maximum(a[..., 0:rot:2], a[..., 1:rot:2])
        s[..., 0:rot:2] = s[..., 1:rot:2] = m
    else:
        m = np.maximum(a[..., :rot // 2], a[..., rot // 2:rot])
        s[..., :rot // 2] = s[..., rot // 2:rot] = m
    return s


def check_bf16(got, want, slack):
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + slack).all(), np.abs(got - want).max()


def check_stored(kind, cache, side, at, want, slack):
    """The rows at slots `at` are those of `want`, rounded to what the cache holds."""
    page, place = at // 16, at % 16
    if kind == "bf16":
        check_bf16(bf16_to_f32(raw(cache)[side].view(np.uint16)[page, :, place]).astype(np.float64), want, slack)
        return
    pools = raw(cache)
    codes, byte = pools[side][page, :, place], pools[2 + side][page, :, place]
    if kind == "fp8":
        most, least, grid, width, load = 448.0, 3, O.e4m3_values(), want.shape[-1], O.fp8_load
    else:
        most, least, grid, width, load = 6.0, 1, np.concatenate([O.E2M1, -O.E2M1]), 32, O.fp4_load
    scale = np.exp2(byte.astype(np.float64).reshape(*want.shape[:-1], -1) - 127.0)
    top = np.abs(want).reshape(*scale.shape, width).max(-1)
    loose = np.abs(slack).reshape(*scale.shape, width).max(-1)
    assert (top - loose <= most * scale).all() and ((top + loose > most / 2 * scale) | (scale == 2.0 ** (least - 127))).all()
    each = np.repeat(scale, width, -1)
    grid = np.unique(grid[np.isfinite(grid)])
    y = want / each
    i = np.clip(np.searchsorted(grid, y), 1, len(grid) - 1)
    nearest = np.minimum(np.abs(y - grid[i - 1]), np.abs(y - grid[i]))
    assert (np.abs(load(codes, byte) / each - y) <= nearest + 2 * slack / each).all()


CASES = [(64, 64, False), (64, 64, True), (128, 128, False), (128, 128, True), (128, 64, True), (128, 64, False), (128, 32, False), (128, 90, False), (128, 90, True), (64, 2, False),
         (64, 34, False), (64, 16, True), (128, 126, False)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d,rot,interleaved", CASES)
@pytest.mark.parametrize("hq,h,n", [(8, 2, 33), (5, 1, 1), (40, 8, 3)])
def test_rows_are_turned_and_written(hq, h, n, d, rot, interleaved, kind):
    rng = np.random.default_rng(rot + d + n)
    model, pages = Model(hq, h, d, 8), n // 16 + 3
    ctx, cache = B.Context(model, 0), empty(kind, model, pages)
    q, k, v = rows(rng, n, hq, d), rows(rng, n, h, d), rows(rng, n, h, d)
    joint = torch.cat([R.bf16_tensor(x, DEV) for x in (q, k, v)], 1)
    at = rng.integers(0, 100000, n).astype(np.int32)
    slots = rng.permutation(pages * 16)[:n].astype(np.int64)
    if n > 2:
        slots[1] = -1
    before = [x.copy() for x in raw(cache)]
    rope = B.Rope(rot, base=1e4, interleaved=interleaved, scaling="parts", factor=16.0, original=4096)
    out, status = torch.full((n, hq, d), 7.0, dtype=torch.bfloat16, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    to = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    ctx.lr_rope_write(rope, to(at), cache, joint[:, hq:hq + h], joint[:, hq + h:], to(slots), joint[:, :hq], out, status)
    f, amplitude = O.rope_frequencies(rot, 1e4, "parts", 16.0, 4096.0, 1.0, 32.0)
    q, k, v = (bf16_to_f32(x).astype(np.float64) for x in (q, k, v))
    check_bf16(bf16_to_f32(R.bf16_bits(out)).astype(np.float64), O.rope(q, at, f, amplitude, interleaved), SLACK * amplitude * pair_size(q, rot, interleaved))
    keep = slots >= 0
    check_stored(kind, cache, 0, slots[keep], O.rope(k, at, f, amplitude, interleaved)[keep], SLACK * amplitude * pair_size(k, rot, interleaved)[keep])
    check_stored(kind, cache, 1, slots[keep], v[keep], np.zeros_like(v[keep]))
    other = np.ones(pages * 16, dtype=bool)
    other[slots[keep]] = False
    for was, now in zip(before, raw(cache)):  # the slots and nothing else
        assert np.array_equal(was[np.flatnonzero(other) // 16, :, np.flatnonzero(other) % 16], now[np.flatnonzero(other) // 16, :, np.flatnonzero(other) % 16])
    assert status.tolist() == [0, 0] and ctx.launch_count == 1
    ctx.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 2, 1500, 20000])
def test_many_tokens_and_values_bit_for_bit(kind, n):
    """V, and K without rotation, are what the caches' own writes leave, whatever number of tokens a CTA takes."""
    rng = np.random.default_rng(n)
    model = Model(8, 4, 128, 8)
    pages = n // 16 + 2
    ctx = B.Context(model, 0)
    x = R.bf16_tensor(rows(rng, 2 * n, 4, 128), DEV)
    k, v = x[:n], x[n:]
    slots = torch.from_numpy(rng.permutation(pages * 16)[:n].astype(np.int64)).to(DEV)
    a, b = empty(kind, model, pages), empty(kind, model, pages)
    at = torch.from_numpy(rng.integers(-(1 << 20), 1 << 20, n).astype(np.int32)).to(DEV)
    ctx.lr_rope_write(None, None, a, k, v, slots)
    ctx.lr_rope_write(B.Rope(128), at, b, k, v, slots)
    if kind == "bf16":
        want = torch.full_like(a.k, 7.0)
        want[slots // 16, :, slots % 16] = k
        assert torch.equal(a.k, want)
        want[slots // 16, :, slots % 16] = v
        assert torch.equal(a.v, want) and torch.equal(b.v, want)
    else:
        c = empty(kind, model, pages)
        (ctx.lr_fp8_write if kind == "fp8" else ctx.lr_fp4_write)(c, k, v, slots)
        pools = [raw(y) for y in (a, b, c)]
        assert all(np.array_equal(p, r) for p, r in zip(pools[0], pools[2]))
        assert np.array_equal(pools[1][1], pools[2][1]) and np.array_equal(pools[1][3], pools[2][3])
    # some of the keys
    some = np.unique(rng.integers(0, n, 40))
    f, _ = O.rope_frequencies(128, 1e4)
    kk = bf16_to_f32(R.bf16_bits(k[some])).astype(np.float64)
    check_stored(kind, b, 0, slots.cpu().numpy()[some], O.rope(kk, at.cpu().numpy()[some], f), SLACK * pair_size(kk, 128, False))
    ctx.close()


@pytest.mark.parametrize("scaling", ["none", "linear", "smooth", "parts"])
def test_far_positions_keep_their_angles(scaling):
    rng = np.random.default_rng(5)
    model = Model(4, 1, 64, 8)
    ctx, at = B.Context(model, 0), np.array([0, 1, -1, 131071, 10_000_019, (1 << 31) - 1, -(1 << 31), 77777], dtype=np.int32)
    n = len(at)
    kw = dict(scaling=scaling, factor=1.0 if scaling == "none" else 7.0, original=2048.0, lo=1.0, hi=8.0)
    rope = B.Rope(64, base=5e5, **kw)
    q, k = rows(rng, n, 4, 64), rows(rng, n, 1, 64)
    cache, out = empty("bf16", model, 2), torch.zeros((n, 4, 64), dtype=torch.bfloat16, device=DEV)
    ctx.lr_rope_write(rope, torch.from_numpy(at).to(DEV), cache, R.bf16_tensor(k, DEV), R.bf16_tensor(k, DEV), torch.arange(n, device=DEV), R.bf16_tensor(q, DEV), out)
    f, amplitude = O.rope_frequencies(64, 5e5, **kw)
    q = bf16_to_f32(q).astype(np.float64)
    # the angle itself: 2^31 radians to 2^-53 of it, here and in the oracle
    check_bf16(bf16_to_f32(R.bf16_bits(out)).astype(np.float64), O.rope(q, at, f, amplitude), (SLACK + 2.0 ** -20) * amplitude * pair_size(q, 64, False))
    ctx.close()


@pytest.mark.parametrize("rot,interleaved", [(128, False), (128, True), (90, False), (32, True)])
def test_queries_may_be_turned_where_they_are(rot, interleaved):
    rng = np.random.default_rng(6)
    model, n = Model(8, 2, 128, 8), 700
    ctx, cache = B.Context(model, 0), empty("fp4", model, 50)
    q, k = R.bf16_tensor(rows(rng, n, 8, 128), DEV), R.bf16_tensor(rows(rng, n, 2, 128), DEV)
    at, slots = torch.arange(n, dtype=torch.int32, device=DEV), torch.arange(n, device=DEV)
    rope, out = B.Rope(rot, interleaved=interleaved), torch.zeros_like(q)
    ctx.lr_rope_write(rope, at, cache, k, k.clone(), slots, q, out)
    ctx.lr_rope_write(rope, at, cache, k, k.clone(), slots, q, q)
    assert torch.equal(q, out)
    ctx.close()


@pytest.mark.parametrize("kind", KINDS)
def test_rows_that_are_not_finite(kind):
    model = Model(2, 1, 64, 8)
    ctx, cache = B.Context(model, 0), empty(kind, model, 1)
    x = torch.ones((4, 1, 64), dtype=torch.bfloat16, device=DEV)
    x[0, 0, 3], x[1, 0, 60], x[2, 0, 1] = float("inf"), float("nan"), -float("inf")  # channels 0..15 are turned
    ctx.lr_rope_write(B.Rope(16), torch.full((4,), 5, dtype=torch.int32, device=DEV), cache, x, x, torch.arange(4, device=DEV))
    if kind == "bf16":
        got = cache.k[0, 0, :4].float()
        assert not bool(torch.isfinite(got[0, [3, 11]]).any()) and bool(torch.isnan(got[1, 60])) and bool(torch.isfinite(got[3]).all())
        assert int(torch.isfinite(got[0]).sum()) == 62 and int(torch.isfinite(got[1]).sum()) == 63
        assert torch.equal(cache.v[0, 0, :4].view(torch.int16), x[:, 0].view(torch.int16))
    else:
        codes, scale = raw(cache)[0], raw(cache)[2]
        assert not codes[0, 0, :3].any() and (scale[0, 0, :3] == 255).all() and (scale[0, 0, 3] != 255).all()
    ctx.close()


def test_more_heads_than_a_cta_takes():
    rng = np.random.default_rng(7)
    model, n = Model(96, 48, 64, 8), 5
    for kind in KINDS:
        ctx, cache = B.Context(model, 0), empty(kind, model, 2)
        q, k, v = rows(rng, n, 96, 64), rows(rng, n, 48, 64), rows(rng, n, 48, 64)
        at, slots, out = np.arange(n, dtype=np.int32) * 1000, np.arange(n) * 3, torch.zeros((n, 96, 64), dtype=torch.bfloat16, device=DEV)
        to = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
        ctx.lr_rope_write(B.Rope(64), to(at), cache, R.bf16_tensor(k, DEV), R.bf16_tensor(v, DEV), to(slots), R.bf16_tensor(q, DEV), out)
        f, _ = O.rope_frequencies(64, 1e4)
        qq, kk, vv = (bf16_to_f32(x).astype(np.float64) for x in (q, k, v))
        check_bf16(bf16_to_f32(R.bf16_bits(out)).astype(np.float64), O.rope(qq, at, f), SLACK * pair_size(qq, 64, False))
        check_stored(kind, cache, 0, slots, O.rope(kk, at, f), SLACK * pair_size(kk, 64, False))
        check_stored(kind, cache, 1, slots, vv, np.zeros_like(vv))
        ctx.close()


def test_slots_beyond_the_cache_are_skipped_and_reported():
    model = Model(4, 2, 64, 8)
    ctx, x = B.Context(model, 0), torch.ones((5, 2, 64), dtype=torch.bfloat16, device=DEV)
    for kind in KINDS:
        cache = empty(kind, model, 3)
        before = raw(cache)
        slots = torch.tensor([-1, 48, -(1 << 62), 1 << 50, -5], device=DEV)
        status, out = torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros((5, 4, 64), dtype=torch.bfloat16, device=DEV)
        q = torch.ones((5, 4, 64), dtype=torch.bfloat16, device=DEV)
        ctx.lr_rope_write(B.Rope(64), torch.zeros(5, dtype=torch.int32, device=DEV), cache, x, x, slots, q, out, status)
        assert status.tolist()[0] == -5 and status.tolist()[1] in (1, 3)
        assert all(np.array_equal(a, b) for a, b in zip(before, raw(cache)))
        assert torch.equal(out, q)  # position 0 turns nothing; queries without a slot are turned all the same
        ctx.lr_rope_write(B.Rope(64), torch.zeros(5, dtype=torch.int32, device=DEV), cache, x, x, slots)  # without a status word as well
    ctx.close()


def test_refusals():
    model = Model(4, 2, 64, 8)
    ctx, L = B.Context(model, 0), B.lib()
    cache, rope = empty("bf16", model, 3), B.Rope(64)
    joint = torch.zeros((3, 8, 64), dtype=torch.bfloat16, device=DEV)
    q, k, v = joint[:, :4], joint[:, 4:6], joint[:, 6:]
    at, slots, out = torch.zeros(3, dtype=torch.int32, device=DEV), torch.arange(3, device=DEV), torch.zeros((3, 4, 64), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(B.LrError) as e:
        ctx.lr_rope_write(B.Rope(66), at, cache, k, v, slots)
    assert e.value.status == -1 and "rot_dim" in str(e.value)
    with pytest.raises(ValueError):
        ctx.lr_rope_write(rope, at, cache, k, v, slots, q, q)  # its rows have a stride
    for args in ((at.cpu(), k, v, slots, q, out), (at, k.float(), v, slots, q, out), (at, k, v, slots.int(), q, out), (at, k, v, slots, q, None), (at, k, v, slots, q.cpu(), out),
                 (at, k, v, slots, q, out.cpu()), (None, k, v, slots, q, out)):
        with pytest.raises(ValueError):
            ctx.lr_rope_write(rope, args[0], cache, *args[1:])
    with pytest.raises(ValueError):
        ctx.lr_rope_write(rope, at, empty("fp8", Model(4, 4, 64, 8), 3), k, v, slots)
    good = [ctx.handle, rope.handle, cache.any, at.data_ptr(), q.data_ptr(), 512, out.data_ptr(), k.data_ptr(), 512, v.data_ptr(), 512, slots.data_ptr(), 3, None, None]
    for i, bad in ((0, None), (2, None), (3, None), (4, q.data_ptr() + 2), (5, 508), (5, 248), (6, None), (6, out.data_ptr() + 8), (6, q.data_ptr()), (7, None), (8, 120), (10, 132), (11, None), (12, -1)):
        args = list(good)
        args[i] = bad
        assert L.lr_rope_write(*args) == -1, (i, bad)
    assert ctx.launch_count == 0
    ctx.lr_rope_write(rope, at[:0], cache, k[:0], v[:0], slots[:0], q[:0], out[:0])
    assert ctx.launch_count == 0
    assert L.lr_rope_write(*good) == 0
    torch.cuda.synchronize()
    ctx.close()


def test_on_a_stream_of_its_own_and_replayed_with_other_positions():
    rng = np.random.default_rng(8)
    model, n = Model(8, 2, 128, 8), 60
    ctx, rope = B.Context(model, 0), B.Rope(128, base=5e5)
    cache, q, k = empty("bf16", model, 5), rows(rng, n, 8, 128), rows(rng, n, 2, 128)
    qd, kd, at, slots = R.bf16_tensor(q, DEV), R.bf16_tensor(k, DEV), torch.arange(n, dtype=torch.int32, device=DEV), torch.arange(n, device=DEV)
    out, side = torch.zeros_like(qd), torch.cuda.Stream()
    torch.cuda.synchronize()
    ctx.lr_rope_write(rope, at, cache, kd, kd, slots, qd, out, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.lr_rope_write(rope, at, cache, kd, kd, slots, qd, out)
    rope.close()  # the graph has what it needs
    f, _ = O.rope_frequencies(128, 5e5)
    q, k = (bf16_to_f32(x).astype(np.float64) for x in (q, k))
    for first in (0, 5000):
        at.copy_(torch.arange(first, first + n, device=DEV))
        graph.replay()
        p = np.arange(first, first + n)
        check_bf16(bf16_to_f32(R.bf16_bits(out)).astype(np.float64), O.rope(q, p, f), SLACK * pair_size(q, 128, False))
        check_stored("bf16", cache, 0, np.arange(n), O.rope(k, p, f), SLACK * pair_size(k, 128, False))
    ctx.close()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,h,d,rot,n", [(8, 2, 128, 90, 5000), (4, 4, 64, 34, 6000), (3, 1, 128, 126, 2500), (96, 48, 128, 90, 7), (96, 48, 128, 128, 7), (96, 48, 64, 2, 5)])
def test_halves_that_start_anywhere(hq, h, d, rot, n, kind):
    """Several tokens to a CTA, more heads than it takes, the most shared memory; what is not turned keeps its bits."""
    rng = np.random.default_rng(rot + n)
    model, pages = Model(hq, h, d, 8), n // 16 + 1
    ctx, cache = B.Context(model, 0), empty(kind, model, pages)
    q, k, v = rows(rng, n, hq, d), rows(rng, n, h, d), rows(rng, n, h, d)
    at, slots = rng.integers(0, 1 << 20, n).astype(np.int32), rng.permutation(pages * 16)[:n].astype(np.int64)
    to = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    out = torch.zeros((n, hq, d), dtype=torch.bfloat16, device=DEV)
    ctx.lr_rope_write(B.Rope(rot), to(at), cache, R.bf16_tensor(k, DEV), R.bf16_tensor(v, DEV), to(slots), R.bf16_tensor(q, DEV), out)
    f, _ = O.rope_frequencies(rot, 1e4)
    assert np.array_equal(R.bf16_bits(out)[:, :, rot:], q[:, :, rot:])
    qq, kk, vv = (bf16_to_f32(x).astype(np.float64) for x in (q, k, v))
    check_bf16(bf16_to_f32(R.bf16_bits(out)).astype(np.float64), O.rope(qq, at, f), SLACK * pair_size(qq, rot, False))
    check_stored(kind, cache, 0, slots, O.rope(kk, at, f), SLACK * pair_size(kk, rot, False))
    check_stored(kind, cache, 1, slots, vv, np.zeros_like(vv))
    ctx.close()


def test_rows_that_are_not_finite_beside_halves_that_start_anywhere():
    model = Model(2, 1, 128, 8)
    ctx, cache = B.Context(model, 0), empty("bf16", model, 1)
    x = torch.ones((2, 1, 128), dtype=torch.bfloat16, device=DEV)
    x.view(torch.int16)[0, 0, 100] = 0x7FA5  # a NaN of its own bits, not turned
    x[1, 0, 3] = float("inf")
    q = torch.cat([x, x], 1)
    ctx.lr_rope_write(B.Rope(90), torch.full((2,), 5, dtype=torch.int32, device=DEV), cache, x, x, torch.arange(2, device=DEV), q, q)
    for got in (cache.k[0, 0, :2], q[:, 0], q[:, 1]):
        assert got.view(torch.int16)[0, 100] == 0x7FA5 and int(torch.isfinite(got[0].float()).sum()) == 127
        assert not bool(torch.isfinite(got[1, [3, 48]].float()).any()) and int(torch.isfinite(got[1].float()).sum()) == 126
    ctx.close()
