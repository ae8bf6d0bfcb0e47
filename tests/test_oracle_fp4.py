"""Pins for the oracle's 4-bit cache and rotary positions, and the refusals of their entry points that need no device."""
import ctypes as C
import math
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from fp4_util import as_bf16
from lr_workloads import Model, bf16_round, bf16_to_f32
from oracle import lr_oracle as O
from paper_2506_19830_b200 import binding as B
from paper_2506_19830_b200.build import build_library


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()


# ---- the 4-bit cache ---------------------------------------------------------------------------------------------------------
def test_codes_are_the_bits_of_a_small_floating_point_number():
    """Sign, two bits of exponent with a bias of 1, one of fraction; the word's order of channels."""
    codes = np.arange(256, dtype=np.uint8)[:, None].repeat(16, 1)  # 32 channels of the same two codes
    x = O.fp4_load(codes, np.full((256, 1), 127, dtype=np.uint8))

    def value(n):
        e, m = n >> 1 & 3, n & 1
        return (-1) ** (n >> 3) * ((1 + m / 2) * 2.0 ** (e - 1) if e else m / 2)

    for byte in range(256):
        low, high = value(byte & 15), value(byte >> 4)
        assert np.array_equal(x[byte, :8], [low, low, high, high] * 2)
    one = np.zeros((8, 16), dtype=np.uint8)  # a code of 1 for each channel of the second word in turn
    for c in range(8):
        bit = 4 * (c // 2) + 16 * (c % 2)
        one[c, 4 + bit // 8] = 2 << bit % 8
    assert np.array_equal(O.fp4_load(one, np.full((8, 1), 127, dtype=np.uint8))[:, 8:16], np.eye(8))


def test_codes_are_the_nearest_and_scales_the_smallest_that_hold_their_group():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((400, 64)) * np.exp(rng.uniform(-60, 60, (400, 1))) * np.exp(rng.uniform(-3, 3, (400, 64)))
    bits = bf16_round(x.astype(np.float32))
    want = bf16_to_f32(bits).astype(np.float64)
    codes, byte = O.fp4_store(bits)
    got, scale = O.fp4_load(codes, byte), np.exp2(byte.astype(np.float64) - 127).repeat(32, -1)
    top = np.abs(want).reshape(400, 2, 32).max(-1)
    assert (top <= 6 * scale[:, ::32]).all() and ((top > 3 * scale[:, ::32]) | (byte == 1)).all()
    grid = np.concatenate([O.E2M1, -O.E2M1])
    assert np.array_equal(np.abs(got - want), np.abs(want[..., None] - grid * scale[..., None]).min(-1))
    assert np.array_equal(bf16_to_f32(as_bf16(codes, byte)).astype(np.float64), got)  # no second rounding


def test_ties_go_to_the_even_code():
    row = np.zeros((1, 32))
    row[0, :15] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5]
    got = O.fp4_load(*O.fp4_store(bf16_round(row.astype(np.float32))))[0, :15]
    assert np.array_equal(got, [6, 0, 1, 1, 2, 2, 4, 4, 0, -1, -1, -2, -2, -4, -4]) and np.signbit(got[8])


def test_rows_that_are_not_finite_and_the_ends_of_the_range():
    bits = bf16_round(np.random.default_rng(3).standard_normal((6, 64)).astype(np.float32))
    bits[0, 3], bits[1, 40], bits[2, 0] = 0x7FC0, 0x7F80, 0xFF80
    bits[3] = 0x0001  # the smallest number there is: half a code of the least scale is 2^-128
    bits[4] = 0x7F7F  # the largest
    bits[5] = 0x8000
    codes, byte = O.fp4_store(bits)
    assert (byte[:3] == 255).all() and not codes[:3].any() and np.isnan(O.fp4_load(codes, byte)[:3]).all()
    assert (byte[3] == 1).all() and not O.fp4_load(codes, byte)[3].any()
    assert (byte[4] == 253).all() and (O.fp4_load(codes, byte)[4] == 2.0 ** 128).all()
    assert (codes[5] == 0x88).all() and (byte[5] == 1).all()


# ---- rotary positions ----------------------------------------------------------------------------------------------------------
SCALINGS = [dict(scaling="none"), dict(scaling="linear", factor=4.0), dict(scaling="parts", factor=16.0, original=4096.0, lo=1.0, hi=32.0),
            dict(scaling="smooth", factor=8.0, original=8192.0, lo=1.0, hi=4.0)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("kw", SCALINGS)
def test_scores_depend_on_how_far_apart_positions_are(kw, interleaved):
    rng = np.random.default_rng(1)
    f, amplitude = O.rope_frequencies(32, 1e4, **kw)
    q, k = rng.standard_normal((2, 1, 1, 64))
    score = lambda p, r: float((O.rope(q, [p], f, amplitude, interleaved) * O.rope(k, [r], f, amplitude, interleaved)).sum())  # noqa: E731
    near = [score(p, p - 7) for p in (7, 100, 70000)]
    assert np.ptp(near) < 1e-9 and abs(score(9, 1) - near[0]) > 1e-3
    turned = O.rope(q, [12345], f, amplitude, interleaved)
    assert np.array_equal(turned[..., 32:], q[..., 32:]) and np.array_equal(O.rope(q, [0], f, 1.0, interleaved), q)
    assert math.isclose(np.square(turned[..., :32]).sum(), amplitude ** 2 * np.square(q[..., :32]).sum(), rel_tol=1e-12)


def test_the_two_layouts_are_one_rotation_of_other_channels():
    rng = np.random.default_rng(2)
    f, _ = O.rope_frequencies(48, 1e4)
    x = rng.standard_normal((5, 2, 64))
    order = np.concatenate([np.arange(48).reshape(2, 24).T.reshape(-1), np.arange(48, 64)])  # channel c of the interleaved layout
    a = O.rope(x, range(5), f)
    b = O.rope(x[..., order], range(5), f, interleaved=True)
    assert np.array_equal(a[..., order], b)


def test_frequencies_that_are_stretched_and_kept():
    plain, one = O.rope_frequencies(128, 5e5)
    assert one == 1.0 and plain[0] == 1.0 and math.isclose(plain[64 - 1], 5e5 ** (-126 / 128))
    smooth, _ = O.rope_frequencies(128, 5e5, "smooth", 8.0, 8192.0, 1.0, 4.0)
    turns = 8192.0 * plain / (2 * math.pi)
    assert np.array_equal(smooth[turns >= 4], plain[turns >= 4]) and np.allclose(smooth[turns <= 1], plain[turns <= 1] / 8, rtol=1e-15)
    between = (turns > 1) & (turns < 4)
    assert between.any() and (smooth[between] < plain[between]).all() and (smooth[between] > plain[between] / 8).all()
    parts, amplitude = O.rope_frequencies(64, 1e4, "parts", 16.0, 4096.0, 1.0, 32.0)
    plain = O.rope_frequencies(64, 1e4)[0]
    turns = 4096.0 * plain / (2 * math.pi)
    first, last = int(np.argmax(turns < 32)) - 1, int(np.argmax(turns < 1))
    assert np.array_equal(parts[:first + 1], plain[:first + 1]) and np.allclose(parts[last:], plain[last:] / 16, rtol=1e-15)
    assert math.isclose(amplitude, 1 + math.log(16) / 10)


@pytest.mark.parametrize("rot,base", [(2, 10.0), (64, 1e4), (128, 5e5), (90, 1e6)])
@pytest.mark.parametrize("kw", SCALINGS)
def test_the_librarys_frequencies_are_the_oracles(kw, rot, base):
    r = B.Rope(rot, base=base, **kw)
    f, amplitude = r.frequencies()
    want, a = O.rope_frequencies(rot, base, **{"factor": 1.0, "original": 0.0, **kw})
    assert np.allclose(f, want, rtol=1e-14, atol=0) and math.isclose(amplitude, a, rel_tol=1e-15)
    assert B.Rope(rot, base=base, **kw, amplitude=1.25).frequencies()[1] == 1.25
    r.close()


@pytest.mark.parametrize("bad", [
    dict(rot_dim=0), dict(rot_dim=-2), dict(rot_dim=7), dict(rot_dim=130), dict(base=1.0), dict(base=0.0), dict(base=float("nan")), dict(base=float("inf")),
    dict(scaling="linear", factor=0.5), dict(scaling="linear", factor=float("nan")), dict(scaling="parts", factor=2.0, original=0.0),
    dict(scaling="smooth", factor=2.0, original=100.0, lo=0.0), dict(scaling="smooth", factor=2.0, original=100.0, lo=4.0, hi=4.0),
    dict(scaling="parts", factor=2.0, original=float("inf")), dict(amplitude=float("nan")),
])
def test_rotary_positions_that_cannot_be_are_refused(bad):
    with pytest.raises(B.LrError) as e:
        B.Rope(**dict(dict(rot_dim=64), **bad))
    assert e.value.status == -1 and "lr_rope_create" in str(e.value)


def test_rope_handles():
    L, h = B.lib(), C.c_void_p(5)
    spec = B.lr_rope_spec(9, 0, 0, 1e4, 1.0, 0.0, 1.0, 4.0, 0.0)
    assert L.lr_rope_create(C.byref(h), C.byref(spec)) == -1 and h.value is None
    assert L.lr_rope_create(None, C.byref(spec)) == -1 and L.lr_rope_create(C.byref(h), None) == -1
    spec.scaling = 4
    spec.rot_dim = 8
    assert L.lr_rope_create(C.byref(h), C.byref(spec)) == -1
    assert L.lr_rope_destroy(None) == -1 and L.lr_rope_frequencies(None, None, None) == -1
    with pytest.raises(ValueError):
        B.Rope(64, scaling="any")


# ---- refusals -------------------------------------------------------------------------------------------------------------
def _cache(kind=None, **kw):
    a = dict(dict(k_d=1 << 20, v_d=2 << 20, k_scale_d=3 << 20, v_scale_d=4 << 20, n_pages=8), **kw)
    return B.lr_fp4_cache(**a) if kind is None else B.lr_kv_cache(kind, *(a[n] for n in ("k_d", "v_d", "k_scale_d", "v_scale_d", "n_pages")))


BAD = [(dict(k_d=None), "null"), (dict(v_d=None), "null"), (dict(k_scale_d=None), "null"), (dict(v_scale_d=None), "null"),
       (dict(k_d=(1 << 20) + 8), "aligned"), (dict(v_scale_d=(4 << 20) + 4), "aligned"), (dict(n_pages=0), "page"), (dict(n_pages=-3), "page"),
       (dict(n_pages=1 << 50), "pages"), (dict(v_d=1 << 20), "share"), (dict(v_scale_d=3 << 20), "share")]


@pytest.mark.parametrize("bad,words", BAD)
def test_a_cache_that_cannot_be_one_is_refused(bad, words):
    L, c = B.lib(), _cache(**bad)
    at = C.addressof(c)
    calls = [lambda: L.lr_fp4_write(None, at, 16, 8, 16, 8, 8, 1, None, None), lambda: L.lr_fp4_read(None, at, 8, 1, 16, 8, 16, 8, None, None),
             lambda: L.lr_verify_attention_fp4(None, 16, at, 16, None, 0.0, None), lambda: L.lr_compact_fp4(None, 4, 4, 4, at, 4, 4, None)]
    for kind in (B.KV_FP8, B.KV_FP4):
        any_kind = _cache(kind, **bad)
        calls.append(lambda c=any_kind: L.lr_rope_write(None, None, C.addressof(c), None, None, 0, None, 16, 8, 16, 8, 8, 1, None, None))
    for call in calls:
        assert call() == -1
        assert words in L.lr_last_error().decode()


@pytest.mark.parametrize("kind,bad", [(-1, {}), (3, {}), (B.KV_BF16, dict(k_d=None)), (B.KV_BF16, dict(v_d=(2 << 20) + 2)), (B.KV_BF16, dict(n_pages=0)), (B.KV_BF16, dict(v_d=1 << 20))])
def test_a_cache_of_no_kind_is_refused(kind, bad):
    L, c = B.lib(), _cache(kind, **bad)
    assert L.lr_rope_write(None, None, C.addressof(c), None, None, 0, None, 16, 8, 16, 8, 8, 1, None, None) == -1
    assert "cache" in L.lr_last_error().decode()


def test_null_handles_are_refused():
    L, c = B.lib(), _cache()
    at, kv = C.addressof(c), _cache(B.KV_FP4)
    for null_cache in (None, at):
        assert L.lr_fp4_write(None, null_cache, 16, 8, 16, 8, 8, 1, None, None) == -1
        assert L.lr_fp4_read(None, null_cache, 8, 1, 16, 8, 16, 8, None, None) == -1
        assert L.lr_verify_attention_fp4(None, 16, null_cache, 16, None, 0.0, None) == -1
        assert L.lr_compact_fp4(None, 4, 4, 4, null_cache, 4, 4, None) == -1
    assert L.lr_rope_write(None, None, C.addressof(kv), None, None, 0, None, 16, 8, 16, 8, 8, 1, None, None) == -1
    assert L.lr_copy_pages(None, C.addressof(kv), C.addressof(kv), 1, 4, 4, 1, None, None) == -1


def test_tensors_that_are_no_cache_are_refused():
    codes, scale = torch.zeros((3, 2, 16, 32), dtype=torch.uint8), torch.zeros((3, 2, 16, 2), dtype=torch.uint8)
    c = B.Fp4Cache(codes, codes.clone(), scale, scale.clone())
    assert c.head_dim == 64 and c.heads == 2 and c.n_pages == 3
    B.Fp4Cache(codes, codes.clone(), scale.view(torch.float8_e8m0fnu), scale)
    for args in ((codes, codes[:2], scale, scale), (codes, codes, scale[:, :1], scale), (codes[..., :16], codes[..., :16], scale, scale),
                 (codes.float(), codes, scale, scale), (codes, codes, scale, codes), (codes[:, :, :8], codes[:, :, :8], scale[:, :, :8], scale[:, :, :8]),
                 (codes.transpose(0, 1), codes.transpose(0, 1), scale.transpose(0, 1), scale.transpose(0, 1)), (codes, codes, scale[..., 0], scale[..., 0])):
        with pytest.raises(ValueError):
            B.Fp4Cache(*args)
    pool = torch.zeros((3, 2, 16, 64), dtype=torch.bfloat16)
    B.Bf16Cache(pool, pool.clone())
    for args in ((pool, pool[:2]), (pool.float(), pool.float()), (pool[:, :, :8], pool[:, :, :8]), (pool[0], pool[0]), (pool[..., ::2], pool[..., ::2])):
        with pytest.raises(ValueError):
            B.Bf16Cache(*args)


def test_a_cache_of_another_kind_is_not_taken_for_one():
    ctx = SimpleNamespace(model=Model(4, 2, 64, 8), device=-1, cache_kind=(2, 64, None))
    for make, kind in ((B.Fp4Cache, B.Fp8Cache), (B.Fp8Cache, B.Fp4Cache)):
        cache = make.empty(ctx.model, 3, "cpu")
        with pytest.raises(ValueError, match=kind.__name__):
            B._of_kind(cache, kind)
        assert B._of_kind(cache, make) is cache


def test_rope_takes_tensors_for_what_they_are():
    ctx = SimpleNamespace(model=Model(4, 2, 64, 8), device=-1)
    joint = torch.zeros((5, 8, 64), dtype=torch.bfloat16)
    q, out, at = joint[:, :4], torch.zeros((5, 4, 64), dtype=torch.bfloat16), torch.zeros(5, dtype=torch.int32)
    assert B._check_rope(ctx, 5, at, q, out, True) == 512
    assert B._check_rope(ctx, 5, at, None, None, True) == 0 and B._check_rope(ctx, 5, None, q, out, False) == 512
    for args in ((at.long(), q, out), (at[:4], q, out), (None, q, out), (torch.zeros(10, dtype=torch.int32)[::2], q, out), (at, q, None), (at, None, out), (at, q.float(), out),
                 (at, q[:4], out), (at, joint[:, ::2], out), (at, q.transpose(1, 2), out), (at, q, out.half()), (at, q, out[:4]), (at, q, joint[:, :4])):
        with pytest.raises(ValueError, match="lr_rope_write"):
            B._check_rope(ctx, 5, *args, True)


def test_a_closed_rope_does_not_leave_rows_as_they_are():
    cache = B.Fp4Cache.empty(Model(4, 2, 64, 8), 3, "cpu")
    ctx = SimpleNamespace(model=Model(4, 2, 64, 8), device=-1, cache_kind=cache.kind, handle=None)
    rows, slots, at = torch.zeros((2, 2, 64), dtype=torch.bfloat16), torch.arange(2), torch.zeros(2, dtype=torch.int32)
    rope = B.Rope(64)
    rope.close()
    with pytest.raises(ValueError, match="closed"):
        B.Context.lr_rope_write(ctx, rope, at, cache, rows, rows, slots)
