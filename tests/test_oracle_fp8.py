"""Pins for the oracle's 8-bit cache, and the refusals of its entry points that need no device."""
import ctypes as C

import numpy as np
import pytest
import torch

from fp8_util import as_bf16
from lr_workloads import bf16_round, bf16_to_f32
from oracle import lr_oracle as O
from paper_2506_19830_b200 import binding as B
from paper_2506_19830_b200.build import build_library


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()


def test_the_code_table_is_torchs():
    got = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(got, O.e4m3_values(), equal_nan=True)


def test_codes_are_torchs_rounding_of_the_scaled_row():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((64, 5, 128)) * np.exp(rng.uniform(-80, 80, (64, 5, 1)))
    bits = bf16_round(x.astype(np.float32))
    codes, byte = O.fp8_store(bits)
    y = torch.from_numpy(bf16_to_f32(bits).astype(np.float64) * np.exp2(127.0 - byte.astype(np.float64))[..., None])
    assert np.array_equal(y.float().to(torch.float8_e4m3fn).view(torch.uint8).numpy(), codes)


def test_scales_are_the_smallest_that_hold_the_row():
    rng = np.random.default_rng(1)
    top = np.concatenate([np.ldexp(1.0 + np.arange(0, 128, 3) / 128.0, rng.integers(-120, 127, 43)), [448.0, 450.0, 1.75, 1.7578125, 0.0]])
    rows = np.zeros((len(top), 64))
    rows[:, 7] = -top
    codes, byte = O.fp8_store(bf16_round(rows.astype(np.float32)))
    scale = np.exp2(byte.astype(np.float64) - 127)
    assert (top <= 448 * scale).all()
    assert ((top > 224 * scale) | (byte == 3)).all()


def test_a_value_is_off_by_half_a_step_and_needs_no_second_rounding():
    rng = np.random.default_rng(2)
    x = bf16_round((rng.standard_normal((300, 128)) * np.exp(rng.uniform(-60, 60, (300, 1)))).astype(np.float32))
    codes, byte = O.fp8_store(x)
    v, want = O.fp8_load(codes, byte), bf16_to_f32(x).astype(np.float64)
    scale = np.exp2(byte.astype(np.float64) - 127)[:, None]
    # normal codes: half a step is 2^-4 of the value; below 2^-6 of the scale: half of 2^-9
    assert (np.abs(v - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * scale)).all()
    assert np.array_equal(bf16_to_f32(as_bf16(codes, byte)).astype(np.float64), v)


def test_rows_that_are_not_finite_and_the_ends_of_the_range():
    bits = bf16_round(np.random.default_rng(3).standard_normal((6, 64)).astype(np.float32))
    bits[0, 3], bits[1, 9], bits[2, 0] = 0x7FC0, 0x7F80, 0xFF80
    bits[3] = 0x0001  # the smallest number there is
    bits[4] = 0x7F7F  # the largest
    bits[5] = 0x8000
    codes, byte = O.fp8_store(bits)
    assert (byte[:3] == 255).all() and not codes[:3].any()
    assert np.isnan(O.fp8_load(codes, byte)[:3]).all()
    assert byte[3] == 3 and (O.fp8_load(codes, byte)[3] == 2.0 ** -133).all()
    assert byte[4] == 127 + 120 and (O.fp8_load(codes, byte)[4] == 2.0 ** 128).all() and (codes[4] == 0x78).all()
    assert (codes[5] == 0x80).all()


def test_drafted_acceptance_is_exact_sampling():
    """Integrating over both uniforms, the emitted token is distributed as the target, whatever the draft model is."""
    rng = np.random.default_rng(4)
    V, n = 5, 400
    target, drafter = bf16_round(rng.standard_normal((2, V)).astype(np.float32)), bf16_round(rng.standard_normal((1, V)).astype(np.float32) * 2)
    P, Q = O.target_probs(target[0], 0.8), O.target_probs(drafter[0], 1.1)
    u = (np.arange(n) + 0.5) / n
    got = np.zeros(V)
    for d in range(V):  # the drafted token, with probability Q(d)
        accepted = np.array([O.accept_sample_drafted(target, drafter, [d], [0, 1], 0.8, 1.1, [x], [0.5])[0][0] for x in u])
        got[d] += Q[d] * accepted.mean()
        if accepted.mean() < 1:
            first = [O.accept_sample_drafted(target, drafter, [d], [0, 1], 0.8, 1.1, [0.999999], [x])[1][0] for x in u]
            got += Q[d] * (1 - accepted.mean()) * np.bincount(first, minlength=V) / n
    assert np.abs(got - P).max() <= V * 2.0 / n  # a grid of n points misplaces a border by 1/n at most, in each of the V terms twice


def test_drafted_acceptance_with_the_targets_own_drafts_and_with_none():
    rng = np.random.default_rng(5)
    rows = bf16_round(rng.standard_normal((4, 50)).astype(np.float32))
    drafts = [3, 49, 7]
    n, f, p, q = O.accept_sample_drafted(rows, rows[:3], drafts, [0, 3], 1.0, 1.0, [0.9, 0.99, 0.999], [0.3])
    assert n[0] == 3 and np.array_equal(p, q) and f[0] == O.sample_inverse_cdf(O.target_probs(rows[3], 1.0), 0.3)
    n, f, p, q = O.accept_sample_drafted(rows[:2], rows[:0], [], [0, 0, 0], 1.0, 1.0, [], [0.3, 0.7])
    assert (n == 0).all() and f[1] == O.sample_inverse_cdf(O.target_probs(rows[1], 1.0), 0.7)


# ---- refusals -------------------------------------------------------------------------------------------------------------
def _cache(**kw):
    return B.lr_fp8_cache(**dict(dict(k_d=1 << 20, v_d=2 << 20, k_scale_d=3 << 20, v_scale_d=4 << 20, n_pages=8), **kw))


@pytest.mark.parametrize("bad,words", [
    (dict(k_d=None), "null"), (dict(v_d=None), "null"), (dict(k_scale_d=None), "null"), (dict(v_scale_d=None), "null"),
    (dict(k_d=(1 << 20) + 8), "aligned"), (dict(v_scale_d=(4 << 20) + 4), "aligned"), (dict(n_pages=0), "page"), (dict(n_pages=-3), "page"),
    (dict(n_pages=1 << 50), "pages"), (dict(v_d=1 << 20), "share"), (dict(v_scale_d=3 << 20), "share"),
])
def test_a_cache_that_cannot_be_one_is_refused(bad, words):
    L, c = B.lib(), _cache(**bad)
    calls = [lambda: L.lr_fp8_write(None, C.addressof(c), 16, 8, 16, 8, 8, 1, None, None), lambda: L.lr_fp8_read(None, C.addressof(c), 8, 1, 16, 8, 16, 8, None, None),
             lambda: L.lr_verify_attention_fp8(None, 16, C.addressof(c), 16, None, 0.0, None), lambda: L.lr_compact_fp8(None, 4, 4, 4, C.addressof(c), 4, 4, None)]
    for call in calls:
        assert call() == -1
        assert words in L.lr_last_error().decode()


def test_null_handles_are_refused():
    L, c = B.lib(), _cache()
    at = C.addressof(c)
    for null_cache in (None, at):
        assert L.lr_fp8_write(None, null_cache, 16, 8, 16, 8, 8, 1, None, None) == -1
        assert L.lr_fp8_read(None, null_cache, 8, 1, 16, 8, 16, 8, None, None) == -1
        assert L.lr_verify_attention_fp8(None, 16, null_cache, 16, None, 0.0, None) == -1
        assert L.lr_compact_fp8(None, 4, 4, 4, null_cache, 4, 4, None) == -1


def test_tensors_that_are_no_cache_are_refused():
    codes, scale = torch.zeros((3, 2, 16, 64), dtype=torch.uint8), torch.zeros((3, 2, 16), dtype=torch.uint8)
    B.Fp8Cache(codes, codes.clone(), scale, scale.clone())
    B.Fp8Cache(codes.view(torch.float8_e4m3fn), codes, scale.view(torch.float8_e8m0fnu), scale)
    for args in ((codes, codes[:2], scale, scale), (codes, codes, scale[:, :1], scale), (codes[..., :32], codes[..., :32], scale, scale),
                 (codes.float(), codes, scale, scale), (codes, codes, scale, codes), (codes[:, :, :8], codes[:, :, :8], scale[:, :, :8], scale[:, :, :8]),
                 (codes.transpose(0, 1), codes.transpose(0, 1), scale.transpose(0, 1), scale.transpose(0, 1))):
        with pytest.raises(ValueError):
            B.Fp8Cache(*args)


def test_drafted_acceptance_is_refused_without_a_device():
    L = B.lib()
    good = [None, 16, 104, 16, 104, 16, 16, 1, 3, 1.0, 1.0, 16, 16, 16, 16, None, None, 16, None]
    for at, bad in ((9, 0.0), (9, float("nan")), (10, -1.0), (10, float("inf")), (7, -1), (7, 4), (1, None)):
        args = list(good)
        args[at] = bad
        assert L.lr_accept_sample_drafted(*args) == -1
    assert L.lr_accept_sample_drafted(*good) == -1 and "null" in L.lr_last_error().decode()
