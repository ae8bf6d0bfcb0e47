"""Sines and cosines of rotary positions as the pairs (1, 0) and (0, 1) give them, which nothing but the last rounding touches."""
import numpy as np
import pytest
import torch

from lr_workloads import Model, bf16_to_f32
from oracle import lr_oracle as O
from paper_2506_19830_b200 import binding as B
from paper_2506_19830_b200 import runner as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# Of a number of 1 at the most: its rounding to fp32 (half a step, 2^-25), the series' end (x^12 / 12! < 2^-32 for x <= pi / 4), and the angle's own roundings here and there
# (of 10^6 radians at the most, three of 2^-53: below 2^-31).
SLACK = 2.0 ** -25 + 2.0 ** -32 + 2.0 ** -31


@pytest.mark.parametrize("interleaved,rot", [(False, 128), (True, 128), (False, 90)])
@pytest.mark.parametrize("second", [0, 1])
def test_sines_and_cosines_are_rounded_once(second, interleaved, rot):
    n, h, d = 32768, 2, 128
    rng = np.random.default_rng(rot + second)
    at = rng.integers(0, 1000000, n).astype(np.int32)
    first = np.arange(0, rot, 2) if interleaved else np.arange(rot // 2)
    other = first + 1 if interleaved else first + rot // 2
    x = torch.zeros((n, h, d), dtype=torch.bfloat16, device=DEV)
    x[..., torch.from_numpy(other if second else first).to(DEV)] = 1.0
    ctx = B.Context(Model(h, h, d, 8), 0)
    cache = B.Bf16Cache(*torch.zeros((2, n // 16, h, 16, d), dtype=torch.bfloat16, device=DEV))
    out = torch.zeros_like(x)
    ctx.lr_rope_write(B.Rope(rot, base=1e4, interleaved=interleaved), torch.from_numpy(at).to(DEV), cache, x, x, torch.arange(n, device=DEV), x, out)
    angle = at[:, None].astype(np.float64) * O.rope_frequencies(rot, 1e4)[0]
    want = np.zeros((n, d))
    want[:, first], want[:, other] = (-np.sin(angle), np.cos(angle)) if second else (np.cos(angle), np.sin(angle))
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(want), 2.0 ** -126))) - 7)
    for got in (R.bf16_bits(out), R.bf16_bits(cache.k.transpose(1, 2).reshape(n, h, d))):
        assert (np.abs(bf16_to_f32(got).astype(np.float64) - want[:, None]) <= (step / 2 + SLACK)[:, None]).all()
    ctx.close()
