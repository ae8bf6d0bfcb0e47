"""The 4-bit cache in the tests: the pools of a workload as the oracle stores them, on the device and as what they stand for."""
import numpy as np
import torch

from fp8_util import u8
from lr_workloads import bf16_round
from oracle import lr_oracle as O
from paper_2506_19830_b200 import binding as B


def store_pools(k_bits, v_bits):
    """(k codes, v codes, k scales, v scales) of two bf16 pools [pages, heads, 16, head size]."""
    (kc, ks), (vc, vs) = O.fp4_store(k_bits), O.fp4_store(v_bits)
    return kc, vc, ks, vs


def poison_slack(batch, pools, rng):
    """Anything at all in the slots that no span of the batch uses: scales of NaN among it."""
    used = np.zeros((batch.n_pool_pages, 16), dtype=bool)
    for first, n in list(zip(batch.span_slot, batch.span_len)) + list(zip(batch.br_own_slot, batch.br_own_len)):
        for t in range(int(n)):
            used[batch.page_ids[int(first) + t // 16], t % 16] = True
    free = ~used[:, None, :, None]
    for i, pool in enumerate(pools):
        x = rng.integers(0, 256, pool.shape, dtype=np.uint8)
        if i >= 2:
            x[rng.random(pool.shape) < 0.3] = 255
        pool[:] = np.where(free, x, pool)
    return pools


def on_device(pools, dev="cuda:0"):
    kc, vc, ks, vs = (u8(p, dev) for p in pools)
    return B.Fp4Cache(kc, vc, ks.view(torch.float8_e8m0fnu), vs.view(torch.float8_e8m0fnu))


def back(cache):
    return [t.view(torch.uint8).cpu().numpy() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]


def as_bf16(codes, scale):
    """What stored rows stand for, as bf16 bits: exact for what the write leaves (NaN stays NaN)."""
    with np.errstate(over="ignore", invalid="ignore"):  # (poison beside the spans)
        return bf16_round(O.fp4_load(codes, scale).astype(np.float32))
