"""The 8-bit cache in the tests: the pools of a workload as the oracle stores them, on the device and as what they stand for."""
import numpy as np
import torch

from lr_workloads import bf16_round
from oracle import lr_oracle as O
from paper_2506_19830_b200 import binding as B


def u8(a, dev="cuda:0"):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.uint8)).to(dev)


def store_pools(k_bits, v_bits):
    """(k codes, v codes, k scales, v scales) of two bf16 pools [pages, heads, 16, head size]."""
    (kc, ks), (vc, vs) = O.fp8_store(k_bits), O.fp8_store(v_bits)
    return kc, vc, ks, vs


def poison_slack(batch, pools, rng):
    """Anything at all in the slots that no span of the batch uses: NaN codes and NaN scales among it."""
    used = np.zeros((batch.n_pool_pages, 16), dtype=bool)
    spans = list(zip(batch.span_slot, batch.span_len)) + list(zip(batch.br_own_slot, batch.br_own_len))
    for first, n in spans:
        for t in range(int(n)):
            used[batch.page_ids[int(first) + t // 16], t % 16] = True
    free = ~used
    kc, vc, ks, vs = pools
    for codes, scale in ((kc, ks), (vc, vs)):
        x = rng.integers(0, 256, codes.shape, dtype=np.uint8)
        x[rng.random(codes.shape) < 0.3] = 0x7F
        codes[:] = np.where(free[:, None, :, None], x, codes)
        y = rng.integers(0, 256, scale.shape, dtype=np.uint8)
        y[rng.random(scale.shape) < 0.3] = 255
        scale[:] = np.where(free[:, None, :], y, scale)
    return pools


def on_device(pools, dev="cuda:0"):
    kc, vc, ks, vs = pools
    return B.Fp8Cache(u8(kc, dev).view(torch.float8_e4m3fn), u8(vc, dev).view(torch.float8_e4m3fn), u8(ks, dev).view(torch.float8_e8m0fnu),
                      u8(vs, dev).view(torch.float8_e8m0fnu))


def back(cache):
    return [t.view(torch.uint8).cpu().numpy() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]


def as_bf16(codes, scale):
    """What stored rows stand for, as bf16 bits: exact for what the write leaves (NaN stays NaN)."""
    with np.errstate(over="ignore"):  # (poison beside the spans)
        return bf16_round(O.fp8_load(codes, scale).astype(np.float32))
