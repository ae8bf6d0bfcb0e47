"""Attention over the 8-bit cache against the fp64 oracle, which is given the bf16 pools that the stored rows stand for (they stand for
bf16 numbers exactly, so both see the same keys and values)."""
import numpy as np
import pytest
import torch

from fp8_util import as_bf16, on_device, poison_slack, store_pools
from gpu_util import REL_LARGE, check_attention
from lr_workloads import Model, make_config, make_random_mid, make_random_small, make_random_tree, make_tree
from lr_workloads.gen import _finish
from oracle import lr_oracle as O
from paper_2506_19830_b200 import binding as B
from paper_2506_19830_b200 import runner as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PATHS = [B.PATH_GENERIC, B.PATH_TENSOR_CORE]


def stored(w, seed=0):
    """The workload's pools in 8 bits, anything in unused slots, and the bf16 pools they stand for."""
    pools = poison_slack(w.batch, store_pools(w.tensors.k_pool, w.tensors.v_pool), np.random.default_rng(seed))
    return pools, as_bf16(pools[0], pools[2]), as_bf16(pools[1], pools[3])


def run(w, pools, path, scale=0.0, lse=True, stream=None):
    b = w.batch
    ctx = B.Context(b.model, 0)
    plan = B.Plan(ctx, b)
    plan.lr_plan_set_attention_path(path)
    q, cache = R.bf16_tensor(w.tensors.q, DEV), on_device(pools)
    n, guard = q.numel(), 4096
    buf = torch.full((n + 2 * guard,), -7.0, dtype=torch.bfloat16, device=DEV)
    out = buf[guard:guard + n].view(q.shape)
    l = torch.full(q.shape[:2], -7.0, device=DEV) if lse else None
    plan.lr_verify_attention_fp8(q, cache, out, l, scale, stream)
    assert plan.lr_poll_status(stream) == 0
    assert bool((buf[:guard] == -7.0).all()) and bool((buf[guard + n:] == -7.0).all())
    plan.close()
    ctx.close()
    return out, l


def check(w, path, rel_large=0.0, scale=0.0, branches=None):
    pools, k, v = stored(w)
    out, lse = run(w, pools, path, scale)
    o_ref, l_ref = O.verify_attention(w.batch, w.tensors.q, k, v, scale if scale > 0 else None, branches=branches)
    rows = None if branches is None else np.concatenate([np.arange(w.batch.cu_q[i], w.batch.cu_q[i + 1]) for i in branches])
    return check_attention(out, lse, o_ref, l_ref, rows, rel_large)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("cfg", [1, 2])
def test_configurations(cfg, path):
    check(make_config(cfg, with_logits=False), path)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("seed", range(10))
def test_ragged_small(seed, path):
    check(make_random_small(9000 + seed), path, REL_LARGE)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("seed", range(6))
def test_irregular_trees(seed, path):
    check(make_random_tree(9100 + seed), path, REL_LARGE)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("prefix,q", [(0, 1), (1, 1), (15, 1), (16, 1), (127, 1), (128, 1), (129, 2), (700, 1)])
def test_single_tokens(d, prefix, q, path):
    rng = np.random.default_rng(prefix + d)
    w = _finish("token", 11, Model(10, 2, d, 16), [{"P": prefix, "segs": [], "branches": [(0, q, q, q)]} for _ in range(3)], rng, 0.3, 0.6, False, True, "nan")
    check(w, path, REL_LARGE)


@pytest.mark.parametrize("cfg,branches", [(3, [0, 5, 15]), (4, [0, 5]), (5, [0, 20, 40])])
def test_large_configurations_on_the_tensor_cores(cfg, branches):
    """Two M-tiles a piece, several pieces a CTA, results merged from many."""
    w = make_config(cfg, with_logits=False)
    check(w, B.PATH_TENSOR_CORE, branches=[b for b in branches if b < w.batch.n_branch])


@pytest.mark.parametrize("seed", range(12))
def test_both_sides_of_the_grouping_switch(seed):
    check(make_random_mid(seed), B.PATH_TENSOR_CORE, REL_LARGE)


@pytest.mark.parametrize("W,size", [(2, "tiny"), (3, "tiny"), (2, "layer")])
def test_full_trees(W, size):
    check(make_tree(W, 2, size=size, with_logits=False), B.PATH_TENSOR_CORE, REL_LARGE)
