"""Acceptance at temperatures so low that a logit over the temperature passes what fp32 tells apart: the distributions are those of the definition, which
are all on the largest logits of a row."""
import numpy as np
import pytest
import torch

from lr_workloads import Model, bf16_round, bf16_to_f32
from oracle import lr_oracle as O
from paper_2506_19830_b200 import binding as B
from paper_2506_19830_b200 import runner as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
COLD = [1e-6, 1e-8, 3e-10, 1e-12, 1e-20, 1e-30, 1e-37, 2e-39]


def rows(rng, n, vocab, size):
    """Logits with the largest of a row there once, twice or three times, anywhere."""
    x = bf16_to_f32(bf16_round((size * rng.standard_normal((n, vocab))).astype(np.float32)))
    for i in range(n):
        top = x[i].max()
        for j in rng.choice(vocab, i % 3, replace=False):
            x[i, j] = top
    return bf16_round(x)


def f32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DEV)


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def padded(bits, vocab):
    stride = (vocab + 7) // 8 * 8
    t = torch.zeros((bits.shape[0], stride), dtype=torch.bfloat16, device=DEV)
    t[:, :vocab] = R.bf16_tensor(bits, DEV)
    return t[:, :vocab]


def draws(bits, temperature, u):
    """Where a uniform number falls among a row's largest logits, and its distance from the nearest border."""
    x = bf16_to_f32(bits).astype(np.float64)
    w = np.exp(np.maximum((x - x.max(axis=1, keepdims=True)) / temperature, -1e4))
    c = np.cumsum(w, axis=1)
    goal = u * c[:, -1]
    return np.array([int(np.argmax(c[i] > goal[i])) for i in range(len(u))]), np.array([np.abs(c[i] - goal[i]).min() for i in range(len(u))])


@pytest.mark.parametrize("size", [0.01, 30.0, -20000.0])
@pytest.mark.parametrize("vocab", [37, 5003, 70000])
@pytest.mark.parametrize("temperature", COLD)
def test_samples_of_rows_without_drafts(temperature, vocab, size):
    rng = np.random.default_rng(vocab)
    n = 9
    bits = rows(rng, n, vocab, abs(size))
    if size < 0:  # all of them far below 0
        bits = bf16_round(bf16_to_f32(bits) + np.float32(8 * size))
    u = rng.random(n).astype(np.float32)
    want, far = draws(bits, float(np.float32(temperature)), u.astype(np.float64))
    assert (far > 1e-4).all()
    ctx = B.Context(Model(4, 1, 64, vocab), 0)
    logits, cu, none = padded(bits, vocab), i32(np.zeros(n + 1)), i32(np.zeros(1))
    got = []
    for call in ("plain", "drafted", "filtered"):
        n_accept, final = (torch.full((n,), -1, dtype=torch.int32, device=DEV) for _ in range(2))
        u0, u1 = f32(np.zeros(1)), f32(u)
        if call == "plain":
            ctx.lr_accept_sample(logits, none, cu, temperature, u0, u1, n_accept, final, ctx.accept_sample_scratch(n))
        elif call == "filtered":
            ctx.lr_accept_sample_filtered(logits, none, cu, temperature, 0, 1.0, u0, u1, n_accept, final, ctx.accept_sample_filtered_scratch(n))
        else:
            ctx.lr_accept_sample_drafted(logits, logits[:0], none[:0], cu, temperature, 1.0, u0[:0], u1, n_accept, final, ctx.accept_sample_drafted_scratch(n))
        got.append((call, n_accept.cpu().numpy(), final.cpu().numpy()))
    ctx.close()
    for call, a, f in got:
        assert (a == 0).all() and np.array_equal(f, want), (call, f, want)


@pytest.mark.parametrize("temperature", COLD)
def test_drafts_against_a_drafter_that_is_cold_too(temperature):
    """The target's largest logit is where the drafter's is (the draft is taken), or it is not (it is refused and the target's comes)."""
    vocab, n_branch, L = 9001, 6, 4
    rng = np.random.default_rng(2)
    x = (12 * rng.standard_normal((n_branch * (L + 1), vocab))).astype(np.float32)
    y = (12 * rng.standard_normal((n_branch * L, vocab))).astype(np.float32)
    top, drafts, n_want, final_want = rng.integers(0, vocab, n_branch * (L + 1)), np.zeros(n_branch * L, np.int32), [], []
    for r in range(n_branch * (L + 1)):
        x[r, top[r]] = 100.0
    for b in range(n_branch):
        for i in range(L):
            right = top[b * (L + 1) + i]
            drafts[b * L + i] = right if i < b else (right + 1) % vocab
            y[b * L + i, drafts[b * L + i]] = 100.0
        n_want.append(min(b, L))
        final_want.append(int(top[b * (L + 1) + min(b, L)]))
    ctx = B.Context(Model(4, 1, 64, vocab), 0)
    lx, ly = padded(bf16_round(x), vocab), padded(bf16_round(y), vocab)
    n_accept, final = (torch.full((n_branch,), -1, dtype=torch.int32, device=DEV) for _ in range(2))
    p, q = (torch.full((n_branch * L,), -1.0, device=DEV) for _ in range(2))
    ctx.lr_accept_sample_drafted(lx, ly, i32(drafts), i32(np.arange(n_branch + 1) * L), temperature, temperature, f32(rng.random(n_branch * L)), f32(rng.random(n_branch)),
                                 n_accept, final, ctx.accept_sample_drafted_scratch(lx.shape[0]), p, q)
    got = n_accept.cpu().tolist(), final.cpu().tolist(), p.cpu().numpy(), q.cpu().numpy()
    ctx.close()
    assert got[0] == n_want and got[1] == final_want
    assert (got[3] == 1.0).all() and np.array_equal(got[2], (drafts == np.concatenate([top[b * (L + 1):b * (L + 1) + L] for b in range(n_branch)])).astype(np.float32))
