"""lr_accept_sample_drafted against the fp64 oracle.

The kernel computes probabilities in fp32, the oracle in 64 bits.  A probability: the exponential's argument is rounded once behind an exact
difference (24 bits, |argument| < 20 base 2 where it matters: 20 * 2^-24 * ln 2 = 8e-7), the exponential is off by 2^-22, the row's sum by
as much, and two products round: below 3e-6 in all.  So a walk may go either way where |u Q - P| < EPS (P + u Q), EPS = 1e-5, and the
final token where its target lies within EPS of the mass of P and Q that the cumulated weights are differences of.  Such branches are
counted (they must be rare) and the answer has to be one of the valid ones."""
import numpy as np
import pytest
import torch

from lr_workloads import Model, bf16_round
from oracle import lr_oracle as O
from paper_2506_19830_b200 import binding as B
from paper_2506_19830_b200 import runner as R

pytestmark = pytest.mark.gpu
DEV, EPS = "cuda:0", 1e-5


def _rows(bits, pad=8):
    n, vocab = bits.shape
    padded = np.full((max(1, n), (vocab + 7) // 8 * 8 + pad), 0x7F80, dtype=np.uint16)  # +inf behind the vocabulary: must be ignored
    padded[:n, :vocab] = bits
    return R.bf16_tensor(padded, DEV)[:n, :vocab]


def _t(a, dt):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dt)).to(DEV)


def _run(p_bits, q_bits, drafts, cu, T, Tq, ua, uf):
    ctx = B.Context(Model(1, 1, 64, p_bits.shape[1]), 0)
    nb, n = len(cu) - 1, len(drafts)
    fin, n_acc = torch.full((nb,), -7, dtype=torch.int32, device=DEV), torch.full((nb,), -7, dtype=torch.int32, device=DEV)
    pd, qd = torch.full((n + 1,), -1.0, device=DEV), torch.full((n + 1,), -1.0, device=DEV)
    scratch = ctx.accept_sample_drafted_scratch(len(p_bits))
    first = None
    for _ in range(2):  # twice on the same scratch: the same answer
        ctx.lr_accept_sample_drafted(_rows(p_bits), _rows(q_bits), _t(drafts, np.int32), _t(cu, np.int32), T, Tq, _t(ua, np.float32), _t(uf, np.float32),
                                     n_acc, fin, scratch, pd, qd)
        got = [t.cpu().numpy() for t in (n_acc, fin, pd, qd)]
        assert first is None or all(np.array_equal(a, b, equal_nan=True) for a, b in zip(first, got))
        first = got
    assert got[2][n] == -1 and got[3][n] == -1
    ctx.close()
    return got[0], got[1], got[2][:n], got[3][:n]


def _check(p_bits, q_bits, drafts, cu, T, Tq, ua, uf, most_unsure=1):
    got_n, got_f, got_p, got_q = _run(p_bits, q_bits, drafts, cu, T, Tq, ua, uf)
    T, Tq = float(np.float32(T)), float(np.float32(Tq))
    ua, uf = np.asarray(ua, dtype=np.float32).astype(np.float64), np.asarray(uf, dtype=np.float32).astype(np.float64)
    n_ref, f_ref, p_ref, q_ref = O.accept_sample_drafted(p_bits, q_bits, drafts, cu, T, Tq, ua, uf)
    for got, ref in ((got_p, p_ref), (got_q, q_ref)):
        # (far below the largest, the argument is larger: 2^-24 ln 2 of it, twice)
        far = -np.log2(np.maximum(ref, 1e-300))
        assert (np.abs(got - ref) <= ref * (3e-6 + far * 2.0 ** -23) + 1e-37).all()
    unsure = 0
    V = p_bits.shape[1]
    for b in range(len(cu) - 1):
        d0, L = int(cu[b]), int(cu[b + 1] - cu[b])
        n = int(got_n[b])
        assert 0 <= n <= L
        if n != n_ref[b]:
            i = d0 + min(n, int(n_ref[b]))
            assert abs(ua[i] * q_ref[i] - p_ref[i]) <= EPS * (p_ref[i] + ua[i] * q_ref[i]), b
            unsure += 1
            continue
        if got_f[b] == f_ref[b]:
            continue
        P = O.target_probs(p_bits[d0 + b + n], T)
        Q = O.target_probs(q_bits[d0 + n], Tq) if n < L else np.zeros(V)
        w = np.maximum(P - Q, 0.0)
        c, f = np.cumsum(w), int(got_f[b])
        assert 0 <= f < V
        slack = EPS * ((P + Q) * (w > 0)).sum()
        assert c[f] - w[f] - slack <= uf[b] * c[-1] <= c[f] + slack, (b, f, int(f_ref[b]))
        unsure += 1
    assert unsure <= most_unsure, unsure
    return got_n, got_f


def _models(rng, n_rows, cu, V, spread=3.0, noise=0.6):
    """Peaked target rows, draft rows near them, drafts sampled from those."""
    p = rng.standard_normal((n_rows, V)) * spread
    at = np.array([i + b for b in range(len(cu) - 1) for i in range(cu[b], cu[b + 1])], dtype=np.int64)
    q_bits = bf16_round((p[at] + noise * rng.standard_normal((len(at), V))).astype(np.float32))
    drafts = np.array([O.sample_inverse_cdf(O.target_probs(r, 1.0), rng.random()) for r in q_bits], dtype=np.int32)
    return bf16_round(p.astype(np.float32)), q_bits, drafts


@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 255, 256, 2047, 2048, 2049, 5003, 40001, 152064])
@pytest.mark.parametrize("T,Tq", [(1.0, 1.0), (0.6, 0.9)])
def test_ragged_branches(V, T, Tq):
    rng = np.random.default_rng(V)
    lens = [3, 0, 1, 9] if V > 10000 else [0, 1, 5, 40, 0, 70, 2]  # more rows than a cluster has warps
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    p, q, drafts = _models(rng, int(cu[-1]) + len(lens), cu, V)
    for u_low in (0.0, 1.0):
        ua = rng.random(len(drafts)) * rng.choice([1.0, u_low], len(drafts))
        _check(p, q, drafts, cu, T, Tq, ua, rng.random(len(lens)))
    ua = np.zeros(len(drafts))  # everything that the target can say is accepted
    n, _ = _check(p, q, drafts, cu, T, Tq, ua, rng.random(len(lens)))
    assert np.array_equal(n, lens)


@pytest.mark.parametrize("n_branch,most", [(2, 70), (40, 6), (40, 20)])
def test_few_and_many_branches_of_short_and_of_long_drafts(n_branch, most):
    """An SM for each CTA or several CTAs to one; rows for every CTA alone or for the cluster's warps in turn."""
    rng = np.random.default_rng(n_branch + most)
    V = 1027
    lengths = rng.integers(most // 2, most + 1, n_branch)
    lengths[0], lengths[1] = most, 0
    cu = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    p, q, d = _models(rng, int(cu[-1]) + n_branch, cu, V, noise=0.1)
    n, _ = _check(p, q, d, cu, 0.8, 0.8, rng.random(int(cu[-1])) * 0.9, rng.random(n_branch), most_unsure=2)
    assert n.max() > most // 3


def test_no_drafts_at_all_and_one_branch():
    rng = np.random.default_rng(1)
    p, q, _ = _models(rng, 3, np.zeros(4, dtype=np.int32), 500)
    n, _ = _check(p, q, np.zeros(0, np.int32), np.zeros(4, np.int32), 1.0, 1.0, [], [0.0, 0.5, 0.999])
    assert (n == 0).all()
    p, q, d = _models(rng, 2, np.array([0, 1], dtype=np.int32), 33)
    _check(p, q, d, np.array([0, 1], dtype=np.int32), 1.0, 1.0, [0.3], [0.25])


def test_the_drafters_own_row_leaves_nothing_and_the_target_is_drawn_from():
    # a draft is refused there by rounding alone; a uniform beyond 1 stands for that, and P - Q is 0 everywhere
    rng = np.random.default_rng(2)
    p, _, d = _models(rng, 2, np.array([0, 1], dtype=np.int32), 900)
    n, f, pd, qd = _run(p, p[:1], d, np.array([0, 1], dtype=np.int32), 0.7, 0.7, [1.5], [0.4])
    assert n[0] == 0 and np.array_equal(pd, qd)
    P = O.target_probs(p[0], float(np.float32(0.7)))
    c = np.cumsum(P)
    assert c[f[0]] - P[f[0]] - EPS <= np.float32(0.4) <= c[f[0]] + EPS


def test_special_values_and_drafts_outside_the_vocabulary():
    rng = np.random.default_rng(3)
    V, L = 3001, 6
    cu = np.array([0, L, 2 * L, 3 * L], dtype=np.int32)
    p, q, d = _models(rng, 3 * L + 3, cu, V)
    p[:, 100:300], q[:, 200:500] = 0xFF80, 0xFF80
    p[:, 700:720], q[:, 710:740] = 0x7FC0, 0xFFC0  # NaN counts as -inf
    d[0], d[1] = V, -1
    d[L], d[L + 1] = 450, 250  # Q = 0 < P: accepted whatever u is; both 0: refused
    d[2 * L] = 17
    ua = np.full(3 * L, 0.2)
    ua[L] = 0.999
    n, f = _check(p, q, d, cu, 1.0, 1.0, ua, [0.1, 0.6, 0.9])
    assert n[0] == 0 and n[1] == 1
    # a drafter's row of -inf: Q is 0, the draft is accepted if the target can say it; a target's: some token of the vocabulary
    q[2 * L] = 0xFF80
    p[0] = 0xFF80
    n, f, pd, qd = _run(p, q, d, cu, 1.0, 1.0, ua, [0.1, 0.6, 0.9])
    assert n[0] == 0 and 0 <= f[0] < V and n[2] >= 1 and qd[2 * L] == 0 and not np.isnan(pd).any() and not np.isnan(qd).any()


@pytest.mark.parametrize("T", [0.05, 0.6])
@pytest.mark.parametrize("offset", [0.0, 100.0, -1000.0])
def test_large_logits_over_small_temperatures(T, offset):
    rng = np.random.default_rng(int(offset) + 2000)
    V, L = 4003, 3
    cu = (np.arange(9) * L).astype(np.int32)
    x = np.full((8 * (L + 1), V), -64.0)
    lead = rng.integers(0, V // 8, len(x))
    for r in range(len(x)):
        x[r, lead[r] + V // 8 * np.arange(8)] = 24.0 - T * rng.uniform(0, 6, 8)
    at = np.array([b * (L + 1) + i for b in range(8) for i in range(L)])
    y = x[at].copy()
    for r in range(len(y)):
        y[r, lead[at[r]] + V // 8 * np.arange(8)] = 24.0 - T * rng.uniform(0, 6, 8)
    _check(bf16_round((x + offset).astype(np.float32)), bf16_round((y + offset).astype(np.float32)), lead[at].astype(np.int32), cu, T, T, rng.random(8 * L),
           rng.random(8))


def test_final_tokens_over_the_whole_range_of_the_uniform():
    """Flat rows: every token is a candidate, the draws land in all steps and CTAs."""
    rng = np.random.default_rng(5)
    V, nb = 70001, 64
    cu = np.arange(nb + 1, dtype=np.int32)
    p = bf16_round(rng.standard_normal((1, V)).astype(np.float32) * 0.3)
    q = bf16_round(rng.standard_normal((1, V)).astype(np.float32) * 0.3)
    p_all, q_all = np.repeat(p, 2 * nb, axis=0), np.repeat(q, nb, axis=0)
    uf = (np.arange(nb) + rng.random(nb)) / nb
    uf[0], uf[-1] = 0.0, np.float32(1.0 - 2.0 ** -24)
    drafts = np.full(nb, int(np.argmax(O.target_probs(q[0], 1.0) - O.target_probs(p[0], 1.0))))
    n, f = _check(p_all, q_all, drafts, cu, 1.0, 1.0, np.full(nb, 0.9999), uf, most_unsure=nb)
    assert (n == 0).all() and (np.diff(f) >= 0).all()


def test_a_vocabulary_beyond_the_sums_of_a_step_each():
    V = 256 * 8 * 4096 + 1003  # a step is 512 tokens there
    rng = np.random.default_rng(6)
    p, q = (bf16_round(rng.standard_normal((n, V)).astype(np.float32) * 3) for n in (2, 1))
    d = np.array([int(np.argmax(q[0].astype(np.int16)))])
    _check(p, q, d, np.array([0, 1], dtype=np.int32), 1.0, 1.0, [0.97], [0.83])
    _check(p, q, d, np.array([0, 1], dtype=np.int32), 1.0, 1.0, [0.0], [0.31])


def test_on_another_stream_two_at_once_and_replayed():
    rng = np.random.default_rng(7)
    cu = np.array([0, 4, 9], dtype=np.int32)
    data = [_models(rng, 11, cu, 6007) for _ in range(2)]
    us = [(rng.random(9), rng.random(2)) for _ in range(2)]
    want = [_run(p, q, d, cu, 1.0, 1.0, ua, uf) for (p, q, d), (ua, uf) in zip(data, us)]
    ctx = B.Context(Model(1, 1, 64, 6007), 0)
    streams, calls = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for (p, q, d), (ua, uf) in zip(data, us):
        outs = [torch.zeros(2, dtype=torch.int32, device=DEV) for _ in range(2)] + [torch.zeros(9, device=DEV) for _ in range(2)]
        calls.append((_rows(p), _rows(q), _t(d, np.int32), _t(cu, np.int32), 1.0, 1.0, _t(ua, np.float32), _t(uf, np.float32), outs[0], outs[1],
                      ctx.accept_sample_drafted_scratch(11), outs[2], outs[3]))
    torch.cuda.synchronize()
    for _ in range(3):
        for s, c in zip(streams, calls):
            ctx.lr_accept_sample_drafted(*c, stream=s)
    torch.cuda.synchronize()
    results = lambda c: [c[i].cpu().numpy() for i in (8, 9, 11, 12)]  # noqa: E731
    for c, w in zip(calls, want):
        assert all(np.array_equal(a, b) for a, b in zip(results(c), w))
    graph, other = torch.cuda.CUDAGraph(), calls[1]
    with torch.cuda.graph(graph):
        ctx.lr_accept_sample_drafted(*other)
    for i in (0, 1, 2, 6, 7):  # the first call's inputs in the second one's buffers
        other[i].copy_(calls[0][i])
    graph.replay()
    torch.cuda.synchronize()
    assert all(np.array_equal(a, b) for a, b in zip(results(other), want[0]))
    ctx.close()


def test_refusals():
    ctx = B.Context(Model(1, 1, 64, 100), 0)
    z = torch.zeros(4096, dtype=torch.int64, device=DEV).data_ptr()
    good = [ctx.handle, z, 104, z, 104, z, z, 1, 3, 1.0, 1.0, z, z, z, z, None, None, z, None]
    for at, bad, code in ((1, None, -1), (1, z + 8, -1), (2, 96, -1), (2, 108, -1), (3, None, -1), (3, z + 2, -1), (4, 96, -1), (4, 101, -1), (5, None, -1), (6, None, -1),
                          (7, 4, -1), (7, -1, -1), (8, 0, -1), (9, 0.0, -1), (9, float("nan"), -1), (9, float("inf"), -1), (10, -1.0, -1), (11, None, -1), (12, None, -1),
                          (13, None, -1), (14, None, -1), (17, None, -1), (17, z + 4, -1), (8, 65536, -2)):
        args = list(good)
        args[at] = bad
        assert B.lib().lr_accept_sample_drafted(*args) == code, (at, bad)
    none = list(good)
    none[7], none[8] = 0, 0
    assert B.lib().lr_accept_sample_drafted(*none) == 0
    assert ctx.launch_count == 0
    ctx.close()
