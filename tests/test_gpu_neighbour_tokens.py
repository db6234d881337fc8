"""Search results as token distributions, against a plain computation in 64 bits.

Tolerance.  e = 2^-24: t = (d_min - d) / T is off by 3 e |t|, a weight by 4 e of itself more, and a sum of up to k of them by k e;
a log-probability is the difference of two logarithms of such sums: e (2 k + 16 + 4 |log-probability| + 8 |t|)."""
import math

import numpy as np
import pytest
import torch

import synth_inputs as si

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


@pytest.fixture(scope="module")
def P():
    import paper_2301_06672_amd as pkg
    pkg.lib()
    return pkg


def reference(ids, dists, table, temperature):
    nq, k = ids.shape
    tokens, logprobs = np.full((nq, k), -1, np.int32), np.full((nq, k), -np.inf)
    for q in range(nq):
        groups = {}
        for i, d in zip(ids[q].tolist(), dists[q].astype(np.float64).tolist()):
            if 0 <= i < len(table) and math.isfinite(d) and table[i] >= 0:
                groups.setdefault(int(table[i]), []).append(-d / temperature)
        if not groups:
            continue
        most = max(max(v) for v in groups.values())
        total = math.fsum(math.exp(x - most) for v in groups.values() for x in v)
        for at, (token, v) in enumerate(groups.items()):
            high = max(v)
            tokens[q, at] = token
            logprobs[q, at] = high - most + math.log(math.fsum(math.exp(x - high) for x in v)) - math.log(total)
    return tokens, logprobs


def check(P, ids, dists, table, temperature):
    got_tokens, got = P.ivfpq_neighbour_tokens(torch.from_numpy(ids).cuda(), torch.from_numpy(dists).cuda(), torch.from_numpy(table).cuda(), temperature)
    tokens, want = reference(ids, dists, table, temperature)
    np.testing.assert_array_equal(got_tokens.cpu().numpy(), tokens)
    got = got.cpu().double().numpy()
    there = tokens >= 0
    assert np.all(got[~there] == -np.inf)
    k = ids.shape[1]
    t = 0.0
    if there.any():
        usable = dists[np.isfinite(dists)].astype(np.float64)
        t = (usable.max() - usable.min()) / temperature
    tol = E * (2 * k + 16 + 4 * np.abs(want[there]) + 8 * min(t, 1e4))
    assert np.all(np.abs(got[there] - want[there]) <= tol)


@pytest.mark.parametrize("k", [1, 2, 10, 63, 64, 65, 100, 128, 129, 256, 257, 700, 1024])
@pytest.mark.parametrize("vocab", [3, 400, 100000])
def test_against_the_definition(P, k, vocab):
    rng = np.random.default_rng(k * vocab)
    nq, n_ids = 9, 5000
    table = rng.integers(0, vocab, n_ids).astype(np.int32)
    table[::50] = -1
    ids = rng.integers(0, n_ids, (nq, k))
    dists = np.cumsum(rng.random((nq, k), np.float32) * 20, axis=1, dtype=np.float32) + 1000
    ids[1, k // 2:], dists[1, k // 2:] = -1, np.inf          # as a search pads short rows
    ids[2] = -1
    ids[3, ::3] = n_ids + 5
    dists[4, k // 3] = np.nan
    dists[5] = dists[5, ::-1]                                # not in ascending order
    dists[6] = dists[6, 0]
    check(P, ids, dists, table, 30.0)
    check(P, ids, dists, table, 1e4)


def test_far_neighbours_keep_their_log_probabilities(P):
    ids = np.arange(6)[None].repeat(2, 0)
    table = np.array([0, 1, 1, 2, 0, 1], np.int32)
    dists = np.array([[0, 500, 501, 90, 3, 700], [5, 3000, 3001, 2000, 2500, 1e30]], np.float32)
    check(P, ids, dists, table, 1.0)
    tokens, logprobs = P.ivfpq_neighbour_tokens(torch.from_numpy(ids).cuda(), torch.tensor([[0.0, 3e38, 3e38, 1, 1, 1]] * 2, device="cuda"),
                                                torch.from_numpy(table).cuda(), 1e-3)
    assert not torch.isnan(logprobs).any()


def test_no_queries_and_no_table(P):
    empty = P.ivfpq_neighbour_tokens(torch.empty((0, 4), dtype=torch.int64, device="cuda"), torch.empty((0, 4), device="cuda"),
                                     torch.zeros(3, dtype=torch.int32, device="cuda"), 1.0)
    assert empty[0].shape == (0, 4)
    tokens, logprobs = P.ivfpq_neighbour_tokens(torch.zeros((2, 4), dtype=torch.int64, device="cuda"), torch.zeros((2, 4), device="cuda"),
                                                torch.empty(0, dtype=torch.int32, device="cuda"), 1.0)
    assert (tokens == -1).all() and torch.isinf(logprobs).all()


def test_on_search_results(P):
    w = si.WORKLOADS["tiny"].with_(n=3000, n_lists=16)
    data, queries = si.dataset(w), si.queries(w, 40)
    index = P.Index.ivfpq_build_device(data, w.n_lists, w.pq_dim, w.pq_bits, 4, seed=3).ivfpq_upload()
    ids, dists = index.ivfpq_search(queries, 4, 32, P.LUT_FP32)
    table = np.random.default_rng(0).integers(0, 50, 3000).astype(np.int32)
    check(P, ids.cpu().numpy(), dists.cpu().numpy(), table, 0.05)
    index.ivfpq_free()
