"""The router at far logits, and the sizes that send it through every kernel
and past the first pass of its loops, against the fp64 oracle.

Bounds as in test_gpu_router, whose cases these continue; u = 2^-24. Gates by
their last bits: an exponential within 4 u, a score (one addition, one
reciprocal) within 7 u, a sum over registers and lanes within 8 u more, the
quotient u: 7 + 7 + 8 + 1 = 23 u. (Logits are multiples of 2^-6, so that their
differences are exact.)
"""
import numpy as np
import pytest
import torch

import oracle.foremoe_step as S
import test_gpu_router as base

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _grid(T, E, seed, low, high):
    rng = np.random.default_rng(seed)
    return rng.integers(int(low * 64), int(high * 64), (T, E)).astype(np.float64) / 64, rng


@pytest.mark.parametrize("score,renorm", [("softmax", True), ("sigmoid", False), ("sigmoid", True)])
@pytest.mark.parametrize("E,K", [(24, 8), (200, 20), (300, 8)])
def test_gates_to_the_last_bits(gpu, score, renorm, E, K):
    """Replayed picks with scores down to e^-80 of the largest."""
    from paper_2606_11867_amd import api
    l, rng = _grid(40, E, E, -80, 1)
    ids = np.argsort(rng.random((40, E)), axis=1)[:, :K].astype(np.int32)
    x = torch.from_numpy(l.astype(np.float32)).to(gpu)
    ref = S.router_forward(l, K, score=score, renorm=renorm, ids=ids)
    for stats in (False, True):
        r = api.router_fwd(x, K, score=score, renorm=renorm, ids=torch.from_numpy(ids).to(gpu), stats=stats)
        rel = np.abs(r.gates.double().cpu().numpy() / ref["gates"] - 1)
        assert rel.max() <= 24 * U, rel.max() / U


@pytest.mark.parametrize("E,K", [(24, 8), (200, 20), (300, 8)])
@pytest.mark.parametrize("where", ["all", "some"])
def test_sigmoid_scores_too_small_for_fp32(gpu, E, K, where):
    """Rows whose every logit is below -90, where a score is subnormal or 0 in
    fp32: shares and gates are ratios all the same."""
    from paper_2606_11867_amd import api
    T = 23
    l, rng = _grid(T, E, E + 1, -400, -90)
    l = np.where(np.arange(E) % 2 == 0, l, -90 - rng.integers(0, 640, (T, E)) / 64)
    if where == "some":
        l[::2] += 90
        l[1] += np.where(np.arange(E) == 3, 95, 0)
    l[5, :] = -np.inf
    l[7, : E // 2] = -np.inf
    x = torch.from_numpy(l.astype(np.float32)).to(gpu)
    dg = rng.standard_normal((T, K)).astype(np.float32)
    coef = 0.7
    rel = U * (2 * 400 + E / 8 + 64)
    ids = np.argsort(rng.random((T, E)), axis=1)[:, :K].astype(np.int32)
    for replay in (None, ids):
        for renorm in (True, False):
            kw = dict(score="sigmoid", renorm=renorm, scale=1.5)
            ref = S.router_forward(l, K, ids=replay, **kw)
            r = api.router_fwd(x, K, ids=None if replay is None else torch.from_numpy(ids).to(gpu), **kw)
            assert np.array_equal(r.ids.cpu().numpy(), ref["ids"])
            assert np.array_equal(r.counts.cpu().numpy(), ref["counts"])
            base._check("gates", r.gates, ref["gates"], rel * ref["gates"] + 1e-37)
            base._check("prob_mean", r.prob_mean, ref["prob_mean"], rel * ref["prob_mean"] + 1e-37)
            base._check("balance_loss", r.balance_loss, np.array([ref["balance_loss"]]),
                        (rel + U * (E + 64)) * ref["balance_loss"])
            lone = api.router_fwd(x, K, ids=r.ids, stats=False, **kw)
            assert torch.equal(lone.gates, r.gates)
            c = coef * E / max(1, ref["n_tokens"]) * ref["counts"] / max(1, ref["counts"].sum())
            for cf, d in ((0.0, dg), (coef, dg), (coef, None)):
                want = S.router_backward(l, ref["ids"], d, counts=ref["counts"], n_tokens=ref["n_tokens"],
                                         balance_coef=cf, **kw)
                got = api.router_bwd(x, r.ids, None if d is None else torch.from_numpy(d).to(gpu), counts=r.counts,
                                     n_tokens=r.n_tokens, balance_coef=cf, **kw)
                size = (0.0 if d is None else 1.5 * np.abs(d).max()) + (c.max() if cf else 0.0)
                base._check("dlogits", got, want, 8 * rel * size)
            if renorm:  # none of it is lost
                assert np.abs(ref["gates"].sum(1)[ref["ids"][:, 0] >= 0] - 1.5).max() < 1e-9
                assert np.abs(want).max() > 0


def test_counts_of_many_ranks(gpu):
    """Counts that fit 32 bits each, their total not."""
    from paper_2606_11867_amd import api
    T, E, K = 50, 40, 4
    x, rng = base._logits(T, E, torch.float32, seed=9)
    counts = rng.integers(1 << 28, (1 << 31) - 1, E).astype(np.int32)
    counts[3] = 0
    n = (1 << 31) - 1
    l = x.double().numpy()
    for score in ("softmax", "sigmoid"):
        want = S.router_backward(l, np.zeros((T, K), np.int32), None, score=score, counts=counts.astype(np.int64),
                                 n_tokens=n, balance_coef=1e9)
        got = api.router_bwd(x.to(gpu), torch.zeros(T, K, dtype=torch.int32, device=gpu), None, score=score,
                             counts=torch.from_numpy(counts).to(gpu),
                             n_tokens=torch.tensor([n], dtype=torch.int32, device=gpu), balance_coef=1e9)
        c = 1e9 * E / n * counts / counts.astype(np.int64).sum()
        base._check("dlogits", got, want, 8 * base._rel(l, E) * c.max())


MORE = [
    # T, E, K, dtype, score, renorm, bias, mask, replay, disabled, pad: places over several registers, few experts
    (70, 100, 40, "f32", "softmax", True, False, True, False, 0, 0),
    (50, 256, 64, "bf16", "softmax", True, False, False, False, 0, 0),
    (33, 20, 20, "f32", "sigmoid", True, False, False, False, 0, 3),
    (33, 20, 20, "bf16", "softmax", False, False, True, True, 5, 0),
    (61, 128, 17, "f32", "sigmoid", False, False, False, True, 0, 1),
    (61, 129, 33, "bf16", "sigmoid", True, False, False, False, 90, 0),
    (45, 255, 48, "f32", "softmax", False, False, False, False, 0, 0),
    (45, 250, 64, "f32", "softmax", True, False, True, True, 3, 2),
]


@pytest.mark.parametrize("case", MORE, ids=lambda c: "T{}-E{}-K{}-{}-{}".format(*c[:5]))
def test_many_places(gpu, case):
    base.test_router_forward_and_backward(gpu, case)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,E,K", [(37, 300, 8), (21, 1000, 20), (90, 100, 6), (31, 90, 30), (29, 256, 40)])
def test_picks_by_score_plus_bias(gpu, dt, T, E, K):
    """Biases and scores that keep the sums of a token apart by more than
    their rounding."""
    from paper_2606_11867_amd import api
    dtype = torch.bfloat16 if dt == "bf16" else torch.float32
    rng = np.random.default_rng(E + K)
    # biases 2^-10 apart in a random order, scores within 2^-11 of one half; and a few that stand out
    bias = (rng.permutation(E) - E / 2).astype(np.float32) * np.float32(2.0 ** -10)
    x = torch.from_numpy((rng.random((T, E)) * 0.0015).astype(np.float32))
    for t in range(T):
        x[t, rng.integers(0, E)] = 3.0
        x[t, rng.integers(0, E, 5)] = -np.inf
    x[1] = -np.inf
    x = x.to(dtype)
    l = x.double().numpy()
    key = np.where(l > -np.inf, 1 / (1 + np.exp(-l)) + bias.astype(np.float64), -100.0 - np.arange(E))
    key = np.sort(key, axis=1)
    assert np.diff(key, axis=1)[:, -K - 1:].min() > 8 * 2.0 ** -23
    mask = np.arange(T) % 5 != 2
    for renorm in (True, False):
        kw = dict(score="sigmoid", renorm=renorm, scale=2.5)
        ref = S.router_forward(l, K, bias=bias.astype(np.float64), mask=mask, **kw)
        r = api.router_fwd(x.to(gpu), K, bias=torch.from_numpy(bias).to(gpu), mask=torch.from_numpy(mask).to(gpu), **kw)
        assert np.array_equal(r.ids.cpu().numpy(), ref["ids"])
        assert np.array_equal(r.counts.cpu().numpy(), ref["counts"])
        rel = base._rel(l, E)
        base._check("gates", r.gates, ref["gates"], rel * ref["gates"] + 1e-30)
        base._check("prob_mean", r.prob_mean, ref["prob_mean"], (rel + 65 * U) * ref["prob_mean"] + 1e-30)


@pytest.mark.parametrize("T,E,K,dt", [(33003, 8, 2, "f32"), (20000, 24, 3, "bf16"), (5000, 300, 2, "bf16")])
@pytest.mark.parametrize("replay", [False, True])
def test_statistics_past_the_first_pass(gpu, T, E, K, dt, replay):
    """More tokens than the workgroups that leave statistics take at once."""
    from paper_2606_11867_amd import api
    print(f"\n[case] statistics T={T} E={E} replay={replay}", flush=True)
    x, rng = base._logits(T, E, torch.bfloat16 if dt == "bf16" else torch.float32, seed=T)
    l = x.double().numpy()
    ids = rng.integers(0, E, (T, K)).astype(np.int32) if replay else None
    mask = rng.random(T) < 0.9
    ref = S.router_forward(l, K, ids=ids, mask=mask)
    r = api.router_fwd(x.to(gpu), K, ids=None if ids is None else torch.from_numpy(ids).to(gpu),
                       mask=torch.from_numpy(mask).to(gpu))
    assert np.array_equal(r.ids.cpu().numpy(), ref["ids"])
    assert np.array_equal(r.counts.cpu().numpy(), ref["counts"])
    assert int(r.n_tokens) == ref["n_tokens"]
    rel = base._rel(l, E)
    sums = rel + U * (T / 256 + 64)
    base._check("gates", r.gates, ref["gates"], rel * ref["gates"] + 1e-30)
    base._check("prob_mean", r.prob_mean, ref["prob_mean"], sums * ref["prob_mean"])
    base._check("balance_loss", r.balance_loss, np.array([ref["balance_loss"]]),
                (sums + U * (E + 64)) * ref["balance_loss"])


@pytest.mark.parametrize("T,E,K,most", [(140000, 8, 2, 131072), (33000, 260, 3, 32768)])
def test_backward_past_the_first_pass(gpu, T, E, K, most):
    """More tokens than the backward's workgroups take at once: rows from the
    start, around the end of the first pass and from the end."""
    from paper_2606_11867_amd import api
    x, rng = base._logits(T, E, torch.float32, seed=T)
    ids = rng.integers(0, E, (T, K)).astype(np.int32)
    dg = rng.standard_normal((T, K)).astype(np.float32)
    counts = rng.integers(0, 1000, E).astype(np.int32)
    rows = np.concatenate([np.arange(40), np.arange(most - 40, most + 40), np.arange(T - 40, T),
                           rng.integers(0, T, 60)])
    n = 777
    got = api.router_bwd(x.to(gpu), torch.from_numpy(ids).to(gpu), torch.from_numpy(dg).to(gpu),
                         counts=torch.from_numpy(counts).to(gpu),
                         n_tokens=torch.tensor([n], dtype=torch.int32, device=gpu), balance_coef=0.5)
    l = x.double().numpy()[rows]
    want = S.router_backward(l, ids[rows], dg[rows], counts=counts, n_tokens=n, balance_coef=0.5)
    size = np.abs(dg).max() + 0.5 * E / n
    base._check("dlogits", got[torch.from_numpy(rows).to(gpu)], want, 8 * base._rel(l, E) * size)
    assert torch.all(got.double().sum(1).abs() < 1e-5)  # every row: a softmax's gradients sum to 0


@pytest.mark.parametrize("E", [12, 128, 700])
def test_sigmoid_of_nan_and_infinity(gpu, E):
    """A NaN makes the shares NaN and a gate only where it enters; the score
    of +inf is 1, that of -inf is out of service."""
    from paper_2606_11867_amd import api
    K = 4
    x, _ = base._logits(6, E, torch.float32, seed=E)
    x[1, 3] = float("nan")
    x[2, 5] = float("inf")
    x[3, 1::2] = -float("inf")
    l = x.double().numpy()
    for renorm in (True, False):
        r = api.router_fwd(x.to(gpu), K, score="sigmoid", renorm=renorm)
        ids, g = r.ids.cpu().numpy(), r.gates.double().cpu().numpy()
        assert 3 not in ids[1] and ids[2, 0] == 5 and np.all(ids[3] % 2 == 0) and ids.min() >= 0 and ids.max() < E
        assert torch.isnan(r.prob_mean).all()
        rows = [0, 2, 3, 4, 5]
        ref = S.router_forward(l[rows], K, score="sigmoid", renorm=renorm)
        assert np.array_equal(ids[rows], ref["ids"])
        assert np.all(np.abs(g[rows] / ref["gates"] - 1) <= 24 * U)
        assert np.isfinite(g[1]).all()  # the NaN was not picked
        clean = api.router_fwd(x[rows].to(gpu), K, score="sigmoid", renorm=renorm)
        base._check("prob_mean", clean.prob_mean, ref["prob_mean"], (base._rel(l, E) + 65 * U) * ref["prob_mean"])
        d = api.router_bwd(x.to(gpu), r.ids, torch.ones(6, K, device=gpu), score="sigmoid", renorm=renorm).cpu()
        assert torch.isfinite(d[rows]).all()
        replay = torch.zeros(6, K, dtype=torch.int32, device=gpu) + torch.tensor([3, 0, 2, 4], device=gpu)
        q = api.router_fwd(x.to(gpu), K, score="sigmoid", renorm=renorm, ids=replay.int(), stats=False).gates.cpu()
        assert torch.isnan(q[1, 0]) and torch.isfinite(q[[0, 2, 4, 5]]).all()
