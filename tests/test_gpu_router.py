"""The router on the GPU against the fp64 oracle: picking and replaying,
statistics, the balance loss and the gradient; ids and counts are equal, the
rest is within bounds derived from fp32 rounding.

Bounds, u = 2^-24. A score is an exponential of x - max, or of -x: its
argument carries a rounding of u |x|, the function a few u, the sum of E
positive scores in a fixed tree less than (E / 16 + 16) u, the quotient 2 u.
With |x| <= X: gates and pi are within rel = u (X + E / 8 + 64) of their
values. Sums over T tokens, at most T / 512 of them one after another, add
u (T / 256 + 64). A gradient is a sum of products of those with dgates and the
balance coefficients: at most 8 rel times the largest magnitude that enters
it; in bf16 it is the rounding of a number that near.
"""
import numpy as np
import pytest
import torch

import oracle.foremoe_step as S
from workload import bf16_round

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
INF = float("inf")


def _logits(T, E, dtype, seed, disabled=0, pad=0, spread=2.0):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy((rng.standard_normal((T, E + pad)) * spread).astype(np.float32)).to(dtype)
    if disabled:
        x[:, rng.permutation(E)[:disabled]] = -INF
    return x[:, :E], rng


def _rel(x, E):
    x = x[np.isfinite(x)]
    return U * ((np.abs(x).max() if x.size else 0.0) * 2 + E / 8 + 64)


def _check(name, got, ref, tol):
    rounded = got.dtype == torch.bfloat16
    got = got.detach().float().cpu().numpy().astype(np.float64)
    assert got.shape == ref.shape, name
    if rounded:  # rounding keeps order
        bad = ~((got >= bf16_round((ref - tol).astype(np.float32))) & (got <= bf16_round((ref + tol).astype(np.float32))))
    else:
        bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), f"{name}: {np.abs(got - ref).max():.3g} off"


CASES = [
    # T, E, K, dtype, score, renorm, bias, mask, replay, disabled, pad
    (1, 8, 2, "f32", "softmax", True, False, False, False, 0, 0),
    (1, 1, 1, "bf16", "softmax", False, False, False, False, 0, 0),
    (2, 3, 3, "f32", "sigmoid", True, False, False, False, 0, 1),
    (5, 13, 5, "bf16", "softmax", True, False, True, False, 9, 0),
    (33, 60, 4, "bf16", "sigmoid", False, True, False, False, 3, 7),
    (67, 64, 6, "f32", "softmax", False, False, True, True, 0, 2),
    (130, 128, 8, "f32", "softmax", True, False, True, True, 0, 0),
    (131, 128, 8, "bf16", "softmax", True, False, False, False, 0, 0),
    (257, 160, 6, "f32", "softmax", True, False, True, False, 40, 3),
    (300, 256, 8, "bf16", "sigmoid", True, True, True, False, 0, 0),
    (301, 256, 8, "f32", "sigmoid", True, False, False, True, 10, 1),
    (64, 257, 64, "bf16", "softmax", True, False, False, False, 0, 0),
    (40, 512, 10, "f32", "softmax", False, False, False, False, 500, 0),
    (21, 1000, 17, "bf16", "sigmoid", True, False, True, False, 0, 24),
    (19, 1024, 64, "f32", "softmax", True, False, False, True, 0, 0),
    (4099, 24, 3, "bf16", "softmax", True, False, True, False, 1, 0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "T{}-E{}-K{}-{}-{}".format(*c[:5]))
def test_router_forward_and_backward(gpu, case):
    from paper_2606_11867_amd import api
    T, E, K, dt, score, renorm, with_bias, with_mask, replay, disabled, pad = case
    dtype = torch.bfloat16 if dt == "bf16" else torch.float32
    print(f"\n[case] router {case}", flush=True)
    x, rng = _logits(T, E, dtype, seed=T * 1000 + E, disabled=disabled, pad=pad)
    l = x.float().numpy().astype(np.float64)
    if T > 4:
        x[2] = -INF  # a token that no expert takes
        l[2] = -INF
    bias = (0.3 * rng.standard_normal(E)).astype(np.float32) if with_bias else None
    mask = rng.random(T) < 0.8 if with_mask else None
    ids = None
    if replay:
        ids = np.argsort(rng.random((T, E)), axis=1)[:, :K].astype(np.int32)
        ids[rng.random((T, K)) < 0.1] = -1
        ids[T // 2, 0] = E + 5
        if K > 1:
            ids[T // 3, 1] = ids[T // 3, 0]
    dgates = rng.standard_normal((T, K)).astype(np.float32)
    scale, coef = 1.7, 0.9
    dev = lambda a: None if a is None else torch.from_numpy(a).to(gpu)  # noqa: E731
    xg = torch.full((T, E + pad), 7.0, dtype=dtype, device=gpu)[:, :E]
    xg.copy_(x)
    ws = api.router_workspace(E, gpu)
    kw = dict(score=score, renorm=renorm, scale=scale)
    ref = S.router_forward(l, K, bias=None if bias is None else bias.astype(np.float64), mask=mask, ids=ids, **kw)
    rel = _rel(l, E)
    for again in range(2):  # the workspace is ready for the next call
        r = api.router_fwd(xg, K, bias=dev(bias), mask=dev(mask), ids=dev(ids), ws=ws, **kw)
        assert np.array_equal(r.ids.cpu().numpy(), ref["ids"])
        assert np.array_equal(r.counts.cpu().numpy(), ref["counts"])
        assert int(r.n_tokens) == ref["n_tokens"]
        _check("gates", r.gates, ref["gates"], rel * np.abs(ref["gates"]) + 1e-30)
        sums = rel + U * (T / 256 + 64)
        _check("prob_mean", r.prob_mean, ref["prob_mean"], sums * ref["prob_mean"] + 1e-30)
        _check("balance_loss", r.balance_loss, np.array([ref["balance_loss"]]),
               (sums + U * (E + 64)) * ref["balance_loss"] + 1e-30)
    lone = api.router_fwd(xg, K, bias=dev(bias), mask=dev(mask), ids=dev(ids), stats=False, **kw)
    assert lone.counts is None
    assert torch.equal(lone.ids, r.ids) and torch.equal(lone.gates, r.gates)

    kept = r.ids.cpu().numpy()
    c = coef * E / max(1, ref["n_tokens"]) * ref["counts"] / max(1, ref["counts"].sum())
    for cf in (coef, 0.0):
        want = S.router_backward(l, kept, dgates, mask=mask, counts=ref["counts"], n_tokens=ref["n_tokens"],
                                 balance_coef=cf, **kw)
        got = api.router_bwd(xg, r.ids, dev(dgates), mask=dev(mask), counts=r.counts, n_tokens=r.n_tokens,
                             balance_coef=cf, **kw)
        size = scale * np.abs(dgates).max() + (c.max() if cf else 0.0)
        _check("dlogits", got, want, 8 * rel * size)
        twice = api.router_bwd(xg, r.ids, dev(dgates), mask=dev(mask), counts=r.counts, n_tokens=r.n_tokens,
                               balance_coef=cf, **kw)
        assert torch.equal(got, twice)
    # balance alone, then in place
    want = S.router_backward(l, kept, None, mask=mask, counts=ref["counts"], n_tokens=ref["n_tokens"],
                             balance_coef=coef, **kw)
    only = api.router_bwd(xg, r.ids, None, mask=dev(mask), counts=r.counts, n_tokens=r.n_tokens, balance_coef=coef,
                          **kw)
    _check("dlogits", only, want, 8 * rel * c.max() + 1e-30)
    out = api.router_bwd(xg, r.ids, dev(dgates), mask=dev(mask), out=xg, **kw)
    assert out is xg and torch.equal(xg, got)
    if pad:
        assert torch.all(xg.as_strided((T, pad), (E + pad, 1), E) == 7.0)  # nothing beside the rows


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("E", [7, 128, 300])
def test_router_ties_take_the_lower_id(gpu, dtype, E):
    from paper_2606_11867_amd import api
    rng = np.random.default_rng(E)
    K = 5
    l = rng.integers(-1, 2, size=(50, E)).astype(np.float32)
    l[0], l[1], l[2] = 0.0, -0.0, torch.finfo(dtype).min
    l[3, ::2] = -0.0  # equal to 0
    l[4] = np.where(np.arange(E) == E - 1, np.float32(torch.finfo(dtype).max), np.float32(torch.finfo(dtype).min))
    r = api.router_fwd(torch.from_numpy(l).to(dtype).to(gpu), K, stats=False)
    l = torch.from_numpy(l).to(dtype).double().numpy()
    ref = S.router_forward(l, K)
    assert np.array_equal(r.ids.cpu().numpy(), ref["ids"])
    _check("gates", r.gates, ref["gates"], 1e-5)


@pytest.mark.parametrize("E", [12, 128, 700])
def test_router_nan_and_infinity_stay_in_range(gpu, E):
    """NaN and +inf logits: ids in range and distinct, NaN where the formula
    has it, other tokens untouched."""
    from paper_2606_11867_amd import api
    K = 4
    x, _ = _logits(6, E, torch.float32, seed=E)
    x[1, 3] = float("nan")
    x[2, :] = float("nan")
    x[3, 5] = INF
    r = api.router_fwd(x.to(gpu), K, renorm=False)
    ids = r.ids.cpu().numpy()
    assert ids.min() >= -1 and ids.max() < E
    assert np.all(ids[2] == -1) and 3 not in ids[1] and ids[3, 0] == 5
    g = r.gates.cpu()
    assert torch.isnan(g[1]).all() and torch.isnan(g[3]).all() and torch.isfinite(g[[0, 4, 5]]).all()
    assert torch.isnan(r.prob_mean).all() and int(r.n_tokens) == 6
    d = api.router_bwd(x.to(gpu), r.ids, torch.ones(6, K, device=gpu), renorm=False)
    assert torch.isfinite(d[[0, 4, 5]]).all()


def test_router_nothing_to_do(gpu):
    from paper_2606_11867_amd import api
    r = api.router_fwd(torch.empty(0, 16, device=gpu), 2)
    assert r.ids.shape == (0, 2) and r.counts.sum() == 0 and int(r.n_tokens) == 0
    assert float(r.balance_loss) == 0.0 and torch.all(r.prob_mean == 0)
    x = torch.randn(9, 16, device=gpu)
    r = api.router_fwd(x, 2, mask=torch.zeros(9, dtype=torch.bool, device=gpu))
    assert torch.all(r.ids == -1) and torch.all(r.gates == 0) and float(r.balance_loss) == 0.0
    d = api.router_bwd(x, r.ids, torch.ones(9, 2, device=gpu), mask=torch.zeros(9, dtype=torch.bool, device=gpu),
                       counts=r.counts, n_tokens=r.n_tokens, balance_coef=1.0)
    assert torch.all(d == 0)


def test_router_feeds_the_dispatch(gpu):
    """The router's ids are what the layer's histogram counts."""
    from paper_2606_11867_amd import api
    x, _ = _logits(777, 32, torch.bfloat16, seed=3)
    mask = torch.arange(777, device=gpu) % 3 > 0
    r = api.router_fwd(x.to(gpu), 4, mask=mask)
    counts = api.histogram(r.ids, 32, api.workspace(777, 4, 32, gpu))
    assert torch.equal(counts, r.counts)


def test_router_on_another_stream_and_twice(gpu):
    """Two runs are bitwise equal, also beside each other on two streams with
    their own workspaces."""
    from paper_2606_11867_amd import api
    x, _ = _logits(20000, 128, torch.float32, seed=4)
    x = x.to(gpu)
    one = api.router_fwd(x, 8, ws=api.router_workspace(128, gpu))
    wss = [api.router_workspace(128, gpu) for _ in range(2)]
    streams = [torch.cuda.Stream(gpu) for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(api.router_fwd(x, 8, ws=wss[i % 2]))
    torch.cuda.synchronize()
    for o in outs:
        for a, b in zip(o, one):
            assert torch.equal(a, b)


def test_router_in_a_graph(gpu):
    from paper_2606_11867_amd import api
    x, rng = _logits(600, 64, torch.bfloat16, seed=8)
    x = x.to(gpu)
    dg = torch.randn(600, 6, device=gpu)
    ws = api.router_workspace(64, gpu)

    def step():
        r = api.router_fwd(x, 6, ws=ws)
        return (*r, api.router_bwd(x, r.ids, dg, counts=r.counts, n_tokens=r.n_tokens, balance_coef=0.3))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        x.copy_(torch.from_numpy(rng.standard_normal((600, 64)).astype(np.float32)))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, step()):
            assert torch.equal(a, b), i
