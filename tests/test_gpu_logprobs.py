"""Token log-probabilities on the GPU against the fp64 oracle.

Bounds, u = 2^-24, Y = the largest |logit / temperature|. log-probabilities
and lse are sums of terms up to 2 Y + log V, each rounded a few times, and the
logarithm of a sum of V positive terms, of which at most V / 256 are added one
after another: within tol = u (16 Y + V / 256 + 128). An entropy is
log s - t / s with both terms positive and t a sum of products (y - max) e^(y -
max): within tol (2 + H). A gradient is dlogp, dentropy (each over the
temperature) times p, p log p and p H: p is within rel = 2 tol, so within
4 tol times the magnitudes that enter it; in bf16 it is the rounding of a
number that near.
"""
import numpy as np
import pytest
import torch

import oracle.foremoe_step as S
from workload import bf16_round

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
INF = float("inf")


def _close(name, got, ref, tol):
    rounded = got.dtype == torch.bfloat16
    got = got.detach().float().cpu().numpy().astype(np.float64)
    assert got.shape == ref.shape, name
    same = (got == ref) | (np.isnan(got) & np.isnan(ref))
    with np.errstate(invalid="ignore"):
        off = np.abs(got - ref)
    near = off <= tol
    if rounded:  # rounding keeps order
        near = (got >= bf16_round((ref - tol).astype(np.float32))) & (got <= bf16_round((ref + tol).astype(np.float32)))
    assert np.all(same | near), f"{name}: {np.nanmax(np.where(same, 0, off)):.3g} off"


def _inputs(N, V, dtype, seed, pad=0, offset=0, masked=0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((N, V)).astype(np.float32) * 3
    for i in range(N):  # likely tokens
        x[i, rng.integers(0, V, 3)] += 9
    if masked:
        x[:, V - masked:] = -INF
    x = torch.from_numpy(x).to(dtype)
    return x, rng


def _on_gpu(x, gpu, pad, offset):
    """x as rows `pad` apart in a larger buffer, `offset` elements from its
    start; the rest holds 5."""
    N, V = x.shape
    buf = torch.full((offset + N * (V + pad),), 5.0, dtype=x.dtype, device=gpu)
    t = buf[offset:].view(N, V + pad)[:, :V]
    t.copy_(x)
    return buf, t


CASES = [
    # N, V, dtype, n_top, temperature, ignored, pad, offset, masked
    (1, 1, "f32", 1, 1.0, False, 0, 0, 0),
    (1, 2, "bf16", 2, 1.0, False, 0, 1, 0),
    (3, 5, "bf16", 5, 0.5, True, 1, 0, 3),
    (2, 31, "f32", 31, 2.0, False, 0, 3, 0),
    (7, 255, "bf16", 3, 1.0, True, 0, 0, 0),
    (5, 256, "f32", 32, 1.0, True, 4, 0, 250),
    (9, 1021, "bf16", 20, 0.7, True, 3, 5, 0),
    (64, 4096, "f32", 5, 1.0, True, 0, 0, 0),
    (33, 4099, "bf16", 0, 1.3, True, 0, 0, 1),
    (1, 32003, "f32", 20, 0.8, False, 0, 0, 0),
    (4, 65537, "bf16", 32, 1.0, False, 8, 1, 17),
    (1, 131072, "bf16", 20, 0.8, False, 0, 0, 0),
    (2, 150001, "bf16", 1, 1.0, True, 7, 0, 0),
    (700, 523, "f32", 4, 1.0, True, 0, 0, 0),
    (1100, 2050, "bf16", 0, 1.0, True, 0, 0, 0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "N{}-V{}-{}-top{}".format(*c[:4]))
@pytest.mark.parametrize("split", [True, False], ids=["ws", "no-ws"])
def test_logprobs_forward_and_backward(gpu, case, split):
    from paper_2606_11867_amd import api
    N, V, dt, n_top, temp, ignored, pad, offset, masked = case
    dtype = torch.bfloat16 if dt == "bf16" else torch.float32
    print(f"\n[case] logprobs {case} split={split}", flush=True)
    x, rng = _inputs(N, V, dtype, seed=N * 7 + V, masked=masked)
    if N > 4:
        x[3] = -INF  # nothing left
        x[4] = torch.finfo(dtype).min  # the type's lowest value everywhere: even odds
    l = x.double().numpy()
    t = rng.integers(0, max(1, V - masked), N).astype(np.int32)
    if N > 4:
        t[1] = V - 1  # -inf where the end is masked
    if ignored:
        t[rng.random(N) < 0.3] = -1
        t[0] = V  # outside as well
    buf, xg = _on_gpu(x, gpu, pad, offset)
    tg = torch.from_numpy(t).to(gpu)
    ws = api.logprobs_workspace(gpu) if split else None
    ref = S.token_logprobs(l, t, temperature=temp, n_top=n_top)
    fin = np.abs(l[np.isfinite(l) & (np.abs(l) < 1e30)])
    Y = (fin.max() if fin.size else 0.0) / temp
    big = np.where(np.abs(np.where(np.isfinite(l), l, 0)).max(1) > 1e30, np.abs(l[4]).max() if N > 4 else 0, 0) / temp
    tol = U * (16 * Y + V / 256 + 128) * np.ones(N)
    for again in range(2):
        r = api.token_logprobs(xg, tg, temperature=temp, n_top=n_top, ws=ws)
        if n_top:
            assert np.array_equal(r.top_ids.cpu().numpy(), ref["top_ids"])
            sel = big == 0
            _close("top_logp", r.top_logp[torch.from_numpy(sel)], ref["top_logp"][sel], tol[sel][:, None])
        else:
            assert r.top_ids is None
        # a row of the lowest value: lse is that value, its distance to the logits is lost in fp32
        _close("lse", r.lse, ref["lse"].astype(np.float32).astype(np.float64), tol + 4 * U * big)
        _close("logp", r.logp, np.where(big > 0, r.logp.double().cpu().numpy(), ref["logp"]), tol)
        _close("entropy", r.entropy, ref["entropy"], tol * (2 + ref["entropy"]))
    every = api.token_logprobs(xg, temperature=temp, n_top=n_top, ws=ws)
    assert every.logp is None
    eref = S.token_logprobs(l, None, temperature=temp, n_top=n_top)
    _close("lse", every.lse, eref["lse"].astype(np.float32).astype(np.float64), tol + 4 * U * big)

    a, b = rng.standard_normal(N).astype(np.float32), rng.standard_normal(N).astype(np.float32)
    rows = np.nonzero(big == 0)[0]
    ag, bg = torch.from_numpy(a).to(gpu), torch.from_numpy(b).to(gpu)
    for da, db in ((a, b), (a, None), (None, b)):
        want = S.token_logprobs_backward(l[rows], t[rows], None if da is None else da[rows],
                                         None if db is None else db[rows], temperature=temp)
        got = api.token_logprobs_bwd(xg, tg, r.lse, None if da is None else ag, entropy=None if db is None else r.entropy,
                                     dentropy=None if db is None else bg, temperature=temp)
        size = (np.abs(a) + np.abs(b) * (2 + ref["entropy"]) * 2)[rows, None] / temp
        _close("dlogits", got[torch.from_numpy(rows)], want, 4 * tol[rows, None] * size)
    d = api.token_logprobs_bwd(xg, None, every.lse, None, entropy=every.entropy, dentropy=bg, temperature=temp)
    want = S.token_logprobs_backward(l[rows], None, None, b[rows], temperature=temp)
    size = (np.abs(b) * (2 + eref["entropy"]) * 2)[rows, None] / temp
    _close("dlogits", d[torch.from_numpy(rows)], want, 4 * tol[rows, None] * size)
    # in place, nothing beside the rows
    out = api.token_logprobs_bwd(xg, tg, r.lse, None, entropy=r.entropy, dentropy=bg, temperature=temp, out=xg)
    assert out is xg and torch.equal(xg, got)
    if pad:
        assert torch.all(buf[offset:].view(N, V + pad)[:, V:] == 5.0)
    assert torch.all(buf[:offset] == 5.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("order", ["equal", "falling", "rising", "one-lane", "few-values", "zeros"])
@pytest.mark.parametrize("N,V", [(1, 70001), (3, 2500), (300, 1300)])
def test_top_alternatives_in_awkward_orders(gpu, dtype, order, N, V):
    """Orders that send every element, or all the large ones of one lane,
    past a threshold; ties everywhere."""
    from paper_2606_11867_amd import api
    rng = np.random.default_rng(V)
    j = np.arange(V)
    row = {"equal": np.zeros(V), "falling": -j / V * 8, "rising": j / V * 8,
           "one-lane": np.where(j % 64 == 5, j % 997 / 100, -4.0), "few-values": rng.integers(0, 3, V),
           "zeros": np.where(rng.random(V) < 0.5, 0.0, -0.0)}[order]
    l = np.repeat(row[None].astype(np.float32), N, 0)
    x = torch.from_numpy(l).to(dtype)
    for n_top in (1, 7, 32):
        r = api.token_logprobs(x.to(gpu), n_top=n_top, ws=api.logprobs_workspace(gpu))
        l = x[:1].double().numpy()
        want = np.lexsort((j, -l[0]))[:n_top]
        assert np.array_equal(r.top_ids.cpu().numpy(), np.repeat(want[None], N, 0)), n_top


@pytest.mark.parametrize("V", [9, 3000, 80000])
def test_logprobs_nan_and_infinity(gpu, V):
    from paper_2606_11867_amd import api
    x, _ = _inputs(4, V, torch.float32, seed=V)
    x[1, V // 2] = float("nan")
    x[2, V - 1] = INF
    t = torch.zeros(4, dtype=torch.int32, device=gpu)
    for ws in (None, api.logprobs_workspace(gpu)):
        r = api.token_logprobs(x.to(gpu), t, n_top=3, ws=ws)
        for v in (r.logp, r.entropy, r.lse):
            assert torch.isnan(v[[1, 2]]).all() and torch.isfinite(v[[0, 3]]).all()
        ids = r.top_ids.cpu().numpy()
        assert ids.min() >= 0 and ids.max() < V and ids[2, 0] == V - 1 and V // 2 not in ids[1]
        d = api.token_logprobs_bwd(x.to(gpu), t, r.lse, torch.ones(4, device=gpu))
        assert torch.isnan(d[[1, 2]]).all() and torch.isfinite(d[[0, 3]]).all()


def test_logprobs_nothing_to_do(gpu):
    from paper_2606_11867_amd import api
    r = api.token_logprobs(torch.empty(0, 10, device=gpu), torch.empty(0, dtype=torch.int32, device=gpu), n_top=2)
    assert r.logp.shape == (0,) and r.top_ids.shape == (0, 2)
    assert api.token_logprobs_bwd(torch.empty(0, 10, device=gpu), torch.empty(0, dtype=torch.int32, device=gpu),
                                  torch.empty(0, device=gpu), torch.empty(0, device=gpu)).shape == (0, 10)
    x = torch.randn(6, 50, device=gpu)
    r = api.token_logprobs(x, torch.full((6,), -100, dtype=torch.int32, device=gpu), n_top=2)
    for v in (r.logp, r.entropy, r.lse):
        assert torch.all(v == 0)
    assert torch.all(r.top_ids == -1) and torch.all(r.top_logp == -INF)


def test_logprobs_large_offsets(gpu):
    """Rows that start past 2^32 bytes and 2^31 elements."""
    from paper_2606_11867_amd import api
    ld, V = (1 << 30) + 64, 1500
    buf = torch.zeros(2 * ld + V, dtype=torch.bfloat16, device=gpu)
    x = buf.as_strided((3, V), (ld, 1))
    x.copy_(torch.randn(3, V, generator=torch.Generator().manual_seed(1)) * 3)
    t = torch.tensor([3, 1499, 700], dtype=torch.int32, device=gpu)
    r = api.token_logprobs(x, t, n_top=4, ws=api.logprobs_workspace(gpu))
    q = api.token_logprobs(x.contiguous(), t, n_top=4, ws=api.logprobs_workspace(gpu))
    for a, b in zip(r, q):
        assert torch.equal(a, b)
    w = torch.tensor([1.0, -2.0, 0.5], device=gpu)
    d = api.token_logprobs_bwd(x, t, r.lse, w)
    api.token_logprobs_bwd(x, t, r.lse, w, out=x)
    assert torch.equal(d, x) and torch.all(buf[V:ld] == 0)


def test_logprobs_repeat_and_streams(gpu):
    from paper_2606_11867_amd import api
    for N, V in ((1, 131072), (12, 9001), (2500, 700)):
        x = (torch.randn(N, V, device=gpu) * 3).to(torch.bfloat16)
        t = torch.randint(0, V, (N,), device=gpu, dtype=torch.int32)
        one = api.token_logprobs(x, t, n_top=9, ws=api.logprobs_workspace(gpu))
        wss = [api.logprobs_workspace(gpu) for _ in range(2)]
        streams = [torch.cuda.Stream(gpu) for _ in range(2)]
        torch.cuda.synchronize()
        outs = []
        for i in range(8):
            with torch.cuda.stream(streams[i % 2]):
                outs.append(api.token_logprobs(x, t, n_top=9, ws=wss[i % 2]))
        torch.cuda.synchronize()
        for o in outs:
            for a, b in zip(o, one):
                assert torch.equal(a, b)


def test_logprobs_in_a_graph(gpu):
    from paper_2606_11867_amd import api
    x = torch.randn(3, 40000, device=gpu)
    t = torch.tensor([1, 2, 39999], dtype=torch.int32, device=gpu)
    w = torch.randn(3, device=gpu)
    ws = api.logprobs_workspace(gpu)

    def step():
        r = api.token_logprobs(x, t, n_top=6, ws=ws)
        return (*r, api.token_logprobs_bwd(x, t, r.lse, w, entropy=r.entropy, dentropy=w))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, step()):
            assert torch.equal(a, b), i


@pytest.mark.parametrize("N,V,dt", [(8200, 100003, "bf16"), (1400, 30001, "f32")], ids=["1.6GB-bf16", "168MB-f32"])
def test_logprobs_larger_than_the_cache(gpu, N, V, dt):
    """Logits and gradients that are kept out of the cache: rows from the
    start, the middle and the end against the oracle, every row's gradient
    summing to zero."""
    from paper_2606_11867_amd import api
    dtype = torch.bfloat16 if dt == "bf16" else torch.float32
    print(f"\n[case] logprobs N={N} V={V} {dt}", flush=True)
    gen = torch.Generator(device=gpu).manual_seed(N)
    x = torch.empty(N, V, dtype=dtype, device=gpu)
    for a in range(0, N, 1024):
        x[a:a + 1024] = 3 * torch.randn(min(1024, N - a), V, generator=gen, device=gpu)
    t = torch.randint(0, V, (N,), generator=gen, device=gpu).to(torch.int32)
    t[5::7] = -1
    a, b = torch.randn(N, generator=gen, device=gpu), torch.randn(N, generator=gen, device=gpu)
    rows = np.array([0, 1, 5, N // 2, N // 2 + 1, N - 2, N - 1])
    pick = torch.from_numpy(rows).to(gpu)
    l, tt = x[pick].double().cpu().numpy(), t[pick].cpu().numpy()
    ref = S.token_logprobs(l, tt)
    tol = U * (16 * np.abs(l).max() + V / 256 + 128)
    r = api.token_logprobs(x, t, ws=api.logprobs_workspace(gpu))
    _close("lse", r.lse[pick], ref["lse"], tol)
    _close("logp", r.logp[pick], ref["logp"], tol)
    _close("entropy", r.entropy[pick], ref["entropy"], tol * (2 + ref["entropy"]))
    an, bn = a[pick].cpu().numpy(), b[pick].cpu().numpy()
    want = S.token_logprobs_backward(l, tt, an, bn)
    size = (np.abs(an) + np.abs(bn) * (2 + ref["entropy"]) * 2)[:, None]
    d = api.token_logprobs_bwd(x, t, r.lse, a, entropy=r.entropy, dentropy=b, out=x)
    _close("dlogits", d[pick], want, 4 * tol * size)
    assert torch.all(d[5::7] == 0)
    # the terms of a row, each within 2^-8 of itself, have magnitudes that sum to less than
    # 2 |a| + |b| sum p |log p + H| <= 2 |a| + 2 |b| H
    H = r.entropy.abs()
    assert torch.all(d.float().sum(1).abs() <= 2.0 ** -8 * (2 * a.abs() + 2 * b.abs() * H) + 1e-3)
