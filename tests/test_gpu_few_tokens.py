"""The expert layer for a few tokens on the GPU against the oracle.

Tolerances: a sum of n products in fp32 is within n u of the sum of their
magnitudes (u = 2^-24), whatever its order; bf16 weights and values of 4-bit
ones are exact factors. The hidden rows are kept in fp32, or as two or three
bf16 each, every one half a step of 2^-8 of what those before leave: 2^-16, and
2^-24 where the output is fp32. bf16 outputs: half a step of 2^-8.
"""
import numpy as np
import pytest
import torch

import oracle.foremoe_rollout as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
DT = {"bf16": BF16, "f32": F32}


def _np(t):
    return t.detach().double().cpu().numpy()


def _weights(rng, gpu, kind, W, r, n):
    """(what the call takes, its values)"""
    from paper_2606_11867_amd import api
    t = torch.from_numpy((rng.standard_normal((W, r, n)) * n ** -0.5).astype(np.float32)).to(gpu)
    if kind == "mxfp4":
        q = api.mxfp4_quantize(t)
        return q, R.mxfp4_values(q.codes.cpu().numpy(), q.scales.cpu().numpy(), n)
    t = t.to(DT[kind])
    return t, _np(t)


def _limit(x, ids, gates, gu, dn, widx, ref, out):
    """|y - ref| that the fp32 sums, and the output's rounding, allow."""
    W, d, F = dn.shape
    lim = np.zeros_like(ref)
    for t in range(x.shape[0]):
        for k in range(ids.shape[1]):
            e = ids[t, k]
            w = (e if widx is None else widx[e]) if 0 <= e < (W if widx is None else len(widx)) else -1
            if not 0 <= w < W:
                continue
            au = gu[w] @ x[t]
            a, u = au[:F], au[F:]
            err = d * U * (np.abs(gu[w]) @ np.abs(x[t]))
            h = R.silu(a) * u
            eh = 1.1 * err[:F] * (np.abs(u) + err[F:]) + np.abs(a) * err[F:] + (16 * U + (2.0 ** -16 if out == "bf16" else U)) * np.abs(h)
            mag = np.abs(dn[w]) @ (np.abs(h) + eh)
            lim[t] += abs(gates[t, k]) * (np.abs(dn[w]) @ eh + (2 * F + ids.shape[1] + 2) * U * mag)
    if out == "bf16":
        lim += 2.0 ** -8 * (np.abs(ref) + lim)
    return lim + 1e-37


def _case(rng, gpu, *, T, d, F, E, W, K, x="bf16", w="bf16", pad=0, dead=0.0, widx=True):
    gu, gu_v = _weights(rng, gpu, w, W, 2 * F, d)
    dn, dn_v = _weights(rng, gpu, w, W, d, F)
    xt = torch.from_numpy(rng.standard_normal((T, d + pad)).astype(np.float32)).to(gpu).to(DT[x])[:, :d]
    ids = np.stack([rng.permutation(E)[:K] for _ in range(T)]).astype(np.int32) if T else np.zeros((0, K), np.int32)
    ids[rng.random(T) < dead] = -1
    at = np.full(E, -1, dtype=np.int32)
    at[rng.permutation(E)[:W]] = np.arange(min(W, E), dtype=np.int32)
    gates = rng.random((T, K)).astype(np.float32)
    return dict(x=xt, ids=ids, gates=gates, gu=gu, dn=dn, gu_v=gu_v, dn_v=dn_v, widx=at if widx else None)


def _run(c, gpu, out, **kw):
    from paper_2606_11867_amd import api
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(gpu)  # noqa: E731
    return api.few_tokens_ffn(c["x"], dev(c["ids"]), dev(c["gates"]), c["gu"], c["dn"], expert_widx=dev(c["widx"]),
                              out_dtype=DT[out], **kw)


def _check(c, y, out):
    x = _np(c["x"])
    args = (x, c["ids"], c["gates"].astype(np.float64), c["gu_v"], c["dn_v"], c["widx"])
    ref = R.few_tokens(*args)
    lim = _limit(*args, ref, out)
    assert y.dtype == DT[out]
    got = _np(y)
    assert np.all(np.abs(got - ref) <= lim), float(np.max(np.abs(got - ref) - lim))
    none = ~((c["ids"] >= 0).any(1))
    assert not got[none].any()


SIZES = {
    "one": dict(T=1, d=256, F=128, E=16, W=16, K=4),
    "one-of-one": dict(T=1, d=32, F=32, E=1, W=1, K=1, widx=False),
    "24": dict(T=24, d=512, F=192, E=32, W=32, K=8, dead=0.2),
    "share": dict(T=64, d=320, F=96, E=64, W=8, K=6, pad=8),
    "crowded": dict(T=128, d=160, F=64, E=3, W=3, K=2, widx=False),  # more than 64 tokens an expert
    "wide": dict(T=3, d=1056, F=1120, E=5, W=5, K=5),
    "pairs": dict(T=128, d=64, F=32, E=40, W=40, K=16),  # 2048 pairs
    "long-rows": dict(T=12, d=8192, F=64, E=3, W=3, K=2),  # past what the LDS holds
    "wide-pairs": dict(T=128, d=2304, F=64, E=40, W=40, K=16),  # 2048 pairs, more than 8 columns a CU
    "wide-share": dict(T=70, d=4128, F=192, E=32, W=4, K=4, dead=0.2),
    "long-and-crowded": dict(T=40, d=2048, F=72 * 32, E=2, W=2, K=2, dead=0.1),
    "many-experts": dict(T=5, d=64, F=64, E=1024, W=1024, K=3, widx=False),
}


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("w", ["bf16", "f32", "mxfp4"])
@pytest.mark.parametrize("name", list(SIZES))
def test_few_tokens(gpu, name, w, out):
    print(f"\n[case] few {name} {w} {out}", flush=True)
    rng = np.random.default_rng(len(name) * 7 + len(w))
    c = _case(rng, gpu, x="f32" if w == "f32" else "bf16", w=w, **SIZES[name])
    _check(c, _run(c, gpu, out), out)


@pytest.mark.parametrize("w", ["bf16", "f32"])
@pytest.mark.parametrize("d,F,pad", [(1, 1, 0), (7, 3, 2), (33, 9, 0), (64, 31, 1), (65, 64, 0), (130, 257, 6), (104, 56, 8),
                                     (96, 1, 0), (2, 100, 0), (4101, 33, 0)])
def test_odd_sizes(gpu, w, d, F, pad):
    print(f"\n[case] few odd {w} d={d} F={F} pad={pad}", flush=True)
    rng = np.random.default_rng(d * 31 + F)
    c = _case(rng, gpu, T=11, d=d, F=F, E=6, W=6, K=3, x=w, w=w, pad=pad, dead=0.2)
    _check(c, _run(c, gpu, "f32"), "f32")


def test_ids_that_name_nothing(gpu):
    """Padding, ids past E, experts that are elsewhere or whose weights are out
    of range: their places count as 0, whatever their gates hold; the same
    expert twice counts twice."""
    rng = np.random.default_rng(8)
    c = _case(rng, gpu, T=7, d=64, F=64, E=6, W=4, K=4)
    c["widx"] = np.array([0, 1, -1, 4, 2, 1], dtype=np.int32)  # 2: elsewhere, 3: out of range, 5: expert 1's weights
    c["ids"] = np.array([[0, 1, 4, 5], [2, 3, 6, -1], [-1, -1, -1, 0], [1, 1, 5, 5], [1 << 30, -7, 2, 4], [2, 2, 2, 2],
                         [0, 0, 0, 0]], dtype=np.int32)
    c["gates"][1] = np.nan
    c["gates"][5] = np.inf
    c["gates"][4, :3] = np.nan
    y = _run(c, gpu, "f32")
    assert bool(torch.isfinite(y).all()) and not y[[1, 5]].any()
    c["gates"] = np.nan_to_num(c["gates"], nan=0.0, posinf=0.0)
    _check(c, y, "f32")


def test_values_that_are_not_finite(gpu):
    """A token's NaN and an expert's infinity reach those that they meet only."""
    rng = np.random.default_rng(9)
    c = _case(rng, gpu, T=20, d=64, F=64, E=5, W=5, K=2, widx=False)
    c["ids"] = np.array([[t % 4, (t + 1) % 4] for t in range(20)], dtype=np.int32)
    good = _run(c, gpu, "f32")
    c["x"][3, 10] = float("nan")
    c["gu"][4] = float("inf")  # nobody's
    y = _run(c, gpu, "f32")
    assert bool(torch.isnan(y[3]).all())
    rest = [t for t in range(20) if t != 3]
    assert torch.equal(y[rest], good[rest])


def test_shared_workspace_and_streams(gpu):
    """Calls of different sizes with one workspace, on a stream that is not the
    tensors' own, captured and replayed with other ids: bit for bit the same."""
    from paper_2606_11867_amd import api
    rng = np.random.default_rng(10)
    ws = api.few_tokens_workspace(128, 16, 256, 256, gpu).fill_(0xFF)
    cases = [_case(rng, gpu, T=T, d=d, F=F, E=16, W=16, K=K, w=w) for T, d, F, K, w in
             ((128, 64, 256, 16, "bf16"), (1, 256, 32, 2, "mxfp4"), (17, 96, 40, 3, "bf16"))]
    alone = [_run(c, gpu, "bf16") for c in cases]
    side = torch.cuda.Stream(gpu)
    side.wait_stream(torch.cuda.current_stream(gpu))
    with torch.cuda.stream(side):
        for c, ref in list(zip(cases, alone)) * 2:
            assert torch.equal(_run(c, gpu, "bf16", ws=ws), ref)
    torch.cuda.synchronize()
    c = cases[2]
    ids, gates = torch.from_numpy(c["ids"]).to(gpu), torch.from_numpy(c["gates"]).to(gpu)
    run = lambda: api.few_tokens_ffn(c["x"], ids, gates, c["gu"], c["dn"], ws=ws)  # noqa: E731
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    g, h = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = run()
    with torch.cuda.graph(h):  # a second graph with the same workspace, replayed in turn
        z = run()
    for seed in range(4):
        ids.copy_(torch.from_numpy(np.random.default_rng(seed).integers(-1, 16, ids.shape).astype(np.int32)))
        (g if seed % 2 == 0 else h).replay()
        torch.cuda.synchronize()
        got = (y if seed % 2 == 0 else z).clone()
        assert torch.equal(run(), got)


def test_no_tokens(gpu):
    rng = np.random.default_rng(11)
    for w in ("bf16", "mxfp4"):
        c = _case(rng, gpu, T=0, d=64, F=32, E=4, W=4, K=2, w=w)
        assert _run(c, gpu, "bf16").shape == (0, 64)


def test_refused(gpu):
    from paper_2606_11867_amd import ForeMoEError, api
    rng = np.random.default_rng(12)
    c = _case(rng, gpu, T=4, d=64, F=32, E=4, W=4, K=2)
    ids, gates = torch.from_numpy(c["ids"]).to(gpu), torch.from_numpy(c["gates"]).to(gpu)
    call = lambda x=c["x"], i=ids, g=gates, gu=c["gu"], dn=c["dn"], **kw: api.few_tokens_ffn(x, i, g, gu, dn, **kw)  # noqa: E731
    q = api.mxfp4_quantize(c["gu"])
    for bad in (lambda: call(x=c["x"].float()), lambda: call(i=ids.long()), lambda: call(i=ids[:3]),
                lambda: call(g=gates.double()), lambda: call(g=gates[:, :1]), lambda: call(dn=c["dn"][:3]),
                lambda: call(gu=c["gu"].transpose(1, 2)), lambda: call(gu=q), lambda: call(ws=torch.empty(8, device="cpu")),
                lambda: call(out_dtype=torch.float64), lambda: call(gu=q, dn=api.mxfp4_quantize(c["dn"]), x=c["x"].float())):
        with pytest.raises((TypeError, ValueError)):
            bad()
    with pytest.raises(ForeMoEError):
        call(ws=torch.empty(64, dtype=torch.uint8, device=gpu))


@pytest.mark.parametrize("w", ["bf16", "f32"])
def test_far_weights(gpu, w):
    """Weights past 2^32 bytes: the last matrix gives what it gives alone."""
    from paper_2606_11867_amd import api
    W, d, F = 100, 7168, 2048
    print(f"\n[case] few {w}, {W} matrices of {d} x {F}", flush=True)
    g = torch.Generator(device=gpu).manual_seed(8)
    gu, dn = (torch.zeros(W, *s, dtype=DT[w], device=gpu) for s in ((2 * F, d), (d, F)))
    pick = [0, W - 1]
    for t in (gu, dn):
        for i in pick:
            t[i] = torch.randn(t.shape[1:], generator=g, device=gpu) * t.shape[2] ** -0.5
    x = torch.randn(3, d, generator=g, device=gpu).to(DT[w])
    ids = torch.tensor([[0, 1], [1, 0], [1, -1]], dtype=I32, device=gpu)
    gates = torch.rand(3, 2, generator=g, device=gpu)
    y = api.few_tokens_ffn(x, ids, gates, gu, dn, expert_widx=torch.tensor(pick, dtype=I32, device=gpu))
    assert bool(y.any()) and torch.equal(y, api.few_tokens_ffn(x, ids, gates, gu[pick], dn[pick]))
