"""4-bit quantisation and the expert FFN in 4 bits, on the GPU against the oracle.

Codes, scales and the values that they stand for are equal bit for bit. The
FFN: products of 4-bit values are exact, so a sum of n of them is within n u of
the sum of their magnitudes (u = 2^-24), whatever the order. A hidden element
that lies within such an error of a rounding border may get the other code, and
a block whose largest lies so near to where its scale changes the other scale:
the oracle finds those, and y may be off by what they weigh. y is then rounded
to bf16, half a step of 2^-8.
"""
import numpy as np
import pytest
import torch

import oracle.foremoe_rollout as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32
DT = {"bf16": BF16, "f32": F32}


def _np(t):
    return t.detach().double().cpu().numpy()


def _same(q, codes, scales):
    assert np.array_equal(q.codes.cpu().numpy(), codes)
    assert np.array_equal(q.scales.cpu().numpy(), scales)


def _hard(rng, rows, cols):
    """Values of all sizes, ties, zeros, blocks of one value."""
    x = rng.standard_normal((rows, cols)) * np.exp(4 * rng.standard_normal((rows, 1)))
    x[rng.random((rows, cols)) < 0.1] = 0.0
    tie = rng.random((rows, cols)) < 0.2
    x[tie] = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, -0.25, -5.0], size=int(tie.sum()))
    x[0] = 0.0
    if rows > 2:
        x[1] = 2.0 ** -130
        x[2] = 3.3e38 * np.sign(rng.standard_normal(cols))
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (5, 31, 0), (7, 32, 3), (4, 33, 0), (33, 64, 8), (3, 1155, 9),
                                           (257, 256, 0), (9, 2048, 1), (64, 2048, 64)])
def test_quantize(gpu, dtype, rows, cols, pad):
    from paper_2606_11867_amd import api
    print(f"\n[case] quantize {dtype} {rows}x{cols}+{pad}", flush=True)
    rng = np.random.default_rng(rows * 1000 + cols)
    x = torch.from_numpy(_hard(rng, rows, cols + pad).astype(np.float32)).to(gpu).to(DT[dtype])[:, :cols]
    q = api.mxfp4_quantize(x)
    codes, scales = R.mxfp4_quantize(_np(x))
    _same(q, codes, scales)
    ref = R.mxfp4_values(codes, scales, cols)
    for out in ("bf16", "f32"):
        buf = torch.full((rows, cols + pad + 2), 9.0, dtype=DT[out], device=gpu)
        v = api.mxfp4_values(q, cols, out=buf[:, :cols])
        assert np.array_equal(_np(v), ref)
        assert bool(torch.all(buf[:, cols:] == 9.0))
    whole = api.mxfp4_values(q)
    assert whole.shape == (rows, q.scales.shape[1] * 32) and not whole[:, cols:].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_bf16_value(gpu, dtype):
    """Every finite bf16 value beside each of several largest ones, and alone."""
    from paper_2606_11867_amd import api
    print(f"\n[case] every bf16 value, {dtype}", flush=True)
    v = torch.arange(1 << 16, dtype=torch.int32, device=gpu).to(torch.int16).view(BF16)
    v = v[torch.isfinite(v.float())]
    x = torch.zeros(v.numel(), 64, dtype=BF16, device=gpu)
    x[:, 5] = v
    x[:, 40] = v
    x[:, 63] = (v.float() * 3.7).clamp(-3e38, 3e38).to(BF16)
    x = x.to(DT[dtype])
    q = api.mxfp4_quantize(x)
    codes, scales = R.mxfp4_quantize(_np(x))
    _same(q, codes, scales)
    assert np.array_equal(_np(api.mxfp4_values(q)), R.mxfp4_values(codes, scales))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_blocks_that_are_not_finite(gpu, dtype):
    from paper_2606_11867_amd import api
    x = torch.ones(4, 96, dtype=DT[dtype], device=gpu)
    x[0, 3], x[1, 40], x[2, 95] = float("nan"), float("inf"), -float("inf")
    q = api.mxfp4_quantize(x)
    _same(q, *R.mxfp4_quantize(_np(x)))
    for out in (BF16, F32):
        v = api.mxfp4_values(q, dtype=out)
        assert torch.isnan(v).view(4, 3, 32).all(-1).tolist() == [[True, False, False], [False, True, False],
                                                                  [False, False, True], [False] * 3]


def test_rows_past_the_count_are_left(gpu):
    from paper_2606_11867_amd import api
    x = torch.randn(50, 64, device=gpu)
    full = api.mxfp4_quantize(x)
    for n in (0, 1, 17, 50, 80, -3):
        out = api.MXFP4(torch.full_like(full.codes, 7), torch.full_like(full.scales, 7))
        api.mxfp4_quantize(x, n_rows=torch.tensor([n], dtype=torch.int32, device=gpu), out=out)
        k = min(max(n, 0), 50)
        assert torch.equal(out.codes[:k], full.codes[:k]) and torch.equal(out.scales[:k], full.scales[:k])
        assert bool((out.codes[k:] == 7).all()) and bool((out.scales[k:] == 7).all())


def test_more_dimensions_and_none(gpu):
    from paper_2606_11867_amd import api
    x = torch.randn(3, 5, 40, device=gpu)
    q = api.mxfp4_quantize(x)
    assert q.codes.shape == (3, 5, 32) and q.scales.shape == (3, 5, 2)
    flat = api.mxfp4_quantize(x.view(15, 40))
    assert torch.equal(q.codes.view(15, 32), flat.codes) and torch.equal(q.scales.view(15, 2), flat.scales)
    assert api.mxfp4_values(q, 40, dtype=BF16).shape == (3, 5, 40)
    e = api.mxfp4_quantize(x[:0])
    assert e.codes.shape == (0, 5, 32) and api.mxfp4_values(e).shape == (0, 5, 64)
    with pytest.raises(ValueError):
        api.mxfp4_quantize(x[:, :, :20])  # rows apart in more than two dimensions
    with pytest.raises(Exception):
        api.mxfp4_quantize(torch.randn(4, 0, device=gpu))


# ---------------------------------------------------------------------------
# The FFN
# ---------------------------------------------------------------------------
def _other_rounding(h, tol):
    """|difference| that a hidden element's value may have where its rounding,
    or its block's scale, could go the other way."""
    lo = R.mxfp4_values(*R.mxfp4_quantize(h), h.shape[1])
    blocks = lambda t: t.reshape(t.shape[0], -1, 32)  # noqa: E731
    a, t = np.abs(blocks(h)), blocks(tol)
    top, slack = a.max(-1), t.max(-1)
    out = np.zeros_like(a)
    e0, e1 = R.mx_exponent(np.maximum(top - slack, 0)), R.mx_exponent(top + slack)
    for e in (e0, e1):
        s = 2.0 ** e[..., None]
        for d in (-1, 1):
            place, _ = R.mx_round(np.maximum(a + d * t, 0) / s)
            out = np.maximum(out, np.abs(R.GRID[place] * s - np.abs(blocks(lo))))
    return out.reshape(h.shape)


def _weights(rng, gpu, W, r, n):
    from paper_2606_11867_amd import api
    q = api.mxfp4_quantize(torch.from_numpy((rng.standard_normal((W, r, n)) * n ** -0.5).astype(np.float32)).to(gpu))
    return q, R.mxfp4_values(q.codes.cpu().numpy(), q.scales.cpu().numpy())


def _check_slot(x, gu, dn, y):
    """One slot's rows against the oracle."""
    d, F = x.shape[1], dn.shape[1]
    h, ref = R.ffn_mxfp4(x, gu, dn)
    a, u = x @ gu[:F].T, x @ gu[F:].T
    ea, eu = (d * U * (np.abs(x) @ np.abs(w).T) for w in (gu[:F], gu[F:]))
    # |silu'| <= 1.1, |silu(a)| <= |a|; its own operations a few u
    th = 1.1 * ea * (np.abs(u) + eu) + np.abs(a) * eu + 16 * U * np.abs(h) + 1e-37
    q = np.abs(R.mxfp4_values(*R.mxfp4_quantize(h), F))
    off = _other_rounding(h, th)
    lim = off @ np.abs(dn).T + F * U * ((q + off) @ np.abs(dn).T)
    lim += 2.0 ** -8 * (np.abs(ref) + lim) + 1e-37
    assert np.all(np.abs(y - ref) <= lim), float(np.max(np.abs(y - ref) - lim))


@pytest.mark.parametrize("d,F,rows,widx", [
    (128, 128, [1], [0]),
    (128, 128, [128, 129, 0, 127], [0, 1, 2, 0]),
    (384, 256, [5, 0, 300, 64], [2, 1, 0, 1]),
    (256, 640, [33, 257], [1, 1]),
    (1152, 128, [70, 3], [0, 1]),
    (640, 384, [2] * 70, [i % 3 for i in range(70)]),
])
def test_grouped_ffn(gpu, d, F, rows, widx):
    from paper_2606_11867_amd import api
    print(f"\n[case] ffn4 d={d} F={F} slots={len(rows)}", flush=True)
    rng = np.random.default_rng(d + F)
    W, n, extra = 3, sum(rows), 19
    gu, gu_v = _weights(rng, gpu, W, 2 * F, d)
    dn, dn_v = _weights(rng, gpu, W, d, F)
    x = torch.from_numpy(rng.standard_normal((n + extra, d)).astype(np.float32)).to(gpu).to(BF16)
    off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    off_t, widx_t = torch.from_numpy(off).to(gpu), torch.tensor(widx, dtype=torch.int32, device=gpu)
    xq = api.mxfp4_quantize(x)
    y = api.grouped_ffn_mxfp4_fwd(xq, off_t, widx_t, gu, dn)
    xv = R.mxfp4_values(xq.codes.cpu().numpy(), xq.scales.cpu().numpy())
    for j, w in enumerate(widx):
        r = slice(off[j], off[j + 1])
        if rows[j]:
            _check_slot(xv[r], gu_v[w], dn_v[w], _np(y[r]))
    # again, with a workspace that holds something else: the same bits
    ws = api.ffn_mxfp4_workspace(n + extra, F, gpu).fill_(0xAB)
    assert torch.equal(api.grouped_ffn_mxfp4_fwd(xq, off_t, widx_t, gu, dn, ws=ws)[:n], y[:n])


@pytest.mark.parametrize("d,F,rows,extra", [
    (384, 128, [i % 4 for i in range(260)], 0),  # scales word by word, every tile short
    (1152, 640, [(7 * i) % 131 for i in range(90)], 0),
    (512, 256, [130, 0, 257, 128], 20000),  # a padded batch
    (4096, 640, [1300, 5, 129], 7000),  # a matrix past an L2: row tiles by eights
])
def test_large_tiles(gpu, d, F, rows, extra):
    """Where rows and slots may need more tiles than the GPU has CUs."""
    from paper_2606_11867_amd import api
    print(f"\n[case] ffn4 large tiles d={d} F={F} slots={len(rows)}", flush=True)
    rng = np.random.default_rng(d * 3 + F)
    W, n = 2, sum(rows)
    gu, gu_v = _weights(rng, gpu, W, 2 * F, d)
    dn, dn_v = _weights(rng, gpu, W, d, F)
    x = torch.zeros(n + extra, d, dtype=BF16, device=gpu)
    x[:n] = torch.from_numpy(rng.standard_normal((n, d)).astype(np.float32)).to(gpu)
    off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    widx = np.arange(len(rows), dtype=np.int32) % W
    off_t = torch.from_numpy(off).to(gpu)
    xq = api.mxfp4_quantize(x, n_rows=off_t[-1:])
    y = api.grouped_ffn_mxfp4_fwd(xq, off_t, torch.from_numpy(widx).to(gpu), gu, dn)
    xv = R.mxfp4_values(xq.codes[:n].cpu().numpy(), xq.scales[:n].cpu().numpy())
    for w in range(W):  # all rows of a matrix at once
        at = np.concatenate([np.arange(off[j], off[j + 1]) for j in range(len(rows)) if widx[j] == w])
        _check_slot(xv[at], gu_v[w], dn_v[w], _np(y[torch.from_numpy(at).to(gpu)]))


def test_rows_outside_slots_are_left(gpu):
    """Through the C call, on a y that holds something."""
    from paper_2606_11867_amd import _lib, api
    rng = np.random.default_rng(4)
    d, F, W, n = 256, 128, 2, 200
    gu, _ = _weights(rng, gpu, W, 2 * F, d)
    dn, _ = _weights(rng, gpu, W, d, F)
    x = api.mxfp4_quantize(torch.from_numpy(rng.standard_normal((n, d)).astype(np.float32)).to(gpu))
    # slot 1 names no weights, slot 3's rows end behind the buffer
    off = torch.tensor([10, 40, 90, 150, 400], dtype=torch.int32, device=gpu)
    widx = torch.tensor([0, 2, -1, 1], dtype=torch.int32, device=gpu)
    y = torch.full((n, d), 7.0, dtype=BF16, device=gpu)
    ws = api.ffn_mxfp4_workspace(n, F, gpu)
    p = lambda t: t.data_ptr()  # noqa: E731
    _lib.check(_lib.load().foremoe_grouped_ffn_mxfp4_fwd(
        p(x.codes), p(x.scales), d, F, 4, p(off), p(widx), W, p(gu.codes), p(gu.scales), p(dn.codes), p(dn.scales), n,
        p(y), p(ws), ws.numel(), torch.cuda.current_stream(gpu).cuda_stream), "ffn")
    assert bool((y[:10] == 7).all()) and bool((y[40:150] == 7).all())
    two = torch.tensor([0, 30, 80], dtype=torch.int32, device=gpu)
    pick = torch.cat([torch.arange(10, 40), torch.arange(150, 200)]).to(gpu)
    ref = api.grouped_ffn_mxfp4_fwd(api.MXFP4(x.codes[pick], x.scales[pick]), two,
                                    torch.tensor([0, 1], dtype=torch.int32, device=gpu), gu, dn)
    assert torch.equal(y[pick], ref)


def test_no_rows_and_no_slots(gpu):
    from paper_2606_11867_amd import api
    rng = np.random.default_rng(5)
    gu, _ = _weights(rng, gpu, 1, 256, 128)
    dn, _ = _weights(rng, gpu, 1, 128, 128)
    x = api.mxfp4_quantize(torch.zeros(4, 128, device=gpu))
    i32 = dict(dtype=torch.int32, device=gpu)
    api.grouped_ffn_mxfp4_fwd(x, torch.zeros(1, **i32), torch.zeros(0, **i32), gu, dn)
    api.grouped_ffn_mxfp4_fwd(x, torch.zeros(2, **i32), torch.zeros(1, **i32), gu, dn)
    e = api.MXFP4(x.codes[:0], x.scales[:0])
    assert api.grouped_ffn_mxfp4_fwd(e, torch.zeros(2, **i32), torch.zeros(1, **i32), gu, dn).shape == (0, 128)
    # a row that is not finite stays its own
    v = torch.randn(40, 128, device=gpu)
    off, w = torch.tensor([0, 40], **i32), torch.zeros(1, **i32)
    good = api.grouped_ffn_mxfp4_fwd(api.mxfp4_quantize(v), off, w, gu, dn)
    v[7, 100] = float("inf")
    bad = api.grouped_ffn_mxfp4_fwd(api.mxfp4_quantize(v), off, w, gu, dn)
    assert bool(torch.isnan(bad[7]).all())
    rest = [i for i in range(40) if i != 7]
    assert torch.equal(bad[rest], good[rest])


def test_captured(gpu):
    """Quantisation and FFN in a graph, replayed on other rows and loads."""
    from paper_2606_11867_amd import api
    rng = np.random.default_rng(6)
    d, F, n = 256, 256, 300
    gu, _ = _weights(rng, gpu, 2, 2 * F, d)
    dn, _ = _weights(rng, gpu, 2, d, F)
    x = torch.randn(n, d, device=gpu).to(BF16)
    off = torch.tensor([0, 100, 200], dtype=torch.int32, device=gpu)
    widx = torch.tensor([0, 1], dtype=torch.int32, device=gpu)
    ws = api.ffn_mxfp4_workspace(n, F, gpu)
    run = lambda: api.grouped_ffn_mxfp4_fwd(api.mxfp4_quantize(x, n_rows=off[-1:]), off, widx, gu, dn, ws=ws)  # noqa: E731
    side = torch.cuda.Stream(gpu)
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = run()
    for loads in ([0, 100, 200], [0, 0, 300], [0, 257, 258], [0, 0, 0]):
        x.copy_(torch.randn(n, d, device=gpu))
        off.copy_(torch.tensor(loads, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(run()[:loads[-1]], y[:loads[-1]])


def test_far_rows(gpu):
    """More than 2^31 elements: the last rows are those of a call of their own."""
    from paper_2606_11867_amd import api
    rows, cols = (1 << 20) + 5, 2080
    print(f"\n[case] quantize {rows}x{cols}", flush=True)
    x = torch.empty(rows, cols, dtype=BF16, device=gpu)
    x[:7].normal_(), x[7:-7].fill_(1.0), x[-7:].normal_()
    q, tail, head = api.mxfp4_quantize(x), api.mxfp4_quantize(x[-7:]), api.mxfp4_quantize(x[:7])
    for at, ref in ((slice(-7, None), tail), (slice(0, 7), head)):
        assert torch.equal(q.codes[at], ref.codes) and torch.equal(q.scales[at], ref.scales)
    v = api.mxfp4_values(q, dtype=BF16)
    assert torch.equal(v[-7:], api.mxfp4_values(tail, dtype=BF16)) and bool((v[7:-7] == 1).all())


def test_far_weights(gpu):
    """Weights past 2^31 bytes: the last matrix gives what it gives alone."""
    from paper_2606_11867_amd import api
    W, d, F = 160, 7168, 2048
    print(f"\n[case] ffn4 and few, {W} matrices of {d} x {F}", flush=True)
    g = torch.Generator(device=gpu).manual_seed(7)
    make = lambda r, n: api.MXFP4(  # noqa: E731
        torch.randint(0, 256, (W, r, n // 2), generator=g, device=gpu, dtype=torch.uint8),
        torch.randint(116, 120, (W, r, n // 32), generator=g, device=gpu, dtype=torch.uint8))
    gu, dn = make(2 * F, d), make(d, F)
    x = torch.randn(40, d, generator=g, device=gpu).to(BF16)
    xq = api.mxfp4_quantize(x)
    off = torch.tensor([0, 25, 40], dtype=torch.int32, device=gpu)
    pick = [0, W - 1]
    few_of = lambda q: api.MXFP4(q.codes[pick], q.scales[pick])  # noqa: E731
    y = api.grouped_ffn_mxfp4_fwd(xq, off, torch.tensor(pick, dtype=torch.int32, device=gpu), gu, dn)
    ref = api.grouped_ffn_mxfp4_fwd(xq, off, torch.tensor([0, 1], dtype=torch.int32, device=gpu), few_of(gu), few_of(dn))
    assert bool(torch.isfinite(y).all()) and torch.equal(y, ref)
    ids = torch.tensor([[0, 1], [1, 0], [1, -1]], dtype=torch.int32, device=gpu)
    gates = torch.rand(3, 2, generator=g, device=gpu)
    widx = torch.tensor(pick, dtype=torch.int32, device=gpu)
    y = api.few_tokens_ffn(x[:3], ids, gates, gu, dn, expert_widx=widx)
    ref = api.few_tokens_ffn(x[:3], ids, gates, few_of(gu), few_of(dn))
    assert bool(torch.isfinite(y).all()) and torch.equal(y, ref)
