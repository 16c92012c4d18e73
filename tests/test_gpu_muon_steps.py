"""Muon where u has directions that are empty or next to it, over all numbers of
steps, against the exact iteration.

A side of at most 64: all of X is fp64, rounded once to the fp32 parameter
(2^-24 of an element). The iteration multiplies what fp64 leaves in an empty
direction by a every step: from |X0| = 1 at most 2^-53 sqrt(64) a^steps of it here,
and as much in the oracle. So X is within 2^-23 of its norm and 2^-49 a^steps,
which the largest of these (a = 3.4445, 16 steps) makes 7e-7.
"""
import numpy as np
import pytest
import torch

import oracle.foremoe_rollout as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
USUAL, CUBIC, SLOW = (3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0), (1.875, -1.25, 0.375)
BF16, F32 = torch.bfloat16, torch.float32


def _np(t):
    return t.detach().double().cpu().numpy()


def matrix(rng, shape, kind):
    """fp32 values in float64. rank r: a product, rounded; whole r: of whole
    numbers, so that its rank is r to the last bit; steep: singular values from 1
    to 1e-6; rows: the second half is zero; full: Gaussian."""
    m = min(shape)
    word, _, r = kind.partition(" ")
    r = int(r or 0)
    if word == "rank":
        a = rng.standard_normal((shape[0], r)) @ rng.standard_normal((r, shape[1]))
    elif word == "whole":
        a = (rng.integers(-3, 4, (shape[0], r)) @ rng.integers(-3, 4, (r, shape[1]))).astype(np.float64)
        a[0, 0] += not a.any()
    elif word == "steep":
        u, v = (np.linalg.qr(rng.standard_normal((n, m)))[0] for n in shape)
        a = (u * np.logspace(0, -6, m)) @ v.T
    else:
        a = rng.standard_normal(shape)
        if word == "rows":
            a[(shape[0] + 1) // 2:] = 0.0
    return a.astype(np.float32).astype(np.float64)


KINDS = ["rank 1", "rank 5", "whole 1", "whole 5", "steep", "rows", "full"]
SMALL = [(64, 64), (4, 4), (8, 256), (128, 16), (60, 1000), (17, 70), (1, 300), (3, 2)]


def bound(exact, coef, steps):
    return 2.0 ** -23 * np.linalg.norm(exact) + 2.0 ** -49 * coef[0] ** steps


@pytest.mark.parametrize("steps", [1, 5, 6, 7, 8, 10, 12, 16])
@pytest.mark.parametrize("coef", [USUAL, CUBIC, SLOW], ids=["usual", "cubic", "slow"])
def test_small_sides(gpu, coef, steps):
    from paper_2606_11867_amd.optimizer import Muon
    rng = np.random.default_rng(100 * steps + len(coef))
    print(f"\n[case] muon, {steps} steps of {coef}", flush=True)
    us = [(s, k, matrix(rng, s, k)) for s in SMALL for k in KINDS]
    gs = [torch.from_numpy(u.astype(np.float32)).to(gpu) for _, _, u in us]
    ps = [torch.zeros_like(g) for g in gs]
    Muon(ps, gs, lr=1.0, momentum=0.0, nesterov=False, scale=-1.0, eps=0.0, steps=steps, coefficients=coef).step()
    for (s, k, u), p in zip(us, ps):
        exact = R.newton_schulz(u / np.linalg.norm(u), coef, steps)
        off = np.linalg.norm(_np(p) - exact)
        assert off <= bound(exact, coef, steps), (s, k, off, np.linalg.norm(exact))


@pytest.mark.parametrize("masters", [False, True])
@pytest.mark.parametrize("nesterov", [False, True])
def test_small_sides_whole_step(gpu, nesterov, masters):
    """13 steps, more than G is carried through at once: m, the parameters and
    cleared gradients as in a short step, batches and odd widths among them."""
    from paper_2606_11867_amd.optimizer import Muon
    print(f"\n[case] muon, 13 steps, nesterov={nesterov} masters={masters}", flush=True)
    rng = np.random.default_rng(31)
    shapes = [(2, 40, 70), (3, 2, 90, 33), (7, 1), (64, 31), (1, 1), (2, 9, 513), (5, 128, 16)]
    t = lambda a: torch.from_numpy(a.astype(np.float32)).to(gpu)  # noqa: E731
    ps = [t(rng.standard_normal(s) * 0.1).to(BF16 if masters else F32) for s in shapes]
    gs = [t(rng.standard_normal(s) * 1e-3) for s in shapes]
    opt = Muon(ps, gs, lr=0.05, momentum=0.9, nesterov=nesterov, weight_decay=0.1, scale=0.5, masters=masters,
               zero_grads=True, steps=13)
    clip = torch.full((1,), 0.7, device=gpu)
    mu, k = float(np.float32(0.9)), float(np.float32(0.7))
    f32 = lambda a: a.astype(np.float32).astype(np.float64)  # noqa: E731
    for step in range(2):
        if step:
            for g, s in zip(gs, shapes):
                g.copy_(t(rng.standard_normal(s) * 1e-3))
        fp, fm, fg = ([_np(v) for v in vs] for vs in (opt.masters or ps, opt.states, gs))
        opt.step(grad_scale=clip)
        for i, s in enumerate(shapes):
            g = f32(fg[i] * k)
            m = _np(opt.states[i])
            assert np.all(np.abs(m - (mu * fm[i] + g)) <= U * np.abs(m) + 1e-44)
            u = f32(mu * m + g) if nesterov else m
            got = _np((opt.masters or ps)[i])
            move = ((fp[i] * (1 - 0.05 * 0.1) - got) / (0.05 * 0.5)).reshape(-1, *s[-2:])
            # decay, move and their sum: 4 roundings of fp32
            slack = (4 * U * (np.abs(fp[i]) + np.abs(got)) / (0.05 * 0.5)).reshape(-1, *s[-2:])
            for mv, uu, sl in zip(move, u.reshape(-1, *s[-2:]), slack):
                exact = R.newton_schulz(uu / np.linalg.norm(uu), USUAL, 13)
                lim = 2.0 ** -22 * np.linalg.norm(exact) + 2.0 ** -49 * USUAL[0] ** 13 + np.linalg.norm(sl)
                assert np.linalg.norm(mv - exact) <= lim, (s, np.linalg.norm(mv - exact), lim)
            if masters:
                assert torch.equal(ps[i], opt.masters[i].to(BF16))
            assert not gs[i].any()


def test_small_sides_captured(gpu):
    """Several stages in a graph, replayed: what a call gives."""
    from paper_2606_11867_amd.optimizer import Muon
    rng = np.random.default_rng(8)
    shapes = [(2, 40, 100), (130, 20)]
    new = lambda: [torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(gpu) for s in shapes]  # noqa: E731
    start = [torch.randn(s, device=gpu) for s in shapes]

    def make():
        ps = [t.clone() for t in start]
        gs = [torch.zeros_like(t) for t in ps]
        return ps, gs, Muon(ps, gs, lr=0.01, zero_grads=True, steps=16)

    (pa, ga, a), (pb, gb, b) = make(), make()
    side = torch.cuda.Stream(gpu)
    side.wait_stream(torch.cuda.current_stream(gpu))
    with torch.cuda.stream(side):
        a.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    for t, s in zip(pa, start):
        t.copy_(s)
    for t in a.states:
        t.zero_()
    for _ in range(3):
        for g, h, v in zip(ga, gb, new()):
            g.copy_(v)
            h.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        b.step()
        for x, y in zip((*pa, *a.states, *ga), (*pb, *b.states, *gb)):
            assert torch.equal(x, y)


@pytest.mark.parametrize("coef,steps", [((15.0, 0.0, 0.0), 2), ((1.0, 125.0, 125.0), 1), ((4.0, -5.0, 2.03), 2)])
def test_large_sides_up_to_the_range_of_fp16(gpu, coef, steps):
    """The largest coefficients that are not refused, on the singular values that
    they drive furthest: 1 alone, and 200 of up to 1."""
    from paper_2606_11867_amd.optimizer import Muon
    print(f"\n[case] muon, {steps} steps of {coef}", flush=True)
    rng = np.random.default_rng(11)
    for kind in ("rank 1", "steep", "full"):
        u = matrix(rng, (200, 330), kind)
        g = torch.from_numpy(u.astype(np.float32)).to(gpu)
        p = torch.zeros_like(g)
        Muon([p], [g], lr=1.0, momentum=0.0, nesterov=False, scale=-1.0, steps=steps, coefficients=coef).step()
        u = u / np.linalg.norm(u)
        exact, held = R.newton_schulz(u, coef, steps), R.newton_schulz_held(u, coef, steps)
        # the format's roundings and fp32 sums in another order, as in test_gpu_muon.py
        lim = 3 * np.linalg.norm(held - exact) + 2.0 ** -18 * np.linalg.norm(exact)
        assert np.linalg.norm(_np(p) - exact) <= lim and lim <= 2.0 ** -8 * np.linalg.norm(exact), (kind, lim)


@pytest.mark.parametrize("steps", [5, 6, 8, 10, 12, 16])
@pytest.mark.parametrize("shape", [(130, 300), (300, 130), (256, 256), (66, 70)])
def test_large_sides(gpu, shape, steps):
    """Both sides above 64: within what the header says, 2^-8 of the norm, twice
    that after 16 steps, and 2^-22 a^steps for the rounding of X in directions
    that u does not have; within three times what the oracle's model
    of the format gives as long as that is small; and always a matrix whose
    singular values the iteration bounds (by 1.2024)."""
    from paper_2606_11867_amd.optimizer import Muon
    print(f"\n[case] muon {shape}, {steps} steps", flush=True)
    rng = np.random.default_rng(steps)
    for kind in KINDS:
        u = matrix(rng, shape, kind)
        g = torch.from_numpy(u.astype(np.float32)).to(gpu)
        p = torch.zeros_like(g)
        Muon([p], [g], lr=1.0, momentum=0.0, nesterov=False, scale=-1.0, eps=0.0, steps=steps).step()
        got, u = _np(p), u / np.linalg.norm(u)
        exact, held = R.newton_schulz(u, USUAL, steps), R.newton_schulz_held(u, USUAL, steps)
        n, fill = np.linalg.norm(exact), 2.0 ** -22 * USUAL[0] ** steps
        off = np.linalg.norm(got - exact)
        assert off <= 2.0 ** -8 * (1 + steps / 16) * n + fill, (kind, off, n)
        if fill < 2.0 ** -6 * n:
            assert off <= 3 * np.linalg.norm(held - exact) + 2.0 ** -18 * n, (kind, off, n)
        assert np.linalg.norm(got, 2) <= 1.2024 * (1 + 2.0 ** -6), kind


@pytest.mark.parametrize("eps", [0.0, 5e-324, 1e-310, 1e-200, 1e-100, 1e-7, 1e300])
@pytest.mark.parametrize("shape", [(3, 40, 50), (3, 90, 70)])
def test_nothing_does_not_move_whatever_eps(gpu, shape, eps):
    """The inverse of the least eps is infinite, and that of others squared; the
    matrices beside the empty one go by the larger of their norm and eps."""
    from paper_2606_11867_amd.optimizer import Muon
    print(f"\n[case] muon {shape} eps={eps}", flush=True)
    rng = np.random.default_rng(4)
    u = np.stack([matrix(rng, shape[1:], "full") for _ in range(3)])
    u[1] = 0.0
    for steps in (0, 5, 13):
        g = torch.from_numpy(u.astype(np.float32)).to(gpu)
        p = torch.ones(shape, device=gpu)
        Muon([p], [g], lr=1.0, momentum=0.0, nesterov=False, scale=-1.0, eps=eps, steps=steps).step()
        assert bool((p[1] == 1.0).all())
        for i in (0, 2):
            exact = R.newton_schulz(u[i] / max(np.linalg.norm(u[i]), eps), USUAL, steps)
            # X of its format, and p = 1 + X in fp32
            lim = 2.0 ** -7 * np.linalg.norm(exact) + 2.0 ** -23 * np.linalg.norm(1 + exact)
            assert np.linalg.norm(_np(p[i]) - 1 - exact) <= lim, (steps, i)


def test_coefficients_are_three(gpu):
    """Two would leave the last at 0."""
    from paper_2606_11867_amd.optimizer import Muon
    p, g = torch.ones(8, 8, device=gpu), torch.ones(8, 8, device=gpu)
    for bad in ((1.5, -0.5), (1.0, 2.0, 3.0, 4.0)):
        with pytest.raises(ValueError):
            Muon([p], [g], coefficients=bad)
        opt = Muon([p], [g])
        opt.coefficients = bad
        with pytest.raises(ValueError):
            opt.step()
    assert bool((p == 1).all())
