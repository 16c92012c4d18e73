"""The AdamW step at the ends of fp32's range and at the last bit of its
reciprocals and square roots.

Bounds, u = 2^-24: a move is a quotient of the stored moments times two
factors rounded to fp32: within 32 u of itself, as for ordinary values.
"""
import numpy as np
import pytest
import torch

import oracle.foremoe_step as S

U = 2.0 ** -24
F32 = torch.float32


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param", ["f32", "bf16"])
@pytest.mark.parametrize("big", [1e20, -3e38])
def test_finite_gradient_whose_square_is_not(gpu, bits, param, big):
    """v is infinite, m finite: m / inf = 0, so the parameter stays."""
    from paper_2606_11867_amd.optimizer import AdamW
    p = torch.ones(1000, device=gpu, dtype=torch.bfloat16 if param == "bf16" else F32)
    g = torch.full((1000,), 0.1, device=gpu)
    g[300] = big
    opt = AdamW([p], [g], lr=0.1, state_bits=bits)
    opt.step()
    where = torch.arange(1000, device=gpu) == 300
    for t in [p, *(opt.masters or ())]:
        assert torch.isfinite(t).all() and t[300] == 1.0 and torch.all(t[~where] < 0.95)
    if bits == 32:
        assert torch.isfinite(opt.states[0][0]).all() and torch.isinf(opt.states[0][1][300])
        opt.step()
        assert torch.isfinite(p).all() and p[300] == 1.0


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_second_moments_below_the_normal_numbers(gpu, bits):
    """eps = 0 and gradients whose squares are subnormal: the move is about lr
    all the same. Where the square is 0 in fp32, so is the denominator, and
    the element does not move."""
    from paper_2606_11867_amd.optimizer import AdamW
    sizes = np.array([1e-18, 5e-19, 1e-19, 3e-20, 1e-21, 1e-22, 1e-25, 0.0], dtype=np.float32)
    signs = np.where(np.arange(1024) % 3 == 0, -1, 1).astype(np.float32)
    gn = np.repeat(sizes, 128) * signs
    g = torch.from_numpy(gn).to(gpu)
    p = torch.zeros(1024, device=gpu)
    lr, b1, b2 = 0.1, 0.9, 0.95
    opt = AdamW([p], [g], lr=lr, betas=(b1, b2), eps=0.0, state_bits=bits)
    opt.step()
    f = np.float32
    m, v = gn * f(1 - b1), (gn * gn) * f(1 - b2)
    if bits == 32:
        assert np.array_equal(opt.states[0][1].cpu().numpy(), v)
    m, v = m.astype(np.float64), v.astype(np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        want = np.where(v > 0, -lr * m / (1 - b1) / np.sqrt(v / (1 - b2)), 0.0)
    assert np.count_nonzero(v) == 5 * 128 and np.abs(want[v > 0]).min() > 0.09
    got = p.double().cpu().numpy()
    assert np.all(np.abs(got - want) <= 32 * U * np.abs(want)), np.abs(got - want).reshape(8, 128).max(1)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_eps_below_the_normal_numbers(gpu, bits):
    from paper_2606_11867_amd.optimizer import AdamW
    eps = 1e-40
    g = torch.zeros(600, device=gpu)
    g[::3] = 1e-3
    p = torch.zeros(600, device=gpu)
    opt = AdamW([p], [g], lr=0.1, eps=eps, state_bits=bits)
    opt.step()
    want = torch.zeros(600, device=gpu)
    want[::3] = -0.1
    assert torch.all((p - want).abs() <= 64 * U * want.abs())


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_no_gradient_and_no_eps_is_no_move(gpu, bits):
    from paper_2606_11867_amd.optimizer import AdamW
    ps = [torch.zeros(n, device=gpu) for n in (1, 255, 256, 700)]
    gs = [torch.zeros_like(p) for p in ps]
    opt = AdamW(ps, gs, lr=0.5, eps=0.0, state_bits=bits)
    for _ in range(2):
        opt.step()
    for p in ps:
        assert torch.all(p == 0)


# ---------------------------------------------------------------------------
# The last bit. A quotient 1 / x and a square root of fp32 numbers, taken in
# 64 bits and rounded to 32, are correctly rounded (64 bits have more than
# twice the digits of 32, and two more).
# ---------------------------------------------------------------------------
BLOCK = 256
CHUNK = 1 << 15  # blocks of a call


def _rounded_codes(x, shift, one, least):
    """Codes of ratios x >= 0, to nearest, ties to even patterns."""
    b = x.view(torch.int32)
    c = ((b + ((1 << (shift - 1)) - 1) + ((b >> shift) & 1)) >> shift) - ((0x3F800000 >> shift) - one)
    return torch.where(x > 0, c.clamp(least, one), torch.zeros_like(c)).to(torch.uint8)


def _beside_the_boundaries(scale, table):
    """[blocks, 256]: the scale, then numbers at its ratios halfway between
    two codes and one step to either side."""
    mid = (table[1:-1] + table[2:]) / 2
    mid = torch.from_numpy(np.sort(mid[np.linspace(0, len(mid) - 1, 85).astype(int)])).to(scale.device)
    a = (scale.double()[:, None] * mid).float()
    bits = a.view(torch.int32)
    return torch.cat([scale[:, None], a, (bits - 1).view(F32), (bits + 1).view(F32)], 1)


def test_boundaries_tell_a_neighbouring_reciprocal():
    """On the CPU: a reciprocal that is off by one unit in the last place
    gives other codes of the blocks below, the all-ones significand's too."""
    rng = np.random.default_rng(5)
    bits = np.concatenate([rng.integers(0x3F800001, 0x40000000, 200), [0x3FFFFFFF, 0x3F800001]]).astype(np.int32)
    scale = torch.from_numpy(bits.view(np.float32))
    a = _beside_the_boundaries(scale, S.TABLE_M)
    right = (1.0 / scale.double()).float()
    for step in (-1, 1):
        off = (right.view(torch.int32) + step).view(F32)
        same = (_rounded_codes(a * right[:, None], 20, 127, 0) == _rounded_codes(a * off[:, None], 20, 127, 0)).all(1)
        assert not same.any()


@pytest.mark.gpu
def test_reciprocal_of_every_significand(gpu):
    """Blocks whose scale has each of the 2^23 significands, with elements at
    the boundaries of the codes: codes as with 1 / scale rounded once. The
    method's known exception, a significand of all ones, is among them."""
    from paper_2606_11867_amd.optimizer import AdamW
    g = torch.empty(CHUNK * BLOCK, device=gpu)
    p = torch.zeros_like(g)
    opt = AdamW([p], [g], lr=0.0, betas=(0.0, 0.0), state_bits=8)  # m = g
    for first in range(0, 1 << 23, CHUNK):
        if first % (CHUNK * 64) == 0:
            print(f"[case] significands from {first}", flush=True)
        # exponents from 2^-60 to 2^60 in turn
        i = torch.arange(first, first + CHUNK, device=gpu, dtype=torch.int32)
        scale = (i | ((127 - 60 + (first // CHUNK) % 121) << 23)).view(F32)
        a = _beside_the_boundaries(scale, S.TABLE_M)
        g.copy_(a.reshape(-1))
        opt.step()
        want = _rounded_codes((a * (1.0 / scale.double()).float()[:, None]), 20, 127, 0)
        assert torch.equal(opt.states[0][2], scale)
        assert torch.equal(opt.states[0][0], want.reshape(-1)), first


@pytest.mark.gpu
def test_square_root_of_every_significand(gpu):
    """Every second moment from 1 to 4 (each significand at both parities of
    the exponent), and as many spread over the exponents, made exactly from an
    old moment and a gradient; its root is the block's scale."""
    from paper_2606_11867_amd.optimizer import AdamW
    g = torch.zeros(CHUNK, BLOCK, device=gpu)
    p = torch.zeros(CHUNK * BLOCK, device=gpu)
    opt = AdamW([p], [g.view(-1)], lr=0.0, betas=(0.0, 0.5), state_bits=8)
    m, v, ms, vs = opt.states[0]
    missed = 0
    for first in range(0, 1 << 24, CHUNK):
        if first % (CHUNK * 128) == 0:
            print(f"[case] patterns from {first}", flush=True)
        i = torch.arange(first, first + CHUNK, device=gpu, dtype=torch.int32)
        for spread in (False, True):
            e = 2 * (((first // CHUNK) * 37) % 100 - 42) if spread else 0  # 2^-84 to 2^114
            target = (i + 0x3F800000).view(F32) * 2.0 ** e
            # (s^2 + g^2) / 2, each square rounded
            s = torch.sqrt(2 * target.double()).float()
            s = torch.where(s * s > 2 * target, (s.view(torch.int32) - 1).view(F32), s)
            rest = 2 * target - s * s
            small = torch.sqrt(rest.double()).float()
            made = (s * s) * 0.5 + (small * small) * 0.5
            missed += int((made != target).sum())
            v.zero_()
            v.view(CHUNK, BLOCK)[:, 0] = 255
            vs.copy_(s)
            g[:, 0] = small
            opt.step()
            assert torch.equal(vs, torch.sqrt(made.double()).float()), (first, spread)
    assert missed == 0
