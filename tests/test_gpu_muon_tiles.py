"""Muon over batches for which the step takes 256-wide tiles, whole steps: decay,
clipping, masters, cleared gradients, sides of either order, odd widths.

m: a product and a sum in fp32. X of a Gaussian matrix is off by about 2^-9 of its
norm, by roundings of fp16 that are independent from element to element: eight
times their spread, 2^-6 of the elements' root mean square, holds for every one of
some 10^7. An element from another place is off by more than its own size.
"""
import pytest
import torch

from test_gpu_muon_steps import USUAL

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def iterate(u):
    """The exact iteration on one matrix, on the GPU."""
    a, b, c = USUAL
    x = u.t().contiguous() if u.shape[0] > u.shape[1] else u
    x = x / x.norm()
    for _ in range(5):
        g = x @ x.t().contiguous()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.t() if u.shape[0] > u.shape[1] else x


def padded(shape, tile):
    """The least workspace of this padding."""
    b, (m, n) = shape[0], (-(-s // tile) * tile for s in sorted(shape[1:]))
    return b * (8 * m * n + 4 * m * m)


# (all products by 256-wide tiles, or all but G and P)
SHAPES = [(64, 500, 700), (64, 700, 500), (60, 505, 509), (60, 509, 505), (40, 513, 770), (43, 767, 501),
          (64, 767, 255)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("param,masters,grad", [(F32, False, F32), (BF16, True, F32), (BF16, False, BF16)],
                         ids=["f32", "bf16-masters", "bf16"])
def test_wide_tiles(gpu, shape, param, masters, grad):
    from paper_2606_11867_amd.optimizer import Muon
    print(f"\n[case] muon {shape} {param} masters={masters} {grad}", flush=True)
    gen = torch.Generator(device=gpu).manual_seed(shape[1])
    randn = lambda: torch.randn(shape, generator=gen, device=gpu)  # noqa: E731
    p, g, m = (0.1 * randn()).to(param), (1e-3 * randn()).to(grad), 1e-2 * randn()
    fp = p.double() if not masters else None
    opt = Muon([p], [g], lr=0.5, momentum=0.9, weight_decay=0.1, scale=2.0, masters=masters, states=[m], zero_grads=True)
    assert opt.ws.numel() >= padded(shape, 256)
    if masters:
        fp = opt.masters[0].double()
        assert torch.equal(fp, p.double())
        opt.masters[0].add_(1e-5 * randn())
        fp = opt.masters[0].double()
    fm, fg = m.double(), g.double()
    clip = torch.full((1,), 0.7, device=gpu)
    opt.step(grad_scale=clip)
    k, mu = float(clip), float(torch.tensor(0.9))
    assert bool(((m.double() - (mu * fm + k * fg)).abs() <= 4 * U * (fm.abs() + fg.abs())).all())
    got = (opt.masters[0] if masters else p).double()
    for i in range(shape[0]):
        x = iterate(k * fg[i] + mu * m[i].double())
        rms = float(x.norm()) / x.numel() ** 0.5
        want = fp[i] * (1 - 0.5 * 0.1) - x
        lim = 2.0 ** -6 * rms + 4 * U * (fp[i].abs() + want.abs())
        if param is BF16 and not masters:
            lim = lim + 2.0 ** -8 * want.abs() * (1 + 2.0 ** -6)
        assert bool(((got[i] - want).abs() <= lim).all()), (i, float(((got[i] - want).abs() - lim).max()))
    if masters:
        assert torch.equal(p, opt.masters[0].to(BF16))
    assert not g.any()


def test_far_matrices_to_the_last_bit(gpu):
    """More than 2^31 elements: the first and the last matrix move as they do
    alone. A matrix by itself takes the same tiles (256 everywhere), each of which
    sums in the order of its own k axis."""
    from paper_2606_11867_amd.optimizer import Muon
    shape = (130, 4096, 4100)
    print(f"\n[case] muon {shape}", flush=True)
    g = torch.zeros(shape, device=gpu)
    gen = torch.Generator(device=gpu).manual_seed(3)
    for i in (0, 129):
        g[i].normal_(generator=gen)
    p = torch.zeros(shape, device=gpu)
    Muon([p], [g], lr=1.0, momentum=0.0, nesterov=False, scale=-1.0).step()
    assert not p[1:129].any()
    for i in (0, 129):
        q = torch.zeros(shape[1:], device=gpu)
        Muon([q], [g[i]], lr=1.0, momentum=0.0, nesterov=False, scale=-1.0).step()
        assert torch.equal(p[i], q)
        x = iterate(g[i].double())
        # every element, as above
        assert float((q.double() - x).abs().max()) <= 2.0 ** -6 * float(x.norm()) / x.numel() ** 0.5
        del x, q
