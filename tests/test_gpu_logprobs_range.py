"""Log-probabilities of rows far from zero, and of more rows than one launch
takes, against the fp64 oracle.

Bounds, u = 2^-24. Where logits are so large that a scaled one has no fraction
left, differences from the row's maximum are taken before they are scaled:
exact, or rounded once, then scaled by a constant rounded once. A
log-probability d - log s is then within 8 u |d| + u (V / 256 + 128), an
entropy within that times (2 + H), lse within 8 u of itself.
"""
import numpy as np
import pytest
import torch

import oracle.foremoe_step as S
import test_gpu_logprobs as base

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
INF = float("inf")


def _far_rows(V, dtype, rng):
    """Rows of one value, of values a few steps of the type apart, and of far
    values beside a masked half."""
    rows = []
    top = float(torch.finfo(dtype).max)
    for base_value in (-1e4, -1e7, -1e8, -1e9, -1e12, -1e30, -top, 1e6, 3e7, 1e10, 1e20, top):
        v = float(torch.tensor(base_value).to(dtype))
        rows.append(np.full(V, v))
        step = 2.0 ** (np.floor(np.log2(abs(v))) - (7 if dtype == torch.bfloat16 else 23))
        rows.append(v - np.sign(v) * step * rng.integers(0, 4, V))
        rows.append(np.where(np.arange(V) % 2 == 0, v, -INF))
    return np.stack(rows)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [5, 3001, 40003])
@pytest.mark.parametrize("temperature", [1.0, 0.7, 1.3, 50.0])
@pytest.mark.parametrize("split", [True, False], ids=["ws", "no-ws"])
def test_rows_far_from_zero(gpu, dtype, V, temperature, split):
    from paper_2606_11867_amd import api
    rng = np.random.default_rng(V)
    x = torch.from_numpy(_far_rows(V, dtype, rng).astype(np.float32)).to(dtype)
    l = x.double().numpy()
    N = len(l)
    T = float(np.float32(temperature))
    l = l[np.abs(np.where(np.isfinite(l), l, 0)).max(1) / T <= np.finfo(np.float32).max]  # x / T in fp32's range
    x = torch.from_numpy(l).to(dtype)
    assert len(l) >= N - 6
    N = len(l)
    t = np.array([2 * rng.integers(0, (V + 1) // 2) for _ in range(N)], dtype=np.int32)
    n_top = min(V, 3)
    ref = S.token_logprobs(l, t, temperature=T, n_top=n_top)
    ws = api.logprobs_workspace(gpu) if split else None
    r = api.token_logprobs(x.to(gpu), torch.from_numpy(t).to(gpu), temperature=temperature, n_top=n_top, ws=ws)
    tol = U * (V / 256 + 128)
    base._close("logp", r.logp, ref["logp"], tol + 8 * U * np.abs(ref["logp"]))
    base._close("entropy", r.entropy, ref["entropy"], (tol + 64 * U) * (2 + ref["entropy"]))
    base._close("lse", r.lse, ref["lse"], tol + 8 * U * np.abs(ref["lse"]))
    assert np.array_equal(r.top_ids.cpu().numpy(), ref["top_ids"])
    near = np.where(np.isfinite(ref["top_logp"]), ref["top_logp"], 0.0)
    base._close("top_logp", r.top_logp, ref["top_logp"], tol + 8 * U * np.abs(near))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("temperature", [1.0, 0.7, 1.3, 50.0])
def test_gradients_of_rows_far_from_zero_are_bounded(gpu, dtype, temperature):
    """An fp32 lse of 1e9 does not hold the logarithm of a sum any more, and
    a gradient from it is not the formula's; but no p exceeds 1, so it stays
    within the formula's largest terms."""
    from paper_2606_11867_amd import api
    V = 1001
    rng = np.random.default_rng(3)
    l = _far_rows(V, dtype, rng)
    l = l[np.abs(np.where(np.isfinite(l), l, 0)).max(1) / temperature <= np.finfo(np.float32).max]
    x = torch.from_numpy(l).to(dtype).to(gpu)
    N = len(l)
    t = torch.zeros(N, dtype=torch.int32, device=gpu)
    a = torch.from_numpy(rng.standard_normal(N).astype(np.float32)).to(gpu)
    b = torch.from_numpy(rng.standard_normal(N).astype(np.float32)).to(gpu)
    r = api.token_logprobs(x, t, temperature=temperature)
    d = api.token_logprobs_bwd(x, t, r.lse, a, entropy=r.entropy, dentropy=b, temperature=temperature).float()
    # |dlogp| (1 + p) + |dentropy| (p |log p| + p H), p |log p| <= 1 / e
    most = (2 * a.abs() + b.abs() * (0.5 + r.entropy)) / temperature
    assert torch.isfinite(d).all()
    assert torch.all(d.abs() <= 1.01 * most[:, None])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N", [70001, (1 << 22) + 1003])
def test_more_rows_than_a_launch_takes(gpu, dtype, N):
    """Short rows past the backward's 65535 and the forward's 2^22: rows from
    the start, around every end of a launch and from the end."""
    from paper_2606_11867_amd import api
    print(f"\n[case] logprobs rows N={N}", flush=True)
    V = 9
    gen = torch.Generator(device=gpu).manual_seed(N)
    x = (torch.randn(N, V, generator=gen, device=gpu) * 3).to(dtype)
    t = torch.randint(-1, V, (N,), generator=gen, device=gpu).to(torch.int32)
    a, b = torch.randn(N, generator=gen, device=gpu), torch.randn(N, generator=gen, device=gpu)
    r = api.token_logprobs(x, t, n_top=2, ws=api.logprobs_workspace(gpu))
    d = api.token_logprobs_bwd(x, t, r.lse, a, entropy=r.entropy, dentropy=b)
    ends = [0, N] + list(range(65535, N, 65535))[:3] + list(range(65535, N, 65535))[-3:] + [1 << 22]
    rows = np.unique(np.concatenate([np.arange(e - 20, e + 20) for e in ends]))
    rows = rows[(rows >= 0) & (rows < N)]
    pick = torch.from_numpy(rows).to(gpu)
    l, tt, an, bn = x[pick].double().cpu().numpy(), t[pick].cpu().numpy(), a[pick].cpu().numpy(), b[pick].cpu().numpy()
    ref = S.token_logprobs(l, tt, n_top=2)
    tol = U * (16 * np.abs(l).max() + V / 256 + 128)
    base._close("logp", r.logp[pick], ref["logp"], tol)
    base._close("entropy", r.entropy[pick], ref["entropy"], tol * (2 + ref["entropy"]))
    assert np.array_equal(r.top_ids[pick].cpu().numpy(), ref["top_ids"])
    want = S.token_logprobs_backward(l, tt, an, bn)
    size = (np.abs(an) + np.abs(bn) * (2 + ref["entropy"]) * 2)[:, None]
    base._close("dlogits", d[pick], want, 4 * tol * size)
    # every row: the gradients of a softmax sum to 0, each within 2^-8 of itself at worst
    assert torch.all(d.float().sum(1).abs() <= 2.0 ** -8 * (2 * a.abs() + 2 * b.abs() * r.entropy.abs()) + 1e-4)
