"""The layer for a few tokens where weights of the second product are infinite or
NaN: hidden rows are held in two or three bf16 planes, of which the later ones may
be 0 or of the other sign. The sum is what the exact one is; the columns
beside it, and the tokens of other experts, keep their bits."""
import numpy as np
import pytest
import torch

import oracle.foremoe_rollout as R
from test_gpu_few_tokens import BF16, _case, _np, _run

pytestmark = pytest.mark.gpu

# (8 or 16 columns of a tile; few and many pairs; parts of the k axis; long rows)
SIZES = [dict(T=1, d=256, F=128, E=16, W=16, K=4), dict(T=24, d=512, F=200, E=32, W=32, K=8),
         dict(T=40, d=2304, F=72, E=6, W=6, K=3), dict(T=128, d=2312, F=64, E=8, W=8, K=6),
         dict(T=3, d=1056, F=1121, E=5, W=5, K=5)]


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("w", ["bf16", "f32"])
@pytest.mark.parametrize("size", range(len(SIZES)))
def test_infinite_weights(gpu, size, w, out):
    print(f"\n[case] few, infinite weights {SIZES[size]} {w} {out}", flush=True)
    rng = np.random.default_rng(size)
    c = _case(rng, gpu, x=w, w=w, **SIZES[size])
    c["gates"] = (c["gates"] + 0.1).astype(np.float32)
    W, d, F = c["dn_v"].shape
    # hidden elements of exactly 0 have no sum: none here is below fp32's normal numbers
    x = _np(c["x"])
    clean = _run(c, gpu, out)
    at = np.full(len(c["widx"]), -1) if c["widx"] is None else c["widx"]
    cols = rng.choice(d, 12, replace=False)
    for n, col in enumerate(cols):
        e = int(rng.integers(W))
        # one of an expert's row, several of one sign, one of each of two experts, a NaN among others
        for v in ([np.inf], [-np.inf], [np.inf, np.inf], [np.inf, -np.inf], [np.nan], [np.inf, np.nan])[n % 6]:
            f = int(rng.integers(F))
            c["dn"][e, col, f] = v
            c["dn_v"][e, col, f] = v
            e = (e + n // 6) % W
    got = _run(c, gpu, out)
    with np.errstate(invalid="ignore"):
        ref = R.few_tokens(x, c["ids"], c["gates"].astype(np.float64), c["gu_v"], c["dn_v"], at)
    bad = ~np.isfinite(ref)
    assert bad.any() and np.isinf(ref).any()
    g = _np(got)
    assert np.array_equal(np.isnan(g), np.isnan(ref))
    assert np.array_equal(g[np.isinf(ref)], ref[np.isinf(ref)])
    keep = torch.from_numpy(~bad).to(gpu)
    bits = torch.int16 if got.dtype is BF16 else torch.int32
    assert torch.equal(got.view(bits)[keep], clean.view(bits)[keep])
