"""Coefficients of a Muon step that fp16 cannot hold are refused before any launch,
where a matrix has both sides above 64."""
import ctypes
import os

import numpy as np
import pytest

FAKE = 0x10000  # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    import paper_2606_11867_amd as fm
    if not os.path.exists(fm.LIB_PATH):
        from paper_2606_11867_amd import build
        build.build()
    return fm.load()


def call(lib, coef, steps, *shapes):
    """-2: refused for its coefficients; -1: not, only for want of a workspace."""
    from paper_2606_11867_amd import _lib
    recs = (_lib.MuonTensor * len(shapes))(*(_lib.MuonTensor(FAKE, FAKE, None, FAKE, 1, r, c, 0.0, 1.0)
                                             for r, c in shapes))
    return lib.foremoe_muon_step(recs, len(shapes), 0, 0, 1e-3, 0.9, 1, steps, (ctypes.c_double * 3)(*coef), 1e-7, None,
                                 0, None, 0, None)


def most(coef, steps):
    """The largest s^2 and |b s^2 + c s^4| on the way, over 10^5 singular values in [0, 1]."""
    a, b, c = coef
    s, top = np.linspace(0, 1, 100001), 0.0
    with np.errstate(all="ignore"):
        for _ in range(steps):
            # of the whole interval that they have reached
            s = np.linspace(0, np.abs(s).max(), 100001)
            top = max(top, (s * s).max(), np.abs(b * s ** 2 + c * s ** 4).max())
            s = a * s + b * s ** 3 + c * s ** 5
    return top


USUAL = (3.4445, -4.7750, 2.0315)


@pytest.mark.parametrize("coef", [USUAL, (1.5, -0.5, 0.0), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375), (15.0, 0.0, 0.0),
                                  (1.0, 125.0, 125.0), (1.0, 126.0, 125.0), (4.0, -5.0, 2.03), (-3.0, 4.0, -1.5),
                                  (1.0, 1500.0, -1500.0), (0.0, 0.0, 0.0), (0.0, 3.0, 0.0), (2.0, 0.0, -1.0),
                                  (1e300, -1e300, 1e300), (0.0, 1e300, -1e300)])
def test_coefficients(lib, coef):
    for steps in range(17):
        top = most(coef, steps)
        assert not 249.9 < top < 250.1 or coef == (1.0, 125.0, 125.0)
        want = -1 if top <= 250.0 else -2
        assert call(lib, coef, steps, (65, 65)) == want, (steps, top)
        assert call(lib, coef, steps, (64, 3), (3, 700), (70, 900)) == want
        assert call(lib, coef, steps, (64, 3000), (3000, 64), (1, 1)) == -1  # fp64
    if -2 in [call(lib, coef, s, (65, 65)) for s in (1, 16)]:
        assert b"coef" in lib.foremoe_last_error()
    if coef == USUAL:
        assert call(lib, coef, 16, (4096, 4100)) == -1


def test_workspace_of_small_matrices(lib):
    """By their tiles of 16: a batch of as many tiny ones as are accepted fits beside them."""
    from paper_2606_11867_amd import _lib

    def size(batch, r, c):
        return lib.foremoe_muon_workspace_size((_lib.MuonTensor * 1)(_lib.MuonTensor(None, None, None, None, batch, r, c,
                                                                                    0.0, 1.0)), 1)

    for (r, c), t, pieces in (((1, 1), 1, 1), ((16, 64), 1, 1), ((17, 65), 2, 2), ((64, 64), 4, 1), ((1000, 60), 4, 16),
                              ((5, 1 << 20), 1, 64)):
        for batch in (1, 7) if c > 100 else (1, 7, 1 << 19):
            if batch == 1 << 19 and r > 256:
                continue
            need = batch * (2048 * (pieces * (t * (t + 1) // 2) + t * t) + 8 + 8 * r * c)
            assert need <= size(batch, r, c) <= need + 4 * 256
