"""What the entry points of 4-bit floats, the layer for a few tokens and Muon
refuse, on the host, before any launch."""
import ctypes
import os

import pytest
import torch

FAKE = 0x10000  # never dereferenced: validation fails first
NAN = float("nan")


@pytest.fixture(scope="module")
def lib():
    import paper_2606_11867_amd as fm
    if not os.path.exists(fm.LIB_PATH):
        from paper_2606_11867_amd import build
        build.build()
    return fm.load()


def test_quantize_refuses(lib):
    ok = dict(x=FAKE, dtype=1, ld=64, rows=4, cols=64, n_rows=None, codes=FAKE, scales=FAKE)

    def call(**kw):
        return lib.foremoe_mxfp4_quantize(*{**ok, **kw}.values(), None)

    for kw in (dict(dtype=2), dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=1 << 31, ld=1 << 31),
               dict(ld=63), dict(ld=(1 << 32) + 1), dict(x=None), dict(codes=None), dict(scales=None), dict(x=FAKE + 1),
               dict(dtype=0, x=FAKE + 2), dict(codes=FAKE + 8), dict(n_rows=FAKE + 2)):
        assert call(**kw) == -1, kw
    assert b"mxfp4_quantize" in lib.foremoe_last_error()
    assert call(rows=0, x=None, codes=None, scales=None) == 0


def test_values_refuses(lib):
    ok = dict(codes=FAKE, scales=FAKE, rows=4, cols=64, out=FAKE, dtype=0, ld=64)

    def call(**kw):
        return lib.foremoe_mxfp4_values(*{**ok, **kw}.values(), None)

    for kw in (dict(dtype=5), dict(rows=-1), dict(cols=0), dict(ld=60), dict(codes=None), dict(scales=None),
               dict(out=None), dict(out=FAKE + 2), dict(codes=FAKE + 4)):
        assert call(**kw) == -1, kw
    assert call(rows=0, out=None) == 0


def test_grouped_ffn_mxfp4_refuses(lib):
    n = lib.foremoe_ffn_mxfp4_workspace_size(100, 256)
    assert n >= 100 * 256 * 17 // 32
    for bad in ((-1, 256), (1 << 31, 256), (10, 0), (10, 100)):
        assert lib.foremoe_ffn_mxfp4_workspace_size(*bad) == 0
    ok = dict(xc=FAKE, xs=FAKE, d=128, F=256, S=2, off=FAKE, widx=FAKE, W=2, gc=FAKE, gs=FAKE, dc=FAKE, ds=FAKE,
              n_cap=100, y=FAKE, ws=FAKE, ws_bytes=n)

    def call(**kw):
        return lib.foremoe_grouped_ffn_mxfp4_fwd(*{**ok, **kw}.values(), None)

    for kw in (dict(d=0), dict(F=0), dict(S=-1), dict(S=1025), dict(W=0), dict(n_cap=-1), dict(n_cap=1 << 31),
               dict(xc=None), dict(ws=None), dict(y=None), dict(ws_bytes=n - 1), dict(ws=FAKE + 128),
               dict(xc=FAKE + 8), dict(gs=FAKE + 2), dict(y=FAKE + 8), dict(off=FAKE + 1)):
        assert call(**kw) == -1, kw
    for kw in (dict(d=64), dict(F=192), dict(d=1 << 17, F=1 << 14)):
        assert call(**kw) == -2, kw
    assert call(S=0) == 0 and call(n_cap=0) == 0


@pytest.mark.parametrize("mx", [False, True])
def test_few_tokens_refuses(lib, mx):
    n = lib.foremoe_few_workspace_size(8, 4, 96)
    assert n >= 8 * 4 * 96 * 4
    for bad in ((-1, 4, 96), (129, 4, 96), (8, 0, 96), (8, 65, 96), (128, 17, 96), (8, 4, 0)):
        assert lib.foremoe_few_workspace_size(*bad) == 0
    assert lib.foremoe_few_workspace_size(0, 4, 96) == 256
    ok = dict(x=FAKE, dtype=1, ld=64, T=8, d=64, F=96, ids=FAKE, gates=FAKE, K=4, E=16, widx=None, W=16, gu=FAKE,
              gus=FAKE, dn=FAKE, dns=FAKE, y=FAKE, out=1, ws=FAKE, ws_bytes=n)

    def call(**kw):
        c = {**ok, **kw}
        for k in (("dtype",) if mx else ("gus", "dns")):
            c.pop(k)
        return (lib.foremoe_few_tokens_ffn_mxfp4 if mx else lib.foremoe_few_tokens_ffn)(*c.values(), None)

    for kw in (dict(T=-1), dict(T=129), dict(K=0), dict(K=65), dict(T=128, K=17), dict(E=0), dict(E=1025),
               dict(W=0), dict(W=1025), dict(E=17), dict(d=0), dict(F=0), dict(ld=63), dict(d=1 << 16, F=1 << 14, ld=1 << 16),
               dict(out=2), dict(x=None), dict(ids=None), dict(gates=None), dict(gu=None), dict(dn=None), dict(y=None),
               dict(ws=None), dict(ws_bytes=n - 1), dict(ws=FAKE + 64), dict(x=FAKE + 1), dict(gu=FAKE + 8),
               dict(out=0, y=FAKE + 2)):
        assert call(**kw) == -1, kw
    n = lib.foremoe_few_workspace_size(8, 4, 1 << 25)
    for kw in (dict(d=1 << 25, F=1, ld=1 << 25), dict(d=1, F=1 << 25), dict(ld=1 << 30)):
        assert call(ws_bytes=n, **kw) == -2, kw
    if mx:
        assert call(d=48, ld=64) == -2 and call(F=80) == -2
        assert call(x=FAKE + 2) == -1 and call(ld=65) == -1 and call(gus=None) == -1
    else:
        assert call(dtype=2) == -1 and call(dtype=0, x=FAKE + 2) == -1
    assert call(T=0, x=None, ids=None, ws=None, ws_bytes=0) == 0


def test_muon_refuses(lib):
    from paper_2606_11867_amd import _lib

    def rec(**kw):
        r = dict(param=FAKE, grad=FAKE, master=None, m=FAKE, batch=2, rows=5, cols=7, weight_decay=0.0, scale=1.0)
        return _lib.MuonTensor(*{**r, **kw}.values())

    def size(*recs):
        return lib.foremoe_muon_workspace_size((_lib.MuonTensor * len(recs))(*recs), len(recs))

    assert size(rec(rows=100, cols=200)) >= 2 * (4 * 128 * 256 + 2 * 128 * 128) * 2
    for r in (rec(), rec(rows=100, cols=200)):
        assert size(*[r] * 24) == size(*[r] * 30)  # more share it, launch after launch
    for kw in (dict(batch=-1), dict(batch=(1 << 30) + 1), dict(rows=0), dict(cols=0), dict(rows=(1 << 20) + 1),
               dict(rows=16385, cols=16385), dict(batch=1 << 30, rows=64, cols=64)):
        assert size(rec(**kw)) == 0, kw
    assert size() == 256 and lib.foremoe_muon_workspace_size(None, 1) == 0
    ok = dict(n=1, pd=1, gd=0, lr=1e-3, momentum=0.9, nesterov=1, steps=5, coef=(3.4445, -4.775, 2.0315), eps=1e-7,
              gs=None, zero=0, ws=FAKE, ws_bytes=1 << 40)

    def call(r=None, **kw):
        c = {**ok, **kw}
        c["coef"] = (ctypes.c_double * 3)(*c["coef"]) if c["coef"] else None
        arr = (_lib.MuonTensor * 1)(rec() if r is None else r)
        return lib.foremoe_muon_step(arr, *c.values(), None)

    for kw in (dict(n=-1), dict(pd=2), dict(gd=2), dict(lr=NAN), dict(lr=-1.0), dict(momentum=1.0), dict(momentum=-0.1),
               dict(momentum=NAN), dict(steps=-1), dict(steps=17), dict(coef=None), dict(coef=(1.0, NAN, 0.0)),
               dict(eps=-1.0), dict(eps=NAN), dict(gs=FAKE + 1), dict(ws=None), dict(ws=FAKE + 64),
               dict(ws_bytes=size(rec()) - 1)):
        assert call(**kw) == -1, kw
    for kw in (dict(param=None), dict(grad=None), dict(m=None), dict(weight_decay=NAN), dict(scale=NAN),
               dict(param=FAKE + 1), dict(grad=FAKE + 2), dict(m=FAKE + 2), dict(master=FAKE + 2), dict(rows=-1)):
        assert call(rec(**kw)) == -1, kw
    assert call(rec(batch=1 << 30, rows=64, cols=64)) == -2
    assert call(rec(master=FAKE), pd=0) == -1  # a master goes with bf16 parameters
    assert call(n=0, ws=None) == 0 and call(rec(batch=0, param=None), ws=None) == 0
    assert lib.foremoe_muon_step(None, 1, 1, 0, 1e-3, 0.9, 1, 5, (ctypes.c_double * 3)(), 1e-7, None, 0, None, 0, None) == -1


def test_host_tensors_are_refused():
    from paper_2606_11867_amd import api
    from paper_2606_11867_amd.optimizer import Muon
    x = torch.zeros(4, 64)
    q = api.MXFP4(torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8))
    w = api.MXFP4(torch.zeros(1, 4, 32, dtype=torch.uint8), torch.zeros(1, 4, 2, dtype=torch.uint8))
    ids = torch.zeros(4, 2, dtype=torch.int32)
    for call in (lambda: api.mxfp4_quantize(x), lambda: api.mxfp4_quantize(x[None]), lambda: api.mxfp4_values(q),
                 lambda: api.grouped_ffn_mxfp4_fwd(q, ids, ids, w, w),
                 lambda: api.few_tokens_ffn(x, ids, x, torch.zeros(1, 4, 64), torch.zeros(1, 64, 2)),
                 lambda: Muon([x], [x])):
        with pytest.raises((ValueError, TypeError)):
            call()
