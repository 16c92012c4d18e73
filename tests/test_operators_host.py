"""What the entry points of the router, the token log-probabilities and the
AdamW step refuse, on the host, before any launch."""
import ctypes
import os

import pytest
import torch

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: validation fails first
NAN = float("nan")


@pytest.fixture(scope="module")
def lib():
    import paper_2606_11867_amd as fm
    if not os.path.exists(fm.LIB_PATH):
        from paper_2606_11867_amd import build
        build.build()
    return fm.load()


def test_router_fwd_refuses(lib):
    ok = dict(logits=FAKE, dtype=1, ld=64, T=10, E=64, K=8, score=0, renorm=1, scale=1.0, bias=None, mask=None,
              ids_in=None, ids=FAKE, gates=FAKE, counts=None, n_tokens=None, prob_mean=None, loss=None, ws=None,
              ws_bytes=0)

    def call(**kw):
        return lib.foremoe_router_fwd(*{**ok, **kw}.values(), None)

    for kw in (dict(dtype=7), dict(E=0), dict(E=1025, ld=2000), dict(K=0), dict(K=65), dict(E=4, K=5), dict(T=-1),
               dict(T=1 << 30), dict(ld=63), dict(score=2), dict(scale=NAN), dict(logits=None), dict(ids=None),
               dict(gates=None), dict(bias=FAKE), dict(counts=FAKE), dict(logits=0x1001),
               dict(dtype=0, logits=0x1002)):
        assert call(**kw) == -1, kw
    stats = dict(counts=FAKE, n_tokens=FAKE, prob_mean=FAKE, loss=FAKE)
    n = lib.foremoe_router_workspace_size(64)
    assert n > 0 and n % 256 == 0
    assert call(**stats) == -1  # no workspace
    assert call(**stats, ws=FAKE, ws_bytes=n - 1) == -1
    assert b"workspace too small" in lib.foremoe_last_error()
    assert call(**stats, ws=0x1010, ws_bytes=n) == -1
    assert call(T=0, logits=None, ids=None, gates=None) == 0  # nothing to do, nothing launched
    assert lib.foremoe_router_workspace_size(0) == 0 and lib.foremoe_router_workspace_size(1025) == 0


def test_router_bwd_refuses(lib):
    ok = dict(logits=FAKE, dtype=1, ld=64, T=10, E=64, K=8, score=0, renorm=1, scale=1.0, mask=None, ids=FAKE,
              dgates=FAKE, counts=None, n_tokens=None, coef=0.0, dlogits=0x9000, ld_out=64)

    def call(**kw):
        return lib.foremoe_router_bwd(*{**ok, **kw}.values(), None)

    for kw in (dict(dtype=3), dict(K=70), dict(coef=0.5), dict(coef=0.5, counts=FAKE), dict(coef=NAN, counts=FAKE,
               n_tokens=FAKE), dict(ld_out=60), dict(dlogits=None), dict(ids=None), dict(dlogits=0x9001),
               dict(dlogits=0x1000, ld_out=65)):
        assert call(**kw) == -1, kw
    assert call(T=0, logits=None, dlogits=None) == 0


def test_token_logprobs_refuses(lib):
    ok = dict(logits=FAKE, dtype=0, ld=100, N=4, V=100, targets=FAKE, temperature=1.0, n_top=0, logp=FAKE, entropy=FAKE,
              lse=FAKE, top_ids=None, top_logp=None, ws=None, ws_bytes=0)

    def call(**kw):
        return lib.foremoe_token_logprobs(*{**ok, **kw}.values(), None)

    n = lib.foremoe_logprobs_workspace_size()
    assert n > 0 and n % 256 == 0
    for kw in (dict(dtype=2), dict(V=0), dict(V=1 << 31, ld=1 << 31), dict(N=-1), dict(N=1 << 31), dict(ld=99),
               dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=NAN), dict(temperature=float("inf")),
               dict(temperature=1e-45), dict(n_top=-1), dict(n_top=33, top_ids=FAKE, top_logp=FAKE),
               dict(V=3, n_top=4, top_ids=FAKE, top_logp=FAKE), dict(n_top=2), dict(n_top=2, top_ids=FAKE),
               dict(targets=None), dict(logits=None), dict(logits=0x1002), dict(ws_bytes=16),
               dict(ws=FAKE, ws_bytes=n - 1), dict(ws=0x1040, ws_bytes=n)):
        assert call(**kw) == -1, kw
    assert call(N=0, logits=None) == 0


def test_token_logprobs_bwd_refuses(lib):
    ok = dict(logits=FAKE, dtype=0, ld=100, N=4, V=100, targets=FAKE, temperature=1.0, lse=FAKE, entropy=None,
              dlogp=FAKE, dentropy=None, dlogits=0x9000, ld_out=100)

    def call(**kw):
        return lib.foremoe_token_logprobs_bwd(*{**ok, **kw}.values(), None)

    for kw in (dict(dtype=2), dict(temperature=0.0), dict(lse=None), dict(dlogits=None), dict(targets=None),
               dict(dentropy=FAKE), dict(ld_out=99), dict(dlogits=0x9002), dict(dlogits=0x1000, ld_out=101)):
        assert call(**kw) == -1, kw
    assert call(N=0) == 0


def test_adamw_refuses(lib):
    from paper_2606_11867_amd._lib import AdamWTensor as R
    good = R(0x1000, 0x2000, None, 0x3000, 0x4000, None, None, 10, 0.0)
    ok = dict(tensors=(R * 1)(good), n=1, pdt=0, gdt=0, bits=32, lr=1e-3, b1=0.9, b2=0.95, eps=1e-8, step=1,
              grad_scale=None, zero=0)

    def call(**kw):
        return lib.foremoe_adamw_step(*{**ok, **kw}.values(), None)

    for kw in (dict(pdt=2), dict(gdt=-1), dict(bits=16), dict(n=-1), dict(tensors=None), dict(lr=NAN), dict(lr=-1.0),
               dict(b1=1.0), dict(b2=-0.1), dict(eps=NAN), dict(eps=-1.0), dict(step=0), dict(grad_scale=0x1001)):
        assert call(**kw) == -1, kw
    for bad in (R(None, 0x2000, None, 0x3000, 0x4000, None, None, 10, 0.0),
                R(0x1000, 0x2000, 0x5000, 0x3000, 0x4000, None, None, 10, 0.0),  # a master beside fp32 parameters
                R(0x1000, 0x2000, None, 0x3000, 0x4000, None, None, -1, 0.0),
                R(0x1000, 0x2000, None, 0x3000, 0x4000, None, None, 10, NAN),
                R(0x1002, 0x2000, None, 0x3000, 0x4000, None, None, 10, 0.0),
                R(0x1000, 0x2000, None, 0x3001, 0x4000, None, None, 10, 0.0)):
        assert call(tensors=(R * 2)(good, bad), n=2) == -1
    assert call(bits=8) == -1  # no scales
    assert call(n=0, tensors=None) == 0
    empty = R(None, None, None, None, None, None, None, 0, 0.0)
    assert call(tensors=(R * 1)(empty)) == 0
    f = lib.foremoe_adamw_state_values
    assert f(FAKE, FAKE, FAKE, FAKE, -1, FAKE, FAKE, None) == -1
    assert f(FAKE, None, FAKE, FAKE, 5, FAKE, FAKE, None) == -1
    assert f(None, None, None, None, 0, None, None, None) == 0


def test_binding_refuses_what_is_not_on_the_device():
    from paper_2606_11867_amd import api
    from paper_2606_11867_amd.optimizer import AdamW
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        api.router_fwd(x, 2)
    with pytest.raises(ValueError):
        api.token_logprobs(x)
    with pytest.raises(ValueError):
        AdamW([x], [x])
    with pytest.raises(ValueError):
        AdamW([], [])
    with pytest.raises(ValueError):
        AdamW([x], [x, x])
    with pytest.raises(ValueError):
        AdamW([x], [x], state_bits=4)


@pytest.mark.gpu
def test_binding_refuses_wrong_tensors(gpu):
    from paper_2606_11867_amd import ForeMoEError, api
    from paper_2606_11867_amd.optimizer import AdamW
    x = torch.zeros(4, 8, device=gpu)
    i4 = torch.zeros(4, dtype=torch.int32, device=gpu)
    for bad in (lambda: api.router_fwd(x.t(), 2), lambda: api.router_fwd(x[0], 2),
                lambda: api.router_fwd(x[:1].expand(4, 8), 2),
                lambda: api.router_fwd(x, 2, score="tanh"), lambda: api.router_fwd(x, 2, mask=i4[:3].bool()),
                lambda: api.router_fwd(x, 2, ids=torch.zeros(4, 3, dtype=torch.int32, device=gpu)),
                lambda: api.router_fwd(x, 2, score="sigmoid", bias=torch.zeros(8)),
                lambda: api.token_logprobs(x, i4[:3]),
                lambda: api.token_logprobs_bwd(x, i4, x[0], x[:, 0].contiguous()),
                lambda: api.token_logprobs_bwd(x, i4, x[:, 0].contiguous(), None, out=x[:3]),
                lambda: AdamW([x], [x], masters=[x]), lambda: AdamW([x], [x[:2]]),
                lambda: AdamW([x], [x], weight_decay=[1.0, 2.0]), lambda: AdamW([x], [x], states=[(x,)])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: api.router_fwd(x, 2, mask=i4), lambda: api.router_fwd(x.half(), 2),
                lambda: api.token_logprobs(x, i4.long()), lambda: AdamW([x], [x], states=[(i4, i4)])):
        with pytest.raises((TypeError, ValueError)):
            bad()
    for bad in (lambda: api.router_fwd(x, 9), lambda: api.router_fwd(x, 2, bias=x[0].contiguous()),
                lambda: api.token_logprobs(x, i4, temperature=0.0), lambda: api.token_logprobs(x, n_top=9),
                lambda: AdamW([x], [x], betas=(1.0, 0.9)).step()):
        with pytest.raises(ForeMoEError):
            bad()
