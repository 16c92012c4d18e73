"""From an update to the rollout, the operators together: a Muon step over the
experts, their quantisation, a prompt through the FFN in 4 bits between router,
permute and combine, and decoding steps of a few tokens, replayed from a graph
after the weights have changed.

Each part is compared with the oracle on the inputs that it was given, with the
tolerances of its own tests; combine adds K products in fp32.
"""
import importlib.util
import os

import numpy as np
import pytest
import torch

import oracle.foremoe_rollout as R
from test_gpu_few_tokens import _limit
from test_gpu_muon import COEF
from test_gpu_mxfp4 import _check_slot

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def _np(t):
    return t.detach().double().cpu().numpy()


class Layer:
    """An expert layer that is trained with Muon and rolled out in 4 bits."""

    def __init__(self, gpu, E=8, d=256, F=128, K=2, seed=0):
        from paper_2606_11867_amd import api
        from paper_2606_11867_amd.optimizer import Muon
        g = torch.Generator(device=gpu).manual_seed(seed)
        randn = lambda *s: torch.randn(s, generator=g, device=gpu)  # noqa: E731
        self.gen, self.gpu, self.E, self.d, self.F, self.K = g, gpu, E, d, F, K
        self.router = randn(E, d) * d ** -0.5
        self.gate_up = (randn(E, 2 * F, d) * d ** -0.5).to(BF16)
        self.down = (randn(E, d, F) * F ** -0.5).to(BF16)
        self.grads = [torch.zeros(t.shape, device=gpu) for t in (self.gate_up, self.down)]
        self.opt = Muon([self.gate_up, self.down], self.grads, lr=0.02, momentum=0.9, weight_decay=0.1, parts=[2, 1],
                        masters=True, zero_grads=True)
        self.q = [api.mxfp4_quantize(t) for t in (self.gate_up, self.down)]
        each = torch.arange(E, dtype=I32, device=gpu)
        self.plan = api.DevicePlan(E=E, S=E, R_max=1, W=E, G=E, slot_expert=each, slot_replica=torch.zeros_like(each),
                                   expert_nrep=torch.ones_like(each), expert_rep_weight=None, slot_widx=each,
                                   slot_gidx=each)

    def tokens(self, T):
        return torch.randn(T, self.d, generator=self.gen, device=self.gpu).to(BF16)

    def update(self):
        from paper_2606_11867_amd import api
        for g in self.grads:
            g.copy_(torch.randn(g.shape, generator=self.gen, device=self.gpu))
        self.opt.step()
        for m, q in zip(self.opt.masters, self.q):
            api.mxfp4_quantize(m, out=q)  # in place: the rollout's graphs read these

    def route(self, x):
        from paper_2606_11867_amd import api
        return api.router_fwd(x.float() @ self.router.t(), self.K, stats=False)

    def prompt(self, x):
        from paper_2606_11867_amd import api
        r = self.route(x)
        ws = api.workspace(x.shape[0], self.K, self.E, self.gpu)
        _, begin, _, offset = api.histogram_assign(r.ids, self.plan, ws)
        x_perm, _, p2r = api.permute(x, r.ids, self.plan, begin, offset, x.shape[0] * self.K, ws)
        xq = api.mxfp4_quantize(x_perm, n_rows=offset[-1:])
        y_perm = api.grouped_ffn_mxfp4_fwd(xq, offset, self.plan.slot_widx, *self.q)
        return r, offset, xq, y_perm, p2r, api.combine(y_perm, p2r, r.gates)


def test_update_prompt_and_decode(gpu):
    from paper_2606_11867_amd import api
    layer = Layer(gpu)
    before = [_np(m) for m in layer.opt.masters]
    layer.update()
    # the update: every expert's gate, up and down matrix moved by lr times its X
    for m, b, state, parts, scale in zip(layer.opt.masters, before, layer.opt.states, (2, 1), layer.opt.scale):
        for e in (0, layer.E - 1):
            rows = m.shape[1] // parts
            for p in range(parts):
                at = (e, slice(p * rows, (p + 1) * rows))
                mom = _np(state)[at]  # after one step m is the gradient, u = (1 + momentum) m
                u = 1.9 * mom
                exact, held = (f(u / np.linalg.norm(u), COEF, 5) for f in (R.newton_schulz, R.newton_schulz_held))
                move = (b[at] * (1 - 0.02 * 0.1) - _np(m)[at]) / (0.02 * scale)
                slack = 8 * U * (np.abs(b[at]) + np.abs(_np(m)[at])) / (0.02 * scale)
                lim = 3 * np.linalg.norm(held - exact) + 2.0 ** -18 * np.linalg.norm(exact) + np.linalg.norm(slack)
                assert np.linalg.norm(move - exact) <= lim, (np.linalg.norm(move - exact), lim)
    assert torch.equal(layer.gate_up, layer.opt.masters[0].to(BF16)) and not layer.grads[0].any()
    # the quantised weights
    values = []
    for m, q in zip(layer.opt.masters, layer.q):
        codes, scales = R.mxfp4_quantize(_np(m))
        assert np.array_equal(q.codes.cpu().numpy(), codes) and np.array_equal(q.scales.cpu().numpy(), scales)
        values.append(R.mxfp4_values(codes, scales, m.shape[-1]))
    # a prompt
    x = layer.tokens(300)
    r, offset, xq, y_perm, p2r, y = layer.prompt(x)
    off = offset.cpu().numpy()
    assert off[-1] == 600
    xv = R.mxfp4_values(xq.codes.cpu().numpy(), xq.scales.cpu().numpy(), layer.d)
    for e in range(layer.E):
        s = slice(off[e], off[e + 1])
        if off[e + 1] > off[e]:
            _check_slot(xv[s], values[0][e], values[1][e], _np(y_perm[s]))
    rows = _np(y_perm)[p2r.cpu().numpy().reshape(300, 2)]
    g = _np(r.gates)
    ref = (g[..., None] * rows).sum(1)
    assert np.all(np.abs(_np(y) - ref) <= 4 * U * (np.abs(g)[..., None] * np.abs(rows)).sum(1) + 1e-37)
    # decoding steps, in bf16 and in 4 bits
    for T in (1, 24):
        xt = x[:T]
        rt = layer.route(xt)
        ids, gates = rt.ids.cpu().numpy(), _np(rt.gates)
        for weights, vals in (((layer.gate_up, layer.down), [_np(layer.gate_up), _np(layer.down)]), (layer.q, values)):
            got = _np(api.few_tokens_ffn(xt, rt.ids, rt.gates, *weights, out_dtype=F32))
            ref = R.few_tokens(_np(xt), ids, gates, *vals)
            lim = _limit(_np(xt), ids, gates, *vals, None, ref, "f32")
            assert np.all(np.abs(got - ref) <= lim)


def test_ranks_add_up(gpu):
    """Two ranks with half of the experts each: their parts add up to the whole
    layer, with bf16 weights and with 4-bit ones."""
    from paper_2606_11867_amd import api
    layer = Layer(gpu, seed=1)
    x = layer.tokens(17)
    r = layer.route(x)
    ids, gates, half = r.ids.cpu().numpy(), _np(r.gates), layer.E // 2
    value = lambda t: _np(api.mxfp4_values(t) if isinstance(t, api.MXFP4) else t)  # noqa: E731
    for w in ((layer.gate_up, layer.down), tuple(layer.q)):
        vals = [value(t) for t in w]
        ref = R.few_tokens(_np(x), ids, gates, *vals)
        total, lim = torch.zeros(17, layer.d, dtype=torch.float64), np.zeros(ref.shape)
        for rank in range(2):
            here = slice(rank * half, (rank + 1) * half)
            widx = torch.full((layer.E,), -1, dtype=I32, device=gpu)
            widx[here] = torch.arange(half, dtype=I32, device=gpu)
            mine = [api.MXFP4(t.codes[here], t.scales[here]) if isinstance(t, api.MXFP4) else t[here] for t in w]
            part = api.few_tokens_ffn(x, r.ids, r.gates, *mine, expert_widx=widx, out_dtype=F32)
            here_vals, at = [v[here] for v in vals], widx.cpu().numpy()
            lim += _limit(_np(x), ids, gates, *here_vals, at, R.few_tokens(_np(x), ids, gates, *here_vals, at), "f32")
            total += part.double().cpu()
        assert np.all(np.abs(total.numpy() - ref) <= lim)


def test_graph_follows_the_weights(gpu):
    """A decoding step in a graph, replayed after updates that quantise into the
    same memory: every replay equals the eager call then, bit for bit."""
    from paper_2606_11867_amd import api
    layer = Layer(gpu, seed=2)
    x = layer.tokens(5)
    ws = api.few_tokens_workspace(5, layer.K, layer.d, layer.F, gpu)
    logits = torch.empty(5, layer.E, device=gpu)

    def step():
        r = api.router_fwd(logits, layer.K, stats=False)
        return api.few_tokens_ffn(x, r.ids, r.gates, *layer.q, ws=ws)

    logits.copy_(x.float() @ layer.router.t())
    side = torch.cuda.Stream(gpu)
    side.wait_stream(torch.cuda.current_stream(gpu))
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream(gpu).wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = step()
    seen = []
    for _ in range(3):
        layer.update()
        x.copy_(layer.tokens(5))
        logits.copy_(x.float() @ layer.router.t())
        g.replay()
        torch.cuda.synchronize()
        seen.append(y.clone())
        assert torch.equal(step(), seen[-1])
    assert not torch.equal(seen[0], seen[1])


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "policy_step.py")
    spec = importlib.util.spec_from_file_location("policy_step", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("muon", [False, True])
def test_example_rolls_out(gpu, example, muon):
    """The example's layer: decoding in bf16, then steps, a refresh into the same
    memory, prompt and decoding in 4 bits, the layer's part against the oracle."""
    model = example.PolicyStep(T=96, d=256, F=128, E=6, K=2, V=301, muon=muon)
    x = model.x[:24]
    assert bool(torch.isfinite(model.decode(x)).all()) and model.rollout is None
    model.step()
    model.refresh()
    first, at = [q.codes.clone() for q in model.rollout], [q.codes.data_ptr() for q in model.rollout]
    before = model.gate_up.clone()
    model.step()
    assert not torch.equal(before, model.gate_up) and not model.d_gate_up.any()
    model.refresh()
    assert at == [q.codes.data_ptr() for q in model.rollout]
    assert not all(torch.equal(a, q.codes) for a, q in zip(first, model.rollout))
    assert model.prompt(x).shape == (24, 301) and bool(torch.isfinite(model.prompt(x)).all())
    r = model._route(x)
    vals = [R.mxfp4_values(q.codes.cpu().numpy(), q.scales.cpu().numpy()) for q in model.rollout]
    for v, m in zip(vals, (model.opts[0].masters or model.opts[0].params)[:2]):
        assert np.array_equal(v, R.mxfp4_values(*R.mxfp4_quantize(_np(m))))
    ids, gates = r.ids.cpu().numpy(), _np(r.gates)
    y = R.few_tokens(_np(x), ids, gates, *vals)
    # the layer's output, its sum with x and the logits are each rounded to bf16
    # (half a step of 2^-8); a product of 256 terms in fp32 is within 256 u of its
    # magnitudes
    lim = _limit(_np(x), ids, gates, *vals, None, y, "bf16")
    hidden = _np(x) + y
    lim += 2.0 ** -8 * (np.abs(hidden) + lim)
    head = _np(model.head)
    ref = hidden @ head.T
    lim = lim @ np.abs(head).T + 256 * U * ((np.abs(hidden) + lim) @ np.abs(head).T)
    lim += 2.0 ** -8 * (np.abs(ref) + lim)
    assert np.all(np.abs(_np(model.decode(x)) - ref) <= lim)
