"""One policy-update step around the expert layer, on one GPU, with the
framework's calls from end to end:

  router -> dispatch -> expert FFN -> combine -> head -> log-probabilities of
  the rollout's tokens -> policy-gradient loss -> the backward of each -> AdamW

The model is one MoE layer between a fixed embedding and a head, with random
weights; the "rollout" is a fixed batch of tokens with advantages, whose
routing the first pass records and every later step replays (Sec. 5). The
experts are updated by AdamW or by Muon; refresh() hands them to a rollout in 4
bits, prompt() and decode() are its two ways through the layer. Run

    python examples/policy_step.py [steps]

to see the loss fall.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_11867_amd import api  # noqa: E402
from paper_2606_11867_amd.optimizer import AdamW, Muon  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


def all_local_plan(E: int, device) -> api.DevicePlan:
    """Every expert in a slot of its own on this GPU, no replicas."""
    each = torch.arange(E, dtype=torch.int32, device=device)
    return api.DevicePlan(E=E, S=E, R_max=1, W=E, G=E, slot_expert=each, slot_replica=torch.zeros_like(each),
                          expert_nrep=torch.ones_like(each), expert_rep_weight=None, slot_widx=each, slot_gidx=each)


class PolicyStep:
    """Weights, workspaces and optimizers of the model, and its step."""

    def __init__(self, T=512, d=256, F=128, E=16, K=4, V=3000, dtype=BF16, state_bits=32, lr=3e-3, seed=0,
                 device="cuda:0", entropy_coef=0.01, balance_coef=0.01, muon=False):
        dev = torch.device(device)
        g = torch.Generator(device=dev).manual_seed(seed)
        self.T, self.d, self.F, self.E, self.K, self.V, self.dtype = T, d, F, E, K, V, dtype
        self.entropy_coef, self.balance_coef = entropy_coef, balance_coef

        def randn(*shape, scale=1.0, dt=dtype):
            return (torch.randn(shape, generator=g, device=dev) * scale).to(dt)

        self.x = randn(T, d)  # the embedded context of every token
        self.tokens = torch.randint(0, V, (T,), generator=g, device=dev).to(torch.int32)
        self.tokens[: T // 8] = -1  # the prompt: no gradient, not read
        self.response = self.tokens >= 0
        self.advantage = torch.randn(T, generator=g, device=dev).abs() + 0.1
        self.router = randn(E, d, scale=d ** -0.5, dt=F32)
        self.gate_up = randn(E, 2 * F, d, scale=d ** -0.5)
        self.down = randn(E, d, F, scale=F ** -0.5)
        self.head = randn(V, d, scale=d ** -0.5)
        self.d_router, self.d_gate_up, self.d_down, self.d_head = (
            torch.zeros(t.shape, dtype=F32, device=dev) for t in (self.router, self.gate_up, self.down, self.head))
        self.plan = all_local_plan(E, dev)
        self.ws, self.rws = api.workspace(T, K, E, dev), api.router_workspace(E, dev)
        self.fws, self.wws, self.lws = api.ffn_workspace(dev), api.wgrad_workspace(d, F, dev), api.logprobs_workspace(dev)
        kw = dict(lr=lr, weight_decay=0.01, state_bits=state_bits, zero_grads=True)
        experts, d_experts = [self.gate_up, self.down], [self.d_gate_up, self.d_down]
        if muon:  # gate and up of an expert are two matrices
            self.opts = [Muon(experts, d_experts, lr=lr, weight_decay=0.01, parts=[2, 1], zero_grads=True),
                         AdamW([self.head], [self.d_head], **kw), AdamW([self.router], [self.d_router], **kw)]
        else:
            self.opts = [AdamW([*experts, self.head], [*d_experts, self.d_head], **kw),
                         AdamW([self.router], [self.d_router], **kw)]
        self.recorded = None  # the rollout's routing
        self.rollout = None   # the rollout's experts, in 4 bits

    def forward(self):
        """Everything the backward needs; the loss is fwd["loss"]."""
        f = {}
        f["router_logits"] = self.x.float() @ self.router.t()
        r = api.router_fwd(f["router_logits"], self.K, ids=self.recorded, ws=self.rws)
        if self.recorded is None:
            self.recorded = r.ids
        _, begin, _, offset = api.histogram_assign(r.ids, self.plan, self.ws)
        f["x_perm"], _, f["p2r"] = api.permute(self.x, r.ids, self.plan, begin, offset, self.T * self.K, self.ws)
        f["h"], f["y_perm"], f["au"] = api.grouped_ffn_fwd(f["x_perm"], offset, self.plan.slot_widx, self.gate_up,
                                                           self.down, ws=self.fws)
        f["hidden"] = self.x + api.combine(f["y_perm"], f["p2r"], r.gates, out_dtype=self.dtype)
        f["logits"] = f["hidden"] @ self.head.t()
        lp = api.token_logprobs(f["logits"], self.tokens, ws=self.lws)
        n = self.response.sum()
        f["loss"] = -(self.advantage * lp.logp).sum() / n - self.entropy_coef * lp.entropy.sum() / n \
            + self.balance_coef * r.balance_loss[0]
        f.update(routing=r, offset=offset, lp=lp, n=n)
        return f

    def backward(self, f):
        """Adds the gradients of the loss into the accumulators."""
        r, offset, dt = f["routing"], f["offset"], self.dtype
        dlogits = api.token_logprobs_bwd(f["logits"], self.tokens, f["lp"].lse, -self.advantage / f["n"],
                                         entropy=f["lp"].entropy,
                                         dentropy=torch.full_like(self.advantage, -self.entropy_coef) / f["n"],
                                         out=f["logits"])  # in place: the logits are the largest tensor
        self.d_head += dlogits.t().float() @ f["hidden"].float()
        dhidden = (dlogits @ self.head).to(dt)
        dy_perm, dgates = api.combine_bwd(dhidden, f["y_perm"], f["p2r"], r.gates)
        d_au, _ = api.grouped_ffn_dgrad(dy_perm, f["au"], offset, self.plan.slot_widx, self.gate_up, self.down,
                                        ws=self.fws)
        api.grouped_ffn_wgrad(f["x_perm"], f["h"], dy_perm, d_au, offset, self.plan.slot_gidx, self.d_gate_up,
                              self.d_down, ws=self.wws)
        d_router_logits = api.router_bwd(f["router_logits"], r.ids, dgates, counts=r.counts, n_tokens=r.n_tokens,
                                         balance_coef=self.balance_coef)
        self.d_router += d_router_logits.t() @ self.x.float()

    def step(self):
        f = self.forward()
        self.backward(f)
        # clip the gradients' norm, on the device
        norm = torch.sqrt(sum(t.square().sum() for t in (self.d_router, self.d_gate_up, self.d_down, self.d_head)))
        scale = torch.clamp(1.0 / (norm + 1e-6), max=1.0).reshape(1)
        for opt in self.opts:
            opt.step(grad_scale=scale)
        return f["loss"]


    def refresh(self):
        """The experts in 4 bits, from the optimizer's masters where it has some;
        into the same memory every time, which a captured rollout reads."""
        experts = list((self.opts[0].masters or self.opts[0].params)[:2])
        if self.rollout is None:
            self.rollout = [api.mxfp4_quantize(t) for t in experts]
        else:
            for t, q in zip(experts, self.rollout):
                api.mxfp4_quantize(t, out=q)

    def _route(self, x):
        return api.router_fwd(x.float() @ self.router.t(), self.K, stats=False)

    def prompt(self, x):
        """Logits of a prompt's tokens x [n, d] (bf16), by the grouped FFN in 4 bits."""
        r, n = self._route(x), x.shape[0]
        ws = api.workspace(n, self.K, self.E, x.device)
        _, begin, _, offset = api.histogram_assign(r.ids, self.plan, ws)
        x_perm, _, p2r = api.permute(x, r.ids, self.plan, begin, offset, n * self.K, ws)
        y_perm = api.grouped_ffn_mxfp4_fwd(api.mxfp4_quantize(x_perm, n_rows=offset[-1:]), offset, self.plan.slot_widx,
                                           *self.rollout)
        return (x + api.combine(y_perm, p2r, r.gates, out_dtype=x.dtype)) @ self.head.t()

    def decode(self, x):
        """Logits of a decoding step's few tokens x [n, d]: the layer in two
        launches, in 4 bits once refresh() has run."""
        r = self._route(x)
        experts = self.rollout or (self.gate_up, self.down)
        return (x + api.few_tokens_ffn(x, r.ids, r.gates, *experts)) @ self.head.t()


def main(steps=20):
    for bits, muon in ((32, False), (8, False), (32, True)):
        model = PolicyStep(state_bits=bits, muon=muon)
        for i in range(steps):
            loss = model.step()
            if i % 5 == 0 or i == steps - 1:
                print(f"{'Muon' if muon else f'{bits}-bit states'}, step {i}: loss {loss.item():.4f}")
    model.refresh()
    picked = model.prompt(model.x)[-4:].argmax(1), model.decode(model.x[-4:]).argmax(1)
    print(f"rollout in 4 bits: {picked[0].tolist()} from the prompt, {picked[1].tolist()} decoding")


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 20)
