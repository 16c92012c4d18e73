"""Cases of the operators around the expert layer: the router that makes its
ids and gates (with the balance loss and the gradient), the log-probabilities
of given tokens (with entropy, top alternatives and the gradient), and the
AdamW step over many tensors with states in 32 or 8 bits.

Where ``own`` is true, run() calls the framework; otherwise it computes the
same operators from elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32
INF = float("inf")
BLOCK = 256  # elements that share a scale in 8-bit optimizer states
DT = {"bf16": BF16, "f32": F32}


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # the router of one decoding step of a rollout: few tokens, the whole call is latency
        dict(name="route-decode", op="router", mode="route", T=24, E=128, K=8, dtype="bf16", score="softmax",
             renorm=True, scale=1.0, bias=False, dead=0.0, disabled=0),
        # recompute of a Qwen3-30B-A3B micro-step: the gates of the recorded ids, padding tokens masked
        dict(name="route-replay-qwen3", op="router", mode="replay", T=16384, E=128, K=8, dtype="f32",
             score="softmax", renorm=True, scale=1.0, bias=False, dead=0.1, disabled=0),
        # policy update of that micro-step: gates of the recorded ids, counts, balance loss, gradient of the logits
        dict(name="route-train-qwen3", op="router", mode="train-replay", T=16384, E=128, K=8, dtype="f32",
             score="softmax", renorm=True, scale=1.0, bias=False, dead=0.1, disabled=0),
        # a DeepSeek-V3 micro-step choosing its experts by sigmoid scores plus a bias, forward and backward
        dict(name="route-train-deepseek", op="router", mode="train", T=32768, E=256, K=8, dtype="bf16",
             score="sigmoid", renorm=True, scale=2.5, bias=True, dead=0.0, disabled=0),
        # one sequence decodes one token and wants the 20 likeliest: a single row, split over the GPU
        dict(name="logprobs-one-token", op="logprobs", mode="top", N=1, V=131072, dtype="bf16", n_top=20,
             temperature=0.8, ignored=0.0, pad=0, masked=0),
        # scoring a few tokens with alternatives; odd vocabulary, padded rows, fp32 logits
        dict(name="logprobs-ragged-f32", op="logprobs", mode="score", N=61, V=50021, dtype="f32", n_top=5,
             temperature=1.0, ignored=0.0, pad=11, masked=21),
        # recompute: log-probabilities and entropies of a chunk of response tokens, prompt tokens ignored
        dict(name="logprobs-recompute", op="logprobs", mode="score", N=8192, V=131072, dtype="bf16", n_top=0,
             temperature=1.0, ignored=0.2, pad=0, masked=0),
        # policy update in fp32 at odd sizes: forward, then the gradient of log-probabilities and entropies
        dict(name="logprobs-train-f32", op="logprobs", mode="train", N=2045, V=32003, dtype="f32", n_top=0,
             temperature=0.7, ignored=0.1, pad=0, masked=0),
        # policy update in bf16, the largest gradient
        dict(name="logprobs-train", op="logprobs", mode="train", N=4096, V=131072, dtype="bf16", n_top=0,
             temperature=1.0, ignored=0.2, pad=0, masked=0),
        # norms, router and other small fp32 tensors, each of its own odd size
        dict(name="adamw-small", op="adamw", tensors=40, n_min=64, n_max=40000, param="f32", grad="f32", bits=32,
             master=False, zero_grads=False, clip=True, sizes=1),
        # the 16 local experts of a Qwen3-30B-A3B share: fp32 accumulators, fp32 masters, bf16 weights
        dict(name="adamw-experts-qwen3", op="adamw", tensors=32, n_min=768 * 2048, n_max=2 * 768 * 2048,
             param="bf16", grad="f32", bits=32, master=True, zero_grads=True, clip=True, sizes=0),
        # many ragged tensors with 8-bit states
        dict(name="adamw-8bit", op="adamw", tensors=60, n_min=3000, n_max=6000000, param="bf16", grad="bf16",
             bits=8, master=True, zero_grads=False, clip=False, sizes=2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["router", "router", "logprobs", "logprobs", "adamw"])
    dtype = rng.choice(["bf16", "f32"])
    if op == "router":
        E, K = rng.choice([(8, 2), (24, 3), (60, 4), (64, 6), (128, 8), (160, 6), (256, 8), (512, 10)])
        mode = rng.choice(["route", "replay", "train", "train-replay"])
        score = rng.choice(["softmax", "softmax", "sigmoid"])
        return dict(op=op, mode=mode, T=_log(rng, 1, 32768), E=E, K=K, dtype=dtype, score=score,
                    renorm=rng.random() < 0.7, scale=rng.choice([1.0, 2.5]),
                    # scores plus a bias are compared after rounding: as logits of 16 bits keep them apart
                    bias=score == "sigmoid" and dtype == "bf16" and rng.random() < 0.5,
                    dead=rng.choice([0.0, 0.0, 0.15]), disabled=rng.choice([0, 0, 1, E // 4]))
    if op == "logprobs":
        mode = rng.choice(["top", "score", "train"])
        c = dict(op=op, mode=mode, N=_log(rng, 1, 8192), V=_log(rng, 1000, 151000), dtype=dtype,
                 n_top=0 if mode == "train" else rng.choice([1, 5, 20]) if mode == "top" else rng.choice([0, 0, 3]),
                 temperature=rng.choice([1.0, 0.7, 1.3]),
                 ignored=0.0 if mode == "top" else rng.choice([0.0, 0.3]), pad=rng.choice([0, 0, 5, 8]),
                 masked=rng.choice([0, 0, 17]))
        while _too_large(c):
            c["N"] = c["N"] * 2 // 3
        return c
    param = rng.choice(["bf16", "f32"])
    c = dict(op=op, tensors=rng.randint(1, 60), n_min=_log(rng, 1, 5000), n_max=_log(rng, 5001, 8000000),
             param=param, grad=dtype, bits=rng.choice([32, 8]), master=param == "bf16" and rng.random() < 0.7,
             zero_grads=rng.random() < 0.5, clip=rng.random() < 0.5, sizes=rng.randint(3, 1 << 20))
    while _too_large(c):
        c["tensors"] = c["tensors"] * 2 // 3
    return c


def _too_large(c):
    n = c["N"] * c["V"] if c["op"] == "logprobs" else sum(_sizes(c))
    # top alternatives: the plain form makes a 64-bit key of every logit
    return work(c)["bytes"] > 2.1e9 or n > (1 << 28 if c.get("n_top") else 1 << 30)


def _sizes(c):
    """Elements of every tensor of an AdamW case."""
    if not c["sizes"]:  # gate/up and down matrices of every expert
        return [c["n_max"], c["n_min"]] * (c["tensors"] // 2)
    rng = random.Random(c["sizes"])
    return [_log(rng, c["n_min"], c["n_max"]) for _ in range(c["tensors"])]


def work(case):
    c = case
    if c["op"] == "router":
        T, E, K, b = c["T"], c["E"], c["K"], 2 if c["dtype"] == "bf16" else 4
        train, replay = c["mode"].startswith("train"), c["mode"].endswith("replay")
        by = T * E * b + T * K * 8 + (T * K * 4 if replay else 0) + T
        if train:  # the gates' gradient in, the logits' gradient out
            by += T * K * 4 + T * E * b + 8 * E
        return dict(bytes=by, flops=T * E * (12 if train else 5))
    if c["op"] == "logprobs":
        b = 2 if c["dtype"] == "bf16" else 4
        n = c["N"] * c["V"]
        read = n * (1 - c["ignored"]) * b
        by = read + c["N"] * (16 + 8 * c["n_top"])
        if c["mode"] == "train":
            by += n * b + c["N"] * 8
        return dict(bytes=by, flops=n * (1 - c["ignored"]) * (12 if c["mode"] == "train" else 5))
    n = sum(_sizes(c))
    p, g = (2 if c["param"] == "bf16" else 4), (2 if c["grad"] == "bf16" else 4)
    by = g + (g if c["zero_grads"] else 0) + (8 + p if c["master"] else 2 * p)
    by += 16 if c["bits"] == 32 else 4 + 8 + 16 / BLOCK  # 8 bits: codes both ways, and the values they stand for
    return dict(bytes=n * by, flops=n * 16)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {"router": _prepare_router, "logprobs": _prepare_logprobs, "adamw": _prepare_adamw}[case["op"]](
        dict(case), g)


def _randn(g, *shape, dtype=F32):
    return torch.randn(*shape, generator=g, device="cuda", dtype=dtype)


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda")


def _prepare_router(c, g):
    T, E, K = c["T"], c["E"], c["K"]
    # a Zipf popularity in a random order, as the synthetic workloads have it
    rank = torch.randperm(E, generator=g, device="cuda").float()
    logits = (_randn(g, T, E) - 1.1 * torch.log(rank + 1))
    if c["score"] == "sigmoid":
        logits = logits + 1.0
    logits = logits.to(DT[c["dtype"]])
    if c["disabled"]:  # experts that are out of service
        off = torch.randperm(E, generator=g, device="cuda")[:min(c["disabled"], E - K)]
        logits[:, off] = -INF
    s = dict(c, logits=logits, mask=None, ids=None, bias_t=None, dgates=None, coef=0.01)
    if c["dead"]:
        s["mask"] = _rand(g, T) >= c["dead"]
    if c["bias"]:
        s["bias_t"] = 0.05 * _randn(g, E)
    if c["mode"].endswith("replay"):
        # recorded by the rollout's weights, which were a little different
        s["ids"] = (logits.float() + 0.1 * _randn(g, T, E)).topk(K, dim=1).indices.to(I32)
    if c["mode"].startswith("train"):
        s["dgates"] = 0.1 * _randn(g, T, K)
    if own:  # the workspace that a program keeps
        from paper_2606_11867_amd import api
        s["ws"] = api.router_workspace(E, logits.device)
    return s


def _prepare_logprobs(c, g):
    N, V = c["N"], c["V"]
    # a few tokens stand out, as they do in a trained model
    logits = torch.empty(N, V + c["pad"], dtype=DT[c["dtype"]], device="cuda")
    for a in range(0, N, 1024):
        b = min(N, a + 1024)
        logits[a:b] = 2.0 * _randn(g, b - a, V + c["pad"])
    logits = logits[:, :V]
    likely = torch.randint(0, V, (N, 8), generator=g, device="cuda")
    logits.scatter_(1, likely, (8.0 + 3.0 * _randn(g, N, 8)).to(logits.dtype))
    if c["masked"]:  # the vocabulary's padding
        logits[:, V - c["masked"]:] = -INF
    s = dict(c, logits=logits, targets=None, dlogp=None, dentropy=None)
    if c["mode"] != "top":
        t = likely[:, 0] if N else likely.new_zeros(0)
        t = t.clamp(max=V - 1 - c["masked"])
        s["targets"] = torch.where(_rand(g, N) < c["ignored"], torch.full_like(t, -1), t).to(I32)
    if c["mode"] == "train":
        s["dlogp"] = _randn(g, N) / N
        s["dentropy"] = 0.01 * _randn(g, N) / N
    if own:
        from paper_2606_11867_amd import api
        s["ws"] = api.logprobs_workspace(logits.device)
    return s


def _prepare_adamw(c, g):
    sizes = _sizes(c)
    starts, at = [], 0
    for n in sizes:  # every tensor starts on a block of its flat buffer
        starts.append(at)
        at += -(-n // BLOCK) * BLOCK
    real = torch.zeros(at, dtype=torch.bool, device="cuda")
    for a, n in zip(starts, sizes):
        real[a:a + n] = True
    p = 0.02 * _randn(g, at) * real
    grad = (1e-3 * _randn(g, at) * real).to(DT[c["grad"]])
    m = 3e-4 * _randn(g, at) * real
    v = (1e-3 * _randn(g, at)).square() * real
    s = dict(c, numel=sizes, starts=starts, grad_t=grad, lr=3e-4, beta1=0.9, beta2=0.95, eps=1e-8, step=100,
             wd=[0.1 if i % 3 else 0.0 for i in range(len(sizes))],
             scale=torch.full((1,), 0.37, device="cuda") if c["clip"] else None)
    s["wd_t"] = torch.tensor(s["wd"], device="cuda")
    s["length"] = torch.tensor([-(-n // BLOCK) * BLOCK for n in sizes], device="cuda")
    s["master_t"] = p if c["master"] else None
    s["param_t"] = p.to(DT[c["param"]])
    if c["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        s["m"], s["m_scale"] = _encode_m(m)
        s["v"], s["v_scale"] = _encode_v(v)
    if own:  # the optimizer that a program keeps
        from paper_2606_11867_amd.optimizer import AdamW
        cut = lambda t, q=1: [t[a // q:a // q + -(-n // q)] for a, n in zip(starts, sizes)]  # noqa: E731
        states = list(zip(cut(s["m"]), cut(s["v"]))) if c["bits"] == 32 else list(
            zip(cut(s["m"]), cut(s["v"]), cut(s["m_scale"], BLOCK), cut(s["v_scale"], BLOCK)))
        s["opt"] = AdamW(cut(s["param_t"]), cut(grad), lr=s["lr"], betas=(s["beta1"], s["beta2"]), eps=s["eps"],
                         weight_decay=s["wd"], state_bits=c["bits"], masters=cut(p) if c["master"] else False,
                         states=states, step=s["step"], zero_grads=c["zero_grads"])
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(state):
    if state["op"] == "router":
        return _router_own(state) if own else _router_plain(state)
    if state["op"] == "logprobs":
        return _logprobs_own(state) if own else _logprobs_plain(state)
    return _adamw_own(state) if own else _adamw_plain(state)


def _router_own(s):
    from paper_2606_11867_amd import api
    kw = dict(score=s["score"], renorm=s["renorm"], scale=s["scale"], mask=s["mask"])
    train = s["dgates"] is not None
    r = api.router_fwd(s["logits"], s["K"], bias=s["bias_t"], ids=s["ids"], stats=train, ws=s["ws"], **kw)
    out = dict(ids=r.ids, gates=r.gates)
    if train:
        out.update(counts=r.counts, n_tokens=r.n_tokens, prob_mean=r.prob_mean, balance_loss=r.balance_loss)
        out["dlogits"] = api.router_bwd(s["logits"], r.ids, s["dgates"], counts=r.counts, n_tokens=r.n_tokens,
                                        balance_coef=s["coef"], **kw)
    return out


def _router_plain(s):
    x = s["logits"].float()
    T, E = x.shape
    K, scale, softmax = s["K"], s["scale"], s["score"] == "softmax"
    alive = (x != -INF).any(1)
    if s["mask"] is not None:
        alive = alive & s["mask"]
    if softmax:
        e = torch.exp(x - x.amax(1, keepdim=True))
        pi = e / e.sum(1, keepdim=True)
    else:
        sig = 1.0 / (1.0 + torch.exp(-x))
        pi = sig / sig.sum(1, keepdim=True)
    if s["ids"] is None:
        key = x if s["bias_t"] is None else torch.where(x == -INF, x, sig + s["bias_t"])
        ids = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :K]
        ids = torch.where(torch.gather(x, 1, ids) == -INF, -1, ids)
    else:
        ids = s["ids"].long()
    ids = torch.where(alive[:, None], ids, -1)
    chosen = ids >= 0
    at = ids.clamp(min=0)
    if softmax and s["renorm"]:
        xs = torch.where(chosen, torch.gather(x, 1, at), -INF)
        q = torch.exp(xs - xs.amax(1, keepdim=True))
        q = torch.where(chosen, q / q.sum(1, keepdim=True), 0.0)
    else:
        q = torch.where(chosen, torch.gather(pi if softmax else sig, 1, at), 0.0)
        if s["renorm"]:
            total = q.sum(1, keepdim=True)
            raw, q = q, torch.where(total > 0, q / total, 0.0)
    out = dict(ids=ids.to(I32), gates=q * scale)
    if s["dgates"] is None:
        return out
    pi = torch.where(alive[:, None], pi, 0.0)
    counts = torch.zeros(E, dtype=I32, device=x.device)
    counts.scatter_add_(0, at.reshape(-1), chosen.reshape(-1).to(I32))
    n = alive.sum()
    mean = pi.sum(0) / n.clamp(min=1)
    f = counts / counts.sum().clamp(min=1)
    out.update(counts=counts, n_tokens=n.to(I32).reshape(1), prob_mean=mean,
               balance_loss=(E * (f * mean).sum()).reshape(1))
    # backward
    dg = torch.where(chosen, s["dgates"], 0.0)
    push = s["coef"] * E * f / n.clamp(min=1)
    spread = lambda t: torch.zeros_like(x).scatter_add_(1, at, t)  # noqa: E731
    if softmax and not s["renorm"]:
        dp = spread(dg * scale) + push
        dl = pi * (dp - (pi * dp).sum(1, keepdim=True))
    else:
        dl = pi * (push - (pi * push).sum(1, keepdim=True))
        if softmax:
            dl = dl + spread(scale * q * (dg - (q * dg).sum(1, keepdim=True)))
        else:
            ds = dg * scale
            if s["renorm"]:
                ds = torch.where(total > 0, (ds - (q * ds).sum(1, keepdim=True)) / total, 0.0)
            dl = (dl + spread(torch.where(chosen, ds * raw, 0.0)) if s["renorm"] else dl + spread(ds * q)) * (1 - sig)
    out["dlogits"] = torch.where(alive[:, None], dl, 0.0).to(s["logits"].dtype)
    return out


def _logprobs_own(s):
    from paper_2606_11867_amd import api
    r = api.token_logprobs(s["logits"], s["targets"], temperature=s["temperature"], n_top=s["n_top"], ws=s["ws"])
    out = dict(entropy=r.entropy, lse=r.lse)
    if s["targets"] is not None:
        out["logp"] = r.logp
    if s["n_top"]:
        out.update(top_ids=r.top_ids, top_logp=r.top_logp)
    if s["mode"] == "train":
        out["dlogits"] = api.token_logprobs_bwd(s["logits"], s["targets"], r.lse, s["dlogp"], entropy=r.entropy,
                                                dentropy=s["dentropy"], temperature=s["temperature"])
    return out


def _logprobs_plain(s):
    raw, t = s["logits"], s["targets"]
    N, V = raw.shape
    x = raw.float() * (1.0 / s["temperature"])
    m = x.amax(1, keepdim=True)
    d = x - m
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    entropy = torch.log(total) - torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True) / total
    del d, e
    keep = None if t is None else ((t >= 0) & (t < V))[:, None]
    out = {}
    if t is not None:
        at = t.long().clamp(0, V - 1)[:, None]
        out["logp"] = torch.where(keep, torch.gather(x, 1, at) - lse, 0.0)[:, 0]
        lse, entropy = torch.where(keep, lse, 0.0), torch.where(keep, entropy, 0.0)
    out.update(entropy=entropy[:, 0], lse=lse[:, 0])
    if s["n_top"]:
        # the logit's order above, the lower id first among equals below
        bits = (raw.float() + 0.0).view(I32)
        key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * (1 << 32)
        key += (1 << 31) - torch.arange(V, device=x.device)
        ids = key.topk(s["n_top"], dim=1).indices
        best = torch.gather(x, 1, ids)
        there = (best != -INF) if keep is None else (best != -INF) & keep
        out["top_ids"] = torch.where(there, ids, -1).to(I32)
        out["top_logp"] = torch.where(there, best - lse, -INF)
    if s["mode"] == "train":
        lp = x - lse
        p = torch.exp(lp)
        dlogp, dh = s["dlogp"][:, None], s["dentropy"][:, None]
        dl = torch.where(p > 0, p * (-dlogp - dh * (lp + entropy)), 0.0)
        dl.scatter_add_(1, at, dlogp)
        out["dlogits"] = torch.where(keep, dl * (1.0 / s["temperature"]), 0.0).to(raw.dtype)
    return out


def _adamw_own(s):
    s["opt"].step(grad_scale=s["scale"])
    return _adamw_out(s, *_state_values(s))


def _state_values(s):
    if s["bits"] == 32:
        return s["m"], s["v"]
    from paper_2606_11867_amd import api
    return api.adamw_state_values(s["m"], s["m_scale"], s["v"], s["v_scale"])


def _adamw_out(s, m, v):
    out = dict(param=s["param_t"], m=m, v=v)
    if s["master"]:
        out["master"] = s["master_t"]
    if s["zero_grads"]:
        out["grad"] = s["grad_t"]
    return out


# 8-bit states. A code of the first moment is a sign and the top bits of |m|
# over its block's largest, as a float with 3 bits behind the binary point, 127
# standing for 1; one of the second moment is sqrt(v) over the block's largest
# with 4 bits behind the point, 255 standing for 1. 0 stands for 0, and a v
# above 0 never becomes 0.
def _blocks(t):
    return t.view(-1, BLOCK)


def _top_bits(x, shift, one):
    """x in [0, 1] to its rounded top bits (ties to even), counted so that 1 is `one`."""
    b = x.view(I32)
    return ((b + ((1 << (shift - 1)) - 1) + ((b >> shift) & 1)) >> shift) - ((0x3F800000 >> shift) - one)


def _of_top_bits(c, shift, one):
    c = c.to(I32)
    return torch.where(c > 0, (c + ((0x3F800000 >> shift) - one)) << shift, 0).view(F32)


def _inverse(scale):
    return torch.where(scale >= 2.0 ** -126, 1.0 / scale, 0.0)


def _encode_m(m):
    a = _blocks(m).abs()
    scale = a.amax(1)
    c = _top_bits(a * _inverse(scale)[:, None], 20, 127).clamp(0, 127)
    c = c + torch.where((_blocks(m) < 0) & (c > 0), 128, 0)
    return c.to(torch.uint8).view(-1), scale


def _decode_m(c, scale):
    c = c.to(I32)
    x = (_blocks(_of_top_bits(c & 127, 20, 127)) * scale[:, None]).view(-1)
    return torch.where(c >= 128, -x, x)


def _encode_v(v):
    u = torch.sqrt(_blocks(v))
    scale = u.amax(1)
    x = u * _inverse(scale)[:, None]
    c = torch.where(x > 0, _top_bits(x, 19, 255).clamp(1, 255), 0)
    return c.to(torch.uint8).view(-1), scale


def _decode_v(c, scale):
    return (_blocks(_of_top_bits(c, 19, 255)) * scale[:, None]).square().view(-1)


def _adamw_plain(s):
    s["step"] += 1
    g = s["grad_t"].float()
    if s["scale"] is not None:
        g = g * s["scale"]
    b1, b2 = s["beta1"], s["beta2"]
    m, v = (s["m"], s["v"]) if s["bits"] == 32 else (_decode_m(s["m"], s["m_scale"]),
                                                     _decode_v(s["v"], s["v_scale"]))
    m.mul_(b1).add_(g * (1 - b1))
    v.mul_(b2).add_((g * g).mul_(1 - b2))
    den = torch.sqrt(v).mul_(1 / math.sqrt(1 - b2 ** s["step"])).add_(s["eps"])
    decay = torch.repeat_interleave(1 - s["lr"] * s["wd_t"], s["length"], output_size=g.numel())
    p = s["master_t"] if s["master"] else s["param_t"].float()
    p = p.mul_(decay).sub_((m / den).mul_(s["lr"] / (1 - b1 ** s["step"])))
    if s["master"] or s["param_t"].dtype != F32:
        s["param_t"].copy_(p)
    if s["zero_grads"]:
        s["grad_t"].zero_()
    if s["bits"] == 8:
        c, scale = _encode_m(m)
        s["m"].copy_(c)
        s["m_scale"].copy_(scale)
        c, scale = _encode_v(v)
        s["v"].copy_(c)
        s["v_scale"].copy_(scale)
        m, v = _decode_m(s["m"], s["m_scale"]), _decode_v(s["v"], s["v_scale"])
    return _adamw_out(s, m, v)


# ---------------------------------------------------------------------------
# The operators' definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"router": _router_exact, "logprobs": _logprobs_exact, "adamw": _adamw_exact}[s["op"]](s)


def _router_exact(s):
    l = s["logits"].double()
    T, E = l.shape
    K = s["K"]
    sig = torch.sigmoid(l)
    lse = torch.logsumexp(l, 1, keepdim=True)
    live = ~torch.isinf(lse[:, 0]) & (True if s["mask"] is None else s["mask"])
    live = live[:, None]
    if s["ids"] is not None:
        ids = s["ids"].long()
    else:
        key = l if s["bias_t"] is None else (sig + s["bias_t"].double()).masked_fill(l == -INF, -INF)
        val, ids = torch.sort(-key, dim=1, stable=True)
        ids = ids[:, :K].masked_fill(val[:, :K] == INF, -1)
    hit = (ids >= 0) & live
    # chosen[t, k, e]: a row of zeros where a place is empty; taken in chunks of tokens
    score = torch.exp(l - lse) if s["score"] == "softmax" else sig
    pi = score / score.sum(1, keepdim=True)
    g = score.gather(1, ids.clamp(min=0)) * hit
    if s["renorm"]:
        tot = g.sum(1, keepdim=True)
        w = torch.where(tot > 0, g / tot, torch.zeros_like(g))
    else:
        w = g
    out = dict(ids=None, gates=s["scale"] * w)
    if s["dgates"] is None:
        return out
    cnt = torch.bincount(ids[hit], minlength=E).double()
    n = max(1, int(live.sum()))
    P = (pi * live).sum(0) / n
    f = cnt / max(1.0, float(cnt.sum()))
    out.update(counts=None, n_tokens=None, prob_mean=P, balance_loss=(E * (f * P).sum()).reshape(1))
    # d loss / d score through the gates, then through pi = score / sum(score), then to the logits
    dw = s["dgates"].double() * s["scale"] * hit
    if s["renorm"]:
        dw = torch.where(tot > 0, (dw - (dw * w).sum(1, keepdim=True)) / tot, torch.zeros_like(dw))
    dscore = torch.zeros_like(l).index_put_((torch.arange(T, device=l.device)[:, None].expand(T, K),
                                             ids.clamp(min=0)), dw * hit, accumulate=True)
    c = (s["coef"] * E / n) * f
    dscore += (c - (pi * c).sum(1, keepdim=True)) / score.sum(1, keepdim=True)
    if s["score"] == "softmax":
        dl = score * (dscore - (score * dscore).sum(1, keepdim=True))
    else:
        dl = dscore * sig * (1 - sig)
    out["dlogits"] = torch.where(live, dl, torch.zeros_like(dl))
    return out


def _logprobs_exact(s):
    raw, t, n_top = s["logits"], s["targets"], s["n_top"]
    N, V = raw.shape
    dev = raw.device
    out = dict(entropy=torch.zeros(N, dtype=F64, device=dev), lse=torch.zeros(N, dtype=F64, device=dev))
    if t is not None:
        out["logp"] = torch.zeros(N, dtype=F64, device=dev)
    if n_top:
        out["top_ids"] = None
        out["top_logp"] = torch.full((N, n_top), -INF, dtype=F64, device=dev)
    if s["mode"] == "train":
        out["dlogits"] = torch.zeros(N, V, dtype=F64, device=dev)
    rows = torch.arange(N, device=dev) if t is None else torch.nonzero((t >= 0) & (t < V))[:, 0]
    step = max(1, (1 << 26) // V)
    for at in range(0, rows.numel(), step):
        r = rows[at:at + step]
        lp = torch.log_softmax(raw[r].double() / s["temperature"], 1)
        p = lp.exp()
        h = -torch.special.xlogy(p, p).sum(1)
        out["entropy"][r] = h
        out["lse"][r] = torch.logsumexp(raw[r].double() / s["temperature"], 1)
        if t is not None:
            tt = t[r].long()
            out["logp"][r] = lp[torch.arange(r.numel(), device=dev), tt]
        if n_top:
            order = torch.sort(-raw[r].double(), dim=1, stable=True).indices[:, :n_top]
            out["top_logp"][r] = lp.gather(1, order)
        if s["mode"] == "train":
            a, b = s["dlogp"][r].double(), s["dentropy"][r].double()
            d = -a[:, None] * p - b[:, None] * (torch.special.xlogy(p, p) + p * h[:, None])
            d[torch.arange(r.numel(), device=dev), tt] += a
            out["dlogits"][r] = d / s["temperature"]
    return out


def _adamw_exact(s):
    n = s["grad_t"].numel()
    if n > 100_000_000:
        return None
    t = s["step"] + 1
    g = s["grad_t"].double() * (1.0 if s["scale"] is None else s["scale"].double())
    if s["bits"] == 32:
        m, v = s["m"].double(), s["v"].double()
    else:
        m = _value(s["m"].long() % 128, 3, 127, s["m_scale"]) * (1 - 2 * (s["m"].long() // 128))
        v = _value(s["v"].long(), 4, 255, s["v_scale"]) ** 2
    m = s["beta1"] * m + (1 - s["beta1"]) * g
    v = s["beta2"] * v + (1 - s["beta2"]) * g * g
    p = (s["master_t"] if s["master"] else s["param_t"]).double()
    wd = torch.zeros(n, dtype=F64, device=g.device)
    for a, k, w in zip(s["starts"], s["numel"], s["wd"]):
        wd[a:a + k] = w
    root = (v / (1 - s["beta2"] ** t)).sqrt() + s["eps"]
    p = p - s["lr"] * wd * p - s["lr"] * (m / (1 - s["beta1"] ** t)) / root
    out = dict(param=p, m=m, v=v)
    if s["bits"] == 8:
        top = m.abs().view(-1, BLOCK).amax(1)
        out["m"] = torch.sign(m) * _nearest(m.abs(), top, 3, 127, 0)
        u = v.sqrt()
        out["v"] = _nearest(u, u.view(-1, BLOCK).amax(1), 4, 255, 1) ** 2
    if s["master"]:
        out["master"] = p
    if s["zero_grads"]:
        out["grad"] = torch.zeros_like(p)
    return out


def _value(code, digits, one, scale):
    """The value of an 8-bit code: 2^e (1 + j / 2^digits) times the scale, `one` being 1."""
    k = code - one
    e = torch.div(k, 1 << digits, rounding_mode="floor")
    x = torch.ldexp(1 + (k - (e << digits)).double() / (1 << digits), e)
    return (torch.where(code > 0, x, torch.zeros_like(x)).view(-1, BLOCK) * scale.double()[:, None]).view(-1)


def _nearest(u, scale, digits, one, least):
    """u over its block's scale, rounded to the nearest of the codes' values."""
    x = u.view(-1, BLOCK) / torch.where(scale > 0, scale, torch.ones_like(scale))[:, None]
    f, e = torch.frexp(x)
    k = torch.round((2 * f - 1) * (1 << digits)).long() + ((e.long() - 1) << digits) + one
    k = torch.where(x > 0, k.clamp(least, one), torch.zeros_like(k))
    return _value(k.view(-1), digits, one, scale)
