"""Cases of the operators that take the experts' weights from an update to the
rollout: the Muon step (momentum, orthogonalised by Newton-Schulz products),
quantisation to microscaled 4-bit floats, the expert FFN over slots in those
(prompts), and the whole expert layer for a few tokens (decoding) with weights
in 32, 16 or 4 bits.

Where ``own`` is true, run() calls the framework; otherwise it computes the
same operators from elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BF16, F32, F64, I32, U8 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.uint8
DT = {"bf16": BF16, "f32": F32}
MX = 32                                       # elements that share a scale
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # what the low three bits of a code stand for
NS = (3.4445, -4.7750, 2.0315)                # coefficients of a Newton-Schulz step


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # the activations of one decoding step, 64 sequences: the whole call is latency
        dict(name="quantize-decode", op="quantize", rows=64, cols=2048, dtype="bf16", pad=0),
        # fp32 rows of an odd width inside a wider buffer
        dict(name="quantize-ragged-f32", op="quantize", rows=3001, cols=1155, dtype="f32", pad=9),
        # the refresh of a rollout engine: 16 updated experts of a Qwen3-30B-A3B share, from their fp32 masters
        dict(name="quantize-experts-qwen3", op="quantize", rows=16 * 2 * 768, cols=2048, dtype="f32", pad=0),
        # a short prompt over many experts: a few rows a slot
        dict(name="ffn4-short", op="ffn4", rows=509, slots=20, weights=16, d=2048, F=768),
        # prompts of a Qwen3-30B-A3B share: 16 experts, 4 replica slots
        dict(name="ffn4-qwen3", op="ffn4", rows=16278, slots=20, weights=16, d=2048, F=768),
        # prompts of a DeepSeek-V3 share
        dict(name="ffn4-deepseek", op="ffn4", rows=8200, slots=10, weights=8, d=7168, F=2048),
        # one sequence decodes one token with all experts on the GPU
        dict(name="few-one-token", op="few", T=1, d=2048, F=768, E=128, W=128, K=8, x="bf16", w="bf16", out="bf16",
             dead=0.0, pad=0),
        # 24 sequences decode with 4-bit experts, a padded batch
        dict(name="few-mxfp4", op="few", T=24, d=2048, F=768, E=128, W=128, K=8, x="bf16", w="mxfp4", out="bf16",
             dead=0.2, pad=0),
        # 64 sequences on a GPU that holds 32 of 256 experts; its part of the sum in fp32
        dict(name="few-share-deepseek", op="few", T=64, d=7168, F=2048, E=256, W=32, K=8, x="bf16", w="bf16",
             out="f32", dead=0.0, pad=64),
        # routers, projections and other small matrices of the same step, each of its own odd size
        dict(name="muon-small", op="muon", kind="ragged", tensors=6, m_min=24, m_max=400, param="f32", grad="f32",
             master=False, nesterov=True, zero_grads=False, clip=True, sizes=1),
        # the 16 local experts of a Qwen3-30B-A3B share: 48 matrices in two tensors
        dict(name="muon-experts-qwen3", op="muon", kind="experts", G=16, F=768, d=2048, param="bf16", grad="f32",
             master=True, nesterov=True, zero_grads=True, clip=True, sizes=0),
        # two experts of a DeepSeek-V3 share: few, large matrices
        dict(name="muon-experts-deepseek", op="muon", kind="experts", G=2, F=2048, d=7168, param="bf16", grad="f32",
             master=True, nesterov=False, zero_grads=True, clip=False, sizes=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "ffn4", "few", "few", "muon", "muon"])
    if op == "quantize":
        c = dict(op=op, rows=_log(rng, 1, 60000), cols=_log(rng, 1, 16000), dtype=rng.choice(["bf16", "f32"]),
                 pad=rng.choice([0, 0, 1, 8, 64]))
        while c["rows"] * c["cols"] > 50e6:
            c["rows"] = c["rows"] * 2 // 3
        return c
    if op == "ffn4":
        W = rng.randint(1, 32)
        c = dict(op=op, rows=_log(rng, 1, 20000), slots=W + rng.randint(0, 6), weights=W,
                 d=128 * _log(rng, 1, 56), F=128 * _log(rng, 1, 20))
        while work(c)["flops"] > 7e11:
            c["rows"] = c["rows"] * 2 // 3
        return c
    if op == "few":
        w = rng.choice(["bf16", "bf16", "mxfp4", "mxfp4", "f32"])
        E, K = rng.choice([(8, 2), (24, 3), (64, 6), (128, 8), (160, 6), (256, 8)])
        step = 32 if w == "mxfp4" else rng.choice([8, 8, 8, 1])
        c = dict(op=op, T=_log(rng, 1, 128), d=step * _log(rng, max(1, 64 // step), 7168 // step),
                 F=step * _log(rng, max(1, 32 // step), 2048 // step), E=E, W=rng.choice([E, max(1, E // 8)]), K=K,
                 x="f32" if w == "f32" else "bf16", w=w, out=rng.choice(["bf16", "f32"]),
                 dead=rng.choice([0.0, 0.0, 0.3]), pad=rng.choice([0, 0, 8]))
        if c["T"] * K * c["W"] < 24 * E:  # some of few tokens' experts are here, and some tokens are not padding
            c.update(W=E, dead=0.0)
        while c["W"] * c["d"] * c["F"] > 32 * 7168 * 2048:
            c["F"] = max(step, c["F"] * 2 // 3 // step * step)
        return c
    param = rng.choice(["bf16", "f32"])
    c = dict(op=op, kind="ragged", tensors=rng.randint(1, 8), m_min=_log(rng, 1, 200), m_max=_log(rng, 201, 2048),
             param=param, grad=rng.choice(["bf16", "f32"]), master=param == "bf16" and rng.random() < 0.7,
             nesterov=rng.random() < 0.7, zero_grads=rng.random() < 0.5, clip=rng.random() < 0.5,
             sizes=rng.randint(2, 1 << 20))
    while work(c)["flops"] > 1.3e12:
        c["tensors"] -= 1
        c["m_max"] = max(c["m_min"], c["m_max"] * 3 // 4)
        c["tensors"] = max(1, c["tensors"])
    return c


def _shapes(c):
    """Matrices of a Muon case: (number, rows, columns) of every tensor, as the step takes them."""
    if c["kind"] == "experts":  # gate and up of an expert are two matrices
        return [(2 * c["G"], c["F"], c["d"]), (c["G"], c["d"], c["F"])]
    rng = random.Random(c["sizes"])
    got = []
    for _ in range(c["tensors"]):
        r, n = _log(rng, c["m_min"], c["m_max"]), _log(rng, c["m_min"], 3 * c["m_max"])
        got.append((rng.choice([1, 1, 2, 5]), *((r, n) if rng.random() < 0.6 else (n, r))))
    return got


def work(case):
    c = case
    if c["op"] == "quantize":  # and the values that the codes stand for, in bf16
        n = c["rows"] * c["cols"]
        return dict(bytes=n * ((2 if c["dtype"] == "bf16" else 4) + 2 * (1 / 2 + 1 / MX) + 2), flops=n * 4)
    if c["op"] == "ffn4":
        n, d, F = c["rows"], c["d"], c["F"]
        return dict(bytes=4 * n * d + min(c["weights"], n) * 3 * d * F * (1 / 2 + 1 / MX), flops=6.0 * n * d * F)
    if c["op"] == "few":
        T, d, F = c["T"] * (1 - c["dead"]), c["d"], c["F"]
        used = c["W"] * (1 - (1 - c["K"] / c["E"]) ** T)  # experts that some token picks
        b = {"bf16": 2, "f32": 4, "mxfp4": 1 / 2 + 1 / MX}[c["w"]]
        return dict(bytes=used * 3 * d * F * b + c["T"] * (6 * d + 8 * c["K"]),
                    flops=6.0 * T * c["K"] * c["W"] / c["E"] * d * F)
    by = 8 + (2 if c["param"] == "bf16" else 4) * (1 if c["master"] else 2) + (8 if c["master"] else 0)
    by += (2 if c["grad"] == "bf16" else 4) * (2 if c["zero_grads"] else 1)
    n = fl = 0
    for b, r, k in _shapes(c):
        n += b * r * k
        m, k = min(r, k), max(r, k)
        fl += b * 5 * (m * m * k + m * m * m + 2 * m * m * k)  # two symmetric products, of which half is enough
    return dict(bytes=n * by, flops=fl)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {"quantize": _prepare_quantize, "ffn4": _prepare_ffn4, "few": _prepare_few, "muon": _prepare_muon}[
        case["op"]](dict(case), g)


def _randn(g, *shape, dtype=F32):
    return torch.randn(*shape, generator=g, device="cuda", dtype=dtype)


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda")


def _prepare_quantize(c, g):
    # channels of different sizes, as activations and weights have them
    x = torch.empty(c["rows"], c["cols"] + c["pad"], dtype=DT[c["dtype"]], device="cuda")
    x.copy_(_randn(g, *x.shape) * torch.exp(_randn(g, x.shape[1])))
    return dict(c, x_t=x[:, :c["cols"]])


def _codes(g, *shape):
    """Random weights in 4 bits: codes [..., n / 2] of Gaussian values and their blocks' scales [..., n / 32]."""
    *lead, n = shape
    v = _randn(g, *lead, n)
    q, e = _quantize(v.view(-1, n))
    code = _code_of(q).view(*lead, n // 2, 2)
    # the scale of a weight of fan-in n
    return code[..., 0] | code[..., 1] << 4, (e.view(*lead, n // MX) + (127 - round(math.log2(n) / 2))).to(U8)


def _prepare_ffn4(c, g):
    n, S, W = c["rows"], c["slots"], c["weights"]
    share = torch.exp(0.7 * _randn(g, S)) + 0.02  # uneven loads; where rows are few some slots are empty
    cut = (share.cumsum(0) / share.sum() * n).round().to(I32)
    off = torch.cat([cut.new_zeros(1), cut])
    off[-1] = n
    widx = (torch.arange(S, device="cuda") % W).to(I32)  # slots past W hold replicas
    gu, dn = _codes(g, W, 2 * c["F"], c["d"]), _codes(g, W, c["d"], c["F"])
    s = dict(c, x_t=_randn(g, n, c["d"]).to(BF16), off=off, widx=widx, gu=gu, dn=dn,
             bounds=off.tolist())  # what the plan says on the host
    if own:
        from paper_2606_11867_amd import api
        s["gu"], s["dn"] = api.MXFP4(*gu), api.MXFP4(*dn)
        s["ws"] = api.ffn_mxfp4_workspace(n, c["F"], off.device)
    return s


def _prepare_few(c, g):
    T, d, F, E, W, K = (c[k] for k in ("T", "d", "F", "E", "W", "K"))
    if c["w"] == "mxfp4":
        gu, dn = _codes(g, W, 2 * F, d), _codes(g, W, d, F)
    else:
        gu, dn = (torch.empty(W, r, n, dtype=DT[c["w"]], device="cuda") for r, n in ((2 * F, d), (d, F)))
        gu.normal_(0, d ** -0.5, generator=g)
        dn.normal_(0, F ** -0.5, generator=g)
    x = _randn(g, T, d + c["pad"]).to(DT[c["x"]])[:, :d]
    logits = _randn(g, T, E)
    top = logits.topk(K, dim=1)
    ids = torch.where(_rand(g, T, 1) < c["dead"], -1, top.indices).to(I32)  # padding tokens pick nothing
    widx = torch.full((E,), -1, dtype=I32, device="cuda")  # weights of the experts that are here
    here = torch.randperm(E, generator=g, device="cuda")[:W]
    widx[here] = torch.arange(W, dtype=I32, device="cuda")
    s = dict(c, x_t=x, ids=ids, gates=torch.softmax(top.values, 1), gu=gu, dn=dn, widx=widx)
    if own:
        from paper_2606_11867_amd import api
        if c["w"] == "mxfp4":
            s["gu"], s["dn"] = api.MXFP4(*gu), api.MXFP4(*dn)
        s["ws"] = api.few_tokens_workspace(T, K, d, F, x.device)
    return s


def _prepare_muon(c, g):
    s = dict(c, lr=3e-4, momentum=0.95, wd=0.1, eps=1e-7,
             clip_t=torch.full((1,), 0.37, device="cuda") if c["clip"] else None)
    s["p"], s["p16"], s["g"], s["m"], shapes = [], [], [], [], _shapes(c)
    for b, r, n in shapes:
        # a bulk and a few directions that stand out, in the gradient and in its mean
        few = min(16, r, n)
        u, v = _randn(g, b, r, few), _randn(g, b, few, n)
        bulk = lambda: _randn(g, b, r, n) + torch.bmm(u * _rand(g, b, 1, few), v)  # noqa: E731
        s["m"].append(1e-3 * bulk())
        s["g"].append((1e-4 * bulk()).to(DT[c["grad"]]))
        p = 0.02 * _randn(g, b, r, n)
        low = p.to(BF16) if c["param"] == "bf16" else None
        s["p"].append(p if c["master"] or low is None else None)
        s["p16"].append(low)
    s["factor"] = [0.2 * math.sqrt(max(r, n)) for _, r, n in shapes]
    if own:  # the optimizer that a program keeps
        from paper_2606_11867_amd.optimizer import Muon
        s["opt"] = Muon(s["p16"] if c["param"] == "bf16" else s["p"], s["g"], lr=s["lr"], momentum=s["momentum"],
                        nesterov=c["nesterov"], weight_decay=s["wd"], eps=s["eps"], coefficients=NS, steps=5,
                        scale=s["factor"], masters=s["p"] if c["master"] else False, states=s["m"],
                        zero_grads=c["zero_grads"])
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(state):
    s = state
    if s["op"] == "quantize":
        return _quantize_own(s) if own else _quantize_plain(s)
    if s["op"] == "ffn4":
        return _ffn4_own(s) if own else _ffn4_plain(s)
    if s["op"] == "few":
        return _few_own(s) if own else _few_plain(s)
    return _muon_own(s) if own else _muon_plain(s)


# Quantisation. 32 consecutive elements of a row share a scale 2^e, e the least
# at which the largest is below 7 * 2^e and so rounds to 6 * 2^e at most; an
# element is rounded to the nearest of GRID times the scale, ties to the even
# code. A row's last block may be short.
def _quantize(x):
    """x [rows, cols] fp32: elements over their scales, rounded [rows, blocks, 32], and e [rows, blocks]."""
    rows, cols = x.shape
    b = torch.nn.functional.pad(x, (0, -cols % MX)).view(rows, -1, MX)
    top = b.abs().amax(-1)
    e = (((top.view(I32) + 0x200000) >> 23) - 129).clamp(min=-127)
    y = b * _power(-e)[..., None]
    a = y.abs()
    r = torch.zeros_like(a)
    r += 0.5 * (a > 0.25) + 0.5 * (a >= 0.75) + 0.5 * (a > 1.25) + 0.5 * (a >= 1.75)
    r += 1.0 * (a > 2.5) + 1.0 * (a >= 3.5) + 2.0 * (a > 5.0)
    return torch.where(y < 0, -r, r), e


def _power(e):
    """2^e, exact, e in [-126, 127]."""
    return ((e + 127) << 23).view(F32)


def _code_of(q):
    """The 4-bit codes of rounded elements: a sign bit over the place in GRID."""
    a = q.abs()
    place = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4))
    return (place + torch.where(q < 0, 8, 0)).to(U8)


def _values(codes, scales, dtype=F32):
    """What codes [..., n / 2] and scales [..., n / 32] stand for."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()
    v = torch.tensor(GRID + tuple(-a for a in GRID), dtype=dtype, device=codes.device)[c]
    v = v.unflatten(-1, (-1, MX)) * _power(scales.to(I32) - 127).to(dtype)[..., None]
    return v.flatten(-2)


def _quantize_own(s):
    from paper_2606_11867_amd import api
    q = api.mxfp4_quantize(s["x_t"])
    return dict(values=api.mxfp4_values(q, s["cols"], dtype=BF16))


def _quantize_plain(s):
    q, e = _quantize(s["x_t"].float())
    return dict(values=(q * _power(e)[..., None]).flatten(1)[:, :s["cols"]].to(BF16))


def _silu(a):
    return a / (1.0 + torch.exp(-a))


def _ffn4_own(s):
    from paper_2606_11867_amd import api
    x = api.mxfp4_quantize(s["x_t"], n_rows=s["off"][-1:])
    return dict(y=api.grouped_ffn_mxfp4_fwd(x, s["off"], s["widx"], s["gu"], s["dn"], ws=s["ws"]))


def _ffn4_plain(s):
    q, e = _quantize(s["x_t"].float())
    x = (q * _power(e)[..., None]).flatten(1)
    F, at, W = s["F"], s["bounds"], s["weights"]
    gu, dn = _values(*s["gu"]), _values(*s["dn"])
    y = torch.empty_like(s["x_t"])
    for j in range(s["slots"]):
        if at[j] < at[j + 1]:
            au = x[at[j]:at[j + 1]] @ gu[j % W].t()
            # the hidden rows are quantised too, before the second product
            q, e = _quantize(_silu(au[:, :F]) * au[:, F:])
            y[at[j]:at[j + 1]] = (q * _power(e)[..., None]).flatten(1) @ dn[j % W].t()
    return dict(y=y)


def _few_own(s):
    from paper_2606_11867_amd import api
    return dict(y=api.few_tokens_ffn(s["x_t"], s["ids"], s["gates"], s["gu"], s["dn"], expert_widx=s["widx"],
                                     out_dtype=DT[s["out"]], ws=s["ws"]))


def _few_plain(s):
    x, ids, F, W = s["x_t"].float(), s["ids"].long(), s["F"], s["W"]
    T, K = ids.shape
    w = torch.where(ids >= 0, s["widx"][ids.clamp(min=0)].long(), -1)
    gates = torch.where(w >= 0, s["gates"], 0.0)
    few = T * K <= W  # the picked experts' weights, or every expert's
    at = w.clamp(min=0).view(-1)
    read = lambda m: _values(*(t[at] if few else t for t in m)) if s["w"] == "mxfp4" else \
        (m[at] if few else m).float()  # noqa: E731
    rows = x.repeat_interleave(K, 0)[:, None, :] if few else x.expand(W, T, -1)
    au = torch.bmm(rows, read(s["gu"]).transpose(1, 2))
    h = _silu(au[..., :F]) * au[..., F:]
    # an expert's output counts by its gate: those of a token's pairs, or of a (token, expert) table
    if few:
        h = h * gates.view(-1, 1, 1)
        y = torch.bmm(h, read(s["dn"]).transpose(1, 2)).view(T, K, -1).sum(1)
    else:
        table = torch.zeros(T, W, device=x.device).scatter_add_(1, w.clamp(min=0), gates)
        y = torch.bmm(h * table.t()[..., None], read(s["dn"]).transpose(1, 2)).sum(0)
    return dict(y=y.to(DT[s["out"]]))


def _muon_own(s):
    s["opt"].step(grad_scale=s["clip_t"])
    return _muon_out(s)


def _muon_out(s):
    out = dict(m=s["m"])
    if s["param"] == "bf16":
        out["param"] = s["p16"]
    if s["master"] or s["param"] == "f32":
        out["master"] = s["p"]
    if s["zero_grads"]:
        out["grad"] = s["g"]
    return out


def _muon_plain(s):
    a, b, c = NS
    for p, p16, grad, m, factor in zip(s["p"], s["p16"], s["g"], s["m"], s["factor"]):
        g = grad.float()
        if s["clip_t"] is not None:
            g = g * s["clip_t"]
        m.mul_(s["momentum"]).add_(g)
        x = g + s["momentum"] * m if s["nesterov"] else m
        tall = x.shape[1] > x.shape[2]
        if tall:
            x = x.transpose(1, 2)
        x = x.contiguous() / torch.sqrt(x.square().sum((1, 2), keepdim=True)).clamp(min=s["eps"])
        for _ in range(5):
            gram = torch.bmm(x, x.transpose(1, 2).contiguous())
            x = a * x + torch.bmm(b * gram + c * torch.bmm(gram, gram), x)
        if tall:
            x = x.transpose(1, 2)
        w = p16.float() if p is None else p
        w.mul_(1 - s["lr"] * s["wd"]).sub_(x, alpha=s["lr"] * factor)
        if p16 is not None:
            p16.copy_(w)
        if s["zero_grads"]:
            grad.zero_()
    return _muon_out(s)


# ---------------------------------------------------------------------------
# The operators' definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"quantize": _quantize_exact, "ffn4": _ffn4_exact, "few": _few_exact, "muon": _muon_exact}[s["op"]](s)


def _nearest4(x):
    """The values that rows of x are held as: the last dimension in blocks of 32."""
    x = x.double()
    n = x.shape[-1]
    x = torch.cat([x, x.new_zeros(*x.shape[:-1], -n % MX)], -1).unflatten(-1, (-1, MX))
    top = x.abs().max(-1, keepdim=True).values
    e = torch.frexp(top / 7).exponent.clamp(min=-127)  # the least e with top / 7 < 2^e
    scale = (e.long() + 1023 << 52).view(F64)
    y = x / scale
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0)).double()
    y = torch.round(y / step) * step * scale
    return y.flatten(-2)[..., :n]


def _quantize_exact(s):
    return dict(values=_nearest4(s["x_t"]))


def _swiglu(au, F):
    return torch.nn.functional.silu(au[..., :F]) * au[..., F:]


def _held(m):
    return _values(*m, dtype=F64)


def _ffn4_exact(s):
    x = _nearest4(s["x_t"])
    y = torch.zeros_like(x)
    for j in range(s["slots"]):
        r, w = slice(*s["bounds"][j:j + 2]), j % s["weights"]
        gu, dn = (_held([t[w] for t in m]) for m in (s["gu"], s["dn"]))
        y[r] = _nearest4(_swiglu(x[r] @ gu.T, s["F"])) @ dn.T
    return dict(y=y)


def _few_exact(s):
    x, ids = s["x_t"].double(), s["ids"].long()
    y = torch.zeros_like(x)
    at = torch.where(ids < 0, ids, s["widx"].long()[ids])
    for w in range(s["W"]):
        t, k = torch.nonzero(at == w, as_tuple=True)
        if t.numel():
            gu, dn = ((_held([v[w] for v in m]) if s["w"] == "mxfp4" else m[w].double()) for m in (s["gu"], s["dn"]))
            y.index_add_(0, t, s["gates"][t, k, None].double() * (_swiglu(x[t] @ gu.T, s["F"]) @ dn.T))
    return dict(y=y)


def _muon_exact(s):
    out = dict(m=[], param=[], master=[], grad=[])
    for p, p16, grad, m, factor in zip(s["p"], s["p16"], s["g"], s["m"], s["factor"]):
        g = grad.double() * (1.0 if s["clip_t"] is None else s["clip_t"].double())
        m = s["momentum"] * m.double() + g
        u = g + s["momentum"] * m if s["nesterov"] else m
        u = u / torch.linalg.norm(u, dim=(1, 2), keepdim=True).clamp(min=s["eps"])
        # an odd polynomial of the singular values: on whichever side the Gram matrix is smaller
        wide = u.shape[1] <= u.shape[2]
        for _ in range(5):
            t = u.mT.contiguous()
            gram = u @ t if wide else t @ u
            poly = NS[1] * gram + NS[2] * (gram @ gram)
            u = NS[0] * u + (poly @ u if wide else u @ poly)
        w = (p16 if p is None else p).double()
        w = w - s["lr"] * s["wd"] * w - s["lr"] * factor * u
        out["m"].append(m)
        out["param"].append(w)
        out["master"].append(w)
        out["grad"].append(torch.zeros_like(w))
    if s["param"] != "bf16":
        del out["param"]
    if not (s["master"] or s["param"] == "f32"):
        del out["master"]
    if not s["zero_grads"]:
        del out["grad"]
    return out
