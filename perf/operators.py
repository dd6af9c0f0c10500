"""The operators of an MoE block that stand beside the DTS-gate layer, as cases that can be timed: the gate's logits,
top-k routing, the residual addition with its root-mean-square norm, and the experts' products in 8 bits.

Every case is one pass of one operator, forward or forward and backward, once in plain torch operations (`own` false) and
once through the entry points of `paper_2112_14397_amd.binding` (`own` true).  Sizes are the layer configurations of this
repository (`synth_inputs.CONFIGS`), ragged ones, and generic ones between them.  Inputs have the distributions of
`synth_inputs`: activations N(0,1), weights and biases N(0, 0.02^2); router logits N(0,1); balance biases N(0, 0.05^2).

8-bit values are e4m3 with one e8m0 scale (a power of two) for 32 neighbours of a row: the scale is the smallest power of
two with which the largest of the 32 stays within 448, at least 2^-127, and the elements are rounded to nearest even.
"""
import math

import torch

own = False

EPS = 1e-6
GROUP = 32               # neighbours that share a scale
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _logits(name, T, d, E, dtype, step):
    return {"op": "logits", "name": name, "T": T, "d": d, "E": E, "dtype": dtype, "step": step}


def _route(name, T, E, k, score, step, groups=1, top_groups=1, group_keys=1, renormalise=True, scale=1.0, bias=False,
           coef=False, padded=0.0):
    """padded: share of the tokens that only fill up the batch, all of whose logits are -inf.  coef: the gradient of a
    balance loss joins the backward."""
    return {"op": "route", "name": name, "T": T, "E": E, "k": k, "score": score, "step": step, "groups": groups,
            "top_groups": top_groups, "group_keys": group_keys, "renormalise": renormalise, "scale": scale, "bias": bias,
            "coef": coef, "padded": padded}


def _norm(name, T, d, dtype, step, residual=True, y=True, eight=False):
    """eight: the norm is also (y) or only written in 8 bits."""
    return {"op": "norm", "name": name, "T": T, "d": d, "dtype": dtype, "step": step, "residual": residual, "y": y,
            "eight": eight}


def _experts(name, T, d, E, F, k, act, skew=0.0):
    """skew: what is added to the log of expert 0's share of the tokens."""
    return {"op": "experts", "name": name, "T": T, "d": d, "E": E, "F": F, "k": k, "act": act, "dtype": "bf16",
            "skew": skew}


def listed():
    return [
        # the GPT-shaped layer's gate, one token for each of 48 sequences: launches and latency
        _logits("logits_gpt_decode", 48, 768, 16, "bf16", False),
        # training the RoBERTa-shaped layer's gate: logits, and their gradients added to the experts' share of dx
        _logits("logits_roberta_step", 16384, 768, 32, "bf16", True),
        # routing a single token: 64 experts in 8 groups, sigmoid scores with a balance bias
        _route("route_one_token", 1, 64, 8, "sigmoid", False, groups=8, top_groups=4, group_keys=2, scale=2.5, bias=True),
        # training the GPT-shaped layer with two experts for a token, softmax scores and the balance loss
        _route("route_gpt_step", 8192, 16, 2, "softmax", True, coef=True),
        # training the large layer: 64 experts in groups, a balance bias, a batch that is partly padding
        _route("route_large_step", 32768, 64, 8, "sigmoid", True, groups=8, top_groups=4, group_keys=2, scale=2.5,
               bias=True, padded=0.03),
        # in front of the GPT-shaped layer while it serves 48 sequences: both outputs, for the gate and for the experts
        _norm("norm_gpt_decode_mx8", 48, 768, "bf16", False, eight=True),
        # a float32 training step of odd sizes, without a residual
        _norm("norm_ragged_f32_step", 777, 260, "f32", True, residual=False),
        # serving prompts, an odd number of tokens
        _norm("norm_gpt_prefill_mx8", 2999, 768, "bf16", False, eight=True),
        # training the large layer
        _norm("norm_large_step", 32768, 1024, "bf16", True),
        # the GPT-shaped experts in 8 bits, from the norm's bf16 rows: single tokens (reading weights is the work),
        # prompts, and the large layer over a whole batch with an expert that is chosen three times as often
        _experts("experts_gpt_decode_mx8", 48, 768, 16, 3072, 1, "gelu"),
        _experts("experts_gpt_prefill_mx8", 2999, 768, 16, 3072, 2, "gelu"),
        _experts("experts_large_mx8", 32768, 1024, 64, 4096, 2, "gelu", skew=1.1),
    ]


def draw(rng):
    """One more case: sizes spread over their logarithm, options as often as they are used."""
    def size(low, high, step=1):
        return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1))) / step)) * step))

    op = rng.choice(("logits", "route", "route", "norm", "norm", "experts"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    step = rng.random() < 0.6
    if op == "logits":
        case = _logits("", size(1, 32768), size(64, 1024, 4 if dtype == "f32" else 8), rng.randint(1, 64), dtype, step)
    elif op == "route":
        groups = rng.choice((1, 1, 2, 4, 8))
        E = groups * rng.randint(1 if groups > 1 else 2, 64 // groups)
        top = rng.randint(1, groups)
        k = rng.randint(1, min(8, E // groups * top))
        case = _route("", size(1, 32768), E, k, rng.choice(("softmax", "sigmoid")), step,
                      groups=groups, top_groups=top, group_keys=rng.choice((1, 2)), renormalise=k > 1 and rng.random() < 0.7,
                      scale=rng.choice((1.0, 2.5)), bias=rng.random() < 0.5, coef=step and rng.random() < 0.4,
                      padded=rng.choice((0.0, 0.0, 0.1)))
    elif op == "norm":
        eight = not step and rng.random() < 0.6
        unit = GROUP if eight else 4 if dtype == "f32" else 8
        case = _norm("", size(1, 32768), size(64, 2048 if dtype == "f32" else 4096, unit), dtype, step,
                     residual=rng.random() < 0.7, y=not eight or rng.random() < 0.5, eight=eight)
        while case["T"] * case["d"] > 32768 * 1024:
            case["T"] = (case["T"] + 1) // 2
    else:
        E = rng.choice((1, 4, 8, 16, 32, 64, rng.randint(2, 64)))
        case = _experts("", size(1, 8192), size(64, 1024, GROUP), E, size(64, 4096, GROUP), rng.randint(1, min(E, 4)),
                        rng.choice(("gelu", "gelu", "relu")), skew=rng.choice((0.0, 0.0, 1.1)))
    del case["name"]
    return case


# ---- inputs --------------------------------------------------------------------------------------

class _State:
    pass


def prepare(case, seed):
    """A program's tensors before the call; where the framework is called, its context and output buffers too."""
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.randn(*shape, generator=g, device=dev, dtype=dtype).mul_(std)

    s = _State()
    s.case = case
    T = case["T"]
    if case["op"] == "logits":
        d, E, dt = case["d"], case["E"], TYPES[case["dtype"]]
        s.x, s.Wg, s.bg = normal(T, d, dtype=dt), normal(d, E, std=0.02), normal(E, std=0.02)
        if case["step"]:
            s.dlogits, s.dx_in = normal(T, E), normal(T, d, dtype=dt)
    elif case["op"] == "route":
        E = case["E"]
        s.logits = normal(T, E)
        if case["padded"]:
            s.logits[torch.rand(T, generator=g, device=dev) < case["padded"]] = -math.inf
        s.bias = normal(E, std=0.05) if case["bias"] else None
        s.dG_pairs = normal(T * case["k"]) if case["step"] else None
        s.coef = normal(E, std=0.1) if case["coef"] else None
    elif case["op"] == "norm":
        d, dt = case["d"], TYPES[case["dtype"]]
        s.x, s.res = normal(T, d, dtype=dt), normal(T, d, dtype=dt) if case["residual"] else None
        s.gamma = normal(d, std=0.1).add_(1.0)
        if case["step"]:
            s.dy, s.dh = normal(T, d, dtype=dt), normal(T, d, dtype=dt)
    else:
        d, E, F, k = case["d"], case["E"], case["F"], case["k"]
        s.x = normal(T, d, dtype=TYPES[case["dtype"]])
        # the weights as they are kept for serving: 8 bits and their scales
        s.W1, s.S1 = _to_mx8(normal(E, F, d, std=0.02))
        s.W2, s.S2 = _to_mx8(normal(E, d, F, std=0.02))
        s.b1, s.b2 = normal(E, F, std=0.02), normal(E, d, std=0.02)
        # k distinct experts for every token; the pairs by expert, by token inside an expert
        share = torch.rand(T, E, generator=g, device=dev).clamp_(1e-7, 1.0 - 6e-8).log_().neg_().log_().neg_()
        share[:, 0] += case["skew"]
        chosen = torch.zeros(T, E, dtype=torch.bool, device=dev).scatter_(1, share.topk(k, dim=1).indices, True)
        expert, token = chosen.t().nonzero(as_tuple=True)
        counts = chosen.sum(0)
        s.offsets = torch.zeros(E + 1, dtype=torch.int32, device=dev)
        s.offsets[1:] = counts.cumsum(0)
        s.pair_token = token.to(torch.int32)
        # the plain form's plan: every expert's pairs in as many places as the fullest expert has
        s.most = int(counts.max().item())
        s.expert, s.place = expert, torch.arange(T * k, device=dev) - s.offsets[expert].long()
    if own:
        _prepare_own(s, case, dev)
    return s


def _prepare_own(s, case, dev):
    from paper_2112_14397_amd import binding as B
    s.ctx = B.Context()
    T, op = case["T"], case["op"]

    def out(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device=dev)

    i32, e4m3, e8m0 = torch.int32, torch.float8_e4m3fn, torch.float8_e8m0fnu
    if op == "logits":
        d, E = case["d"], case["E"]
        s.shape = B.make_shape(T, d, E, d, case["dtype"], "gelu", T)
        s.logits = out(T, E)
        if case["step"]:
            s.dWg, s.dbg, s.dx = out(d, E), out(E), torch.empty_like(s.dx_in)
            s.workspace = out(B.evomoe_workspace_bytes(s.shape), dtype=torch.uint8)
    elif op == "route":
        E, k = case["E"], case["k"]
        s.shape = B.make_shape(T, 64, E, 64, "f32", "gelu", T * k)
        s.topk = B.make_topk(k, case["score"], groups=case["groups"], top_groups=case["top_groups"],
                             group_keys=case["group_keys"], renormalise=case["renormalise"], scale=case["scale"])
        s.scores, s.gate_w, s.mask = out(T, E), out(T, E), out(T, dtype=torch.int64)
        s.counts, s.k = out(E, dtype=i32), out(T, dtype=i32)
        if case["step"]:
            s.hist = out((T + 255) // 256, E, dtype=i32)
            s.offsets, s.pair_token, s.pair_gate = out(E + 1, dtype=i32), out(T * k, dtype=i32), out(T * k)
            s.tok_off, s.tok_rows, s.num_pairs = out(T + 1, dtype=i32), out(T * k, dtype=i32), out(1, dtype=torch.int64)
            s.dlogits = out(T, E)
    elif op == "norm":
        d = case["d"]
        s.shape = B.make_shape(T, d, 1, d, case["dtype"], "gelu", T)
        s.h = torch.empty_like(s.x) if case["residual"] else None
        s.y = torch.empty_like(s.x) if case["y"] else None
        s.q, s.scale = (out(T, d, dtype=e4m3), out(T, d // GROUP, dtype=e8m0)) if case["eight"] else (None, None)
        s.rstd = out(T) if case["step"] else None
        if case["step"]:
            s.dx, s.dgamma = torch.empty_like(s.x), out(d)
            s.workspace = out(B.evomoe_workspace_bytes(s.shape), dtype=torch.uint8)
    else:
        d, E, F, P = case["d"], case["E"], case["F"], T * case["k"]
        s.shape = B.make_shape(T, d, E, F, case["dtype"], case["act"], P)
        s.xq, s.xs = out(T, d, dtype=e4m3), out(T, d // GROUP, dtype=e8m0)
        s.O = out(P, d, dtype=s.x.dtype)
        s.workspace = out(B.evomoe_workspace_bytes_mx8(s.shape), dtype=torch.uint8)


# ---- the framework's calls ---------------------------------------------------------------------------

def _run_own(s):
    from paper_2112_14397_amd import binding as B
    case, op = s.case, s.case["op"]
    if op == "logits":
        B.evomoe_gate_logits(s.ctx, s.shape, s.x, s.Wg, s.bg, s.logits)
        out = {"logits": s.logits}
        if case["step"]:
            B.evomoe_gate_logits_bwd(s.ctx, s.shape, s.dlogits, s.x, s.Wg, s.dx_in, s.dWg, s.dbg, s.dx, s.workspace)
            out.update(dWg=s.dWg, dbg=s.dbg, dx=s.dx)
        return out
    if op == "route":
        B.evomoe_topk_gate(s.ctx, s.shape, s.topk, s.logits, s.bias, s.scores, s.gate_w, s.mask, s.counts, s.k,
                           s.hist if case["step"] else None)
        out = {"scores": s.scores, "gate_w": s.gate_w, "mask": s.mask, "counts": s.counts, "k": s.k}
        if case["step"]:
            B.evomoe_dispatch(s.ctx, s.shape, s.mask, s.gate_w, s.offsets, s.pair_token, s.pair_gate, s.tok_off,
                              s.tok_rows, s.num_pairs, block_hist=s.hist)
            B.evomoe_topk_gate_bwd(s.ctx, s.shape, s.topk, s.dG_pairs, s.tok_off, s.tok_rows, s.logits, s.mask,
                                   s.coef, 1.0, s.dlogits)
            out.update(dlogits=s.dlogits)
        return out
    if op == "norm":
        B.evomoe_add_rmsnorm(s.ctx, s.shape, s.x, s.res, s.gamma, EPS, s.h, s.y, s.rstd, s.q, s.scale)
        out = {"h": s.h, "y": s.y, "q": s.q, "scale": s.scale}
        if case["step"]:
            B.evomoe_add_rmsnorm_bwd(s.ctx, s.shape, s.dy, s.dh, s.h if case["residual"] else s.x, s.gamma, s.rstd, s.dx,
                                     s.dgamma, s.workspace)
            out.update(dx=s.dx, dgamma=s.dgamma)
        return out
    B.evomoe_quantize_mx8(s.ctx, s.x, s.xq, s.xs)
    B.evomoe_expert_ffn_mx8(s.ctx, s.shape, s.xq, s.xs, s.pair_token, s.offsets, s.W1, s.S1, s.b1, s.W2, s.S2, s.b2, s.O,
                            s.workspace)
    return {"O": s.O}


# ---- the plain forms -----------------------------------------------------------------------------------

def _to_mx8(v):
    """float32 [..., n] -> e4m3 [..., n] and e8m0 [..., n/32]."""
    groups = v.float().unflatten(-1, (-1, GROUP))
    amax = groups.abs().amax(-1, keepdim=True)
    mantissa, exponent = torch.frexp(amax)                       # amax = mantissa 2^exponent, 448 = 0.875 * 2^9
    exponent = (exponent - 9 + (mantissa > 0.875)).clamp_(min=-127)
    exponent = torch.where(amax > 0, exponent, -127)
    q = torch.ldexp(groups, -exponent).to(torch.float8_e4m3fn).flatten(-2)
    return q, (exponent.squeeze(-1) + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _from_mx8(q, scale):
    return (q.float().unflatten(-1, (-1, GROUP)) * scale.float().unsqueeze(-1)).flatten(-2)


def _act(h, act):
    return h.clamp(min=0) if act == "relu" else 0.5 * h * (1.0 + torch.erf(h * math.sqrt(0.5)))


def _rank(key):
    """Place of every entry of a row in descending order; equal ones by index."""
    i = torch.arange(key.shape[-1], device=key.device)
    a, b = key.unsqueeze(-1), key.unsqueeze(-2)                  # entry, and what it is compared with
    return ((b > a) | ((b == a) & (i < i.unsqueeze(-1)))).sum(-1)


def _plain_route(s):
    """In 64 bits: which experts are taken is decided between neighbouring values."""
    case = s.case
    T, E, k = case["T"], case["E"], case["k"]
    z = s.logits.double()
    if case["score"] == "softmax":
        top = z.amax(1, keepdim=True)
        e = torch.exp(z - torch.where(top > -math.inf, top, 0.0))
        score = e / e.sum(1, keepdim=True).clamp(min=1e-300)
    else:
        score = 1.0 / (1.0 + torch.exp(-z))
    key = score if s.bias is None else score + s.bias.double()
    key = torch.where(z > -math.inf, key, -math.inf)
    if case["groups"] > 1:
        inside = key.view(T, case["groups"], -1)
        first = (_rank(inside) < case["group_keys"]) & (inside > -math.inf)
        group = torch.where(first, inside, 0.0).sum(2)
        group = torch.where(first.any(2), group, -math.inf)
        kept = (_rank(group) < case["top_groups"]).repeat_interleave(E // case["groups"], 1)
        key = torch.where(kept, key, -math.inf)
    taken = (_rank(key) < k) & (key > -math.inf)
    share = torch.where(taken, score, 0.0)
    if case["renormalise"]:
        share = share / share.sum(1, keepdim=True).clamp(min=1e-300)
    counts = taken.sum(1)
    out = {"scores": score.float(), "gate_w": (case["scale"] * share).float(),
           "mask": (taken.long() << torch.arange(E, device=z.device)).sum(1), "counts": taken.sum(0).int(), "k": counts.int()}
    if case["step"]:
        # the row of a pair: pairs are in the order of experts, of tokens inside an expert
        row = (taken.t().flatten().cumsum(0) - 1).clamp(min=0).view(E, T).t()
        dw = torch.where(taken, s.dG_pairs[row].double(), 0.0)
        coef = 0.0 if s.coef is None else s.coef.double()
        if case["renormalise"]:
            of_weight = case["scale"] * share * (dw - (dw * share).sum(1, keepdim=True))       # score times its gradient
        else:
            of_weight = case["scale"] * score * dw
        ds = of_weight + score * coef
        if case["score"] == "softmax":
            out["dlogits"] = (ds - score * ds.sum(1, keepdim=True)).float()
        else:
            out["dlogits"] = (ds * (1.0 - score)).float()
    return out


def _plain_norm(s):
    case = s.case
    h = s.x if s.res is None else (s.x.float() + s.res.float()).to(s.x.dtype)
    hf = h.float()
    rstd = torch.rsqrt((hf * hf).mean(1, keepdim=True) + EPS)
    unit = hf * rstd
    y = unit * s.gamma
    out = {"h": h if case["residual"] else None, "y": y.to(s.x.dtype) if case["y"] else None}
    out["q"], out["scale"] = _to_mx8(y) if case["eight"] else (None, None)
    if case["step"]:
        dy = s.dy.float()
        du = dy * s.gamma
        out["dx"] = (s.dh.float() + rstd * (du - unit * (du * unit).mean(1, keepdim=True))).to(s.x.dtype)
        out["dgamma"] = (dy * unit).sum(0)
    return out


def run(s):
    if own:
        return _run_own(s)
    case, op = s.case, s.case["op"]
    if op == "logits":
        x = s.x.float()
        out = {"logits": x @ s.Wg + s.bg}
        if case["step"]:
            out.update(dWg=x.t() @ s.dlogits, dbg=s.dlogits.sum(0),
                       dx=(s.dx_in.float() + s.dlogits @ s.Wg.t()).to(s.x.dtype))
        return out
    if op == "route":
        return _plain_route(s)
    if op == "norm":
        return _plain_norm(s)
    x = _from_mx8(*_to_mx8(s.x))
    rows = torch.zeros(case["E"], s.most, case["d"], device=x.device)
    rows[s.expert, s.place] = x[s.pair_token.long()]
    H = torch.bmm(rows, _from_mx8(s.W1, s.S1).transpose(1, 2)) + s.b1.unsqueeze(1)
    A = _from_mx8(*_to_mx8(_act(H, case["act"])))
    O = torch.bmm(A, _from_mx8(s.W2, s.S2).transpose(1, 2)) + s.b2.unsqueeze(1)
    return {"O": O[s.expert, s.place].to(s.x.dtype)}


# ---- what cannot be done without -----------------------------------------------------------------------

def work(case):
    T, op = case["T"], case["op"]
    size = 4 if case.get("dtype") == "f32" else 2
    if op == "logits":
        d, E = case["d"], case["E"]
        nbytes, flops = T * d * size + (d + 1) * E * 4 + T * E * 4, 2 * T * d * E
        if case["step"]:
            nbytes += 2 * T * d * size + T * E * 4 + (d + 1) * E * 4
            flops += 4 * T * d * E
    elif op == "route":
        E, k = case["E"], case["k"]
        nbytes, flops = T * E * 12 + T * 12 + E * 8, 8 * T * E
        if case["step"]:
            nbytes += T * E * 4 + T * k * 4
            flops += 8 * T * E
    elif op == "norm":
        d = case["d"]
        row = d * size
        nbytes = T * row * (1 + 2 * case["residual"] + case["y"]) + d * 4
        nbytes += T * (d + d // GROUP) if case["eight"] else 0
        flops = 5 * T * d
        if case["step"]:
            nbytes += 3 * T * row + d * 4
            flops += 10 * T * d
    else:
        d, E, F, P = case["d"], case["E"], case["F"], T * case["k"]
        used = min(E, P)
        nbytes = T * d * size + used * (2 * d * F * (GROUP + 1) // GROUP + (d + F) * 4) + P * d * size + P * 4
        flops = 4 * P * d * F
    return {"bytes": nbytes, "flops": flops}


# ---- the definitions in 64 bits ------------------------------------------------------------------------

def _exact_mx8(v):
    """The elements and scales as float64 numbers, by arithmetic on them alone."""
    g = v.reshape(*v.shape[:-1], v.shape[-1] // GROUP, GROUP)
    largest = g.abs().max(-1).values
    power = torch.ceil(torch.log2(largest / 448.0)).clamp(min=-127.0)
    power = torch.where(largest * torch.exp2(-power) > 448.0, power + 1, power)                  # (where log2 is off by an ulp)
    power = torch.where((largest * torch.exp2(1 - power) <= 448.0) & (power > -127.0), power - 1, power)
    power = torch.where(largest > 0, power, -127.0)
    g = g * torch.exp2(-power)[..., None]
    step = torch.exp2(torch.floor(torch.log2(g.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(g / step) * step).reshape(v.shape), torch.exp2(power)


def _exact_route(s, case):
    T, E, k, n = case["T"], case["E"], case["k"], case["groups"]
    z = s.logits.double()
    dead = z == -math.inf
    score = torch.softmax(z, 1).nan_to_num(0.0) if case["score"] == "softmax" else torch.sigmoid(z)
    key = (score + (0 if s.bias is None else s.bias.double())).masked_fill(dead, -math.inf)
    if n > 1:
        best = key.reshape(T, n, E // n).sort(dim=2, descending=True).values[..., :case["group_keys"]]
        group = best.clamp(min=-1e30).masked_fill(best == -math.inf, 0).sum(2).masked_fill(best[..., 0] == -math.inf, -math.inf)
        order = group.sort(dim=1, descending=True, stable=True).indices[:, :case["top_groups"]]
        open_ = torch.zeros(T, n, dtype=torch.bool, device=z.device).scatter_(1, order, True)
        key = key.reshape(T, n, E // n).masked_fill(~open_[..., None], -math.inf).reshape(T, E)
    order = key.sort(dim=1, descending=True, stable=True).indices[:, :k]
    taken = torch.zeros_like(dead).scatter_(1, order, True) & (key > -math.inf)
    leaf = s.logits.double().requires_grad_(True)
    with torch.enable_grad():
        again = torch.softmax(leaf.masked_fill(dead.all(1, keepdim=True), 0.0), 1) if case["score"] == "softmax" else torch.sigmoid(leaf)
        again = again.masked_fill(dead, 0.0)
        weight = again * taken
        if case["renormalise"]:
            weight = weight / weight.sum(1, keepdim=True).masked_fill(~taken.any(1, keepdim=True), 1.0)
        weight = weight * case["scale"]
        if case["step"]:
            dw = torch.zeros(E, T, dtype=torch.float64, device=z.device)
            picked = taken.t().contiguous()
            dw[picked] = s.dG_pairs[:int(picked.sum())].double()
            loss = (weight * dw.t()).sum()
            if s.coef is not None:
                loss = loss + (again * s.coef.double()).sum()
            loss.backward()
    out = {"scores": score, "gate_w": weight.detach(), "mask": (taken.long() * (1 << torch.arange(E, device=z.device))).sum(1),
           "counts": taken.sum(0).int(), "k": taken.sum(1).int()}
    if case["step"]:
        out["dlogits"] = leaf.grad.masked_fill(dead, 0.0)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "route":
        return _exact_route(s, case)
    if op == "logits":
        x, W = s.x.double(), s.Wg.double()
        out = {"logits": torch.addmm(s.bg.double(), x, W)}
        if case["step"]:
            dz = s.dlogits.double()
            out.update(dWg=torch.mm(x.t(), dz), dbg=torch.mv(dz.t(), torch.ones_like(dz[:, 0])),
                       dx=torch.addmm(s.dx_in.double(), dz, W.t()))
        return out
    if op == "norm":
        # h is what is stored: the sum rounded to the layer's type
        h = s.x.double() if s.res is None else (s.x.double() + s.res.double()).to(s.x.dtype).double()
        r = 1.0 / torch.sqrt(torch.linalg.vector_norm(h, dim=1, keepdim=True) ** 2 / case["d"] + EPS)
        y = s.gamma.double() * h * r
        out = {"h": h if case["residual"] else None, "y": y if case["y"] else None}
        out["q"], out["scale"] = _exact_mx8(y) if case["eight"] else (None, None)
        if case["step"]:
            dy = s.dy.double()
            inner = torch.einsum("td,td,d->t", dy, h, s.gamma.double()).unsqueeze(1)
            out["dx"] = s.dh.double() + r * dy * s.gamma.double() - h * r ** 3 * inner / case["d"]
            out["dgamma"] = torch.mv((dy * h).t(), r.squeeze(1))
        return out
    # expert by expert
    q, scale = _exact_mx8(s.x.double())
    x = (q.reshape(case["T"], -1, GROUP) * scale[..., None]).reshape(case["T"], -1)
    ends = s.offsets.tolist()
    rows = []
    for e in range(case["E"]):
        W1 = s.W1[e].double() * s.S1[e].double().repeat_interleave(GROUP, 1)
        W2 = s.W2[e].double() * s.S2[e].double().repeat_interleave(GROUP, 1)
        H = torch.addmm(s.b1[e].double(), x[s.pair_token[ends[e]:ends[e + 1]].long()], W1.t())
        A = torch.relu(H) if case["act"] == "relu" else H * torch.special.ndtr(H)
        q, scale = _exact_mx8(A)
        A = q * scale.repeat_interleave(GROUP, 1)
        rows.append(torch.addmm(s.b2[e].double(), A, W2.t()))
    return {"O": torch.cat(rows)}
