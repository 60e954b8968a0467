"""The performance cases of libheinsen's operators for language models, over the range of sizes their users call them at.

Two families: linear attention with a decay for each head (the recurrence S_t = a_t S_{t-1} + k_t v_t^T of a matrix
state, o_t = scale S_t^T q_t: prompts, single tokens, training) and the norms around a block, fused with its gate,
residual scale and residual.  `listed()` names the kinds of use, `draw()` gives more sizes of the same kinds, `run()`
makes one pass in the plain form or through the library, `exact()` evaluates the definitions in float64.
"""
from __future__ import annotations

import math
import random

import torch

own = False  # True: run() calls the library; False: the plain form

# ---- the kinds of use ---------------------------------------------------------------------------------
#
# op      "attention" | "norm"
# step    True: the state is updated in place by one token per sequence; False: prompts of up to n tokens
# train   True: the pass returns the gradients of every input beside the outputs
# ragged  True: sequences of different lengths, none and one among them, packed one after the other
# H, Hk   heads of v and of the state; heads of q and k, each shared by H / Hk of them
# decay   "token": a decay for each token and head; "head": one for each head
# full    norm with residual, residual scale and the norm before the next block; else the norm and gate of heads

_LISTED = [
    # A recurrent model generating one token for one user: latency only.
    dict(name="attention_step_one", op="attention", step=True, train=False, ragged=False, B=1, n=1, H=8, Hk=8, K=128, V=128, bf16=True, decay="token"),
    # The same in a serving loop over a batch: the states are read and written once.
    dict(name="attention_step_batch", op="attention", step=True, train=False, ragged=False, B=64, n=1, H=32, Hk=32, K=128, V=128, bf16=True, decay="token"),
    # Prompts of different lengths that continue from stored states.
    dict(name="attention_prompts", op="attention", step=False, train=False, ragged=True, B=16, n=4096, H=8, Hk=8, K=128, V=128, bf16=True, decay="token"),
    # A wide layer over long sequences.
    dict(name="attention_layer_large", op="attention", step=False, train=False, ragged=False, B=16, n=16384, H=16, Hk=16, K=128, V=128, bf16=True, decay="token"),
    # Very long sequences of few small heads, each with a fixed decay.
    dict(name="attention_long_tracks", op="attention", step=False, train=False, ragged=False, B=2, n=131072, H=2, Hk=2, K=48, V=48, bf16=False, decay="head"),
    # A layer in training: outputs, final states and the gradients of every input.
    dict(name="attention_training", op="attention", step=False, train=True, ragged=False, B=8, n=4096, H=8, Hk=8, K=128, V=128, bf16=True, decay="token"),
    # The same in float32 with smaller heads.
    dict(name="attention_training_float32", op="attention", step=False, train=True, ragged=False, B=8, n=4096, H=16, Hk=16, K=64, V=64, bf16=False, decay="token"),
    # Sizes that are multiples of nothing, queries and keys shared by two heads of values.
    dict(name="attention_training_odd", op="attention", step=False, train=True, ragged=True, B=6, n=3001, H=10, Hk=5, K=55, V=77, bf16=True, decay="token"),
    # Between two blocks of a model that generates tokens.
    dict(name="norm_step", op="norm", train=False, rows=64, D=4096, bf16=True, full=True),
    # Between two blocks in training.
    dict(name="norm_training", op="norm", train=True, rows=8 * 4096, D=1024, bf16=True, full=True),
    # The same at the largest size, in float32.
    dict(name="norm_training_large", op="norm", train=True, rows=16 * 8192, D=2048, bf16=False, full=True),
    # The norm and gate of attention heads of an odd width.
    dict(name="norm_heads", op="norm", train=True, rows=6 * 3001 * 7, D=110, bf16=True, full=False),
]

# Ranges of each kind.  Attention: B, n, H, H / Hk, K, V and the most B n H (K + V) a drawn call has; norm: rows, D, the most rows D.
_RANGES = {
    "attention_step_one": ((1, 4), (1, 1), (2, 16), (1, 2), (32, 128), (32, 128), 1 << 22),
    "attention_step_batch": ((8, 128), (1, 1), (4, 64), (1, 4), (32, 128), (32, 128), 1 << 20),
    "attention_prompts": ((2, 32), (64, 8192), (2, 32), (1, 4), (32, 128), (32, 128), 1 << 27),
    "attention_layer_large": ((1, 32), (1024, 32768), (4, 32), (1, 1), (64, 128), (64, 128), 1 << 29),
    "attention_long_tracks": ((1, 4), (1 << 14, 1 << 17), (1, 4), (1, 1), (16, 128), (16, 128), 1 << 26),
    "attention_training": ((1, 16), (256, 8192), (2, 32), (1, 1), (64, 128), (64, 128), 1 << 26),
    "attention_training_float32": ((1, 16), (256, 8192), (2, 32), (1, 1), (32, 128), (32, 128), 1 << 26),
    "attention_training_odd": ((1, 16), (65, 4095), (2, 16), (1, 4), (17, 127), (17, 127), 1 << 25),
    "norm_step": ((1, 512), (256, 8192), 1 << 21),
    "norm_training": ((1 << 11, 1 << 16), (256, 8192), 1 << 26),
    "norm_training_large": ((1 << 14, 1 << 18), (512, 8192), 1 << 28),
    "norm_heads": ((1 << 12, 1 << 18), (17, 256), 1 << 25),
}
_ROUND = {"attention_step_one", "attention_step_batch", "attention_layer_large", "attention_training", "attention_training_float32",
          "norm_step", "norm_training", "norm_training_large"}  # widths are usually chosen round there


def listed():
    return [dict(c) for c in _LISTED]


def draw(rng):
    """One more call of one of the kinds: sizes log-uniform over the kind's range, round ones and odd ones."""
    def size(lo, hi, unit=1):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return min(max(v // unit * unit if v > unit else v, lo), hi)

    case = dict(rng.choice(_LISTED))
    kind = case.pop("name")
    unit = 16 if kind in _ROUND and rng.random() < 0.8 else 1
    if case["op"] == "norm":
        rows, d, most = _RANGES[kind]
        while True:
            case["rows"], case["D"] = size(*rows), size(*d, unit)
            if case["rows"] * case["D"] <= most:
                return case
    b, n, h, shared, k, v, most = _RANGES[kind]
    while True:
        case["B"], case["n"] = size(*b), size(*n, 64 if rng.random() < 0.5 else 1)
        share = size(*shared)
        case["Hk"] = max(1, size(*h) // share)
        case["H"] = case["Hk"] * share
        case["K"], case["V"] = size(*k, unit), size(*v, unit)
        if case["B"] * case["n"] * case["H"] * (case["K"] + case["V"]) <= most:
            return case


# ---- inputs -------------------------------------------------------------------------------------------

EPS = 1e-6


def _lengths(case, seed):
    """How many tokens each sequence has: all n, or ragged ones with none, one and n among them, in an order of the seed."""
    if not case["ragged"]:
        return [case["n"]] * case["B"]
    rng = random.Random(case["B"] * case["n"])
    some = [0, 1][:max(0, case["B"] - 2)]
    lengths = some + [max(1, int(case["n"] * rng.random() ** 1.5)) for _ in range(case["B"] - 1 - len(some))] + [case["n"]]
    random.Random(seed).shuffle(lengths)
    return lengths


def _tokens(case):
    """Tokens of a pass, of all sequences together."""
    return sum(_lengths(case, 0))


def _attention_inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = torch.bfloat16 if case["bf16"] else torch.float32
    lengths = _lengths(case, seed)
    total, B, H, Hk, K, V = sum(lengths), case["B"], case["H"], case["Hk"], case["K"], case["V"]

    def normal(*size, mean=0.0, std=1.0):
        return torch.empty(size, dtype=torch.float32, device="cuda").normal_(mean, std, generator=g)

    x = {"q": normal(total, Hk, K).to(dtype), "k": normal(total, Hk, K).to(dtype), "v": normal(total, H, V).to(dtype)}
    # logarithms of sigmoid gates; the heads remember from a few to a few hundred tokens
    slow = 0.5 ** (torch.arange(H, device="cuda") % 7).float()
    gates = normal(H, mean=2.0) if case["decay"] == "head" else normal(total, H, mean=2.0)
    x["log_a"] = (torch.nn.functional.logsigmoid(gates) * slow).to(dtype)
    x["s0"] = normal(B, H, K, V)
    if case["train"]:
        x["grad_out"] = normal(total, H, V).to(dtype)
        x["grad_sn"] = normal(B, H, K, V, std=0.1)
    return x, lengths


def _norm_inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = torch.bfloat16 if case["bf16"] else torch.float32
    rows, D = case["rows"], case["D"]

    def normal(*size, mean=0.0, std=1.0):
        return torch.empty(size, dtype=torch.float32, device="cuda").normal_(mean, std, generator=g)

    x = {"u": normal(rows, D).to(dtype), "gate": normal(rows, D).to(dtype), "w_post": normal(D, mean=1.0, std=0.1)}
    if case["full"]:
        x |= {"residual": normal(rows, D, std=2.0).to(dtype), "scale": normal(D, mean=0.5, std=0.1), "w_pre": normal(D, mean=1.0, std=0.1)}
    if case["train"]:
        x["grad_h"] = normal(rows, D).to(dtype)
        if case["full"]:
            x["grad_y"] = normal(rows, D).to(dtype)
    return x


def prepare(case, seed):
    if case["op"] == "norm":
        x = _norm_inputs(case, seed)
        s = {"case": case, **x, "h": torch.empty_like(x["u"])}
        if case["full"]:
            s["y"] = torch.empty_like(x["u"])
        if case["train"]:
            s["grads"] = {n: torch.empty_like(x[n]) for n in ("u", "gate", "residual", "scale", "w_post", "w_pre") if n in x}
        return s
    x, lengths = _attention_inputs(case, seed)
    s = {"case": case, **x, "out": torch.empty_like(x["v"])}
    s["sn"] = x["s0"] if case["step"] else torch.empty_like(x["s0"])
    if case["ragged"]:  # where the sequences start, and where each packed token is among B sequences of n
        s["starts"] = torch.tensor([sum(lengths[:b]) for b in range(len(lengths) + 1)], dtype=torch.int64, device="cuda")
        s["place"] = torch.cat([torch.arange(m, device="cuda") + b * case["n"] for b, m in enumerate(lengths)])
    if case["train"]:
        s["grads"] = {n: torch.empty_like(x[n]) for n in ("q", "k", "v", "log_a", "s0")}
    return s


# ---- one pass -----------------------------------------------------------------------------------------

def run(state):
    norm = state["case"]["op"] == "norm"
    if own:
        return _own_norm(state) if norm else _own_attention(state)
    return _plain_norm_pass(state) if norm else _plain_attention_pass(state)


def _own_attention(s):
    from paper_2311_06281_amd import binding as hs

    c, stream = s["case"], torch.cuda.current_stream()
    flags = (hs.HEINSEN_IN_BF16 if c["bf16"] else 0) | (hs.HEINSEN_DECAY_PER_HEAD if c["decay"] == "head" else 0)
    scale = c["K"] ** -0.5
    hs.heinsen_linear_attention(s["q"], s["k"], s["v"], s["log_a"], s["s0"], s["out"], s["sn"], c["B"], c["n"], c["H"], c["K"], c["V"],
                                scale, flags, stream, Hk=c["Hk"], starts=s.get("starts"))
    if not c["train"]:
        return {"out": s["out"], "sn": s["sn"]}
    g = s["grads"]
    hs.heinsen_linear_attention_backward(s["q"], s["k"], s["v"], s["log_a"], s["s0"], s["grad_out"], s["grad_sn"], g["q"], g["k"], g["v"],
                                         g["log_a"], g["s0"], c["B"], c["n"], c["H"], c["K"], c["V"], scale, flags, stream, Hk=c["Hk"],
                                         starts=s.get("starts"))
    return {"out": s["out"], "sn": s["sn"], "grads": g}


def _own_norm(s):
    from paper_2311_06281_amd import binding as hs

    c, stream = s["case"], torch.cuda.current_stream()
    flags = hs.HEINSEN_IN_BF16 if c["bf16"] else 0
    given = [s["u"], s["gate"]] + [s.get(n) for n in ("residual", "scale", "w_post", "w_pre")]
    hs.heinsen_block_norm(*given, s["h"], s.get("y"), c["rows"], c["D"], EPS, flags, stream)
    outputs = {n: s[n] for n in ("h", "y") if n in s}
    if not c["train"]:
        return outputs
    g = s["grads"]
    hs.heinsen_block_norm_backward(*given, s["grad_h"], s.get("grad_y"), *(g.get(n) for n in ("u", "gate", "residual", "scale", "w_post", "w_pre")),
                                   c["rows"], c["D"], EPS, flags, stream)
    return {**outputs, "grads": g}


CHUNK = 64


def _plain_attention(q, k, v, log_a, s0, scale):
    """out [B, n, H, V] and the final states, in chunks of 64 tokens: products within a chunk, the chunks' own sums of
    k v^T, and the states at their starts as one product with the decays between chunks.  q, k: [B, n, H, K]."""
    B, n, H, V = v.shape
    chunks = -(-n // CHUNK)

    def cut(x):  # [B, n, H, ...] -> [B, H, chunks, CHUNK, ...], zeros after the end
        x = torch.nn.functional.pad(x, (0, 0) * (x.dim() - 2) + (0, chunks * CHUNK - n))
        return x.reshape(B, chunks, CHUNK, *x.shape[2:]).movedim(3, 1)

    q, k, v = cut(q), cut(k), cut(v)
    decay = cut(log_a.unsqueeze(-1)).squeeze(-1).cumsum(-1)
    seen = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=q.device).tril()
    weights = (decay.unsqueeze(-1) - decay.unsqueeze(-2)).masked_fill(~seen, -math.inf).exp()
    within = (q @ k.transpose(-1, -2).contiguous() * weights) @ v
    last = decay[..., -1:]
    sums = (k * (last - decay).exp().unsqueeze(-1)).transpose(-1, -2).contiguous() @ v  # [B, H, chunks, K, V]
    # decay from the end of chunk j to the end of chunk c: sums that start at j, so that they keep their precision
    later = torch.ones(chunks, chunks, dtype=torch.bool, device=q.device).tril(-1)
    between = last.expand(-1, -1, -1, chunks).masked_fill(~later, 0.0).cumsum(-2).masked_fill(later.T, -math.inf).exp()
    ends = (between @ sums.flatten(-2)).view_as(sums) + last.cumsum(-2).exp().unsqueeze(-1) * s0.unsqueeze(2)
    starts = torch.cat([s0.unsqueeze(2), ends[:, :, :-1]], 2)
    out = scale * (within + decay.exp().unsqueeze(-1) * (q @ starts))
    return out.movedim(1, 3).reshape(B, chunks * CHUNK, H, V)[:, :n], ends[:, :, -1]


def _plain_attention_pass(s):
    c = s["case"]
    dtype, B, n, H, share = s["v"].dtype, c["B"], c["n"], c["H"], c["H"] // c["Hk"]
    names = ("q", "k", "v", "log_a", "s0")
    x = {m: s[m].float().requires_grad_(c["train"]) for m in names}
    scale = c["K"] ** -0.5
    if c["step"]:
        q, k = (x[m].repeat_interleave(share, 1) for m in "qk")
        new = x["log_a"].exp()[..., None, None] * x["s0"] + k.unsqueeze(-1) * x["v"].unsqueeze(-2)
        out = scale * (q.unsqueeze(-1) * new).sum(-2)
        s["sn"].copy_(new)
        return {"out": out.to(dtype), "sn": s["sn"]}

    def padded(t):  # packed tokens to [B, n, ...]
        if not c["ragged"]:
            return t.reshape(B, n, *t.shape[1:])
        return torch.zeros(B * n, *t.shape[1:], device=t.device).index_copy(0, s["place"], t).reshape(B, n, *t.shape[1:])

    log_a = x["log_a"].expand(B, n, H) if c["decay"] == "head" else padded(x["log_a"])
    out, sn = _plain_attention(padded(x["q"].repeat_interleave(share, 1)), padded(x["k"].repeat_interleave(share, 1)), padded(x["v"]), log_a,
                               x["s0"], scale)
    out = out.reshape(B * n, *out.shape[2:])
    out = out.index_select(0, s["place"]) if c["ragged"] else out
    if not c["train"]:
        return {"out": out.to(dtype), "sn": sn}
    grads = torch.autograd.grad([out, sn], [x[m] for m in names], [s["grad_out"].float(), s["grad_sn"]])
    return {"out": out.detach().to(dtype), "sn": sn.detach(), "grads": {m: g.to(s[m].dtype) for m, g in zip(names, grads)}}


def _plain_norm_pass(s):
    c, dtype = s["case"], s["u"].dtype
    names = [m for m in ("u", "gate", "residual", "scale", "w_post", "w_pre") if m in s]
    x = {m: s[m].float().detach().requires_grad_(c["train"]) for m in names}
    h = x["u"] * (x["u"].square().mean(-1, keepdim=True) + EPS).rsqrt() * x["w_post"] * (x["gate"] * x["gate"].sigmoid())
    outputs = {"h": h}
    if c["full"]:
        h = x["residual"] + x["scale"] * h
        outputs = {"h": h, "y": h * (h.square().mean(-1, keepdim=True) + EPS).rsqrt() * x["w_pre"]}
    rounded = {m: t.detach().to(dtype) for m, t in outputs.items()}
    if not c["train"]:
        return rounded
    grads = torch.autograd.grad(list(outputs.values()), [x[m] for m in names], [s["grad_" + m].float() for m in outputs])
    return {**rounded, "grads": {m: g.to(s[m].dtype) for m, g in zip(names, grads)}}


# ---- what a pass cannot do without ----------------------------------------------------------------------

def work(case):
    """Inputs read once, outputs written once; a training pass reads the inputs once and returns outputs and gradients.
    Attention: two products and two sums for each entry of a state and token, ten more for the gradients."""
    size = 2 if case["bf16"] else 4
    if case["op"] == "norm":
        elements, arrays, vectors = case["rows"] * case["D"], 5 if case["full"] else 3, 3 if case["full"] else 1
        per = 16 if case["full"] else 8
        if case["train"]:
            arrays += 2 + 3 if case["full"] else 1 + 2
            vectors *= 2
            per *= 3
        return {"bytes": size * arrays * elements + 4 * vectors * case["D"], "flops": per * elements}
    tokens, B, H, Hk, K, V = _tokens(case), case["B"], case["H"], case["Hk"], case["K"], case["V"]
    inputs = 2 * Hk * K + H * V + (H if case["decay"] == "token" else 0)
    arrays = inputs + H * V
    states = 2
    flops = 4
    if case["train"]:
        arrays += inputs + H * V
        states += 2
        flops += 10
    return {"bytes": size * tokens * arrays + 4 * states * B * H * K * V, "flops": flops * tokens * H * K * V}


# ---- the definitions in float64 -------------------------------------------------------------------------

def exact(case, seed):
    return _exact_norm(case, seed) if case["op"] == "norm" else _exact_attention(case, seed)


def _exact_attention(case, seed):
    """The recurrence one token after the other, and its gradients by going back over it."""
    x, lengths = _attention_inputs(case, seed)
    B, n, H, Hk, K = case["B"], case["n"], case["H"], case["Hk"], case["K"]
    share, scale = H // Hk, K ** -0.5
    place = torch.cat([torch.arange(m, device="cuda") * B + b for b, m in enumerate(lengths)])  # [n, B]: a token of all sequences is one piece

    def by_token(t):
        return torch.zeros(n * B, *t.shape[1:], dtype=torch.float64, device="cuda").index_copy_(0, place, t.double()).view(n, B, *t.shape[1:])

    def packed(t):
        return t.flatten(0, 1).index_select(0, place)

    q, k = (by_token(x[m]).repeat_interleave(share, 2) for m in "qk")
    v = by_token(x["v"])
    log_a = x["log_a"].double().expand(n, B, H) if case["decay"] == "head" else by_token(x["log_a"])
    a = log_a.exp()[..., None, None]
    s = x["s0"].double()
    out = torch.empty_like(v)
    if case["train"]:
        d = by_token(x["grad_out"])
        dq = torch.empty_like(q)
    for t in range(n):
        s = torch.addcmul(s * a[t], k[t].unsqueeze(-1), v[t].unsqueeze(-2))
        out[t] = scale * (s * q[t].unsqueeze(-1)).sum(-2)
        if case["train"]:
            dq[t] = scale * (s * d[t].unsqueeze(-2)).sum(-1)
    result = {"out": packed(out), "sn": s}
    if not case["train"]:
        return result
    r = x["grad_sn"].double()
    flow = (r * s).sum((-1, -2))
    dk, dv = torch.empty_like(k), torch.empty_like(v)
    for t in range(n - 1, -1, -1):
        r = torch.addcmul(r, scale * q[t].unsqueeze(-1), d[t].unsqueeze(-2))
        dk[t] = (r * v[t].unsqueeze(-2)).sum(-1)
        dv[t] = (r * k[t].unsqueeze(-1)).sum(-2)
        r = r * a[t]
    # a_t R_t . S_{t-1}: what the tokens from t on take from the state, less what they put into it themselves
    dlog = ((q * dq).sum(-1) - (k * dk).sum(-1)).flip(0).cumsum(0).flip(0) + flow
    shared = lambda t: t.view(n, B, Hk, share, K).sum(3)  # noqa: E731
    dlog = dlog.sum((0, 1)) if case["decay"] == "head" else packed(dlog)
    result["grads"] = {"q": packed(shared(dq)), "k": packed(shared(dk)), "v": packed(dv), "log_a": dlog, "s0": r}
    return result


def _exact_norm(case, seed):
    x = {m: t.double() for m, t in _norm_inputs(case, seed).items()}
    u, gate, w = x["u"], x["gate"], x["w_post"]
    inverse = (u.pow(2).sum(-1, keepdim=True) / case["D"] + EPS).pow(-0.5)
    unit = u * inverse
    sig = 1.0 / (1.0 + torch.exp(-gate))
    act = gate * sig
    scale = x.get("scale", torch.ones((), dtype=torch.float64, device="cuda"))
    h = scale * act * unit * w
    result = {"h": h}
    if case["full"]:
        h = h + x["residual"]
        inverse_h = (h.pow(2).sum(-1, keepdim=True) / case["D"] + EPS).pow(-0.5)
        result = {"h": h, "y": h * inverse_h * x["w_pre"]}
    if not case["train"]:
        return result
    dh, grads = x["grad_h"], {}
    if case["full"]:
        unit_h, dy = h * inverse_h, x["grad_y"]
        grads["w_pre"] = (dy * unit_h).sum(0)
        t = dy * x["w_pre"]
        dh = dh + inverse_h * (t - unit_h * (t * unit_h).mean(-1, keepdim=True))
        grads["residual"] = dh
        grads["scale"] = (dh * act * unit * w).sum(0)
    t = dh * scale
    grads["gate"] = t * unit * w * sig * (1.0 + gate * (1.0 - sig))
    t = t * act
    grads["w_post"] = (t * unit).sum(0)
    t = t * w
    grads["u"] = inverse * (t - unit * (t * unit).mean(-1, keepdim=True))
    return {**result, "grads": grads}
