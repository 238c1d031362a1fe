"""The client's other steps between two delegated products, as a user's program calls them: norms around a block with
its gate and residual, the gated activation of a feed-forward block, and the choice of the next token.

Decoded products come in as field elements with the scales that their weights and activations were quantised by, and the
next product's input goes out as field elements, so results are whole numbers: every step is defined in 32-bit numbers
rounded in a stated order, statistics are formed in more bits and rounded once, and the tokens' weights are integers.  The
plain forms below take the same roundings; 64 bits hold what is summed.
"""
import math
import random

import torch

own = False  # whether run() calls the framework's operators or their plain forms

Q = 15 * 2**27 + 1  # the field of decoded products
FLT_MAX = 3.4028234663852886e38

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "field": torch.int32}


def listed():
    return [
        # one generated token between the attention's output product and the feed-forward block's: all latency
        {"name": "norm_1_token", "op": "norm", "T": 1, "D": 4096, "y": "field", "channel": True, "res": "bf16",
         "post": "none", "pre": "rms", "gate": "none", "weight": "bf16", "out": "field", "dynamic": True, "pad": 0},
        # a batch of generating requests, norms before and after the block, integers by a scale known ahead
        {"name": "norm_64_sandwich", "op": "norm", "T": 64, "D": 8192, "y": "field", "channel": False, "res": "bf16",
         "post": "rms", "pre": "rms", "gate": "none", "weight": "bf16", "out": "field", "dynamic": False, "pad": 0},
        # an odd width and rows off the 16-byte boundaries, everything in 32 bits, a gate of one row
        {"name": "norm_333_odd_f32", "op": "norm", "T": 333, "D": 5001, "y": "f32", "channel": True, "res": "f32",
         "post": "layer", "pre": "rms", "gate": "row", "weight": "f32", "out": "f32", "dynamic": False, "pad": 1},
        # a prompt's chunk, each token with a gate of its own, out of the rows of a wider product
        {"name": "norm_4096_gated_layer", "op": "norm", "T": 4096, "D": 2560, "y": "bf16", "channel": False, "res": "f32",
         "post": "none", "pre": "layer", "gate": "tokens", "weight": "f32", "out": "bf16", "dynamic": False, "pad": 512},
        # the largest: several prompts' tokens to the integers of the next product, each token with its own step
        {"name": "norm_8192_wide", "op": "norm", "T": 8192, "D": 8192, "y": "field", "channel": True, "res": "bf16",
         "post": "none", "pre": "rms", "gate": "none", "weight": "bf16", "out": "field", "dynamic": True, "pad": 0},
        # one generated token inside a feed-forward block: all latency
        {"name": "glu_1_token", "op": "glu", "T": 1, "D": 14336, "x": "field", "channel": True, "gated": True,
         "act": "silu", "out": "field", "dynamic": True, "pad": 0},
        # an odd width without a gate, from a half-precision program
        {"name": "glu_101_odd_f16", "op": "glu", "T": 101, "D": 9731, "x": "f16", "channel": False, "gated": False,
         "act": "gelu", "out": "f16", "dynamic": False, "pad": 3},
        # the largest: a prompt's chunk, gate and up side by side in one product's rows
        {"name": "glu_4096_field", "op": "glu", "T": 4096, "D": 28672, "x": "field", "channel": True, "gated": True,
         "act": "silu", "out": "field", "dynamic": True, "pad": 0},
        # the next token of one conversation
        {"name": "sample_1_top_k_p", "op": "sample", "T": 1, "V": 128000, "x": "field", "channel": True, "k": 50, "p": 0.95,
         "min_p": 0.0, "mixed": False, "banned": False, "spread": 2.0},
        # a small vocabulary with tokens that a grammar forbids
        {"name": "sample_9_min_p_banned", "op": "sample", "T": 9, "V": 32001, "x": "f16", "channel": False, "k": 0, "p": 1.0,
         "min_p": 0.05, "mixed": False, "banned": True, "spread": 1.5},
        # a batch of requests, each with parameters of its own (some of them greedy, some without limits)
        {"name": "sample_64_mixed", "op": "sample", "T": 64, "V": 150001, "x": "bf16", "channel": False, "k": 200, "p": 0.9,
         "min_p": 0.02, "mixed": True, "banned": False, "spread": 2.0},
        # the largest: many sequences drawn from their whole distribution
        {"name": "sample_512_whole", "op": "sample", "T": 512, "V": 128000, "x": "field", "channel": False, "k": 0, "p": 1.0,
         "min_p": 0.0, "mixed": False, "banned": False, "spread": 2.5},
    ]


def _log(rng, lo, hi):
    """A size spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["norm", "glu", "sample"])
    if op == "norm":
        D = _log(rng, 64, 16384)
        if rng.random() < 0.7:
            D = max(64, D // 64 * 64)
        out = rng.choice(["field", "field", "bf16", "f16", "f32"])
        return {"op": op, "T": _log(rng, 1, min(8192, 60_000_000 // D)), "D": D,
                "y": rng.choice(["field", "field", "bf16", "f16", "f32"]), "channel": rng.random() < 0.5,
                "res": rng.choice(["bf16", "f16", "f32"]), "post": rng.choice(["none", "none", "rms", "layer"]),
                "pre": rng.choice(["rms", "rms", "layer"]), "gate": rng.choice(["none", "none", "row", "tokens"]),
                "weight": rng.choice(["bf16", "f32"]), "out": out, "dynamic": out == "field" and rng.random() < 0.5,
                "pad": rng.choice([0, 0, 8, 1, 64])}
    if op == "glu":
        D = _log(rng, 64, 32768)
        if rng.random() < 0.7:
            D = max(64, D // 64 * 64)
        out = rng.choice(["field", "field", "bf16", "f16", "f32"])
        return {"op": op, "T": _log(rng, 1, min(8192, 60_000_000 // D)), "D": D,
                "x": rng.choice(["field", "field", "bf16", "f16", "f32"]), "channel": rng.random() < 0.5,
                "gated": rng.random() < 0.8, "act": rng.choice(["silu", "silu", "gelu", "relu", "sigmoid"]), "out": out,
                "dynamic": out == "field" and rng.random() < 0.5, "pad": rng.choice([0, 0, 8, 1, 64])}
    V = _log(rng, 500, 200000)
    how = rng.choice(["whole", "k", "p", "k p", "min_p", "mixed", "mixed"])
    return {"op": op, "T": _log(rng, 1, min(512, 40_000_000 // V)), "V": V,
            "x": rng.choice(["field", "bf16", "f16", "f32"]), "channel": rng.random() < 0.3,
            "k": _log(rng, 1, 1000) if "k" in how else 0 if how != "mixed" else 100,
            "p": round(rng.uniform(0.3, 0.99), 3) if "p" in how.split() or how == "mixed" else 1.0,
            "min_p": round(rng.uniform(0.005, 0.3), 3) if how in ("min_p", "mixed") else 0.0, "mixed": how == "mixed",
            "banned": rng.random() < 0.25, "spread": round(rng.uniform(0.5, 4.0), 2)}


# ---------------------------------------------------------------- inputs

def _values(g, shape, kind, gain=1.0):
    """A tensor of the type and the scale that takes its values back to about `gain`."""
    x = torch.randn(shape, generator=g, device="cuda")
    if kind == "field":  # a decoded product of quantised weights and activations: integers mod q
        return (x * 40000.0).round_().to(torch.int64).remainder_(Q).to(torch.int32), gain / 40000.0
    return (x * gain).to(_TYPES[kind]), 1.0


def _scales(g, n):
    """Steps of a quantisation, one a token or a channel."""
    return torch.exp(0.3 * torch.randn(n, generator=g, device="cuda"))


def _padded(g, T, D, pad, kind, gain=1.0):
    """T x D values in rows that are `pad` longer, from an odd place on where pad is odd."""
    x, scale = _values(g, (T, D + pad), kind, gain)
    at = pad // 2 if pad % 2 else 0
    return x[:, at:at + D], scale


def _empty(T, D, pad, kind):
    return torch.empty((T, D + pad), dtype=_TYPES[kind], device="cuda")[:, :D]


def _norm_inputs(case, g, s):
    T, D, pad = case["T"], case["D"], case["pad"]
    s["y"], s["y_scale"] = _padded(g, T, D, pad, case["y"], 0.7)
    s["residual"], _ = _padded(g, T, D, pad, case["res"], 1.5)
    s["token_scale"] = _scales(g, T) if case["y"] == "field" else None
    s["channel_scale"] = _scales(g, D) if case["channel"] else None
    s["gate_x"], s["gate_scale"] = None, 1.0
    if case["gate"] != "none":
        kind = case["y"] if case["gate"] == "tokens" else case["weight"]
        s["gate_x"], s["gate_scale"] = _padded(g, T if case["gate"] == "tokens" else 1, D, pad, kind)
    for name in ("post", "pre"):  # weights around 1, with a bias where the mean is taken
        w, _ = _values(g, (D,), case["weight"], 0.2)
        b, _ = _values(g, (D,), case["weight"], 0.1)
        s[name + "_w"], s[name + "_b"] = (w + 1).to(w.dtype), b if case[name] == "layer" else None
    s["residual_out"] = _empty(T, D, pad, case["res"])
    s["out"] = _empty(T, D, pad, case["out"])
    s["out_token_scale"] = torch.empty(T, device="cuda") if case["dynamic"] else None


def _glu_inputs(case, g, s):
    T, D, pad = case["T"], case["D"], case["pad"]
    x, s["x_scale"] = _padded(g, T, 2 * D if case["gated"] else D, pad, case["x"], 1.5)
    s["gate"], s["up"] = x[:, :D], x[:, D:] if case["gated"] else None
    s["token_scale"] = _scales(g, T) if case["x"] == "field" else None
    s["gate_channel"], s["up_channel"] = (_scales(g, D), _scales(g, D)) if case["channel"] else (None, None)
    s["out"] = _empty(T, D, pad, case["out"])
    s["out_token_scale"] = torch.empty(T, device="cuda") if case["dynamic"] else None


def _sample_inputs(case, g, s):
    T, V = case["T"], case["V"]
    l = torch.randn((T, V), generator=g, device="cuda") * case["spread"]
    hot = max(1, min(40, V // 10))  # what the model finds likely: a few tokens above the bulk, each less than the last
    at = torch.randint(0, V, (T, hot), generator=g, device="cuda")
    up = 4 * case["spread"] + 3 - torch.arange(hot, device="cuda") * 0.25 * torch.rand((T, 1), generator=g, device="cuda")
    l.scatter_add_(1, at, up)
    if case["x"] == "field":
        l, s["x_scale"] = (l * 5000.0).round_().to(torch.int64).remainder_(Q).to(torch.int32), 1 / 5000.0
    else:
        l, s["x_scale"] = l.to(_TYPES[case["x"]]), 1.0
    s["logits"] = l
    s["token_scale"] = _scales(g, T) * 0.2 + 0.8 if case["x"] == "field" else None
    s["channel_scale"] = _scales(g, V) * 0.05 + 0.95 if case["channel"] else None
    s["random"] = torch.randint(-2**31, 2**31, (T,), generator=g, device="cuda").to(torch.int32)
    s["t"], s["k"], s["p"], s["min_p"] = 0.8, case["k"], case["p"], case["min_p"]
    if case["mixed"]:  # every request has its own: a quarter leaves each limit out, an eighth is greedy
        u = torch.rand((4, T), generator=g, device="cuda")
        off = torch.rand((4, T), generator=g, device="cuda")
        s["t"] = (0.3 + 1.2 * u[0]).masked_fill(off[0] < 0.125, 0.0)
        s["k"] = (1 + 2 * case["k"] * u[1]).to(torch.int32).masked_fill(off[1] < 0.25, 0)
        s["p"] = (case["p"] + (1 - case["p"]) * u[2]).masked_fill(off[2] < 0.25, 1.0)
        s["min_p"] = (2 * case["min_p"] * u[3]).masked_fill(off[3] < 0.25, 0.0)
    s["allowed"] = None
    if case["banned"]:  # one bit a token: about a third is allowed
        words = torch.randint(-2**31, 2**31, (2, T, (V + 31) // 32), generator=g, device="cuda")
        s["allowed"] = (words[0] & (words[1] | (words[0] >> 16))).to(torch.int32)
    s["token"] = torch.empty(T, dtype=torch.int32, device="cuda")
    s["logprob"] = torch.empty(T, device="cuda")


def _inputs(case, seed):
    """Everything that a case's call reads and writes, from the seed."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = {"case": case}
    {"norm": _norm_inputs, "glu": _glu_inputs, "sample": _sample_inputs}[case["op"]](case, g, s)
    return s


_EPS, _RES, _BRANCH, _STEP, _LIMIT = 1e-6, 0.9, 1.1, 24.0, 127


def prepare(case, seed):
    """The tensors, and with the framework's operators the descriptions of weights and parameters that a program makes once
    and keeps."""
    s = _inputs(case, seed)
    if own:
        import paper_2609_10264_gb300 as pv
        s["pv"] = pv
        if case["op"] == "norm":
            for name in ("post", "pre"):
                s[name] = None if case[name] == "none" else pv.Norm(case[name], s[name + "_w"], s[name + "_b"], eps=_EPS)
        if case["op"] == "sample":
            s["sampling"] = pv.Sampling(s["t"], s["k"], s["p"], s["min_p"])
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    case = s["case"]
    if not own:
        return {"norm": _norm, "glu": _glu, "sample": _sample}[case["op"]](s)
    pv = s["pv"]
    if case["op"] == "norm":
        gate = s["gate_x"] if s["gate_x"] is None else pv.Rows(s["gate_x"], s["gate_scale"])
        pv.pvmvmd_block_norm(pv.Rows(s["y"], s["y_scale"], s["token_scale"], s["channel_scale"]), s["residual"],
                             post=s["post"], gate=gate, residual_scale=_RES, branch_scale=_BRANCH,
                             residual_out=s["residual_out"], pre=s["pre"], out=s["out"], out_scale=_STEP, limit=_LIMIT,
                             out_token_scale=s["out_token_scale"])
        return {"residual": s["residual_out"], "out": s["out"], "token_scale": s["out_token_scale"]}
    if case["op"] == "glu":
        up = s["up"] if s["up"] is None else pv.Rows(s["up"], s["x_scale"], s["token_scale"], s["up_channel"])
        pv.pvmvmd_glu(pv.Rows(s["gate"], s["x_scale"], s["token_scale"], s["gate_channel"]), up, act=case["act"],
                      out=s["out"], out_scale=_STEP, limit=_LIMIT, out_token_scale=s["out_token_scale"])
        return {"out": s["out"], "token_scale": s["out_token_scale"]}
    pv.pvmvmd_sample(pv.Rows(s["logits"], s["x_scale"], s["token_scale"], s["channel_scale"]), s["random"], s["sampling"],
                     allowed=s["allowed"], token=s["token"], logprob=s["logprob"])
    return {"token": s["token"], "logprob": s["logprob"]}


# ---------------------------------------------------------------- plain forms

def _numbers(x):
    """Floating values, or field elements as the centred integers they stand for, in 32 bits."""
    if x.dtype == torch.int32:
        return torch.where(x > (Q - 1) // 2, x - Q, x).float()
    return x.float()


def _read(x, scale, token_scale=None, channel_scale=None):
    """x times (scale token_scale) times channel_scale: each product rounded."""
    c = torch.full((1, 1), scale, device=x.device)
    if token_scale is not None:
        c = c * token_scale[:, None]
    v = _numbers(x) * c
    return v if channel_scale is None else v * channel_scale


def _write(s, z):
    """z in the output's type; integers by a fixed scale, or by each row's largest value, as field elements."""
    case = s["case"]
    if case["out"] != "field":
        return z.to(_TYPES[case["out"]]), None
    m, step = _STEP, None
    if case["dynamic"]:
        big = z.abs().amax(-1, keepdim=True)
        limit = torch.full_like(big, _LIMIT)
        m, step = torch.clamp(limit / big, max=FLT_MAX), (big / limit)[:, 0]
    n = torch.round(torch.clamp(z * m, -_LIMIT, _LIMIT)).to(torch.int32)
    return torch.where(n < 0, n + Q, n), step


def _normed(x, kind, w, b):
    """Root mean square or layer norm: statistics in 64 bits, each rounded to 32 once."""
    if kind == "layer":
        x = x - x.double().mean(-1, keepdim=True).float()
    eps = torch.tensor(_EPS, dtype=torch.float32).double().item()
    inv = (1 / (x.double().square().mean(-1, keepdim=True) + eps).sqrt()).float()
    n = x * inv * w.float()
    return n if b is None else n + b.float()


def _norm(s):
    case = s["case"]
    u = _read(s["y"], s["y_scale"], s["token_scale"], s["channel_scale"])
    if case["post"] != "none":
        u = _normed(u, case["post"], s["post_w"], s["post_b"])
    if s["gate_x"] is not None:
        u = u * _read(s["gate_x"], s["gate_scale"])
    r = s["residual"].float() * _RES + u * _BRANCH
    out, step = _write(s, _normed(r, case["pre"], s["pre_w"], s["pre_b"]))
    return {"residual": r.to(s["residual"].dtype), "out": out, "token_scale": step}


_LOG2E = 1.4426950408889634
# 2^-f for |f| <= 1/2: the polynomial of degree 5 with f(0) = 1 of least relative error (2^-23.4)
_EXP = (-0.6931470036506653, 0.24022242426872253, -0.05550733953714371, 0.009671512991189957, -0.0013264715671539307)


def _exp_parts(d):
    """2^-d as (2^-f, n) with d = n + f, n the nearest whole number: every product and sum rounded to 32 bits."""
    n = torch.round(d)
    f = d - n
    p = f * _EXP[4] + _EXP[3]
    p = p * f + _EXP[2]
    p = p * f + _EXP[1]
    p = p * f + _EXP[0]
    return p * f + 1.0, n.to(torch.int32)


def _one_plus_exp(d):
    """1 + 2^-d."""
    p, n = _exp_parts(torch.clamp(d, -128.0, 125.0))
    return 1.0 + (p.view(torch.int32) - (n << 23)).view(torch.float32)


def _glu(s):
    case = s["case"]
    x = _read(s["gate"], s["x_scale"], s["token_scale"], s["gate_channel"])
    if case["act"] == "relu":
        a = torch.clamp(x, min=0.0)
    elif case["act"] == "sigmoid":
        e = _one_plus_exp(x * _LOG2E)
        a = torch.ones_like(e) / e
    elif case["act"] == "silu":
        a = x / _one_plus_exp(x * _LOG2E)
    else:  # gelu in its tanh form is x sigmoid(2 sqrt(2/pi) (x + 0.044715 x^3))
        c = 2 * math.sqrt(2 / math.pi) * _LOG2E
        a = x / _one_plus_exp((x * x * (0.044715 * c) + c) * x)
    if s["up"] is not None:
        a = a * _read(s["up"], s["x_scale"], s["token_scale"], s["up_channel"])
    out, step = _write(s, a)
    return {"out": out, "token_scale": step}


def _per_row(v, T, dtype):
    return (v if torch.is_tensor(v) else torch.full((T,), v, dtype=dtype, device="cuda")).to(dtype)[:, None]


def _sample(s):
    x = _numbers(s["logits"])
    T, V = x.shape
    t, k = _per_row(s["t"], T, torch.float32), _per_row(s["k"], T, torch.int64)
    p, min_p = _per_row(s["p"], T, torch.float32), _per_row(s["min_p"], T, torch.float32)
    greedy = ~(t > 0)
    m = torch.full((T, 1), s["x_scale"], device="cuda")
    if s["token_scale"] is not None:
        m = m * s["token_scale"][:, None]
    m = torch.where(greedy, m, torch.clamp(m * (torch.full_like(t, _LOG2E) / t), max=FLT_MAX))
    x = x * m
    if s["channel_scale"] is not None:
        x = x * s["channel_scale"]
    x = torch.clamp(x, max=FLT_MAX)
    if s["allowed"] is not None:
        i = torch.arange(V, device="cuda")
        x = x.masked_fill((s["allowed"][:, i // 32] >> (i % 32)) & 1 == 0, -math.inf)
    # weights 2^(x - largest) in units of 2^-40, of 22 bits each
    big = x.amax(-1, keepdim=True)
    e, n = _exp_parts(torch.clamp(big - x, max=63.0).nan_to_num(63.0))
    w = (torch.round(e * 4194304.0).to(torch.int64) << 18) >> n
    # in falling order, equal ones by their index: what top-k and top-p leave
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices
    ws = w.gather(1, order)
    rank = torch.arange(V, device="cuda")
    keep = rank < torch.where((k <= 0) | (k > V), V, k)
    ws = ws * keep
    cum = ws.cumsum(-1)
    total, f = cum[:, -1:], (torch.clamp(p, 0.0, 1.0) * 2147483648.0).to(torch.int64)
    part = f * (total >> 31) + ((f * (total & 0x7fffffff)) >> 31)
    keep &= (rank == 0) | (p >= 1) | (cum - ws < part)
    kept = torch.zeros_like(w).scatter_(1, order, ws * keep)
    kept *= kept >= (torch.clamp(min_p, 0.0, 1.0) * 2147483648.0).to(torch.int64) << 9
    # the first token whose sum in the vocabulary's order is above the random part of the whole
    cum = kept.cumsum(-1)
    total, u = cum[:, -1:], s["random"].to(torch.int64)[:, None] & 0xffffffff
    low = total & 0xffffffff
    at = u * (total >> 32) + ((u * (low >> 16) + ((u * (low & 0xffff)) >> 16)) >> 16)
    token = (cum <= at).sum(-1, keepdim=True)
    token = torch.where(greedy, order[:, :1], token)
    mine = kept.gather(1, token.clamp(max=V - 1)).double()
    logprob = torch.where(greedy, 0.0, -torch.log1p((total - mine) / mine))
    none = big == -math.inf  # nothing is allowed
    return {"token": token.masked_fill(none, -1).to(torch.int32)[:, 0],
            "logprob": logprob.masked_fill(none, -math.inf).float()[:, 0]}


# ---------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    with torch.no_grad():
        r = {"norm": _norm64, "glu": _glu64, "sample": _sample64}[case["op"]](s, case)
    return r if r and any(v is not None for v in r.values()) else None


def _wide(x, scale, token=None, channel=None):
    v = x.double()
    if x.dtype == torch.int32:
        v = v - Q * (v > Q / 2)
    v = v * float(torch.tensor(scale, dtype=torch.float32))
    if token is not None:
        v = v * token.double().unsqueeze(1)
    return v if channel is None else v * channel.double()


def _out64(z, case):
    # integers are those of the roundings' order: a number next to the middle of two has no value of its own in 64 bits
    if case["out"] != "field":
        return z, None
    return None, z.abs().max(dim=1).values / _LIMIT if case["dynamic"] else None


def _norm64(s, case):
    f32 = lambda v: float(torch.tensor(v, dtype=torch.float32))  # noqa: E731

    def norm(v, kind, w, b):
        if kind == "none":
            return v
        if kind == "layer":
            v = v - v.sum(1, keepdim=True) / v.shape[1]
        v = v * torch.rsqrt((v * v).sum(1, keepdim=True) / v.shape[1] + f32(_EPS)) * w.double()
        return v + b.double() if b is not None else v

    u = norm(_wide(s["y"], s["y_scale"], s["token_scale"], s["channel_scale"]), case["post"], s["post_w"], s["post_b"])
    if case["gate"] != "none":
        u = u * _wide(s["gate_x"], s["gate_scale"])
    r = f32(_RES) * s["residual"].double() + f32(_BRANCH) * u
    out, step = _out64(norm(r, case["pre"], s["pre_w"], s["pre_b"]), case)
    return {"residual": r, "out": out, "token_scale": step}


def _glu64(s, case):
    x = _wide(s["gate"], s["x_scale"], s["token_scale"], s["gate_channel"])
    if case["act"] == "gelu":
        a = 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
    else:
        a = {"relu": lambda v: (v + v.abs()) / 2, "sigmoid": torch.sigmoid, "silu": lambda v: v * torch.sigmoid(v)}[case["act"]](x)
    if case["gated"]:
        a = a * _wide(s["up"], s["x_scale"], s["token_scale"], s["up_channel"])
    out, step = _out64(a, case)
    return {"out": out, "token_scale": step}


def _sample64(s, case):
    """Row by row on the host: the tokens' order and limits from the integers that define them, the probability of the
    token that is drawn from those of the tokens kept."""
    import numpy as np

    T, V = case["T"], case["V"]
    if T * V > 50_000_000 and case["k"] + case["p"] + case["min_p"] != 1.0:
        return None
    host = lambda v, t: np.broadcast_to(np.asarray(v.cpu() if torch.is_tensor(v) else v), (T,)).astype(t)  # noqa: E731
    temp, k, p, min_p = host(s["t"], np.float32), host(s["k"], int), host(s["p"], np.float32), host(s["min_p"], np.float32)
    random32 = host(s["random"], np.int64) % 2**32
    tok, lp = np.empty(T, np.int32), np.empty(T)
    c = np.full(T, np.float32(s["x_scale"]))
    if s["token_scale"] is not None:
        c = c * s["token_scale"].cpu().numpy()
    coef = [np.float32(v) for v in reversed(_EXP)]
    with np.errstate(all="ignore"):
        for t in range(T):
            l = s["logits"][t].cpu()
            if case["x"] == "field":
                l = l.numpy().astype(np.int64)
                l = (l - np.where(2 * l > Q, Q, 0)).astype(np.float32)
            else:
                l = l.float().numpy()
            greedy = not temp[t] > 0
            m = c[t] if greedy else min(c[t] * (np.float32(_LOG2E) / temp[t]), np.float32(FLT_MAX))
            x = l * np.float32(m)
            if s["channel_scale"] is not None:
                x = x * s["channel_scale"].cpu().numpy()
            x = np.minimum(x, np.float32(FLT_MAX))
            if s["allowed"] is not None:
                bits = np.unpackbits(s["allowed"][t].cpu().numpy().view(np.uint8), bitorder="little")[:V]
                x = np.where(bits == 1, x, -np.inf).astype(np.float32)
            top = x.max()
            if top == -np.inf:
                tok[t], lp[t] = -1, -np.inf
                continue
            if greedy:
                tok[t], lp[t] = int(np.argmax(x)), 0.0
                continue
            d = np.minimum(top - x, np.float32(63))
            n = np.rint(d)
            f = d - n
            y = np.zeros_like(f)
            for a in coef:
                y = y * f + a
            y = y * f + np.float32(1)
            w = (np.rint(y * np.float32(2**22)).astype(np.int64) * 2**18) >> n.astype(np.int64)
            keep = np.ones(V, bool)
            if 0 < k[t] < V or p[t] < 1:
                order = np.lexsort((np.arange(V), -x.astype(np.float64)))
                last = k[t] if 0 < k[t] < V else V
                run_ = np.cumsum(w[order[:last]])
                if p[t] < 1:  # whole numbers of any length
                    part = int(run_[-1]) * int(float(p[t]) * 2**31) >> 31
                    last = max(1, min(last, int(np.searchsorted(run_, part, side="left")) + 1))
                keep[:] = False
                keep[order[:last]] = True
            keep &= w >= int(float(max(min_p[t], 0)) * 2**31) << 9
            cum = np.cumsum(np.where(keep, w, 0))
            at = int(cum[-1]) * int(random32[t]) >> 32
            tok[t] = int(np.searchsorted(cum, at, side="right"))
            kept = np.exp2(x[keep].astype(np.float64) - float(top))
            lp[t] = float(x[tok[t]]) * math.log(2) - float(top) * math.log(2) - math.log(kept.sum())
    return {"token": torch.from_numpy(tok), "logprob": torch.from_numpy(lp)}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    """Each input read once, each output written once; operations are those of the formulas."""
    size = lambda kind: 2 if kind in ("bf16", "f16") else 4  # noqa: E731
    T = case["T"]
    if case["op"] == "sample":
        V = case["V"]
        bits = T * ((V + 31) // 32) * 4 if case["banned"] else 0
        return {"bytes": T * V * size(case["x"]) + (4 * V if case["channel"] else 0) + bits + 16 * T,
                "flops": 20.0 * T * V}
    D = case["D"]
    rows = 4 * T * ((case["y" if case["op"] == "norm" else "x"] == "field") + case["dynamic"])
    if case["op"] == "glu":
        n = 2 if case["gated"] else 1
        return {"bytes": T * D * (n * size(case["x"]) + size(case["out"])) + rows + (4 * n * D if case["channel"] else 0),
                "flops": 30.0 * T * D}
    gate = {"none": 0, "row": D * size(case["weight"]), "tokens": T * D * size(case["y"])}[case["gate"]]
    norms = sum({"none": 0, "rms": 1, "layer": 2}[case[n]] for n in ("post", "pre"))
    return {"bytes": T * D * (size(case["y"]) + 2 * size(case["res"]) + size(case["out"])) + rows + gate +
            norms * D * size(case["weight"]) + (4 * D if case["channel"] else 0), "flops": 12.0 * T * D}
