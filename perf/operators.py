"""The client's attention between two delegated products, as a user's program
calls it: rotary positions, the append of new tokens to a paged cache, attention
of the new tokens over it, and eviction by accumulated attention weight.

The head layouts are those of the repository's projections (q 4096 or 8192 and
k, v 1024 outputs: 32 or 64 query heads over 8 key heads of 128), and generic
ones beside them (narrower heads, one key head per query head, odd page sizes).
"""
import math
import random

import torch

own = False  # whether run() calls the framework's operators or their plain forms

Q = 15 * 2**27 + 1  # the field of decoded projections

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "field": torch.int32}


def listed():
    return [
        # q and k of one generated token: the smallest call, all latency
        {"name": "rope_1_token", "op": "rope", "T": 1, "H": 40, "D": 128, "rot": 128, "type": "bf16", "inter": False,
         "scaling": "none", "span": 4000},
        # a long prompt, in 32 bits, part of the head, positions scaled for a long context, read out of a wider
        # row (q of a fused projection's output)
        {"name": "rope_4097_partial_f32", "op": "rope", "T": 4097, "H": 32, "D": 96, "rot": 64, "type": "f32",
         "inter": True, "scaling": "ramp", "span": 100000},
        # the paper's eight-token prompt: q, k, v as decode_verify returns them, into an empty cache
        {"name": "append_8_field", "op": "append", "B": 1, "T": 8, "Hq": 32, "Hkv": 8, "D": 128, "rot": 128,
         "type": "field", "cache": "bf16", "page": 16, "inter": False, "scaling": "none", "past": 0, "spread": 1},
        # prompts of several requests at once, ragged, from bf16 projections
        {"name": "append_6001_ragged", "op": "append", "B": 5, "T": 6001, "Hq": 64, "Hkv": 8, "D": 128, "rot": 128,
         "type": "bf16", "cache": "bf16", "page": 32, "inter": False, "scaling": "base", "past": 3000, "spread": 2},
        # one generated token of a short conversation: all latency
        {"name": "decode_1x200", "op": "attend", "B": 1, "T": 1, "Hq": 32, "Hkv": 8, "D": 128, "cache": "bf16",
         "page": 16, "past": 199, "spread": 3, "window": 0, "mass": False},
        # a batch of generating requests of all ages, with the weights that eviction goes by
        {"name": "decode_64_ragged_mass", "op": "attend", "B": 64, "T": 64, "Hq": 64, "Hkv": 8, "D": 128,
         "cache": "bf16", "page": 16, "past": 8191, "spread": 4, "window": 0, "mass": True},
        # one token over a very long context
        {"name": "decode_1x131071_f16", "op": "attend", "B": 1, "T": 1, "Hq": 32, "Hkv": 8, "D": 128, "cache": "f16",
         "page": 64, "past": 131070, "spread": 5, "window": 0, "mass": False},
        # the paper's eight-token prompt over its own keys
        {"name": "chunk_8_of_8", "op": "attend", "B": 1, "T": 8, "Hq": 32, "Hkv": 8, "D": 128, "cache": "bf16",
         "page": 16, "past": 0, "spread": 6, "window": 0, "mass": False},
        # several prompts, odd sizes, narrow heads with keys of their own, a sliding window, pages of 24
        {"name": "chunk_ragged_window_mass", "op": "attend", "B": 6, "T": 3001, "Hq": 16, "Hkv": 16, "D": 64,
         "cache": "f16", "page": 24, "past": 2500, "spread": 7, "window": 1000, "mass": True},
        # the largest: a chunk of a long prompt over what came before
        {"name": "chunk_8192_of_24576", "op": "attend", "B": 1, "T": 8192, "Hq": 32, "Hkv": 8, "D": 128,
         "cache": "bf16", "page": 64, "past": 16384, "spread": 8, "window": 0, "mass": False},
        # one request a little over its budget
        {"name": "evict_1x700", "op": "evict", "B": 1, "Hkv": 8, "D": 128, "cache": "bf16", "page": 16, "past": 700,
         "spread": 9, "budget": 512, "recent": 64},
        # a batch of long ones down to a quarter
        {"name": "evict_16_ragged", "op": "evict", "B": 16, "Hkv": 8, "D": 128, "cache": "bf16", "page": 16,
         "past": 16384, "spread": 10, "budget": 4096, "recent": 256},
    ]


def _log(rng, lo, hi):
    """A size spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["rope", "append", "attend", "attend", "attend", "evict"])
    D = rng.choice([128, 128, 64, 96, 80])
    rot = rng.choice([D, D, D // 2])
    scaling = rng.choice(["none", "linear", "base", "ramp"])
    inter = rng.random() < 0.5
    Hkv = rng.choice([1, 2, 4, 8, 8])
    group = rng.choice([1, 2, 4, 4, 5, 8])
    page = rng.choice([1, 16, 16, 24, 32, 64, 100, 128])
    cache = rng.choice(["bf16", "bf16", "f16"])
    spread = rng.randrange(1 << 30)
    if op == "rope":
        return {"op": op, "T": _log(rng, 1, 8192), "H": rng.choice([1, 7, 8, 32, 40, 64]), "D": D, "rot": rot,
                "type": rng.choice(["bf16", "f16", "f32", "field"]), "inter": inter, "scaling": scaling,
                "span": _log(rng, 10, 1000000)}
    if op == "append":
        T = _log(rng, 1, 8192)
        return {"op": op, "B": _log(rng, 1, min(64, T)), "T": T, "Hq": Hkv * group, "Hkv": Hkv, "D": D, "rot": rot,
                "type": rng.choice([cache, cache, "field"]), "cache": cache, "page": page, "inter": inter,
                "scaling": scaling, "past": rng.choice([0, _log(rng, 1, 4000)]), "spread": spread}
    if op == "evict":
        past = _log(rng, 20, 16384)
        budget = max(1, int(past * rng.uniform(0.1, 1.1)))
        return {"op": op, "B": _log(rng, 1, 16), "Hkv": Hkv, "D": D, "cache": cache, "page": page, "past": past,
                "spread": spread, "budget": budget, "recent": int(budget * rng.uniform(0, 0.9))}
    window = rng.choice([0, 0, 0, _log(rng, 1, 4000)])
    if rng.random() < 0.5:  # single tokens, or the few of a speculated continuation
        B, few = _log(rng, 1, 128), rng.choice([1, 1, 1, 3])
        T, past = B * few, _log(rng, 1, min(131072, 600000 // B))
    else:
        T = _log(rng, 2, 4096)
        B, past = _log(rng, 1, min(16, T)), _log(rng, 1, 16384)
        past = min(past, 1 + 300_000_000 // (T * Hkv * group))  # the plain form holds every score
    return {"op": op, "B": B, "T": T, "Hq": Hkv * group, "Hkv": Hkv, "D": D, "cache": cache, "page": page,
            "past": past, "spread": spread, "window": window, "mass": rng.random() < 0.3}


def _shape(case):
    """New tokens and length of each sequence: of the case alone."""
    rng, B = random.Random(case["spread"]), case["B"]
    T = case.get("T", B)
    if T == B:
        n = [1] * B
    else:  # every sequence one at least, the rest spread unevenly
        w = [rng.random() ** 2 + 0.05 for _ in range(B)]
        n = [1 + int((T - B) * x / sum(w)) for x in w]
        n[0] += T - sum(n)
    # single sequences have the length the case says, batches are of all ages up to it
    past = [case["past"]] if B == 1 else [int(case["past"] * (0.02 + 0.98 * rng.random())) for _ in range(B)]
    if case["op"] == "evict":
        return n, past
    return n, [a + b for a, b in zip(n, past)]


def _thetas(rot, scaling):
    """Angles per position of the pairs, in 64 bits, and the magnitude."""
    r, base, s = rot, 500000.0, 8.0
    if scaling == "base":
        base *= s ** (r / (r - 2))
    th = [base ** (-2 * i / r) for i in range(r // 2)]
    if scaling == "linear":
        th = [t / s for t in th]
    if scaling == "ramp":
        n = [8192 * t / (2 * math.pi) for t in th]
        g = [min(1.0, max(0.0, (x - 1.0) / 31.0)) for x in n]
        th = [t * (a + (1 - a) / s) for t, a in zip(th, g)]
        return th, 0.1 * math.log(s) + 1
    return th, 1.0


_KIND = {"none": {}, "linear": {"scaling": "linear", "factor": 8.0}, "base": {"scaling": "base", "factor": 8.0},
         "ramp": {"scaling": "ramp", "factor": 8.0, "original": 8192, "slow": 1.0, "fast": 32.0,
                  "magnitude": 0.1 * math.log(8.0) + 1}}
_BASE = 500000.0


# ---------------------------------------------------------------- inputs

def _values(g, shape, kind, gain=1.0):
    x = torch.randn(shape, generator=g, device="cuda")
    if kind == "field":  # a decoded product of 16-bit-quantised weights and activations: integers mod q
        v = (x * 40000.0 * gain).round().to(torch.int64) % Q
        return v.to(torch.int32)
    return (x * gain).to(_TYPES[kind])


_FIELD_SCALE = 1.0 / 40000.0


def _inputs(case, seed):
    """Everything that a case's call reads, from the seed."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = dict(case, mass_on=case.get("mass", False))
    if case["op"] == "rope":
        wide = _values(g, (case["T"], case["H"] + 2, case["D"]), case["type"])
        s["x"] = wide[:, 1:-1]  # a part of the rows of a wider projection
        s["pos"] = torch.randint(0, case["span"], (case["T"],), generator=g, device="cuda", dtype=torch.int32)
        s["out"] = torch.empty((case["T"], case["H"], case["D"]), device="cuda",
                               dtype=torch.bfloat16 if case["type"] == "field" else _TYPES[case["type"]])
        return s
    n, lens = _shape(case)
    B, page, D, Hkv = case["B"], case["page"], case["D"], case["Hkv"]
    pages = [-(-x // page) for x in lens]
    total, width = sum(pages) + 3, max(1, max(pages))
    spare = -(-min(case["budget"], max(lens)) // page) if case["op"] == "evict" else 0
    order = torch.randperm(total + B * spare, generator=g, device="cuda").to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(B):
        table[b, :pages[b]] = order[at:at + pages[b]]
        at += pages[b]
    shape = (total + B * spare, page, Hkv, D)
    s["K"], s["V"] = _values(g, shape, case["cache"]), _values(g, shape, case["cache"])
    s["mass"] = torch.zeros((shape[0], Hkv, page), device="cuda")
    s["table"] = table
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    cu = [0]
    for x in n:
        cu.append(cu[-1] + x)
    s["cu"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
    s["max_new"] = max(n)
    T = cu[-1]
    if case["op"] == "append":
        kind, Hq = case["type"], case["Hq"]
        fused = _values(g, (T, Hq + 2 * Hkv, D), kind)  # one projection's output, or three side by side
        s["q"], s["k"], s["v"] = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
        # positions go on behind those of an evicted cache
        s["pos"] = torch.cat([torch.arange(l - m, l, device="cuda") + 100 * b
                              for b, (l, m) in enumerate(zip(lens, n))]).to(torch.int32)
        s["q_out"] = torch.empty((T, Hq, D), dtype=_TYPES[case["cache"]], device="cuda")
    elif case["op"] == "attend":
        s["q"] = _values(g, (T, case["Hq"], D), case["cache"], 1.5)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((T, case["Hq"]), device="cuda")
        # pages hold whatever their last user left behind the sequence's end
        first = torch.arange(width, device="cuda") * page
        slot = first[None, :, None] + torch.arange(page, device="cuda")
        dead = (slot >= s["lens"][:, None, None]) & (table >= 0)[:, :, None]
        b, p, o = dead.nonzero(as_tuple=True)
        s["K"][table[b, p].long(), o] = float("nan")
        s["V"][table[b, p].long(), o] = float("inf")
    else:
        s["mass"] = torch.rand(s["mass"].shape, generator=g, device="cuda") ** 4 * 10
        new = torch.full((B, max(1, spare)), -1, dtype=torch.int32, device="cuda")
        new[:, :spare] = order[total:].view(B, spare)
        s["new_table"], s["new_lens"] = new, torch.empty(B, dtype=torch.int32, device="cuda")
    return s


def prepare(case, seed):
    """The tensors, and what a program makes once and keeps: the frequencies, and with the framework's operators
    the views of its cache and batch."""
    s = _inputs(case, seed)
    if "rot" in case:
        th, s["magnitude"] = _thetas(case["rot"], case["scaling"])
        # in turns, as fractions of 2^64, so that a position's multiple is exact modulo whole turns
        turns = [int(round(t / (2 * math.pi) * 2.0**64)) for t in th]
        s["turns"] = torch.tensor([t - 2**64 if t >= 2**63 else t for t in turns], dtype=torch.int64, device="cuda")
    if own:
        import paper_2609_10264_gb300 as pv
        s["pv"] = pv
        if "rot" in case:
            s["rope"] = pv.pvmvmd_rope_table(case["rot"], base=_BASE, **_KIND[case["scaling"]])
        if case["op"] != "rope":
            s["pool"] = pv.KvPool(s["K"], s["V"], s["mass"])
            s["batch"] = pv.KvBatch(s["table"], s["lens"], None if case.get("T", case["B"]) == case["B"] else s["cu"],
                                    max_new=s["max_new"])
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    op = s["op"]
    if own:
        pv = s["pv"]
        fs = _FIELD_SCALE if s.get("type") == "field" else 1.0
        if op == "rope":
            return pv.pvmvmd_rope(s["x"], s["pos"], s["rope"], out=s["out"], interleaved=s["inter"], scale=fs)
        if op == "append":
            pv.pvmvmd_kv_append(s["pool"], s["batch"], s["k"], s["v"], s["pos"], s["rope"], q=s["q"], q_out=s["q_out"],
                                interleaved=s["inter"], scale=fs)
            return {"q": s["q_out"], "K": s["K"], "V": s["V"], "mass": s["mass"]}
        if op == "attend":
            pv.pvmvmd_paged_attention(s["pool"], s["batch"], s["q"], out=s["out"], lse=s["lse"], window=s["window"],
                                      accumulate=s["mass_on"])
            return _attended(s)
        pv.pvmvmd_kv_evict(s["pool"], s["batch"], s["budget"], s["recent"], new_lens=s["new_lens"],
                           new_table=s["new_table"])
        return {"K": s["K"], "V": s["V"], "mass": s["mass"], "lens": s["new_lens"]}
    return {"rope": _rope, "append": _append, "attend": _attend, "evict": _evict}[op](s)


def _attended(s):
    return {"out": s["out"], "lse": s["lse"], "mass": s["mass"]} if s["mass_on"] else {"out": s["out"],
                                                                                     "lse": s["lse"]}


def _float(x, scale):
    if x.dtype == torch.int32:
        x = torch.where(x > (Q - 1) // 2, x - Q, x)
    return x.float() * scale


def _rotate(s, x, pos):
    """x (T, H, D) in 32 bits, rotated."""
    r = s["rot"]
    frac = (pos.to(torch.int64)[:, None] * s["turns"]).float() * 2.0**-64  # wraps modulo whole turns
    c, d = (f(2 * math.pi * frac)[:, None] * s["magnitude"] for f in (torch.cos, torch.sin))
    y = x.clone()
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if s["inter"] else (x[..., :r // 2], x[..., r // 2:r])
    if s["inter"]:
        y[..., 0:r:2], y[..., 1:r:2] = a * c - b * d, a * d + b * c
    else:
        y[..., :r // 2], y[..., r // 2:r] = a * c - b * d, a * d + b * c
    return y


def _rope(s):
    s["out"].copy_(_rotate(s, _float(s["x"], _FIELD_SCALE if s["type"] == "field" else 1.0), s["pos"]))
    return s["out"]


def _rows(s):
    """Sequence and cache index of every new token."""
    t = torch.arange(s["q"].shape[0], device="cuda")
    b = torch.searchsorted(s["cu"][1:].contiguous(), t.to(torch.int32), right=True)
    n = s["cu"][1:] - s["cu"][:-1]
    return b, t - s["cu"][b], (s["lens"] - n)[b] + t - s["cu"][b]


def _append(s):
    fs = _FIELD_SCALE if s["type"] == "field" else 1.0
    b, _, idx = _rows(s)
    page, off = s["table"][b, idx // s["page"]].long(), idx % s["page"]
    s["q_out"].copy_(_rotate(s, _float(s["q"], fs), s["pos"]))
    s["K"][page, off] = _rotate(s, _float(s["k"], fs), s["pos"]).to(s["K"].dtype)
    s["V"][page, off] = _float(s["v"], fs).to(s["V"].dtype)
    s["mass"][page, :, off] = 0.0
    return {"q": s["q_out"], "K": s["K"], "V": s["V"], "mass": s["mass"]}


def _gathered(s, table, L):
    """Page and offset of the first L cache indexes of every sequence, and which there are."""
    j = torch.arange(L, device="cuda")
    page = table[:, torch.clamp(j // s["page"], max=table.shape[1] - 1)].long().clamp(min=0)
    return page, (j % s["page"])[None].expand_as(page), j[None] < s["lens"][:, None]


def _attend(s):
    B, Hkv, D, G = s["B"], s["Hkv"], s["D"], s["Hq"] // s["Hkv"]
    T, L, N = s["q"].shape[0], s["table"].shape[1] * s["page"], s["max_new"]
    page, off, live = _gathered(s, s["table"], L)
    K = s["K"][page, off].float().masked_fill(~live[:, :, None, None], 0).permute(0, 2, 3, 1)  # B, Hkv, D, L
    V = s["V"][page, off].float().masked_fill(~live[:, :, None, None], 0).permute(0, 2, 1, 3)
    b, i, at = _rows(s)
    q = torch.zeros((B, N, Hkv, G, D), device="cuda")
    q[b, i] = s["q"].float().view(T, Hkv, G, D) * D**-0.5
    S = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, D), K).view(B, Hkv, N, G, L)
    j = torch.arange(L, device="cuda")
    n = s["cu"][1:] - s["cu"][:-1]
    at = (s["lens"] - n)[:, None] + torch.arange(N, device="cuda")  # B, N
    see = live[:, None, :] & (j <= at[:, :, None])
    if s["window"]:
        see &= j > at[:, :, None] - s["window"]
    S.masked_fill_(~see[:, None, :, None, :], float("-inf"))
    m = S.amax(-1, keepdim=True).clamp(min=-1e30)
    P = S.sub_(m).exp_()
    l = P.sum(-1, keepdim=True)
    out = torch.matmul(P.view(B, Hkv, N * G, L), V).view(B, Hkv, N, G, D) / l.clamp(min=1e-30)
    s["out"].copy_(out.permute(0, 2, 1, 3, 4)[b, i].reshape(T, Hkv * G, D))
    s["lse"].copy_((m + torch.log(l)).permute(0, 2, 1, 3, 4)[b, i].reshape(T, Hkv * G))
    if s["mass_on"]:
        real = (torch.arange(N, device="cuda")[None] < n[:, None])[:, None, :, None, None]
        w = (P * (real / l.clamp(min=1e-30))).sum((2, 3))  # B, Hkv, L
        bb, jj = live.nonzero(as_tuple=True)
        s["mass"][page[bb, jj], :, off[bb, jj]] += w[bb, :, jj]
    return _attended(s)


def _evict(s):
    L, keep = s["table"].shape[1] * s["page"], s["budget"]
    page, off, live = _gathered(s, s["table"], L)
    w = s["mass"][page, :, off].permute(0, 2, 1)  # B, Hkv, L
    j = torch.arange(L, device="cuda")
    w = w.masked_fill((j >= s["lens"][:, None] - s["recent"])[:, None], float("inf"))
    w = w.masked_fill(~live[:, None], float("-inf"))
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :keep]
    stays = torch.zeros_like(w, dtype=torch.bool).scatter_(2, order, True) & live[:, None]
    b, h, j = stays.nonzero(as_tuple=True)
    to = (stays.cumsum(-1) - 1)[b, h, j]
    sp, so = page[b, j], off[b, j]
    dp, do = s["new_table"][b, to // s["page"]].long(), to % s["page"]
    s["K"][dp, do, h], s["V"][dp, do, h] = s["K"][sp, so, h], s["V"][sp, so, h]
    s["mass"][dp, h, do] = s["mass"][sp, h, so]
    s["new_lens"].copy_(torch.clamp(s["lens"], max=keep))
    return {"K": s["K"], "V": s["V"], "mass": s["mass"], "lens": s["new_lens"]}


# ---------------------------------------------------------------- work and the exact results

def _visible(case):
    """(pairs of a new token and a key it sees, keys that any sees) over the sequences."""
    pairs = keys = 0
    n, lens = _shape(case)
    for m, l in zip(n, lens):
        w = case["window"] or l + 1
        pairs += sum(min(p + 1, w) for p in range(l - m, l))
        keys += min(l, w + m - 1)
    return pairs, keys


def work(case):
    op, D = case["op"], case["D"]
    size = {"bf16": 2, "f16": 2, "f32": 4, "field": 4}
    if op == "rope":
        n = case["T"] * case["H"] * D
        out = 2 if case["type"] == "field" else size[case["type"]]
        return {"bytes": n * (size[case["type"]] + out) + 4 * case["T"] + 4 * case["rot"],
                "flops": case["T"] * case["H"] * case["rot"] * 3}
    Hkv = case["Hkv"]
    if op == "append":
        n = case["T"] * (case["Hq"] + 2 * Hkv) * D
        return {"bytes": n * (size[case["type"]] + 2) + 4 * case["T"] * (1 + Hkv),
                "flops": case["T"] * (case["Hq"] + Hkv) * case["rot"] * 3}
    if op == "attend":
        pairs, keys = _visible(case)
        T, Hq = case["T"], case["Hq"]
        return {"bytes": keys * Hkv * (4 * D + (8 if case["mass"] else 0)) + T * Hq * (4 * D + 4),
                "flops": 4.0 * D * Hq * pairs}
    lens = _shape(case)[1]
    kept = sum(min(x, case["budget"]) for x in lens)
    return {"bytes": Hkv * (4 * sum(lens) + kept * (8 * D + 4)), "flops": 0}


def _exact_rotate(case, x, pos):
    """Pair by pair as a product of complex numbers, in 64 bits."""
    th, m = _thetas(case["rot"], case["scaling"])
    r = case["rot"]
    at = pos.double()[:, None] * torch.tensor(th, dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.full_like(at, m), at)[:, None]
    y = x.double().clone()
    if case["inter"]:
        z = torch.view_as_complex(y[..., :r].reshape(*y.shape[:2], r // 2, 2).contiguous()) * turn
        y[..., :r] = torch.view_as_real(z).reshape(*y.shape[:2], r)
    else:
        z = torch.complex(y[..., :r // 2].contiguous(), y[..., r // 2:r].contiguous()) * turn
        y[..., :r] = torch.cat([z.real, z.imag], -1)
    return y


def _exact_float(x):
    if x.dtype != torch.int32:
        return x.double()
    v = x.long()
    return torch.where(v * 2 > Q, v - Q, v).double() * _FIELD_SCALE


def exact(case, seed):
    s = _inputs(case, seed)
    op, page = case["op"], case.get("page")
    if op == "rope":
        return _exact_rotate(case, _exact_float(s["x"]), s["pos"])
    K, V, mass = s["K"].double(), s["V"].double(), s["mass"].double()
    n, lens = _shape(case)
    cu = s["cu"].tolist()
    slots = [[(s["table"][b, torch.arange(l, device="cuda") // page].long()),
              torch.arange(l, device="cuda") % page] for b, l in enumerate(lens)]
    if op == "append":
        k, v = _exact_rotate(case, _exact_float(s["k"]), s["pos"]), _exact_float(s["v"])
        for b, (m, l) in enumerate(zip(n, lens)):
            p, o = (x[l - m:] for x in slots[b])
            K[p, o], V[p, o], mass[p, :, o] = k[cu[b]:cu[b + 1]], v[cu[b]:cu[b + 1]], 0.0
        return {"q": _exact_rotate(case, _exact_float(s["q"]), s["pos"]), "K": K, "V": V, "mass": mass}
    if op == "evict":
        for b, l in enumerate(lens):
            p, o = slots[b]
            keep = min(case["budget"], l)
            fixed = min(case["recent"], keep)
            for h in range(case["Hkv"]):
                w = mass[p, h, o]
                best = sorted(range(l - fixed), key=lambda j, w=w.tolist(): (-w[j], j))[:keep - fixed]
                idx = torch.tensor(sorted(best) + list(range(l - fixed, l)), dtype=torch.long, device="cuda")
                to = torch.arange(keep, device="cuda")
                dp, do = s["new_table"][b, to // page].long(), to % page
                K[dp, do, h], V[dp, do, h], mass[dp, h, do] = K[p[idx], o[idx], h], V[p[idx], o[idx], h], w[idx]
        return {"K": K, "V": V, "mass": mass, "lens": None}
    if 8.0 * case["D"] * case["Hq"] * _visible(case)[0] > 1e13:
        return None  # takes too long in 64 bits
    Hkv, G, D = case["Hkv"], case["Hq"] // case["Hkv"], case["D"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(out.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for b, (m, l) in enumerate(zip(n, lens)):
        p, o = slots[b]
        Kb, Vb = K[p, o].transpose(0, 1), V[p, o].transpose(0, 1)  # Hkv, l, D
        j = torch.arange(l, device="cuda")
        step = max(1, 200_000_000 // (l * Hkv * G))
        for t in range(0, m, step):
            e = min(m, t + step)
            qb = s["q"][cu[b] + t:cu[b] + e].double().view(e - t, Hkv, G, D).permute(1, 2, 0, 3)
            S = qb @ Kb.transpose(1, 2)[:, None] / math.sqrt(D)  # Hkv, G, rows, l
            at = torch.arange(l - m + t, l - m + e, device="cuda")[:, None]
            hidden = (j > at) | (j <= at - case["window"] if case["window"] else j < 0)
            S = S.masked_fill(hidden, -math.inf)
            z = torch.logsumexp(S, -1, keepdim=True)
            W = torch.exp(S - z)
            out[cu[b] + t:cu[b] + e] = (W @ Vb[:, None]).permute(2, 0, 1, 3).reshape(e - t, Hkv * G, D)
            lse[cu[b] + t:cu[b] + e] = z[..., 0].permute(2, 0, 1).reshape(e - t, Hkv * G)
            if case["mass"]:
                mass[p, :, o] += W.sum((1, 2)).T
    return {"out": out, "lse": lse, "mass": mass} if case["mass"] else {"out": out, "lse": lse}
