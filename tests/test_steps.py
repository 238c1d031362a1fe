"""The client's other steps between two delegated products (pvmvmd_block_norm, pvmvmd_glu, pvmvmd_sample).

Their results are defined to the last bit: each is compared for equality with the definition in
numpy (steps_plain.py), whose statistics are formed in 64 bits, and floating ones with the formula in 64 bits, within
bounds counted from the roundings.  With e = 2^-24 (half a step of 32 bits) and u half a step of the output's
type, a value that passes n roundings is off by at most n e of itself, and where two values are added by n e of the sum of
their sizes; a type's smallest values add its smallest step."""
import ctypes

import numpy as np
import pytest

import steps_plain as plain

E = 2.0**-24
U = {"bf16": 2.0**-8, "f16": 2.0**-11, "f32": E}
TINY = {"bf16": 2.0**-133, "f16": 2.0**-24, "f32": 2.0**-149}


@pytest.fixture(scope="module")
def pv():
    import __graft_entry__
    __graft_entry__._load_build_module().build()
    import paper_2609_10264_gb300 as pv
    return pv


def _dt(kind):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "field": torch.int32}[kind]


def _dev(a, kind="f32", pad=0, at=0):
    """A numpy matrix on the device, in rows that are pad longer, from value `at` on; and what it holds there."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a))
    t = (t if kind == "field" else t.to(_dt(kind))).cuda()
    if pad:
        wide = torch.zeros(t.shape[0], t.shape[1] + pad, dtype=t.dtype, device="cuda")
        wide[:, at:at + t.shape[1]] = t
        t = wide[:, at:at + t.shape[1]]
    return t


def _host(t):
    return t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _values(rng, shape, kind):
    if kind == "field":
        return plain.field(np.rint(rng.standard_normal(shape) * 30000))
    return rng.standard_normal(shape).astype(np.float32)


def _rounded(z, kind):
    """32-bit values in the type."""
    import torch
    return _host(torch.from_numpy(np.ascontiguousarray(z)).to(_dt(kind)))


# ---------------------------------------------------------------- block norm

def _norm_case(pv, seed, T, D, y="field", res="bf16", out="field", post=None, pre="rms", gate=None, w="bf16", bias=False,
               add=0.0, dynamic=False, pad=0, at=0, token=True, channel=True, limit=127, scale=24.0, keep=0.9, branch=1.1):
    import torch
    rng = np.random.default_rng(seed)
    ts = np.exp(0.3 * rng.standard_normal(T)).astype(np.float32) if token else None
    cs = np.exp(0.3 * rng.standard_normal(D)).astype(np.float32) if channel else None
    s = 1 / 30000 if y == "field" else 1.0
    ynp = _values(rng, (T, D), y) if y else None
    yt = _dev(ynp, y, pad, at) if y else None
    rt = _dev(_values(rng, (T, D), res), res, pad, at) if res else None
    gt = _dev(_values(rng, (T if gate == "tokens" else 1, D), w), w, pad, at) if gate else None
    norms, np_norms = {}, {}
    for name, kind in (("post", post), ("pre", pre)):
        if kind is None:
            norms[name] = np_norms[name] = None
            continue
        wt = _dev(1 + 0.2 * rng.standard_normal(D).astype(np.float32), w) if w else None
        bt = _dev(0.1 * rng.standard_normal(D).astype(np.float32), w) if bias else None
        norms[name] = pv.Norm(kind, wt, bt, eps=1e-5, weight_add=add)
        np_norms[name] = (kind, None if wt is None else _host(wt), None if bt is None else _host(bt), 1e-5, add)
    ot = _dev(np.zeros((T, D), np.int32 if out == "field" else np.float32), out, pad, at) if out else None
    st = torch.zeros(T, device="cuda") if dynamic else None
    dev = lambda v: None if v is None else torch.from_numpy(v).cuda()  # noqa: E731
    r2, o = pv.pvmvmd_block_norm(pv.Rows(yt, s, dev(ts), dev(cs)) if y else None, rt, post=norms["post"], gate=gt,
                                 branch_scale=branch, residual_scale=keep, pre=norms["pre"], out=ot, out_scale=scale,
                                 limit=limit, out_token_scale=st)

    def form(wide):
        t = np.float64 if wide else np.float32
        if y:
            u = plain.read(ynp if y == "field" else _host(yt), s, ts, cs, y == "field", wide)
            size = np.abs(u)
            if np_norms["post"]:
                u = plain.norm(u, *np_norms["post"], wide=wide)
            if gate:
                u = u * _host(gt).astype(t)
            u = u * t(np.float32(branch))
        if res:
            q = _host(rt).astype(t) * t(np.float32(keep))
            r = q + u if y else q
        else:
            r = u
        z = plain.norm(r, *np_norms["pre"], wide=wide) if np_norms["pre"] else r
        return r, z

    return (r2, o, st), form, out, dynamic, scale, limit


NORMS = [
    dict(T=1, D=1, bias=True, pre="layer"),
    dict(T=2, D=7, y="f32", out="f32", post="rms"),
    dict(T=17, D=64, dynamic=True),
    dict(T=3, D=100, y="f16", res="f16", out="f16", gate="tokens", w="f16", pad=4),
    dict(T=300, D=128, y="bf16", out="bf16", post="layer", pre="layer", bias=True, gate="row"),
    dict(T=1300, D=1000, dynamic=True, gate="tokens", w="f32"),
    dict(T=5, D=1024, y="bf16", res="f32", out="f32", pre="layer", token=False, channel=False),
    dict(T=5, D=1025, y="f32", res="f32", out="field", dynamic=True, pad=1),
    dict(T=2, D=1032, res=None, post="rms", out="bf16", add=1.0, w="f32"),
    dict(T=1, D=4096, dynamic=True),
    dict(T=200, D=4096, y=None, out="bf16"),
    dict(T=3, D=5001, y="f16", res="f32", out="field", post="layer", bias=True, pad=5, at=3),
    dict(T=2, D=8200, pre=None, out="f32"),
    dict(T=160, D=8192, post="rms", scale=1e6, limit=1 << 22),
    dict(T=1, D=16384, post="rms", pre="layer", w=None, add=0.5),
    dict(T=153, D=16392, dynamic=True, limit=1),
    dict(T=2, D=2048, dynamic=True, limit=1 << 22),
    dict(T=160, D=2560, y="bf16", out="bf16", gate="tokens", post="rms"),
    dict(T=2, D=40000, y="bf16", out="f16", gate="row", dynamic=False),
    dict(T=153, D=40008, res="f16", dynamic=True, post="layer"),
    dict(T=1, D=131071, dynamic=True, post="rms"),
    dict(T=154, D=131064, y="bf16", out="bf16"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("k", range(len(NORMS)), ids=lambda k: "-".join(f"{a}={b}" for a, b in NORMS[k].items()))
def test_block_norm_is_its_definition(pv, k):
    case = NORMS[k]
    (r2, o, st), form, out, dynamic, scale, limit = _norm_case(pv, k, **case)
    r, z = form(False)
    kind = case.get("res", "bf16") or "bf16"
    assert np.array_equal(_host(r2), _rounded(r, kind))
    if out == "field":
        n, step = plain.integers(z, scale, limit, dynamic)
        assert np.array_equal(o.cpu().numpy(), plain.field(n))
        if dynamic:
            assert np.array_equal(st.cpu().numpy(), step)
            assert np.abs(n).max(-1).min() == limit  # the largest value takes the largest integer
    else:
        assert np.array_equal(_host(o), _rounded(z, out))
    # In 64 bits.  u passes 5 roundings at most (two scales, their product, gate, branch) and a post norm
    # of 6 more on terms of its size, its own statistic's included; r' one more on each part, z again 6.
    r64, z64 = form(True)
    rms = np.sqrt(np.square(r64).mean(-1, keepdims=True) + 1e-5)
    part = np.abs(r64) + 2 * rms * (1 + np.abs(r64 / rms)) * (3 if case.get("gate") or case.get("post") else 1)
    assert (np.abs(r - r64) <= 14 * E * (part + 8)).all()
    size = (np.abs(z64) + 1) * (14 * E * (part + 8) / np.minimum(rms, 1) + 8 * E) * 4
    assert (np.abs(z - z64) <= size).all()


@pytest.mark.gpu
def test_block_norm_in_place(pv):
    """residual_out is residual, out is y; what lies beside the rows and behind them stays."""
    import torch
    rng = np.random.default_rng(5)
    T, D = 70, 2000
    for kind, at in (("bf16", 8), ("f32", 1)):
        y, r = (_dev(_values(rng, (T + 2, D), kind), kind, 16, at) for _ in range(2))
        w = _dev(_values(rng, (1, D), "f32"), "f32")[0]
        n = pv.Norm("rms", w)
        want_r, want = pv.pvmvmd_block_norm(y[:T], r[:T], pre=n, out=torch.empty_like(y[:T].contiguous()))
        whole = [t._base.clone() for t in (y, r)]
        got_r, got = pv.pvmvmd_block_norm(y[:T], r[:T], residual_out=r[:T], pre=n, out=y[:T])
        assert torch.equal(got, want) and torch.equal(got_r, want_r)
        for t, before in zip((y, r), whole):
            mine = torch.zeros_like(before, dtype=torch.bool)
            mine[:T, at:at + D] = True
            assert torch.equal(t._base[~mine], before[~mine])


@pytest.mark.gpu
def test_block_norm_of_nothing_and_of_what_is_not_finite(pv):
    import torch
    n = pv.Norm("rms", eps=1e-6)
    empty = torch.empty(0, 512, device="cuda")
    r, o = pv.pvmvmd_block_norm(empty, empty, pre=n, out=torch.empty(0, 512, dtype=torch.int32, device="cuda"))
    assert o.shape == (0, 512)
    for D in (96, 1500, 4096):
        x = torch.randn(6, D, device="cuda")
        x[1] = 0
        x[2, D // 2] = float("nan")
        x[3, D - 1] = float("inf")
        x[4] *= 1e-30
        out = torch.empty(6, D, dtype=torch.int32, device="cuda")
        step = torch.empty(6, device="cuda")
        pv.pvmvmd_block_norm(None, x, residual_out=False, out=out, out_token_scale=step)
        n, s = plain.integers(_host(x), 1, 127, True)
        assert np.array_equal(out.cpu().numpy(), plain.field(n))
        assert np.array_equal(step.cpu().numpy(), s, equal_nan=True) and np.isnan(s[2:4]).all() and s[1] == 0
        # by a scale known ahead: NaN is 0, infinities are the limits
        pv.pvmvmd_block_norm(None, x, residual_out=False, out=out, out_scale=3.0, limit=5)
        n, _ = plain.integers(_host(x), 3.0, 5, False)
        assert np.array_equal(out.cpu().numpy(), plain.field(n)) and n[2, D // 2] == 0 and n[3, D - 1] == 5
        # a norm of zeros is zeros, one of NaN is NaN, and neither reaches another row
        z = torch.empty(6, D, device="cuda")
        pv.pvmvmd_block_norm(None, x, residual_out=False, pre=pv.Norm("layer", eps=1e-6), out=z)
        z = _host(z)
        assert (z[1] == 0).all() and np.isnan(z[2]).all() and np.isfinite(z[[0, 1, 4, 5]]).all()


@pytest.mark.gpu
def test_norm_of_large_and_small_values(pv):
    """Squares far above and below what 16 bits hold: the definition's values.  (An eps of 2^-126 is 2^-26 of the mean of
    squares of 2^-100, and moves the inverse root by 2^-27 of itself: norms of a row and of the row times 2^-50 need not
    be the same.)"""
    import torch
    x = np.random.default_rng(12).standard_normal((3, 3000)).astype(np.float32)
    for gain in (1, 2.0**50, 2.0**-50):
        z = torch.empty(3, 3000, device="cuda")
        pv.pvmvmd_block_norm(None, _dev(x * np.float32(gain)), residual_out=False, pre=pv.Norm("rms", eps=1e-38), out=z)
        assert np.array_equal(_host(z), plain.norm(x * np.float32(gain), "rms", eps=1e-38))


# ---------------------------------------------------------------- gated activation

GLUS = [
    dict(T=1, D=1, act="silu"), dict(T=3, D=33, act="gelu", x="f32", out="f32"),
    dict(T=1, D=14336, act="silu", dynamic=True), dict(T=7, D=9731, act="gelu", x="f16", out="f16", up=False, pad=3, at=1),
    dict(T=400, D=512, act="relu", x="bf16", out="bf16"), dict(T=155, D=28672, act="silu", dynamic=True),
    dict(T=2, D=50000, act="sigmoid", x="f32", out="f32"), dict(T=2, D=131071, act="silu", dynamic=True, x="bf16"),
    dict(T=20, D=1024, act="none", x="f32", out="field", limit=1000), dict(T=154, D=70000, act="gelu", out="field", dynamic=True),
    dict(T=9, D=4096, act="silu", x="f16", out="bf16", up=True, pad=8),
]


@pytest.mark.gpu
@pytest.mark.parametrize("k", range(len(GLUS)), ids=lambda k: "-".join(f"{a}={b}" for a, b in GLUS[k].items()))
def test_glu_is_its_definition(pv, k):
    import torch
    c = dict(x="field", out="field", up=True, pad=0, at=0, dynamic=False, limit=127)
    c.update(GLUS[k])
    T, D, kind = c["T"], c["D"], c["x"]
    rng = np.random.default_rng(50 + k)
    s = 1 / 12000 if kind == "field" else 1.5
    fused = _dev(_values(rng, (T, 2 * D), kind), kind, c["pad"], c["at"])
    g, u = fused[:, :D], fused[:, D:] if c["up"] else None
    ts = np.exp(0.3 * rng.standard_normal(T)).astype(np.float32)
    gs, us = (np.exp(0.3 * rng.standard_normal(D)).astype(np.float32) for _ in range(2))
    dev = lambda v: torch.from_numpy(v).cuda()  # noqa: E731
    out = _dev(np.zeros((T, D), np.int32 if c["out"] == "field" else np.float32), c["out"], c["pad"], c["at"])
    st = torch.zeros(T, device="cuda") if c["dynamic"] else None
    pv.pvmvmd_glu(pv.Rows(g, s, dev(ts), dev(gs)), None if u is None else pv.Rows(u, s, dev(ts), dev(us)), act=c["act"],
                  out=out, out_scale=20.0, limit=c["limit"], out_token_scale=st)
    f = kind == "field"
    a = plain.act(plain.read(_host(g), s, ts, gs, f), c["act"])
    a64 = plain.act64(plain.read(_host(g), s, ts, gs, f, True), c["act"])
    if u is not None:
        a = a * plain.read(_host(u), s, ts, us, f)
        a64 = a64 * plain.read(_host(u), s, ts, us, f, True)
    if c["out"] == "field":
        n, step = plain.integers(a, 20.0, c["limit"], c["dynamic"])
        assert np.array_equal(out.cpu().numpy(), plain.field(n))
        if st is not None:
            assert np.array_equal(st.cpu().numpy(), step)
    else:
        assert np.array_equal(_host(out), _rounded(a, c["out"]))
    # x and u pass 4 roundings each; an exponent t in base 2 is off by 4 + 4 of its own, which is |t| ln 2 of the
    # power, itself off by 2^-22.3 = 3.3 e; quotient, sum and product round three times.
    x = np.abs(plain.read(_host(g), s, ts, gs, f, True))
    t = (x * x * 0.044715 + 1) * x * 2 if c["act"] == "gelu" else x
    assert (np.abs(a - a64) <= np.abs(a64) * E * (15 + 8 * t) + 2.0**-120).all()


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "relu", "sigmoid", "silu", "gelu"])
def test_glu_at_the_ends_of_its_range(pv, act):
    import torch
    v = np.array([0.0, -0.0, 1e-40, -1e-40, 1e-20, 60, -60, 86.6, -86.6, 87.9, -87.9, 88.8, -88.8, 500, -500, 1e19, -1e19, 1e30,
                  -1e30, 3e38, -3e38, np.inf, -np.inf, np.nan], np.float32)
    x = np.stack([v, v[::-1]])
    out = torch.empty(x.shape, device="cuda")
    pv.pvmvmd_glu(torch.from_numpy(x).cuda(), act=act, out=out)
    got, want = _host(out), plain.act(x, act)
    assert np.array_equal(got, want, equal_nan=True)
    fine = np.isfinite(x) & (np.abs(x) < 1e19)
    with np.errstate(all="ignore"):
        true = plain.act64(x.astype(np.float64), act)
    # below 2^-126 the power is cut: x / 2^128 at most is left of what is smaller
    got, true = got[fine], true[fine]
    assert (np.abs(got - true) <= np.abs(true) * E * (15 + 8 * 90) + 2.0**-115).all()


def _silu_or_gelu(x, act):
    """The definition on the device: each operation is a kernel of its own, and rounds by itself."""
    import math
    import torch
    l = 1.4426950408889634
    c = 2 * math.sqrt(2 / math.pi) * l
    d = (x * x * (0.044715 * c) + c) * x if act == "gelu" else x * l
    d = torch.clamp(d, -128.0, 125.0)
    n = torch.round(d)
    f = d - n
    p = f * float(plain.COEF[0]) + float(plain.COEF[1])
    for k in plain.COEF[2:]:
        p = p * f + float(k)
    p = p * f + 1.0
    return x / (1.0 + (p.view(torch.int32) - (n.nan_to_num().to(torch.int32) << 23)).view(torch.float32))


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_quotients_of_all_numbers(pv, act):
    """Every number of 32 bits: the quotient by the inverse is the quotient of two numbers, rounded once."""
    import torch
    T, D = 1024, 32768
    out = torch.empty(T, D, device="cuda")
    for k in range(2**32 // (T * D)):
        bits = torch.arange(k * T * D, (k + 1) * T * D, device="cuda", dtype=torch.int64)
        x = torch.where(bits >= 2**31, bits - 2**32, bits).to(torch.int32).view(torch.float32).view(T, D)
        pv.pvmvmd_glu(x, act=act, out=out)
        want = _silu_or_gelu(x, act)
        assert bool(((out == want) | (out.isnan() & want.isnan())).all()), k


@pytest.mark.gpu
@pytest.mark.parametrize("T,D", [(3, 700), (2, 12000), (160, 12000), (200, 512)])
def test_glu_in_place(pv, T, D):
    """out is gate, or up, and the step a token's scale that is replaced."""
    import torch
    g, u = (torch.randint(-30000, 30000, (T, D), device="cuda").remainder(plain.Q).to(torch.int32) for _ in range(2))
    ts = torch.rand(T, device="cuda") + 0.5
    for which in (0, 1):
        a, b, s = g.clone(), u.clone(), ts.clone()
        step = torch.empty(T, device="cuda")
        want = pv.pvmvmd_glu(pv.Rows(a, 1e-4, s), pv.Rows(b, 1e-4, s), out_token_scale=step)
        pv.pvmvmd_glu(pv.Rows(a, 1e-4, s), pv.Rows(b, 1e-4, s), out=(a, b)[which], out_token_scale=s)
        assert torch.equal((a, b)[which], want) and torch.equal(s, step) and torch.equal((b, a)[which], (u, g)[which])


def test_power_of_two_within_its_bound():
    """E of the header against 64 bits: 2^-22.3, at a million places and next to the halves where n changes."""
    d = np.concatenate([np.linspace(-127, 125, 1 << 20), np.arange(-126.5, 125, 1)]).astype(np.float32)
    d = np.concatenate([d, np.nextafter(d, np.float32(200)), np.nextafter(d, np.float32(-200))])
    d = d[(d > -127) & (d < 125)]
    got = plain.power(d).astype(np.float64) / np.exp2(-d.astype(np.float64))
    assert np.abs(got - 1).max() <= 2.0**-22.3
    assert plain.power(np.array([0, -128], np.float32)).tolist() == [1, np.inf]


# ---------------------------------------------------------------- the next token

def _sample(pv, l, kind="f32", scale=1.0, ts=None, cs=None, t=1.0, k=0, p=1.0, m=0.0, words=None, allowed=None, pad=0, at=0):
    """The call on logits l (T x V numpy), and the definition row by row."""
    import torch
    T, V = l.shape
    x = _dev(l, kind, pad, at)
    dev = lambda v: torch.from_numpy(np.ascontiguousarray(v)).cuda()  # noqa: E731
    par = [v if np.isscalar(v) else dev(np.asarray(v, np.int32 if i == 1 else np.float32)) for i, v in enumerate((t, k, p, m))]
    words = np.random.default_rng(T * V).integers(0, 2**32, T) if words is None else np.broadcast_to(words, (T,))
    lp = torch.empty(T, device="cuda")
    al = None if allowed is None else dev(allowed.astype(np.uint32).view(np.int32))
    tok = pv.pvmvmd_sample(pv.Rows(x, scale, None if ts is None else dev(ts), None if cs is None else dev(cs)),
                           dev(words.astype(np.uint32).view(np.int32)), pv.Sampling(*par), allowed=al, logprob=lp)
    h = plain.centred(_host(x)).astype(np.float32) if kind == "field" else _host(x)
    row = lambda v, r: v if np.isscalar(v) else v[r]  # noqa: E731
    for r in range(T):
        mul = plain.multiplier(scale, None if ts is None else ts[r], row(t, r))
        a = None if allowed is None else allowed if allowed.ndim == 1 else allowed[r % len(allowed)]
        xs = plain.distances(h[r], mul, cs, a)
        want, wlp = plain.sample(xs, row(t, r), int(row(k, r)), float(np.float32(row(p, r))), float(np.float32(row(m, r))),
                                 words[r])
        got, glp = int(tok[r]), float(lp[r])
        assert got == want, (r, got, want)
        # the quotient of two whole numbers, each rounded, and log1p: three roundings and one unit of the
        # function's own of an argument a; log1p(a) moves by less than a / (1 + a) <= 1 of that
        assert glp == wlp or abs(glp - wlp) <= 4 * E * (1 + abs(wlp)), (r, glp, wlp)
    return tok


def _logits(rng, T, V, spread=3.0, levels=None):
    l = rng.standard_normal((T, V)) * spread
    for r in range(T):
        l[r, rng.integers(0, V, max(1, V // 100))] += 2.5 * spread
    return (np.round(l * levels) / levels if levels else l).astype(np.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [1, 2, 31, 255, 256, 257, 1000, 4097, 20011])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16", "field"])
def test_sample_is_its_definition(pv, V, kind):
    rng = np.random.default_rng(V)
    T = 7
    l = _logits(rng, T, V)
    scale = 1.0
    if kind == "field":
        l, scale = plain.field(np.rint(l * 4000)), 1 / 4000
    off = {"f32": 1, "field": 3, "bf16": 5, "f16": 7}[kind]
    ts = np.exp(0.1 * rng.standard_normal(T)).astype(np.float32)
    cs = np.exp(0.1 * rng.standard_normal(V)).astype(np.float32)
    _sample(pv, l, kind, scale)
    _sample(pv, l, kind, scale, ts, cs, t=0.7, k=5, pad=off, at=off // 2)
    _sample(pv, l, kind, scale, ts, p=0.8, t=1.3)
    _sample(pv, l, kind, scale, cs=cs, m=0.1, pad=off, at=off)
    # each row with its own: greedy, no limit, all of them
    _sample(pv, l, kind, scale, ts, t=np.array([0, 1, 0.5, 2, -1, 0.01, np.nan]), k=np.array([3, 0, 50, V, 1, V + 7, -5]),
            p=np.array([0.5, 1.0, 0.9, 0.3, 0.99, 0.0, 2.0]), m=np.array([0.0, 0.2, 0.01, 1.0, 3.0, -1.0, np.nan]))


@pytest.mark.gpu
@pytest.mark.parametrize("V", [300, 9000])
@pytest.mark.parametrize("levels", [None, 4, 0.2])
def test_sample_with_ties_and_limits(pv, V, levels):
    """Logits of few values: limits that fall among equal ones, which go by their index."""
    rng = np.random.default_rng(V)
    l = _logits(rng, 12, V, levels=levels)
    l[11] = 1.5  # all equal
    for k in (1, 2, 7, V // 3, V - 1):
        _sample(pv, l, k=k)
        _sample(pv, l, k=k, p=0.7, words=2**32 - 1)
    for p in (1e-9, 0.01, 0.5, 0.999):
        _sample(pv, l, p=p)
        _sample(pv, l, p=p, m=0.02, words=0)
        _sample(pv, l, "bf16", p=p, k=200, t=3.0, words=2**32 - 1)


@pytest.mark.gpu
def test_sample_of_flat_rows(pv):
    """Thousands of tokens inside every limit, as at high temperatures."""
    rng = np.random.default_rng(3)
    l = rng.standard_normal((6, 30000)).astype(np.float32)
    _sample(pv, l, t=20.0, p=0.97)
    _sample(pv, l, t=20.0, k=12345, p=0.9)
    _sample(pv, l, t=20.0, k=29999)
    _sample(pv, l, "bf16", t=50.0, k=6000)
    _sample(pv, l * 1e-30, p=0.5, k=9999)


@pytest.mark.gpu
def test_sample_where_likely_tokens_lie_together(pv):
    """The likely ones at the front of the vocabulary, at its end, side by side."""
    rng = np.random.default_rng(4)
    l = rng.standard_normal((4, 50000)).astype(np.float32)
    l[0, :3000] += 12
    l[1, -3000:] += 12
    l[2, 24000:24800] += 15
    l[3, 7] += 40
    for how in (dict(k=1500), dict(k=40, p=0.9), dict(p=0.95), dict(p=0.95, m=0.01), dict(k=2500, p=0.99)):
        _sample(pv, l, "f16", **how)


@pytest.mark.gpu
def test_sample_allowed_tokens_and_values_that_are_not_finite(pv):
    rng = np.random.default_rng(6)
    T, V = 8, 1003
    l = _logits(rng, T, V)
    l[1, ::3] = np.nan
    l[2, ::2] = -np.inf
    l[3, [5, 900]] = np.inf
    l[4] = -np.inf
    l[5] = np.nan
    l[6] = 3e38
    l[7, 10:] = -3e38
    words = (V + 31) // 32
    bits = rng.integers(0, 2**32, (T, words))
    bits[0] = 0  # nothing allowed
    bits[6] = 0
    bits[6, words - 1] = 1 << ((V - 1) % 32)  # the last one alone
    bits[7] = 0
    bits[7, 0] = 1 << 3
    t = np.array([1, 1, 0, 1, 1, 0, 0.5, 1.0])
    for allowed in (None, bits, bits[2]):
        for how in (dict(), dict(k=3), dict(p=0.9, k=100), dict(m=0.3)):
            tok = _sample(pv, l, t=t, allowed=allowed, pad=3, at=1, **how)
            assert int(tok[4]) == int(tok[5]) == -1
            if allowed is bits:
                assert int(tok[0]) == -1 and int(tok[6]) == V - 1 and int(tok[7]) == 3


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V", [131073, 1 << 22])
def test_sample_of_large_vocabularies(pv, V, kind):
    """Up to the largest one, and rows of all equal logits, whose weights come to 2^62."""
    import torch
    rng = np.random.default_rng(V % 1000)
    l = (rng.standard_normal((3, V)) * 1.5).astype(np.float32)
    l[1] = 0.25
    l[2, rng.integers(0, V, 60)] += 12
    x = _dev(l, kind)
    h = _host(x)
    words = np.array([2**32 - 1, 2**31 + 12345, 77777777], np.uint32)
    for t, k, p, m in ((0.8, 0, 1.0, 0.0), (0.8, 40, 0.9, 0.0), (1.0, 0, 0.7, 0.0), (0.7, 100000, 0.95, 0.0), (0.9, 0, 1.0, 0.3),
                       (3.0, 70001, 1.0, 0.001)):
        lp = torch.empty(3, device="cuda")
        tok = pv.pvmvmd_sample(x, torch.from_numpy(words.view(np.int32)).cuda().view(torch.uint32), pv.Sampling(t, k, p, m),
                               logprob=lp)
        for r in range(3):
            want, wlp = plain.sample_long(plain.distances(h[r], plain.multiplier(1.0, None, t)), t, k, p, m, words[r])
            assert int(tok[r]) == want, (r, t, k, p, m)
            assert abs(float(lp[r]) - wlp) <= 4 * E * (1 + abs(wlp))


@pytest.mark.gpu
def test_rows_far_apart(pv):
    """Rows further apart than 2^31 elements."""
    import torch
    V, far = 5000, 2**31 + 64
    flat = torch.empty(far + V, dtype=torch.bfloat16, device="cuda")
    x = flat.as_strided((2, V), (far, 1))
    x.copy_(torch.randn(2, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)))
    near = x.clone()
    word, how = torch.tensor([123456789, -5], dtype=torch.int32, device="cuda"), pv.Sampling(0.9, 200, 0.9)
    assert torch.equal(pv.pvmvmd_sample(x, word, how), pv.pvmvmd_sample(near, word, how))
    n = pv.Norm("layer", eps=1e-5)
    a = pv.pvmvmd_block_norm(near, near, pre=n, out=torch.empty_like(near))
    b = pv.pvmvmd_block_norm(x, x, residual_out=x, pre=n, out=torch.empty_like(near))
    assert torch.equal(a[0], x) and torch.equal(a[1], b[1])
    z = pv.pvmvmd_glu(near, near, out=torch.empty_like(near))
    x.copy_(near)
    pv.pvmvmd_glu(x, x, out=x)
    assert torch.equal(z, x)


@pytest.mark.gpu
def test_sample_frequencies(pv):
    """Random words in even steps draw each token as often as its probability says, to one draw of 4096 and what the
    weights' 22 bits are off."""
    import torch
    rng = np.random.default_rng(8)
    n, V = 4096, 40
    l = rng.standard_normal(V).astype(np.float32) * 2
    words = (np.arange(n, dtype=np.uint64) * (2**32 // n)).astype(np.uint32).view(np.int32)
    tok = pv.pvmvmd_sample(torch.from_numpy(np.tile(l, (n, 1))).cuda(), torch.from_numpy(words).cuda(), pv.Sampling())
    p = np.exp(l.astype(np.float64) - l.max())
    count = np.bincount(tok.cpu().numpy(), minlength=V)
    assert (np.abs(count - n * p / p.sum()) <= 1 + n * 2.0**-20).all()
    assert (np.diff(tok.cpu().numpy()) >= 0).all()


# ---------------------------------------------------------------- streams, graphs, calls at once

def _three(pv, s):
    pv.pvmvmd_block_norm(pv.Rows(s["y"], 1e-4, s["ts"]), s["r"], pre=s["n"], residual_out=s["r2"], out=s["x"],
                         out_token_scale=s["xs"])
    pv.pvmvmd_glu(pv.Rows(s["y"], 1e-4, s["ts"]), s["r2"], out=s["z"], out_token_scale=s["zs"])
    pv.pvmvmd_sample(pv.Rows(s["y"], 1e-3, s["ts"]), s["words"], s["how"], token=s["token"], logprob=s["lp"])
    return [s[k].clone() for k in ("r2", "x", "xs", "z", "zs", "token", "lp")]


def _state(pv, T, D, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"y": (torch.randn(T, D, device="cuda", generator=g) * 9000).to(torch.int64).remainder(plain.Q).to(torch.int32),
         "ts": torch.rand(T, device="cuda", generator=g) + 0.5, "r": torch.randn(T, D, device="cuda", generator=g),
         "words": torch.randint(-2**31, 2**31, (T,), device="cuda", generator=g).to(torch.int32)}
    s["n"] = pv.Norm("rms", torch.rand(D, device="cuda", generator=g))
    s["how"] = pv.Sampling(0.9, 100, 0.9, 0.001)
    s["r2"] = torch.empty(T, D, device="cuda")
    s["x"], s["z"] = (torch.empty(T, D, dtype=torch.int32, device="cuda") for _ in range(2))
    s["xs"], s["zs"], s["lp"] = (torch.empty(T, device="cuda") for _ in range(3))
    s["token"] = torch.empty(T, dtype=torch.int32, device="cuda")
    return s


@pytest.mark.gpu
def test_steps_captured_replayed_and_at_once(pv):
    import torch
    shapes = [(1, 4096), (40, 9000), (200, 2048)]
    states = [_state(pv, T, D, i) for i, (T, D) in enumerate(shapes)]
    want = [_three(pv, s) for s in states]
    again = [_three(pv, s) for s in states]
    for a, b in zip(want, again):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    torch.cuda.synchronize()
    # on streams of their own, at once
    streams = [torch.cuda.Stream() for _ in states]
    got = []
    for st, s in zip(streams, states):
        with torch.cuda.stream(st):
            for _ in range(3):
                r = _three(pv, s)
            got.append(r)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    # captured, with inputs that change under the graph
    graphs = []
    for s in states:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s["kept"] = _three(pv, s)
        graphs.append(g)
    for s, (T, D) in zip(states, shapes):
        other = _state(pv, T, D, 77)
        s["before"] = [s[k].clone() for k in ("y", "words")]
        s["y"].copy_(other["y"])
        s["words"].copy_(other["words"])
    changed = [_three(pv, s) for s in states]
    for s, g, c in zip(states, graphs, changed):
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(s["kept"], c))
    for s, g, w in zip(states, graphs, want):
        s["y"].copy_(s["before"][0])
        s["words"].copy_(s["before"][1])
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(s["kept"], w))


# ---------------------------------------------------------------- refusals

def test_steps_refuse_bad_arguments_before_device_use(pv):
    """Through the C ABI, with addresses that are never used."""
    lib = pv._lib
    R = lambda **k: pv.pvmvmd_rows(**dict(dict(data_dev=64, token=8, scale=1.0, type=pv.PVMVMD_F32), **k))  # noqa: E731
    O = lambda **k: pv.pvmvmd_rows_out(**dict(dict(data_dev=64, token=8, scale=1.0, limit=127, type=pv.PVMVMD_FIELD), **k))  # noqa: E731
    N = lambda **k: pv.pvmvmd_norm(**dict(dict(eps=1e-6, kind=1, type=pv.PVMVMD_F32), **k))  # noqa: E731
    ref = lambda v: None if v is None else ctypes.byref(v)  # noqa: E731
    ARG, SHAPE, PARAM = pv.PVMVMD_E_ARG, pv.PVMVMD_E_SHAPE, pv.PVMVMD_E_PARAM
    F32 = dict(type=pv.PVMVMD_F32)

    def norm(T=1, D=8, y=R(), post=None, gate=None, branch=1.0, residual=R(), keep=1.0, rout=O(**F32), pre=N(), out=O()):
        return lib.pvmvmd_block_norm(T, D, ref(y), ref(post), ref(gate), branch, ref(residual), keep, ref(rout), ref(pre),
                                     ref(out), None)
    inf = float("inf")
    assert norm(T=0) == pv.PVMVMD_OK
    assert norm(T=-1) == norm(D=0) == norm(D=pv.PVMVMD_MAX_K + 1) == SHAPE
    assert norm(y=None, residual=None) == norm(rout=None, out=None, pre=None) == norm(y=None, post=N()) == ARG
    assert norm(out=None) == norm(y=None, gate=R()) == ARG
    assert norm(y=R(data_dev=None)) == norm(y=R(type=9)) == norm(y=R(data_dev=66)) == norm(gate=R(type=0)) == ARG
    assert norm(residual=R(type=pv.PVMVMD_FIELD)) == norm(residual=R(scale=2.0)) == norm(residual=R(token_scale_dev=64)) == ARG
    assert norm(rout=O()) == norm(out=O(type=5)) == norm(out=O(data_dev=None)) == ARG
    assert norm(out=O(token_scale_dev=64, **F32)) == ARG
    assert norm(out=O(limit=0)) == norm(out=O(limit=(1 << 22) + 1)) == norm(out=O(scale=inf)) == PARAM
    assert norm(pre=N(kind=3)) == norm(post=N(kind=0)) == norm(pre=N(weight_dev=64, type=4)) == ARG
    assert norm(y=R(token_scale_dev=66)) == norm(y=R(channel_scale_dev=65)) == norm(pre=N(weight_dev=66)) == ARG
    assert norm(out=O(token_scale_dev=70)) == ARG
    assert norm(pre=N(eps=0.0)) == norm(pre=N(eps=float("nan"))) == norm(post=N(weight_add=inf)) == PARAM
    assert norm(branch=inf) == norm(keep=float("nan")) == norm(y=R(scale=inf)) == PARAM

    def glu(T=1, D=8, gate=R(), act=3, up=R(), out=O()):
        return lib.pvmvmd_glu(T, D, ref(gate), act, ref(up), ref(out), None)
    assert glu(T=0) == pv.PVMVMD_OK
    assert glu(T=-1) == glu(D=0) == glu(D=pv.PVMVMD_MAX_K + 1) == SHAPE
    assert glu(gate=None) == glu(out=None) == glu(act=5) == glu(act=-1) == glu(up=R(data_dev=None)) == ARG
    assert glu(out=O(limit=0)) == glu(gate=R(scale=inf)) == PARAM

    how = pv.pvmvmd_sampling(temperature=1.0, top_p=1.0)

    def sample(T=1, V=8, l=R(), how=how, random=64, token=64):
        return lib.pvmvmd_sample(T, V, ref(l), ref(how), None, 0, random, token, None, None)
    assert sample(T=0) == pv.PVMVMD_OK
    assert sample(T=-1) == sample(V=0) == sample(V=pv.PVMVMD_MAX_V + 1) == SHAPE
    assert sample(l=None) == sample(how=None) == sample(random=None) == sample(token=None) == ARG
    assert sample(random=66) == sample(token=65) == sample(how=pv.pvmvmd_sampling(top_k_dev=2)) == ARG
    assert sample(l=R(type=7)) == sample(l=R(data_dev=None)) == ARG and sample(l=R(scale=inf)) == PARAM


def test_binding_refuses_what_is_no_device_tensor(pv):
    import torch
    x = torch.zeros(2, 8)
    with pytest.raises(TypeError, match="CUDA"):
        pv.pvmvmd_block_norm(x, x)
    with pytest.raises(TypeError, match="CUDA"):
        pv.pvmvmd_glu(pv.Rows(x))
    with pytest.raises(TypeError, match="CUDA"):
        pv.pvmvmd_sample(x, torch.zeros(2, dtype=torch.int32), pv.Sampling())
    with pytest.raises(ValueError, match="there"):
        pv.pvmvmd_block_norm(None, None, residual_out=x)
    with pytest.raises(ValueError, match="act"):
        pv.pvmvmd_glu(x, act="tanh")
    with pytest.raises(ValueError, match="kind"):
        pv.Norm("batch")
    with pytest.raises(TypeError, match="CUDA"):
        pv.Norm("rms", torch.ones(8))
    with pytest.raises(TypeError, match="CUDA"):
        pv.Sampling(torch.ones(2))
    with pytest.raises(OverflowError):
        pv.Sampling(1.0, 1 << 40)


@pytest.mark.gpu
def test_binding_refuses_shapes_types_and_strides(pv):
    import torch
    d = dict(device="cuda")
    x, n = torch.zeros(4, 16, **d), pv.Norm("rms", torch.ones(16, **d))
    out = torch.zeros(4, 16, dtype=torch.int32, **d)
    bad = [
        lambda: pv.pvmvmd_block_norm(x, x[:3], pre=n, out=out), lambda: pv.pvmvmd_block_norm(x, x.t(), pre=n, out=out),
        lambda: pv.pvmvmd_block_norm(x, x, pre=pv.Norm("rms", torch.ones(8, **d)), out=out),
        lambda: pv.pvmvmd_block_norm(pv.Rows(x, 1.0, torch.ones(3, **d)), x), lambda: pv.pvmvmd_block_norm(x[0], x),
        lambda: pv.pvmvmd_block_norm(x, x, gate=x[:2]), lambda: pv.pvmvmd_glu(x, x[:, :8]),
        lambda: pv.pvmvmd_glu(x[:, ::2]), lambda: pv.pvmvmd_glu(x, out=out[:2]),
        lambda: pv.pvmvmd_glu(x, out=out, out_token_scale=torch.ones(5, **d)),
        lambda: pv.pvmvmd_sample(x, out[:3, 0].contiguous(), pv.Sampling()),
        lambda: pv.pvmvmd_sample(x, out[:, 0].contiguous(), pv.Sampling(torch.ones(3, **d))),
        lambda: pv.pvmvmd_sample(x, out[:, 0].contiguous(), pv.Sampling(), allowed=out[:, :2]),
        lambda: pv.Sampling(torch.ones(3, **d), torch.ones(4, dtype=torch.int32, **d)),
        lambda: pv.Norm("rms", torch.ones(4, **d), torch.ones(5, **d)),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    wrong = [lambda: pv.pvmvmd_block_norm(x.double(), x), lambda: pv.pvmvmd_block_norm(x, out),
             lambda: pv.pvmvmd_glu(x, out=x.double()), lambda: pv.pvmvmd_sample(x, x[:, 0].contiguous(), pv.Sampling()),
             lambda: pv.pvmvmd_sample(x, out[:, 0].contiguous(), pv.Sampling(), allowed=x[:, :1]),
             lambda: pv.Norm("rms", torch.ones(4, dtype=torch.int32, **d))]
    for f in wrong:
        with pytest.raises(TypeError):
            f()
    with pytest.raises(pv.PvmvmdError):
        pv.pvmvmd_glu(x, out=out, limit=0)
    with pytest.raises(pv.PvmvmdError):
        pv.pvmvmd_block_norm(x, x, pre=pv.Norm("rms", eps=0.0), out=out)
    # the same gate for all rows, as a row or a vector
    a = pv.pvmvmd_block_norm(x + 1, x, gate=torch.arange(16.0, **d))[0]
    b = pv.pvmvmd_block_norm(x + 1, x, gate=torch.arange(16.0, **d)[None])[0]
    assert torch.equal(a, b) and torch.equal(a[3], torch.arange(16.0, **d))
