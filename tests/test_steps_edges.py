"""The client's other steps at the edges of what their calls take: tensors that are refused, the ends of a norm's range,
and the choice of the next token among many rows."""
import ctypes

import numpy as np
import pytest

import steps_plain as plain
from test_attention import Fake
from test_steps import _dev, _host, _sample, pv  # noqa: F401


# ---------------------------------------------------------------- rows to write that lie on one another

@pytest.mark.parametrize("token", [0, 1, 7, -1, -7])
def test_overlapping_rows_to_write_are_refused(pv, token):
    """Rows closer than they are long would be written by several threads at once.  (A single row has no other.)"""
    R = pv.pvmvmd_rows(data_dev=64, token=8, scale=1.0, type=pv.PVMVMD_F32)
    good = pv.pvmvmd_rows_out(data_dev=64, token=8, scale=1.0, limit=127, type=pv.PVMVMD_F32)
    r, g = ctypes.byref(R), ctypes.byref(good)
    for kind in (pv.PVMVMD_F32, pv.PVMVMD_FIELD):
        bad = ctypes.byref(pv.pvmvmd_rows_out(data_dev=64, token=token, scale=1.0, limit=127, type=kind))
        assert pv._lib.pvmvmd_block_norm(2, 8, r, None, None, 1.0, r, 1.0, g, None, bad, None) == pv.PVMVMD_E_ARG
        assert pv._lib.pvmvmd_glu(2, 8, r, 3, r, bad, None) == pv.PVMVMD_E_ARG
    bad = ctypes.byref(pv.pvmvmd_rows_out(data_dev=64, token=token, scale=1.0, limit=127, type=pv.PVMVMD_F32))
    assert pv._lib.pvmvmd_block_norm(2, 8, r, None, None, 1.0, r, 1.0, bad, None, g, None) == pv.PVMVMD_E_ARG


@pytest.mark.parametrize("stride", [0, 5, 15])
def test_binding_refuses_overlapping_rows_to_write(pv, stride):
    import torch
    x = Fake((3, 16), torch.float32, address=64)
    bad, good = Fake((3, 16), torch.float32, (stride, 1), 64), Fake((3, 16), torch.float32, address=64)
    for call in (lambda: pv.pvmvmd_block_norm(x, x, residual_out=bad, stream=0),
                 lambda: pv.pvmvmd_block_norm(x, x, residual_out=good, out=bad, stream=0),
                 lambda: pv.pvmvmd_glu(x, out=bad, stream=0)):
        with pytest.raises(ValueError, match="on one another"):
            call()


@pytest.mark.gpu
def test_one_row_to_write_of_any_stride(pv):
    import torch
    x = torch.randn(1, 40, device="cuda")
    for stride in (0, 3):
        out = torch.empty(40, device="cuda").as_strided((1, 40), (stride, 1))
        pv.pvmvmd_glu(x, act="relu", out=out)
        assert torch.equal(out, x.clamp(min=0))


# ---------------------------------------------------------------- the ends of a norm's range

def _inverse_bounds(x, eps):
    """1 / sqrt of a row's mean of squares and eps, which is formed within 2^-39 of itself and 2^-146, rounded once: the
    smallest and the largest value that has."""
    M = np.square(x.astype(np.float64)).mean(-1, keepdims=True) + np.float64(np.float32(eps))
    off = M * 2.0**-39 + 2.0**-146
    return (1 / np.sqrt(M + off)).astype(np.float32), (1 / np.sqrt(np.maximum(M - off, 2.0**-149))).astype(np.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [1, 8, 40, 1100])
@pytest.mark.parametrize("lo,hi,eps", [(96, 126, 1e-6), (-30, 30, 1e-6), (-104, -40, 1e-38), (-150, -90, 1e-30), (-150, -90, 1e-38)],
                         ids=["large", "usual", "small", "small-eps", "smallest"])
def test_norm_over_its_range(pv, D, lo, hi, eps):
    """Rows whose squares' sums are 2^lo to just below 2^hi."""
    rng = np.random.default_rng(D)
    T = 20000 if D < 100 else 3000
    x = rng.standard_normal((T, D))
    x *= np.sqrt(np.exp2(rng.uniform(lo, hi - 0.001, (T, 1))) / np.square(x).sum(-1, keepdims=True))
    x = x.astype(np.float32)
    z = _dev(np.zeros((T, D), np.float32))
    pv.pvmvmd_block_norm(None, _dev(x), residual_out=False, pre=pv.Norm("rms", eps=eps), out=z)
    got = np.abs(_host(z))
    low, high = (np.abs(x * v) for v in _inverse_bounds(x, eps))
    bad = ~((got >= low) & (got <= high))
    assert not bad.any(), f"{bad.any(-1).sum()} of {T} rows, of squares' sums from " \
                          f"2^{np.log2(np.square(x.astype(np.float64)).sum(-1)[bad.any(-1)].min()):.1f} on"


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("D", [5, 1500, 9000])
def test_norm_of_zeros_with_any_eps(pv, kind, D):
    """Zeros, also with the smallest number above 0."""
    import torch
    x = torch.zeros(3, D, device="cuda")
    for eps in (1e-45, 1e-42, 1e-40, 1e-38, 1e-30, 1e-6, 1.0, 3e38):
        z = torch.full((3, D), 7.0, device="cuda")
        pv.pvmvmd_block_norm(None, x, residual_out=False, pre=pv.Norm(kind, eps=eps), out=z)
        assert (z == 0).all(), eps


# ---------------------------------------------------------------- what the binding takes

def test_steps_to_no_output_are_refused(pv):
    import torch
    x, s = Fake((3, 16), torch.float32, address=64), Fake((3,), torch.float32, address=64)
    with pytest.raises(ValueError, match="out_token_scale"):
        pv.pvmvmd_block_norm(x, x, residual_out=x, out_token_scale=s, stream=0)



@pytest.mark.gpu
def test_norm_of_no_weights_is_refused(pv):
    """A vector of no values is not the absence of weights, which holds for rows of any length."""
    import torch
    for name in ("weight", "bias"):
        with pytest.raises(ValueError, match="one value"):
            pv.Norm("rms", **{name: torch.empty(0, device="cuda")})



@pytest.mark.gpu
def test_sampling_of_an_empty_batch(pv):
    """Parameters of no rows are for calls of no rows, and those alone."""
    import torch
    d = dict(device="cuda")
    how = pv.Sampling(torch.empty(0, **d), torch.empty(0, dtype=torch.int32, **d), 0.9)
    word = torch.empty(0, dtype=torch.int32, **d)
    assert pv.pvmvmd_sample(torch.empty(0, 50, **d), word, how).shape == (0,)
    with pytest.raises(ValueError, match="of 0 rows"):
        pv.pvmvmd_sample(torch.zeros(1, 50, **d), torch.zeros(1, dtype=torch.int32, **d), how)
    with pytest.raises(ValueError):
        pv.Sampling(torch.empty(0, **d), torch.ones(2, dtype=torch.int32, **d))



@pytest.mark.gpu
def test_residual_as_rows(pv):
    """Rows without scales, as a tensor alone."""
    import torch
    y, r = (torch.randn(3, 40, device="cuda") for _ in range(2))
    want = pv.pvmvmd_block_norm(y, r)[0]
    assert want.dtype == torch.float32 and torch.equal(pv.pvmvmd_block_norm(y, pv.Rows(r))[0], want)
    assert torch.equal(pv.pvmvmd_block_norm(None, pv.Rows(r))[0], r)
    with pytest.raises(pv.PvmvmdError):
        pv.pvmvmd_block_norm(y, pv.Rows(r, 2.0))


# ---------------------------------------------------------------- the next token of many rows: one CTA each

def _many(pv, l, kind, scale=1.0, t=1.0, k=0, p=1.0, m=0.0, seed=0):
    import torch
    T, V = l.shape
    x = _dev(l, kind)
    per = lambda v, d: _dev(np.asarray(v, np.float32)[None])[0].to(d) if not np.isscalar(v) else v  # noqa: E731
    words = np.random.default_rng(seed).integers(0, 2**32, T, dtype=np.uint32)
    words[:2] = 0, 2**32 - 1
    lp = torch.empty(T, device="cuda")
    how = pv.Sampling(per(t, torch.float32), per(k, torch.int32), per(p, torch.float32), per(m, torch.float32))
    tok = pv.pvmvmd_sample(pv.Rows(x, scale), torch.from_numpy(words.view(np.int32)).cuda(), how, logprob=lp).cpu().numpy()
    lp = lp.cpu().numpy()
    h = plain.centred(_host(x)).astype(np.float32) if kind == "field" else _host(x)
    row = lambda v, r: v if np.isscalar(v) else v[r]  # noqa: E731
    for r in range(T):
        tr = row(t, r)
        xs = plain.distances(h[r], plain.multiplier(scale, None, tr))
        if tr > 0:
            want, wlp = plain.sample_long(xs, tr, int(row(k, r)), float(np.float32(row(p, r))), float(np.float32(row(m, r))), words[r])
        else:
            want, wlp = int(np.argmax(xs)), 0.0
        assert tok[r] == want, (r, tok[r], want)
        # the quotient of two whole numbers, each rounded, and log1p of a unit: 2^-23 of 1 and of the value
        assert abs(lp[r] - wlp) <= 2.0**-22 * (1 + abs(wlp)), (r, lp[r], wlp)


MANY = [
    dict(t=20.0, p=0.9), dict(t=20.0, k=1025), dict(t=1.0, k=1024), dict(t=5.0, k=1024, p=0.99), dict(t=8.0, k=7000, p=0.6),
    dict(t=3000.0, p=0.5), dict(t=3000.0, k=6001), dict(t=3000.0, k=6500, p=0.3), dict(t=1.0, p=0.95, m=0.05), dict(t=30.0, m=0.5),
]


@pytest.mark.gpu
@pytest.mark.parametrize("V,kind", [(6000, "f16"), (9001, "field"), (30000, "bf16"), (30011, "f32")])
@pytest.mark.parametrize("k", range(len(MANY)), ids=lambda k: "-".join(f"{a}={b}" for a, b in MANY[k].items()))
def test_tokens_of_many_rows(pv, V, kind, k):
    """More rows than SMs: lists, the histograms of flat rows (whose distances come down to one bin of them), several of
    each limit's ways."""
    rng = np.random.default_rng(V + k)
    l = (rng.standard_normal((160, V)) * 1.5).astype(np.float32)
    l[:40] *= 4
    scale = 1.0
    if kind == "field":
        l, scale = plain.field(np.rint(l * 5000)), 1 / 5000
    _many(pv, l, kind, scale, seed=k, **MANY[k])


@pytest.mark.gpu
@pytest.mark.parametrize("V,kind", [(6500, "f32"), (9001, "bf16"), (30000, "field")])
def test_tokens_of_many_rows_of_equal_values(pv, V, kind):
    """More equal logits than a list takes, and limits among them."""
    rng = np.random.default_rng(V)
    l = np.rint(rng.standard_normal((160, V)) * 0.8).astype(np.float32)
    l[:3] = 2.5 if kind != "field" else 2
    scale = 1.0
    if kind == "field":
        l, scale = plain.field(l.astype(np.int64)), 1.0
    for how in (dict(k=V // 3), dict(p=0.5), dict(t=2.0, k=V - 1, p=0.7), dict(t=0.5, k=1500, p=0.999, m=0.01), dict(k=1), dict(p=1e-7)):
        _many(pv, l, kind, scale, seed=len(how), **how)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["f32", "f16"])
def test_tokens_of_many_rows_of_all_kinds(pv, kind):
    """Rows that take every way in one call."""
    rng = np.random.default_rng(11)
    T, V = 200, 12011
    l = (rng.standard_normal((T, V)) * np.exp2(rng.uniform(-12, 3, (T, 1)))).astype(np.float32)
    off = rng.random((4, T))
    t = np.where(off[0] < 0.15, 0.0, np.exp2(rng.uniform(-2, 4, T)))
    k = np.where(off[1] < 0.3, 0, np.exp2(rng.uniform(0, 13.6, T)).astype(int))
    p = np.where(off[2] < 0.3, 1.0, rng.random(T))
    m = np.where(off[3] < 0.5, 0.0, rng.random(T) * 0.3)
    _many(pv, l, kind, t=t.astype(np.float32), k=k, p=p.astype(np.float32), m=m.astype(np.float32))


def test_results_in_the_random_words_are_refused(pv):
    """Every CTA of a row reads its word, some after another has chosen the row's token."""
    R = ctypes.byref(pv.pvmvmd_rows(data_dev=64, token=8, scale=1.0, type=pv.PVMVMD_F32))
    how = ctypes.byref(pv.pvmvmd_sampling(temperature=1.0, top_p=1.0))
    for token, logprob in ((1024, None), (1028, 4096), (1012, None), (4096, 1024), (4096, 1036), (4096, 1012)):
        assert pv._lib.pvmvmd_sample(4, 8, R, how, None, 0, 1024, token, logprob, None) == pv.PVMVMD_E_ARG, (token, logprob)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [6, 28, 100, 1022, 5004, 12000, 40000])
def test_mean_in_the_middle_of_two_numbers(pv, D):
    """Rows of two neighbouring numbers, as many of each: the mean is the even one of them.  (Sums of D of them and their
    D-th part are exact in 64 bits.)"""
    rng = np.random.default_rng(D)
    T = 400 if D < 5000 else 60
    low = np.exp2(rng.uniform(-3, 3, (T, 1))).astype(np.float32) * rng.choice([-1, 1], (T, 1)).astype(np.float32)
    x = np.repeat(low, D, axis=1)
    for row in x:
        up = rng.permutation(D)[:D // 2]
        row[up] = np.nextafter(row[up], np.float32(np.inf))
    z = _dev(np.zeros((T, D), np.float32))
    pv.pvmvmd_block_norm(None, _dev(x), residual_out=False, pre=pv.Norm("layer", eps=1e-5), out=z)
    assert np.array_equal(_host(z), plain.norm(x, "layer", eps=1e-5))


# ---------------------------------------------------------------- numbers and addresses of any kind

INF, NAN = float("inf"), float("nan")


@pytest.mark.gpu
@pytest.mark.parametrize("T", [5, 160])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_sample_with_any_parameters(pv, kind, T):
    """Scales, temperatures and limits that are zero, negative, tiny, huge or no numbers."""
    rng = np.random.default_rng(T)
    V = 1201
    l = (rng.standard_normal((T, V)) * 2).astype(np.float32)
    l[:, rng.integers(0, V, 20)] = np.array([INF, -INF, NAN, 3e38, -3e38] * 4, np.float32)
    l[0] = rng.standard_normal(V)
    ts, cs = np.ones(T, np.float32), np.ones(V, np.float32)
    ts[:5] = 1, 0, INF, NAN, -1
    cs[[3, 50, 700, 1199]] = 0, INF, NAN, -2
    for scale in (1.0, -1.0, 0.0, 1e-40, 1e30):
        _sample(pv, l, kind, scale, p=0.9, k=100)
    per = lambda *v: np.array([v[(i * 7) % len(v)] for i in range(T)])  # noqa: E731
    t, k = per(1.0, 0.7, 0.0, INF, NAN, 1e-40, -2.0, 1e30), per(0, 1, V, -3, 50, V - 1, 2**31 - 1)
    p, m = per(1.0, 0.9, 0.0, -1.0, NAN, 1e-12, 2.0), per(0.0, 1.0, NAN, 3.0, -1.0, 1e-9)
    for a in ((None, None), (ts, None), (None, cs), (ts, cs)):
        _sample(pv, l, kind, 1.0, *a, t=t, k=k, p=p, m=m)


@pytest.mark.gpu
@pytest.mark.parametrize("at", [1, 2, 3])
def test_scales_and_weights_off_the_16_byte_boundaries(pv, at):
    """Vectors that begin at any value: the same results as from the boundaries, with rows on these."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(at)
    T, D = 30, 4096
    x, y = (torch.randn(T, D, device="cuda", generator=g) for _ in range(2))
    v = [torch.rand(D, device="cuda", generator=g) + 0.5 for _ in range(3)]
    off = []
    for a in v:
        wide = torch.empty(D + at, device="cuda")
        wide[at:] = a
        off.append(wide[at:])
    word = torch.randint(-2**31, 2**31, (T,), device="cuda", generator=g).to(torch.int32)
    got = []
    for c, w, b in (v, off):
        n = pv.Norm("layer", w, b)
        r, o = pv.pvmvmd_block_norm(pv.Rows(x, 0.5, None, c), y, pre=n, out=torch.empty(T, D, dtype=torch.int32, device="cuda"), out_scale=30.0)
        z = pv.pvmvmd_glu(pv.Rows(x, 1.0, None, c), pv.Rows(y, 1.0, None, w), out=torch.empty_like(x))
        got.append((r, o, z, pv.pvmvmd_sample(pv.Rows(x, 1.0, None, c), word, pv.Sampling(0.9, 100, 0.9))))
    assert all(torch.equal(a, b) for a, b in zip(*got))
