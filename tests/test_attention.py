"""The client's attention (pvmvmd_rope, pvmvmd_kv_append, pvmvmd_paged_attention,
pvmvmd_kv_evict) against plain implementations in 64 bits.

Tolerances are bounds: u is the unit roundoff of the output's type (2^-8 for bf16,
2^-11 for fp16, 2^-24 for 32 bits).  An attention output may be off by its own
rounding, u |o|, by that of the probabilities to the type that the tensor cores
take, u sum_j p_j |v_j| (and 2^-24 sum_j |v_j| for fp16's smallest ones), and by
the scores' error in 32 bits, e = 2^-24 (D + 16) max_j |scale| sum_d |q_d k_jd|, which
moves p by the factor 1 + 2 e; the log of the sum by e and its own rounding."""
import ctypes

import numpy as np
import pytest

Q = 2013265921
U = {"bf16": 2.0**-8, "f16": 2.0**-11, "f32": 2.0**-24}


@pytest.fixture(scope="module")
def pv():
    import __graft_entry__
    __graft_entry__._load_build_module().build()
    import paper_2609_10264_gb300 as pv
    return pv


def _dt(name):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "field": torch.int32}[name]


def _dev(a, kind="f32"):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if kind == "field" else t.to(_dt(kind))).cuda()


def _host(t):
    return t.double().cpu().numpy()


# ---------------------------------------------------------------- plain implementations

def thetas(rot, base=10000.0, scaling="none", factor=1.0, original=0.0, slow=1.0, fast=32.0):
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2))
    th = base ** (-2.0 * np.arange(rot // 2) / rot)
    if scaling == "linear":
        th = th / factor
    if scaling == "ramp":
        g = np.clip((original * th / (2 * np.pi) - slow) / (fast - slow), 0, 1)
        th = th * (g + (1 - g) / factor)
    return th


def rotate(x, pos, th, inter, m=1.0):
    r = 2 * len(th)
    ang = np.asarray(pos, np.float64)[:, None] * th
    c, s = m * np.cos(ang)[:, None], m * np.sin(ang)[:, None]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if inter else (x[..., :r // 2], x[..., r // 2:r])
    y = x.copy()
    p, q = a * c - b * s, a * s + b * c
    if inter:
        y[..., 0:r:2], y[..., 1:r:2] = p, q
    else:
        y[..., :r // 2], y[..., r // 2:r] = p, q
    return y


def centred(v):
    v = v.astype(np.int64) & 0xFFFFFFFF
    return np.where(v > (Q - 1) // 2, v - Q, v).astype(np.float64)


def attend(q, K, V, n, scale, causal=True, window=0):
    """q (n, Hq, D), K and V (len, H, D) -> out, lse, mass (H, len), and the bounds' pieces: sum p|v|, sum |v|, e."""
    L, H, D = K.shape
    Hq = q.shape[1]
    out, lse = np.zeros((n, Hq, D)), np.full((n, Hq), -np.inf)
    pabs, vabs, e = np.zeros((n, Hq, D)), np.zeros((n, Hq, D)), np.zeros((n, Hq))
    mass = np.zeros((H, L))
    for t in range(n):
        at = L - n + t
        j = np.arange(L)
        see = np.ones(L, bool)
        if causal:
            see &= j <= at
        if window:
            see &= at - j < window
        if not see.any():
            continue
        for h in range(Hq):
            hk = h // (Hq // H)
            k, v = K[see, hk], V[see, hk]
            s = scale * (k @ q[t, h])
            z = s.max() + np.log(np.exp(s - s.max()).sum())
            p = np.exp(s - z)
            out[t, h], lse[t, h] = p @ v, z
            pabs[t, h], vabs[t, h] = p @ np.abs(v), np.abs(v).sum(0)
            e[t, h] = 2.0**-24 * (D + 16) * (abs(scale) * (np.abs(k) @ np.abs(q[t, h]))).max() + 2.0**-20
            mass[hk, see] += p
    return out, lse, mass, pabs, vabs, e


class Cache:
    """A paged cache on the host (64-bit copies of what the device holds) and on the device."""

    def __init__(self, pv, lens, news, H, D, page, kind, seed, layout="nhd", extra=2, mass=True, garbage=True):
        import torch
        rng = np.random.default_rng(seed)
        self.lens, self.news, self.H, self.D, self.page, self.kind = list(lens), list(news), H, D, page, kind
        B = len(lens)
        need = [-(-x // page) for x in lens]
        total, width = sum(need) + extra, max(1, max(need))
        order = rng.permutation(total)
        table = np.full((B, width + 1), -7, np.int32)
        at = 0
        for b in range(B):
            table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
        shape = (total, page, H, D)
        K, V = rng.standard_normal(shape), rng.standard_normal(shape)
        if layout == "hnd":  # heads outside slots
            self.K, self.V = (_dev(x.transpose(0, 2, 1, 3), kind).transpose(1, 2) for x in (K, V))
        elif layout == "fused":  # keys and values of a slot side by side
            kv = _dev(np.concatenate([K, V], -1), kind)
            self.K, self.V = kv[..., :D], kv[..., D:]
        else:
            self.K, self.V = _dev(K, kind), _dev(V, kind)
        self.mass0 = rng.random((total, H, page)).astype(np.float32)
        self.mass = _dev(self.mass0) if mass else None
        self.tab, self.table = table, _dev(table, "field")[:, :width]
        self.dlens = _dev(np.array(lens, np.int32), "field")
        self.cu_host = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
        self.cu = _dev(self.cu_host, "field")
        if garbage:  # behind the ends, and on pages of nobody
            dead = np.ones((total, page), bool)
            for b in range(B):
                p, o = self.at(b)
                dead[p, o] = False
            d = torch.from_numpy(dead).cuda()
            self.K[d], self.V[d] = float("nan"), float("inf")
        self.pool = pv.KvPool(self.K, self.V, self.mass)
        one = all(x == 1 for x in news)
        self.batch = pv.KvBatch(self.table, self.dlens, None if one else self.cu, max_new=max(news))

    def at(self, b, n=None, table=None):
        j = np.arange(self.lens[b] if n is None else n)
        t = self.tab if table is None else table
        return t[b, j // self.page], j % self.page

    def rows(self, b, what):
        p, o = self.at(b)
        x = _host({"K": self.K, "V": self.V}[what])
        return x[p, o]

    def masses(self, b, m):
        p, o = self.at(b)
        return m[p, :, o].T  # (H, len)


def check_attention(pv, lens, news, Hq, H, D, page, kind, seed, layout="nhd", causal=True, window=0, accumulate=False,
                    gain=1.0, scale=None, strided=False, unknown=False, lse=True):
    import torch
    c = Cache(pv, lens, news, H, D, page, kind, seed, layout)
    if unknown:
        c.batch = pv.KvBatch(c.table, c.dlens, c.cu)
    rng = np.random.default_rng(seed + 1)
    T = sum(news)
    q = _dev(gain * rng.standard_normal((T, Hq + 2 if strided else Hq, D)), kind)
    if strided:
        q = q[:, 1:-1]
    out = torch.full((T, Hq, D + 8 if strided else D), 7.0, dtype=_dt(kind), device="cuda")[..., :D]
    z = torch.full((T, Hq), 7.0, device="cuda") if lse else None
    pv.pvmvmd_paged_attention(c.pool, c.batch, q, out=out, lse=z, scale=scale, causal=causal, window=window,
                              accumulate=accumulate)
    assert pv.pvmvmd_device_status() == 0
    qh, oh, zh, mh = _host(q), _host(out), _host(z) if lse else None, _host(c.mass)
    u = U[kind]
    touched = np.zeros(mh.shape, bool)
    for b, (L, n) in enumerate(zip(lens, news)):
        r = slice(c.cu_host[b], c.cu_host[b + 1])
        o, l, m, pabs, vabs, e = attend(qh[r], c.rows(b, "K"), c.rows(b, "V"), n, D**-0.5 if scale is None else scale,
                                        causal, window)
        tol = u * np.abs(o) + (u + 2 * e[..., None]) * pabs + (2.0**-24 * vabs if kind == "f16" else 0) + 1e-30
        tol = tol * (1 + u)
        bad = np.argwhere(~(np.abs(oh[r] - o) <= tol))
        assert bad.size == 0, (b, len(bad), bad[:4].tolist(), oh[r][tuple(bad[0])], o[tuple(bad[0])])
        if lse:
            same = np.where(np.isinf(l), zh[r] == l, np.abs(zh[r] - np.where(np.isinf(l), 0, l)) <=
                            e + 2.0**-20 * (1 + np.abs(np.where(np.isinf(l), 0, l))))
            assert same.all(), (b, np.argwhere(~same)[:4].tolist())
        if accumulate:
            p, s = c.at(b)
            touched[p, :, s] = True
            got, was = c.masses(b, mh), c.masses(b, c.mass0.astype(np.float64))
            emax = e.max(initial=0.0) if n else 0.0
            tol_m = m * (2 * emax + 2.0**-18) + 2.0**-22 * (was + m)
            assert (np.abs(got - was - m) <= tol_m).all(), (b, np.abs(got - was - m).max())
    if accumulate:
        assert np.array_equal(mh[~touched], c.mass0.astype(np.float64)[~touched])
    else:
        assert np.array_equal(mh, c.mass0.astype(np.float64))
    return c, q, out, z


# ---------------------------------------------------------------- host logic

def test_turns_are_the_frequencies(pv):
    for kw in ({}, {"base": 500000.0}, {"scaling": "linear", "factor": 4.0}, {"scaling": "base", "factor": 8.0},
               {"scaling": "ramp", "factor": 8.0, "original": 8192.0, "slow": 1.0, "fast": 4.0}):
        for rot in (2, 64, 128) if kw.get("scaling") != "base" else (4, 128):
            got = pv.pvmvmd_rope_turns(rot, **kw).astype(np.float64) * 2.0**-64
            exp = thetas(rot, **kw) / (2 * np.pi)
            assert (np.abs(got - exp) <= 2.0**-64 + 2.0**-50 * exp).all()  # the unit, and doubles
    assert pv.pvmvmd_rope_turns(4, base=2.0**-20)[1] > 0  # more than a turn per position: the rest


@pytest.mark.parametrize("kw", [{"rot": 3}, {"rot": 0}, {"base": 0.0}, {"base": float("inf")},
                                {"scaling": "linear", "factor": 0.5}, {"scaling": "linear", "factor": float("nan")},
                                {"rot": 2, "scaling": "base", "factor": 2.0},
                                {"scaling": "ramp", "factor": 2.0, "original": 0.0},
                                {"scaling": "ramp", "factor": 2.0, "original": 100.0, "slow": 4.0, "fast": 4.0}])
def test_turns_refuse(pv, kw):
    with pytest.raises(pv.PvmvmdError) as e:
        pv.pvmvmd_rope_turns(**{"rot": 64, **kw})
    assert e.value.status == pv.PVMVMD_E_PARAM
    with pytest.raises(ValueError):
        pv.pvmvmd_rope_turns(64, scaling="unknown")


def _c_pool(pv, **kw):
    d = dict(K_dev=4096, V_dev=8192, mass_dev=4096, k_page=1024, k_slot=64, k_head=64, v_page=1024, v_slot=64, v_head=64,
             pages=4, page_size=16, heads=1, dim=64, type=pv.PVMVMD_BF16)
    d.update(kw)
    return ctypes.byref(pv.pvmvmd_kv_pool(*[d[f] for f, _ in pv.pvmvmd_kv_pool._fields_]))


def _c_batch(pv, **kw):
    d = dict(table_dev=4096, lens_dev=4096, cu_dev=None, table_stride=4, B=2, T=2, max_pages=4, max_new=0)
    d.update(kw)
    return ctypes.byref(pv.pvmvmd_kv_batch(*[d[f] for f, _ in pv.pvmvmd_kv_batch._fields_]))


def test_refusals_before_any_device_use(pv):
    """Nothing here is dereferenced: every call is refused by its arguments."""
    lib, E = pv._lib, pv
    rows, none = (4096, 64, 64), (None, 0, 0)

    def att(pool=None, batch=None, Hq=2, q=rows, window=0, acc=0, out=rows):
        return lib.pvmvmd_paged_attention(pool or _c_pool(pv), batch or _c_batch(pv), Hq, *q, 1.0, 1, window, acc, *out,
                                          None, None)
    assert att(batch=_c_batch(pv, T=0, cu_dev=4096), q=none, out=none) == E.PVMVMD_OK
    assert lib.pvmvmd_paged_attention(None, _c_batch(pv), 2, *rows, 1.0, 1, 0, 0, *rows, None, None) == E.PVMVMD_E_ARG
    assert lib.pvmvmd_paged_attention(_c_pool(pv), None, 2, *rows, 1.0, 1, 0, 0, *rows, None, None) == E.PVMVMD_E_ARG
    for kw in (dict(K_dev=None), dict(V_dev=None), dict(type=E.PVMVMD_F32), dict(type=0), dict(K_dev=4104),
               dict(k_slot=60), dict(v_head=4), dict(k_page=12)):
        assert att(_c_pool(pv, **kw)) == E.PVMVMD_E_ARG, kw
    for kw in (dict(dim=0), dict(dim=60), dict(dim=136), dict(pages=0), dict(page_size=0), dict(heads=0)):
        assert att(_c_pool(pv, **kw)) == E.PVMVMD_E_SHAPE, kw
    for kw in (dict(B=0), dict(T=-1), dict(T=3), dict(max_pages=0), dict(max_new=-1), dict(max_pages=1 << 30)):
        assert att(batch=_c_batch(pv, **kw)) == E.PVMVMD_E_SHAPE, kw
    for kw in (dict(table_dev=None), dict(lens_dev=None)):
        assert att(batch=_c_batch(pv, **kw)) == E.PVMVMD_E_ARG, kw
    assert att(_c_pool(pv, heads=2), Hq=3) == E.PVMVMD_E_SHAPE
    assert att(Hq=0) == E.PVMVMD_E_SHAPE
    assert att(window=-1) == E.PVMVMD_E_SHAPE
    assert att(_c_pool(pv, mass_dev=None), acc=1) == E.PVMVMD_E_ARG
    for bad in (none, (4100, 64, 64), (4096, 60, 64), (4096, 64, 4)):
        assert att(q=bad) == E.PVMVMD_E_ARG
        assert att(out=bad) == E.PVMVMD_E_ARG

    rope = ctypes.byref(pv.pvmvmd_rope_view(4096, 64, 0, 1.0))

    def app(pool=None, batch=None, r=rope, kind=E.PVMVMD_FIELD, k=rows, v=rows, Hq=0, q=none, qo=none):
        return lib.pvmvmd_kv_append(pool or _c_pool(pv), batch or _c_batch(pv), r, None, kind, 1.0, *k, *v, Hq, *q, *qo,
                                    None)
    assert app(batch=_c_batch(pv, T=0, cu_dev=4096), k=none, v=none) == E.PVMVMD_OK
    assert app(k=none) == app(v=none) == app(kind=9) == app(Hq=2, q=rows) == E.PVMVMD_E_ARG
    assert app(Hq=0, q=rows, qo=rows) == app(batch=_c_batch(pv, T=1)) == E.PVMVMD_E_SHAPE
    for rot in (1, 0, 66):
        assert app(r=ctypes.byref(pv.pvmvmd_rope_view(4096, rot, 0, 1.0))) == E.PVMVMD_E_SHAPE
    assert app(r=ctypes.byref(pv.pvmvmd_rope_view(None, 64, 0, 1.0))) == E.PVMVMD_E_ARG

    def rp(r=rope, pos=4096, T=2, H=2, D=64, x=4096, xt=E.PVMVMD_F32, out=4096, ot=E.PVMVMD_F32):
        return lib.pvmvmd_rope(r, pos, T, H, D, x, xt, 128, 64, 1.0, out, ot, 128, 64, None)
    assert rp(T=0, x=None, out=None, pos=None) == E.PVMVMD_OK
    assert rp(r=None) == rp(pos=None) == rp(x=None) == rp(out=None) == rp(xt=0) == rp(ot=E.PVMVMD_FIELD) == E.PVMVMD_E_ARG
    assert rp(T=-1) == rp(H=0) == rp(D=0) == rp(D=62) == E.PVMVMD_E_SHAPE

    def ev(pool=None, budget=8, recent=2, table=4096, width=4, lens=4096):
        return lib.pvmvmd_kv_evict(pool or _c_pool(pv), _c_batch(pv), budget, recent, table, 4, width, lens, None)
    assert ev(_c_pool(pv, mass_dev=None)) == ev(table=None) == ev(lens=None) == E.PVMVMD_E_ARG
    assert ev(budget=0) == ev(recent=-1) == ev(width=0) == ev(budget=17, width=1) == E.PVMVMD_E_SHAPE


# ---------------------------------------------------------------- rotary positions

class Fake:
    """What the binding looks at of a tensor."""

    def __init__(self, shape, dtype, strides=None, address=0, cuda=True):
        import torch
        self.shape, self.dtype, self.is_cuda, self.address = torch.Size(shape), dtype, cuda, address
        self.strides = strides or torch.empty(shape, device="meta").stride()

    def stride(self):
        return self.strides

    def data_ptr(self):
        return self.address

    def is_contiguous(self):
        return True

    def numel(self):
        return self.shape.numel()


def test_binding_refuses_tensors(pv):
    """What the native binding checks, before the library sees anything (which refuses null pointers)."""
    import torch
    bf, f16, f32, i32 = torch.bfloat16, torch.float16, torch.float32, torch.int32
    pool, batch = object.__new__(pv.KvPool), object.__new__(pv.KvBatch)
    pool.view = pv.pvmvmd_kv_pool(16, 16, None, 1024, 128, 64, 1024, 128, 64, 4, 8, 2, 64, pv.PVMVMD_BF16)
    batch.view = pv.pvmvmd_kv_batch(16, 16, None, 4, 3, 3, 4, 0)
    batch.B, batch.table, batch.lens = 3, Fake((3, 4), i32), Fake((3,), i32)
    for v in (pool, batch):
        v.address = ctypes.addressof(v.view)
    q = Fake((3, 4, 64), bf)

    def refused(kind, match, f, *args, **kw):
        with pytest.raises(kind, match=match):
            f(*args, **{"stream": 0, **kw})

    attend = pv.pvmvmd_paged_attention
    refused(pv.PvmvmdError, None, attend, pool, batch, q, out=q)  # null pointers
    assert batch.view.T == 3
    refused(TypeError, "q must be a CUDA tensor", attend, pool, batch, Fake((3, 4, 64), bf, cuda=False), out=q)
    refused(TypeError, "q must be a CUDA tensor", attend, pool, batch, np.zeros((3, 4, 64)), out=q)
    refused(TypeError, "q must have dtype torch.bfloat16", attend, pool, batch, Fake((3, 4, 64), f16), out=q)
    refused(ValueError, "q must have 3 dimensions", attend, pool, batch, Fake((3, 256), bf), out=q)
    refused(ValueError, "out must be 3 x 4 x 64", attend, pool, batch, q, out=Fake((3, 2, 64), bf))
    refused(ValueError, "the last dimension of q", attend, pool, batch, Fake((3, 4, 64), bf, (512, 128, 2)), out=q)
    refused(ValueError, "lse has 9 elements, expected 12", attend, pool, batch, q, out=q, lse=Fake((3, 3), f32))
    refused(TypeError, "lse must have dtype", attend, pool, batch, q, out=q, lse=Fake((3, 4), f16))
    refused(OverflowError, "window", attend, pool, batch, q, out=q, window=2**31)
    refused(TypeError, None, attend, pool, batch, q, out=q, window=1.5)
    refused(TypeError, None, attend, pool, batch, q, out=q, scale="1")
    append, k = pv.pvmvmd_kv_append, Fake((3, 2, 64), f16)
    refused(pv.PvmvmdError, None, append, pool, batch, k, k)
    refused(TypeError, "k must be a floating or field tensor", append, pool, batch, Fake((3, 2, 64), torch.int64), k)
    refused(TypeError, "v must have dtype", append, pool, batch, k, Fake((3, 2, 64), bf))
    refused(ValueError, "v must be 3 x 2 x 64", append, pool, batch, k, Fake((2, 2, 64), f16))
    refused(TypeError, "q_out must have dtype torch.bfloat16", append, pool, batch, k, k, q=Fake((3, 4, 64), f16),
            q_out=Fake((3, 4, 64), f16))
    refused(TypeError, "positions must have dtype", append, pool, batch, k, k, Fake((3,), torch.int64))
    rope = pv.RopeTable(Fake((32,), torch.int64), 64, 1.0)
    refused(pv.PvmvmdError, None, pv.pvmvmd_rope, q, Fake((3,), i32), rope, out=q)
    refused(ValueError, "positions has 2 elements", pv.pvmvmd_rope, q, Fake((2,), i32), rope, out=q)
    refused(TypeError, "out must be a floating tensor", pv.pvmvmd_rope, q, Fake((3,), i32), rope, out=Fake((3, 4, 64), i32))
    evict = pv.pvmvmd_kv_evict
    refused(pv.PvmvmdError, None, evict, pool, batch, 5)  # no mass
    refused(ValueError, "new_table must be", evict, pool, batch, 5, new_table=Fake((2, 4), i32))
    refused(ValueError, "new_table must be", evict, pool, batch, 5, new_table=Fake((3, 4), i32, (1, 3)))
    refused(ValueError, "new_table must be", evict, pool, batch, 5, new_table=Fake((3, 4), torch.int64))
    refused(ValueError, "new_lens has 4 elements", evict, pool, batch, 5, new_lens=Fake((4,), i32))
    refused(AttributeError, "cuda_stream", attend, pool, batch, q, out=q, stream="s")


@pytest.mark.gpu
@pytest.mark.parametrize("T,H,D,rot,kind,out,inter,strided", [
    (1, 1, 2, 2, "f32", "f32", False, False), (1, 40, 128, 128, "bf16", "bf16", False, False),
    (3, 7, 96, 64, "f32", "f32", True, True), (5, 2, 128, 128, "field", "bf16", False, False),
    (257, 3, 80, 40, "f16", "f16", True, False), (33, 5, 64, 64, "bf16", "f32", False, True),
    (9, 3, 70, 34, "f32", "f16", False, False), (4, 2, 13, 6, "field", "f32", True, False),
    (700, 8, 64, 32, "field", "f16", False, True), (31, 3, 24, 24, "bf16", "bf16", False, False)])
@pytest.mark.parametrize("scaling", ["none", "ramp"])
def test_rope(pv, T, H, D, rot, kind, out, inter, strided, scaling):
    import torch
    rng = np.random.default_rng(T * 131 + D)
    kw = {"base": 500000.0, "scaling": scaling}
    if scaling == "ramp":
        kw.update(factor=8.0, original=8192.0, slow=1.0, fast=4.0)
    m = 1.0 if scaling == "none" else 1.25
    table = pv.pvmvmd_rope_table(rot, magnitude=m, **kw)
    pos = rng.integers(-5, 200000, T).astype(np.int32)
    pos[0] = 2**31 - 1 if T > 4 else 0
    scale = 1.0
    wide = H + (2 if strided else 0)
    if kind == "field":
        v = rng.integers(-40000, 40001, (T, wide, D))
        x, scale = _dev((v % Q).astype(np.int64).astype(np.int32), "field"), 2.0**-15
    else:
        x = _dev(rng.standard_normal((T, wide, D)), kind)
    if strided:
        x = x[:, 1:-1]
    xh = (centred(x.cpu().numpy()) * scale) if kind == "field" else _host(x)
    y = pv.pvmvmd_rope(x, _dev(pos, "field"), table, out=torch.full((T, H, D), 9.0, dtype=_dt(out), device="cuda"),
                       interleaved=inter, scale=scale)
    exp = rotate(xh, pos, thetas(rot, **kw), inter, m)
    # a rotated value: its rounding, and 32-bit arithmetic on the pair (angle, sine, two products and a sum: below
    # 2^-20 of the pair's size); frequencies in double are 2^-52 of a turn off, times the position
    mag = np.abs(rotate(np.abs(xh), pos * 0, thetas(rot, **kw), inter, m)).max(-1, keepdims=True)
    tol = U[out] * np.abs(exp) + 4 * (2.0**-20 + 2.0**-49 * np.abs(pos.astype(np.float64))[:, None, None]) * mag
    if out == "f16":
        tol = tol + 2.0**-25
    assert (np.abs(_host(y) - exp) <= tol).all(), np.abs(_host(y) - exp).max()


@pytest.mark.gpu
def test_rope_in_place_and_empty(pv):
    import torch
    table = pv.pvmvmd_rope_table(64)
    x = torch.randn(50, 3, 64, device="cuda").to(torch.bfloat16)
    pos = torch.arange(50, dtype=torch.int32, device="cuda")
    y = pv.pvmvmd_rope(x, pos, table)
    assert not torch.equal(x, y)
    pv.pvmvmd_rope(x, pos, table, out=x)
    assert torch.equal(x, y)
    e = pv.pvmvmd_rope(x[:0], pos[:0], table)
    assert e.shape == (0, 3, 64)
    # values that are not rotated pass as they are, also those that are not numbers
    x[0, 0, 40] = float("inf")
    z = pv.pvmvmd_rope(x, pos, pv.pvmvmd_rope_table(16))
    assert torch.equal(z[..., 16:], x[..., 16:])


@pytest.mark.gpu
def test_rotation_is_undone_by_the_opposite_positions(pv):
    import torch
    table = pv.pvmvmd_rope_table(128, base=500000.0)
    x = torch.randn(64, 2, 128, device="cuda")
    pos = torch.randint(-2**31, 2**31 - 1, (64,), dtype=torch.int64, device="cuda").to(torch.int32)
    back = pv.pvmvmd_rope(pv.pvmvmd_rope(x, pos, table), -pos, table)
    assert (back - x).abs().max() < 2e-6 * 4  # two passes of 2^-20 of values below 4


# ---------------------------------------------------------------- append

@pytest.mark.gpu
@pytest.mark.parametrize("lens,news,Hq,H,D,page,kind,src,layout,inter,rot", [
    ([8], [8], 32, 8, 128, 16, "bf16", "field", "nhd", False, 128),
    ([1, 1, 5], [1, 1, 1], 4, 2, 64, 16, "f16", "field", "hnd", False, 64),
    ([40, 17, 300], [33, 17, 1], 8, 8, 80, 7, "bf16", "bf16", "nhd", True, 40),
    ([5, 0, 2], [3, 0, 4], 6, 2, 128, 1, "f16", "f16", "fused", False, 128),
    ([1000, 900], [700, 900], 5, 1, 96, 64, "bf16", "f32", "hnd", True, 96),
    ([130, 64], [129, 64], 4, 4, 24, 24, "f16", "f32", "nhd", False, 20)])
@pytest.mark.parametrize("with_q,given", [(True, True), (False, False)])
def test_append(pv, lens, news, Hq, H, D, page, kind, src, layout, inter, rot, with_q, given):
    import torch
    c = Cache(pv, lens, news, H, D, page, kind, 5, layout, garbage=False)
    rng = np.random.default_rng(6)
    T, scale = sum(news), 1.0
    if src == "field":
        x, scale = _dev((rng.integers(-30000, 30001, (T, Hq + 2 * H, D)) % Q).astype(np.int32), "field"), 2.0**-14
        xh = centred(x.cpu().numpy()) * scale
    else:
        x = _dev(rng.standard_normal((T, Hq + 2 * H, D)), src)
        xh = _host(x)
    K0, V0 = _host(c.K), _host(c.V)
    table = pv.pvmvmd_rope_table(rot)
    idx = np.concatenate([np.arange(L - n, L) for L, n in zip(lens, news)]) if T else np.zeros(0)
    pos = (idx + rng.integers(0, 5000, T)).astype(np.int32) if given else idx.astype(np.int32)
    q_out = torch.full((T, Hq, D), 3.0, dtype=_dt(kind), device="cuda") if with_q else None
    pv.pvmvmd_kv_append(c.pool, c.batch, x[:, Hq:Hq + H], x[:, Hq + H:], _dev(pos, "field") if given else None, table,
                        q=x[:, :Hq] if with_q else None, q_out=q_out, interleaved=inter, scale=scale)
    torch.cuda.synchronize()
    th, u = thetas(rot), U[kind]
    m0 = c.mass0.astype(np.float64)

    def near(got, exp, what):
        mag = np.abs(exp).max(-1, keepdims=True) * 2
        assert (np.abs(got - exp) <= u * np.abs(exp) + 2.0**-18 * mag + 2.0**-25).all(), what
    if with_q:
        near(_host(q_out), rotate(xh[:, :Hq], pos, th, inter), "q")
    kr = rotate(xh[:, Hq:Hq + H], pos, th, inter)
    Kg, Vg, mg = _host(c.K), _host(c.V), _host(c.mass)
    for b, (L, n) in enumerate(zip(lens, news)):
        for i in range(n):
            at, t = L - n + i, c.cu_host[b] + i
            if at < 0:
                continue
            p, o = c.tab[b, at // page], at % page
            near(Kg[p, o], kr[t], ("k", b, i))
            near(Vg[p, o], xh[t, Hq + H:], ("v", b, i))
            assert (mg[p, :, o] == 0).all()
            K0[p, o], V0[p, o], m0[p, :, o] = Kg[p, o], Vg[p, o], 0
    assert np.array_equal(Kg, K0) and np.array_equal(Vg, V0) and np.array_equal(mg, m0)  # and nothing else


@pytest.mark.gpu
def test_append_keeps_off_what_is_not_its_own(pv):
    """Page numbers outside the pool, and lengths beyond the table, write nothing."""
    import torch
    c = Cache(pv, [20, 20], [2, 2], 2, 64, 16, "bf16", 1, garbage=False)
    c.table[0, 1] = 1 << 20
    c.table[1, 1] = -1
    K0 = c.K.clone()
    x = torch.ones(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    pv.pvmvmd_kv_append(c.pool, c.batch, x, x)
    assert torch.equal(c.K, K0)
    c.dlens.fill_(10000)  # taken as 32, all that the table holds: slots 30 and 31
    pv.pvmvmd_kv_append(c.pool, c.batch, x, x)
    assert torch.equal(c.K, K0)
    c.dlens.fill_(-5)
    pv.pvmvmd_kv_append(c.pool, c.batch, x, x)
    assert torch.equal(c.K, K0)


# ---------------------------------------------------------------- attention

DECODE = [  # lens, Hq, H, D, page, kind, layout
    ([1], 1, 1, 8, 1, "bf16", "nhd"), ([200], 32, 8, 128, 16, "bf16", "nhd"),
    ([1, 17, 64, 65, 1000, 3], 8, 2, 64, 16, "f16", "hnd"), ([333, 5], 5, 1, 80, 7, "bf16", "nhd"),
    ([2000, 0, 31], 64, 8, 128, 32, "bf16", "fused"), ([4097], 4, 4, 96, 100, "f16", "nhd"),
    ([129] * 40, 16, 2, 128, 64, "bf16", "nhd"), ([700], 20, 1, 128, 16, "f16", "nhd"),
    ([257, 90], 48, 1, 64, 24, "bf16", "hnd"), ([33], 200, 1, 40, 16, "bf16", "nhd")]


@pytest.mark.gpu
@pytest.mark.parametrize("lens,Hq,H,D,page,kind,layout", DECODE)
@pytest.mark.parametrize("accumulate", [False, True])
def test_single_tokens(pv, lens, Hq, H, D, page, kind, layout, accumulate):
    check_attention(pv, lens, [1] * len(lens), Hq, H, D, page, kind, 11, layout, accumulate=accumulate,
                    strided=len(lens) == 2)


CHUNKS = [  # lens, news, Hq, H, D, page, kind, layout
    ([8], [8], 32, 8, 128, 16, "bf16", "nhd"), ([2, 9], [2, 3], 4, 2, 64, 16, "f16", "nhd"),
    ([130, 40, 300], [129, 1, 77], 4, 4, 64, 24, "f16", "hnd"), ([500, 260], [257, 260], 8, 1, 128, 64, "bf16", "nhd"),
    ([70, 0, 5], [70, 0, 9], 6, 2, 80, 1, "bf16", "fused"), ([400], [130], 5, 1, 96, 100, "f16", "nhd"),
    ([1100], [64], 8, 2, 128, 128, "bf16", "hnd"), ([3, 700, 64, 1], [3, 4, 2, 1], 8, 2, 128, 16, "bf16", "nhd"),
    ([385], [300], 1, 1, 128, 16, "f16", "nhd"), ([90], [33], 24, 8, 40, 12, "bf16", "nhd"),
    ([700, 333], [200, 300], 4, 2, 128, 16, "bf16", "fused"), ([600], [200], 16, 16, 8, 32, "f16", "nhd"),
    ([900, 10], [64, 10], 6, 2, 24, 256, "bf16", "hnd"), ([1300, 800, 20], [3, 100, 1], 32, 8, 128, 48, "bf16", "nhd"),
    ([260] * 3, [1, 257, 2], 64, 1, 64, 8, "f16", "nhd"), ([2500], [400], 12, 4, 128, 64, "bf16", "nhd")]


@pytest.mark.gpu
@pytest.mark.parametrize("lens,news,Hq,H,D,page,kind,layout", CHUNKS)
@pytest.mark.parametrize("causal,window,accumulate", [(True, 0, False), (True, 37, True), (False, 0, True)])
def test_chunks(pv, lens, news, Hq, H, D, page, kind, layout, causal, window, accumulate):
    check_attention(pv, lens, news, Hq, H, D, page, kind, 12, layout, causal, window, accumulate,
                    strided=len(lens) == 1, unknown=window == 37)


TOGETHER = [  # lens, news, Hq, H, D, page, kind, layout
    ([3000, 700, 1200, 0], [3, 1, 200, 0], 16, 2, 128, 16, "bf16", "nhd"),    # 24, 8 and 1600 rows a head
    ([6044], [5], 8, 2, 80, 24, "f16", "nhd"), ([2000, 900], [4, 2], 32, 4, 96, 100, "bf16", "hnd"),
    ([9000, 9000], [2, 130], 4, 1, 64, 64, "bf16", "nhd"),                    # the chunk's keys in parts
    ([40 + 7 * (i % 90) for i in range(150)], [1 + 5 * i % 7 for i in range(150)], 8, 1, 64, 16, "f16", "nhd"),
    ([5000, 33, 5000], [1, 30, 4], 8, 1, 40, 1, "bf16", "fused")]


@pytest.mark.gpu
@pytest.mark.parametrize("lens,news,Hq,H,D,page,kind,layout", TOGETHER)
@pytest.mark.parametrize("window,accumulate", [(0, False), (0, True), (300, True)])
def test_few_and_many_rows_together(pv, lens, news, Hq, H, D, page, kind, layout, window, accumulate):
    """Sequences of one tile of rows, of two, and of many, in one call."""
    check_attention(pv, lens, news, Hq, H, D, page, kind, 31, layout, window=window, accumulate=accumulate)


@pytest.mark.gpu
@pytest.mark.parametrize("window", [1, 2, 64, 10**9, 2**31 - 1])
def test_windows(pv, window):
    check_attention(pv, [150, 20], [70, 20], 4, 2, 64, 16, "bf16", 13, window=window, accumulate=True)
    check_attention(pv, [1500, 20], [1, 1], 4, 2, 64, 16, "bf16", 13, window=window, accumulate=True)
    check_attention(pv, [150, 20], [70, 20], 4, 2, 64, 16, "bf16", 13, causal=False, window=window)


@pytest.mark.gpu
@pytest.mark.parametrize("news", [[1], [40]])
@pytest.mark.parametrize("gain", [0.0, 1.0, 40.0])
def test_score_ranges(pv, news, gain):
    """From equal weights to one key that takes them all, with the largest one late or early."""
    check_attention(pv, [1500], news, 4, 1, 128, 16, "bf16", 14, gain=gain, accumulate=True)
    check_attention(pv, [1500], news, 4, 1, 128, 16, "f16", 15, gain=gain, scale=-0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.0, -0.25, 3.0])
@pytest.mark.parametrize("lens,news", [([900, 70], [1, 1]), ([900, 70], [100, 60]), ([300], [12])])
def test_scales(pv, lens, news, scale):
    check_attention(pv, lens, news, 4, 1, 64, 16, "bf16", 24, scale=scale, accumulate=True)


@pytest.mark.gpu
def test_rows_and_lengths_beyond_what_there_is(pv):
    """cu that names rows outside the token tensors, more new tokens than max_new, lengths beyond the table: nothing
    outside is read or written, and what is inside comes out as it should."""
    import torch
    c = Cache(pv, [300, 200], [40, 24], 2, 64, 16, "bf16", 25, garbage=False)
    q = torch.randn(64, 8, 64, device="cuda").to(torch.bfloat16)
    ref = pv.pvmvmd_paged_attention(c.pool, c.batch, q)
    guard = torch.full((64 + 64, 8, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    wild = torch.tensor([0, 40, 1 << 30], dtype=torch.int32, device="cuda")
    pv.pvmvmd_paged_attention(c.pool, pv.KvBatch(c.table, c.dlens, wild), q, out=guard[:64])
    assert torch.equal(guard[:64], ref) and (guard[64:] == 5).all()
    guard.fill_(5.0)
    pv.pvmvmd_paged_attention(c.pool, pv.KvBatch(c.table, c.dlens, c.cu, max_new=24), q, out=guard[:64])
    assert torch.equal(guard[40:64], ref[40:]) and (guard[64:] == 5).all()
    wild = torch.tensor([-70, 40, 64], dtype=torch.int32, device="cuda")
    pv.pvmvmd_paged_attention(c.pool, pv.KvBatch(c.table, c.dlens, wild), q, out=guard[:64], accumulate=True)
    assert torch.equal(guard[:64], ref) and (guard[64:] == 5).all()
    K0 = c.K.clone()
    x = torch.ones(64, 2, 64, dtype=torch.bfloat16, device="cuda")
    pv.pvmvmd_kv_append(c.pool, pv.KvBatch(c.table, c.dlens, wild), x, x)
    c.dlens.fill_(1 << 30)
    pv.pvmvmd_paged_attention(c.pool, c.batch, q, accumulate=True)
    used = torch.zeros(K0.shape[:2], dtype=torch.bool, device="cuda")
    for b, (L, n) in enumerate(((300, 40), (200, 24))):
        p, o = c.at(b)
        used[torch.from_numpy(p[L - n:]).long().cuda(), torch.from_numpy(o[L - n:]).long().cuda()] = True
    assert torch.equal(c.K[~used], K0[~used]) and (c.K[used] == 1).all()
    assert pv.pvmvmd_device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 200])
def test_rows_that_see_nothing(pv, n):
    """New tokens in front of the start of a shorter sequence, and empty sequences: 0 and -inf, mass unchanged."""
    check_attention(pv, [0, 150], [n, n if n == 1 else 190], 4, 2, 128, 16, "bf16", 16, accumulate=True)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 48])
def test_growing_scores_rescale(pv, T):
    """Scores that grow along the keys by far more than any headroom: every tile changes the maximum."""
    import torch
    L, D = 1200, 64
    c = Cache(pv, [L], [T], 1, D, 16, "bf16", 17, garbage=False)
    q = torch.ones(T, 4, D, dtype=torch.bfloat16, device="cuda")
    ramp = torch.linspace(-30, 30, L, device="cuda")
    p, o = c.at(0)
    c.K[torch.from_numpy(p).long().cuda(), torch.from_numpy(o).long().cuda(), 0] = \
        (ramp[:, None] / 8).expand(L, D).to(torch.bfloat16)
    out, z = torch.empty_like(q), torch.empty(T, 4, device="cuda")
    pv.pvmvmd_paged_attention(c.pool, c.batch, q, out=out, lse=z)
    o64, l64, _, pabs, vabs, e = attend(_host(q), c.rows(0, "K"), c.rows(0, "V"), T, D**-0.5)
    assert (np.abs(_host(z) - l64) <= e + 2.0**-20 * (1 + np.abs(l64))).all()
    assert (np.abs(_host(out) - o64) <= 2.0**-8 * np.abs(o64) + (2.0**-8 + 2 * e[..., None]) * pabs).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 40])
def test_same_bits_from_call_to_call(pv, T):
    import torch
    c, q, out, z = check_attention(pv, [5000, 333], [T, T], 8, 2, 128, 16, "bf16", 18, accumulate=True)
    c.mass.zero_()
    pv.pvmvmd_paged_attention(c.pool, c.batch, q, accumulate=True)
    m = c.mass.clone()
    for _ in range(3):
        c.mass.zero_()
        o2, z2 = torch.empty_like(out), torch.empty_like(z)
        pv.pvmvmd_paged_attention(c.pool, c.batch, q, out=o2, lse=z2, accumulate=True)
        assert torch.equal(o2, out) and torch.equal(z2, z) and torch.equal(c.mass, m)


@pytest.mark.gpu
@pytest.mark.parametrize("news", [[1, 1, 1], [70, 40, 33], [200, 3, 150], [9, 130, 1]])
@pytest.mark.parametrize("page", [16, 100, 1])
@pytest.mark.parametrize("lens", [[300, 190, 517], [2000, 1300, 900]])
def test_a_sequence_does_not_depend_on_what_is_not_its_own(pv, news, page, lens):
    """Other numbers behind the ends and in the other sequences leave one's results bit for bit as they were."""
    import torch
    c = Cache(pv, lens, news, 2, 80, page, "bf16", 33)
    q = _dev(3 * np.random.default_rng(5).standard_normal((sum(news), 8, 80)), "bf16")
    r = slice(c.cu_host[1], c.cu_host[2])
    p, o = c.at(1)
    own = torch.zeros(c.K.shape[:2], dtype=torch.bool, device="cuda")
    own[p, o] = True
    seen = []
    for fill in range(3):
        c.mass.zero_()
        out, z = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
        pv.pvmvmd_paged_attention(c.pool, c.batch, q, out=out, lse=z, accumulate=True)
        seen.append((out[r].clone(), z[r].clone(), c.mass[p, :, o].clone()))
        for x in (c.K, c.V):
            x[~own] = (torch.randn_like(x) * 10.0**fill)[~own]
        q[:r.start].mul_(-7.0)
        q[r.stop:].mul_(30.0)
    assert pv.pvmvmd_device_status() == 0
    for s in seen[1:]:
        assert all(torch.equal(x, y) for x, y in zip(s, seen[0]))


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 64])
def test_keys_that_are_not_numbers(pv, T):
    """A NaN key reaches the rows that see it, and no other row, sequence or head."""
    import torch
    c = Cache(pv, [300, 300], [T, T], 2, 64, 16, "bf16", 19, garbage=False)
    q = torch.randn(2 * T, 4, 64, device="cuda").to(torch.bfloat16)
    ref = pv.pvmvmd_paged_attention(c.pool, c.batch, q)
    at = 300 - T // 2 - 1  # seen by the later half of the new tokens
    c.K[c.tab[0, at // 16], at % 16, 0] = float("nan")
    got = pv.pvmvmd_paged_attention(c.pool, c.batch, q)
    bad = torch.zeros(2 * T, 4, dtype=torch.bool, device="cuda")
    bad[max(0, T - T // 2 - 1):T, :2] = True
    assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], ref[~bad])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 150])
def test_pages_outside_the_pool_are_not_seen(pv, T):
    import torch
    c = Cache(pv, [400], [T], 1, 64, 16, "bf16", 20)
    q = torch.randn(T, 4, 64, device="cuda").to(torch.bfloat16)
    c.table[0, 2], c.table[0, 5] = -1, 1 << 30
    out, z = torch.empty_like(q), torch.empty(T, 4, device="cuda")
    pv.pvmvmd_paged_attention(c.pool, c.batch, q, out=out, lse=z, accumulate=True)
    Kh, Vh = c.K.clone(), c.V.clone()
    seen = [j for j in range(400) if j // 16 not in (2, 5)]
    p, o = c.at(0)
    K, V = _host(Kh)[p, o], _host(Vh)[p, o]
    qh = _host(q)
    for t in range(0, T, 29):
        js = [j for j in seen if j <= 400 - T + t]
        s = K[js, 0] @ qh[t].T / 8
        w = np.exp(s - s.max(0))
        o64 = (w / w.sum(0)).T @ V[js, 0]
        assert np.abs(_host(out[t]) - o64).max() < 2.0**-8 * 2 * np.abs(V[js]).max()
        assert np.abs(_host(z[t]) - (s.max(0) + np.log(w.sum(0)))).max() < 1e-4


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 40])
def test_a_pool_beyond_32_bit_offsets(pv, T):
    """Pages more than 2^32 bytes apart."""
    import torch
    far, D, page = 1 << 31, 64, 16  # elements between the pool's two page strides
    buf = torch.empty(far + 4 * page * D, dtype=torch.bfloat16, device="cuda")
    K = buf.as_strided((2, page, 1, D), (far, D, D, 1))
    V = buf[page * D:].as_strided((2, page, 1, D), (far, D, D, 1))
    K.copy_(torch.randn(2, page, 1, D))
    V.copy_(torch.randn(2, page, 1, D))
    tab = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([32], dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    q = torch.randn(T, 2, D, device="cuda").to(torch.bfloat16)
    near = pv.KvPool(K.contiguous(), V.contiguous())
    batch = pv.KvBatch(tab, lens, cu, max_new=T)
    a = pv.pvmvmd_paged_attention(pv.KvPool(K, V), batch, q)
    assert torch.equal(a, pv.pvmvmd_paged_attention(near, batch, q))
    x = torch.ones(T, 1, D, dtype=torch.bfloat16, device="cuda")
    pv.pvmvmd_kv_append(pv.KvPool(K, V), batch, x, x)
    assert (K[1, 16 - min(T, 16):] == 1).all() and (V[1, 16 - min(T, 16):] == 1).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 40])
def test_streams_and_graphs(pv, T):
    """Another stream than torch's current one, two at once, and a captured call replayed over new contents."""
    import torch
    cases = [Cache(pv, [3000, 40], [T, T], 2, 128, 16, "bf16", 21 + i) for i in range(2)]
    qs = [torch.randn(2 * T, 8, 128, device="cuda").to(torch.bfloat16) for _ in cases]
    refs = [pv.pvmvmd_paged_attention(c.pool, c.batch, q, accumulate=True) for c, q in zip(cases, qs)]
    masses = [c.mass.clone() for c in cases]
    for c in cases:
        c.mass.copy_(torch.from_numpy(c.mass0))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [torch.empty_like(r) for r in refs]
    for _ in range(3):
        for c in cases:
            c.mass.copy_(torch.from_numpy(c.mass0))
        torch.cuda.synchronize()
        for c, q, o, s in zip(cases, qs, outs, streams):
            pv.pvmvmd_paged_attention(c.pool, c.batch, q, out=o, accumulate=True, stream=s)
        torch.cuda.synchronize()
    for o, r, c, m in zip(outs, refs, cases, masses):
        assert torch.equal(o, r) and torch.equal(c.mass, m)
    s, c, q, o = streams[0], cases[0], qs[0].clone(), outs[0]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        pv.pvmvmd_paged_attention(c.pool, c.batch, q, out=o)
    for L in (3000, 90, 1):
        c.dlens[0] = L
        q.normal_()
        g.replay()
        assert torch.equal(o, pv.pvmvmd_paged_attention(c.pool, c.batch, q))


@pytest.mark.gpu
def test_refusals_of_tensors(pv):
    import torch
    c = Cache(pv, [20], [2], 2, 64, 16, "bf16", 22)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    ok = pv.pvmvmd_paged_attention
    for bad in (q.half(), q.cpu()):
        with pytest.raises(TypeError):
            ok(c.pool, c.batch, bad)
    for bad in (q[..., :32], q.transpose(1, 2).contiguous().transpose(1, 2), q[0]):
        with pytest.raises(ValueError):
            ok(c.pool, c.batch, bad)
    with pytest.raises(ValueError):
        ok(c.pool, c.batch, q, lse=torch.empty(3, 4, device="cuda"))
    with pytest.raises(TypeError):
        ok(c.pool, c.batch, q, lse=torch.empty(2, 4, device="cuda").half())
    with pytest.raises(pv.PvmvmdError) as e:
        ok(c.pool, c.batch, q[:, :3])
    assert e.value.status == pv.PVMVMD_E_SHAPE
    with pytest.raises(pv.PvmvmdError):  # one token each: as many as sequences
        ok(c.pool, pv.KvBatch(c.table, c.dlens), q)
    with pytest.raises(pv.PvmvmdError) as e:
        ok(pv.KvPool(c.K, c.V), c.batch, q, accumulate=True)
    assert e.value.status == pv.PVMVMD_E_ARG
    with pytest.raises(TypeError):
        pv.KvPool(c.K, c.V.half())
    with pytest.raises(TypeError):
        ok(pv.KvPool(c.K.float(), c.V.float()), c.batch, q)
    with pytest.raises(ValueError):
        pv.KvPool(c.K, c.V, c.mass[:1])
    with pytest.raises(ValueError):
        pv.KvBatch(c.table.long(), c.dlens)
    with pytest.raises(ValueError):
        pv.KvBatch(c.table, c.dlens, c.cu[:1])
    x = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(TypeError):
        pv.pvmvmd_kv_append(c.pool, c.batch, x, x.float())
    with pytest.raises(ValueError):
        pv.pvmvmd_kv_append(c.pool, c.batch, x, x[:1])


# ---------------------------------------------------------------- eviction

def kept_indexes(w, L, budget, recent):
    n = min(L, budget)
    fixed = min(recent, n)
    best = sorted(range(L - fixed), key=lambda j: (np.isnan(w[j]), 0 if np.isnan(w[j]) else -w[j], j))[:n - fixed]
    return np.array(sorted(best) + list(range(L - fixed, L)), np.int64)


@pytest.mark.gpu
@pytest.mark.parametrize("lens,H,D,page,budget,recent,layout,kind", [
    ([1], 1, 8, 1, 1, 0, "nhd", "bf16"), ([700], 8, 128, 16, 512, 64, "nhd", "bf16"),
    ([5, 0, 64, 65, 200], 2, 64, 16, 64, 10, "hnd", "f16"), ([3000, 100], 2, 128, 100, 1000, 0, "fused", "bf16"),
    ([1025, 2049], 4, 80, 7, 1, 0, "nhd", "bf16"), ([300], 1, 64, 64, 50, 90, "nhd", "f16"),
    ([513, 40], 3, 40, 24, 5000, 3, "nhd", "bf16"), ([20000], 1, 64, 32, 19999, 1, "nhd", "bf16")])
@pytest.mark.parametrize("where", ["own", "copy", "new"])
@pytest.mark.parametrize("values", ["any", "ties", "odd"])
def test_evict(pv, lens, H, D, page, budget, recent, layout, kind, where, values):
    import torch
    c = Cache(pv, lens, [1] * len(lens), H, D, page, kind, 31, layout, extra=2 + len(lens) * -(-budget // page) if
              where == "new" else 2, garbage=False)
    rng = np.random.default_rng(32)
    m = c.mass0
    if values == "ties":
        m = rng.integers(0, 3, m.shape).astype(np.float32)
    elif values == "odd":
        m = rng.choice(np.array([0.0, -0.0, 1e-45, 3e38, np.inf, -np.inf, np.nan, -1.0], np.float32), m.shape)
    c.mass.copy_(torch.from_numpy(m))
    K0, V0, m0 = _host(c.K), _host(c.V), m.astype(np.float64)
    table, tab = c.table, c.tab
    new_lens = torch.full((len(lens),), -1, dtype=torch.int32, device="cuda")
    if where == "new":
        used = set(c.tab[c.tab >= 0].tolist())
        free = [p for p in range(c.K.shape[0]) if p not in used]
        w = -(-budget // page)
        tab = np.array(free[:len(lens) * w], np.int32).reshape(len(lens), w)
        table = _dev(tab, "field")
        pv.pvmvmd_kv_evict(c.pool, c.batch, budget, recent, new_lens=new_lens, new_table=table)
        assert c.dlens.tolist() == lens
    elif where == "copy":  # the same pages, under a table of its own
        pv.pvmvmd_kv_evict(c.pool, c.batch, budget, recent, new_lens=new_lens, new_table=table.clone())
    else:
        pv.pvmvmd_kv_evict(c.pool, c.batch, budget, recent)
        new_lens = c.dlens
    assert pv.pvmvmd_device_status() == 0
    assert new_lens.tolist() == [min(L, budget) for L in lens]
    Kg, Vg, mg = _host(c.K), _host(c.V), _host(c.mass)
    for b, L in enumerate(lens):
        p, o = c.at(b)
        n = min(L, budget)
        dp, do = c.at(b, n, tab)
        for h in range(H):
            idx = kept_indexes(m0[p, h, o], L, budget, recent)
            assert np.array_equal(Kg[dp, do, h], K0[p[idx], o[idx], h]), (b, h)
            assert np.array_equal(Vg[dp, do, h], V0[p[idx], o[idx], h]), (b, h)
            assert np.array_equal(mg[dp, h, do], m0[p[idx], h, o[idx]], equal_nan=True), (b, h)


@pytest.mark.gpu
def test_evict_refusals(pv):
    c = Cache(pv, [100], [1], 1, 64, 16, "bf16", 33)
    for kw in ({"budget": 0}, {"budget": 10, "recent": -1}, {"budget": 40, "new_table": c.table[:, :2]}):
        with pytest.raises(pv.PvmvmdError) as e:
            pv.pvmvmd_kv_evict(c.pool, c.batch, **kw)
        assert e.value.status == pv.PVMVMD_E_SHAPE
    with pytest.raises(pv.PvmvmdError) as e:
        pv.pvmvmd_kv_evict(pv.KvPool(c.K, c.V), c.batch, 10)
    assert e.value.status == pv.PVMVMD_E_ARG
    with pytest.raises(ValueError):
        pv.pvmvmd_kv_evict(c.pool, c.batch, 10, new_table=c.table.long())


@pytest.mark.gpu
def test_attention_after_eviction_sees_what_stayed(pv):
    """Append, attend with accumulation, evict, append at later positions, attend: as a client's generation goes."""
    import torch
    H, D, page, Hq = 2, 64, 16, 8
    table = pv.pvmvmd_rope_table(D)
    n0, budget, recent = 150, 64, 8
    width = -(-n0 // page)
    K = torch.zeros(width, page, H, D, dtype=torch.float16, device="cuda")
    V, mass = torch.zeros_like(K), torch.zeros(width, H, page, device="cuda")
    tab = torch.arange(width, dtype=torch.int32, device="cuda")[None]
    lens = torch.tensor([n0], dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, n0], dtype=torch.int32, device="cuda")
    pool = pv.KvPool(K, V, mass)
    x = torch.randn(n0 + 3, Hq + 2 * H, D, device="cuda")
    batch = pv.KvBatch(tab, lens, cu, max_new=n0)
    q = pv.pvmvmd_kv_append(pool, batch, x[:n0, Hq:Hq + H], x[:n0, Hq + H:], None, table, q=x[:n0, :Hq])
    pv.pvmvmd_paged_attention(pool, batch, q, accumulate=True)
    Kh, Vh, mh = (_host(t.reshape(width * page, H, -1) if t.dim() == 4 else t.permute(0, 2, 1).reshape(-1, H))[:n0]
                  for t in (K, V, mass))
    assert abs(mh.sum() - n0 * Hq) < 1e-3 * n0 * Hq  # every row's weights sum to one
    pv.pvmvmd_kv_evict(pool, batch, budget, recent)
    one = pv.KvBatch(tab, lens)
    keys, vals = [], []
    for h in range(H):
        idx = kept_indexes(mh[:, h].astype(np.float32), n0, budget, recent)
        keys.append(Kh[idx, h])
        vals.append(Vh[idx, h])
    for i in range(3):
        lens += 1
        t = n0 + i
        pos = torch.tensor([t], dtype=torch.int32, device="cuda")
        q = pv.pvmvmd_kv_append(pool, one, x[t:t + 1, Hq:Hq + H], x[t:t + 1, Hq + H:], pos, table, q=x[t:t + 1, :Hq])
        out = pv.pvmvmd_paged_attention(pool, one, q, accumulate=True)
        at = budget + i
        for h in range(H):
            keys[h] = np.concatenate([keys[h], _host(K[at // page, at % page, h])[None]])
            vals[h] = np.concatenate([vals[h], _host(V[at // page, at % page, h])[None]])
        o64, _, _, pabs, vabs, e = attend(_host(q), np.stack(keys, 1), np.stack(vals, 1), 1, D**-0.5)
        tol = U["f16"] * np.abs(o64) + (U["f16"] + 2 * e[..., None]) * pabs + 2.0**-24 * vabs
        assert (np.abs(_host(out) - o64) <= tol * 1.001).all()
