"""The client's attention where its ranges end.  Tolerances are those of test_attention.py."""
import numpy as np
import pytest

from test_attention import U, Cache, _dev, _host, check_attention, pv  # noqa: F401


def attend_there(q, K, V, there, n, scale, causal=True, window=0):
    """test_attention.attend over the keys that are there."""
    L, H, D = K.shape
    Hq = q.shape[1]
    out, lse, mass = np.zeros((n, Hq, D)), np.full((n, Hq), -np.inf), np.zeros((H, L))
    pabs, vabs, e = np.zeros((n, Hq, D)), np.zeros((n, Hq, D)), np.zeros((n, Hq))
    j = np.arange(L)
    for t in range(n):
        at = L - n + t
        see = there & (j <= at if causal else True) & (at - j < window if window else True)
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


def check_rows(kind, got, z, ref):
    """Outputs and log sums within the bounds of test_attention.py."""
    o, lse, _, pabs, vabs, e = ref
    u = U[kind]
    tol = (u * np.abs(o) + (u + 2 * e[..., None]) * pabs + (2.0**-24 * vabs if kind == "f16" else 0) + 1e-30) * (1 + u)
    assert (np.abs(got - o) <= tol).all(), np.abs(got - o).max()
    real = np.where(np.isinf(lse), 0, lse)
    assert np.where(np.isinf(lse), z == lse, np.abs(z - real) <= e + 2.0**-20 * (1 + np.abs(real))).all()


# ---------------------------------------------------------------- pages that are not there

@pytest.mark.gpu
@pytest.mark.parametrize("D,kind", [(64, "bf16"), (40, "f16"), (128, "f16"), (96, "bf16")])
@pytest.mark.parametrize("page", [16, 24, 100, 7])  # boxes of 16, 8 and 4 keys, and none
@pytest.mark.parametrize("T,L", [(150, 1500), (150, 620), (40, 2100), (1, 1500), (5, 900)])
@pytest.mark.parametrize("holes", ["first", "middle", "last", "all three"])
def test_missing_pages_in_any_tile(pv, D, kind, page, T, L, holes):
    """Keys on pages outside the pool, in the first, a middle and the last of five to seventeen tiles of 128 keys:
    they have no weight, and every other key has its own."""
    import torch
    c = Cache(pv, [L, 300], [T, T], 1, D, page, kind, 41)
    there = np.ones(L, bool)
    first, middle, last = {0}, {L // 2 // page, L // 2 // page + 1}, {(L - 1) // page}
    gone = {"first": first, "middle": middle, "last": last, "all three": first | middle | last}[holes]
    for i, p in enumerate(sorted(gone)):
        c.table[0, p] = -1 - i if i % 2 else 1 << 30
        there[p * page:(p + 1) * page] = False
    G = 4
    q = _dev(np.random.default_rng(42).standard_normal((2 * T, G, D)), kind)
    out, z = torch.full_like(q, 7.0), torch.full((2 * T, G), 7.0, device="cuda")
    pv.pvmvmd_paged_attention(c.pool, c.batch, q, out=out, lse=z, accumulate=True)
    assert pv.pvmvmd_device_status() == 0
    qh, oh, zh, mh = _host(q), _host(out), _host(z), _host(c.mass)
    touched = np.zeros(mh.shape, bool)
    for b, (n, t) in enumerate(((L, there), (300, np.ones(300, bool)))):
        r = slice(b * T, (b + 1) * T)
        ref = attend_there(qh[r], c.rows(b, "K"), c.rows(b, "V"), t, T, D**-0.5)
        check_rows(kind, oh[r], zh[r], ref)
        m, e = ref[2], ref[5]
        got, was = c.masses(b, mh), c.masses(b, c.mass0.astype(np.float64))
        assert (np.abs(got - was - m) <= m * (2 * e.max() + 2.0**-18) + 2.0**-22 * (was + m)).all()
        p, o = c.at(b)
        touched[p[t], :, o[t]] = True
    assert np.array_equal(mh[~touched], c.mass0.astype(np.float64)[~touched])


# ---------------------------------------------------------------- one sequence with fewer tokens than rows

@pytest.mark.gpu
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("T,n,known", [(40, 2, True), (40, 2, False), (300, 1, True), (300, 1, False), (40, 30, True),
                                       (40, 30, False), (40, 0, False), (9, 3, True), (9, 3, False)])
@pytest.mark.parametrize("L", [700, 90])
def test_one_sequence_of_fewer_tokens_than_rows(pv, T, n, known, L, accumulate):
    """B = 1 and n of the T rows: bounded by max_new, or by a cu that ends before T.  The n come out as they do in a
    call of n rows, and the others are left alone."""
    import torch
    H, G, D = 2, 8, 64
    c = Cache(pv, [L], [max(n, 1)], H, D, 16, "bf16", 43)
    q = _dev(np.random.default_rng(44).standard_normal((T, H * G, D)), "bf16")
    cu = torch.tensor([0, T if known else n], dtype=torch.int32, device="cuda")
    batch = pv.KvBatch(c.table, c.dlens, cu, max_new=n if known else 0)
    out, z = torch.full_like(q, 7.0), torch.full((T, H * G), 7.0, device="cuda")
    pv.pvmvmd_paged_attention(c.pool, batch, q, out=out, lse=z, accumulate=accumulate)
    assert pv.pvmvmd_device_status() == 0
    assert (out[n:] == 7).all() and (z[n:] == 7).all()
    mh = _host(c.mass)
    if n == 0:
        assert np.array_equal(mh, c.mass0.astype(np.float64))
        return
    ref = attend_there(_host(q[:n]), c.rows(0, "K"), c.rows(0, "V"), np.ones(L, bool), n, D**-0.5)
    check_rows("bf16", _host(out[:n]), _host(z[:n]), ref)
    m = ref[2] if accumulate else 0 * ref[2]
    got, was = c.masses(0, mh), c.masses(0, c.mass0.astype(np.float64))
    assert (np.abs(got - was - m) <= m * (2 * ref[5].max() + 2.0**-18) + 2.0**-22 * (was + m)).all()


# ---------------------------------------------------------------- windows

@pytest.mark.gpu
@pytest.mark.parametrize("window", [2**31 - 1, 2**31 - 3, 2**30, 40])
@pytest.mark.parametrize("lens,news", [([5, 700], [9, 1]), ([5, 1700], [20, 2]), ([0, 2100], [16, 1]), ([30], [60])])
@pytest.mark.parametrize("Hq", [1, 3])
def test_windows_over_sequences_shorter_than_their_new_tokens(pv, window, lens, news, Hq):
    """The largest windows, where the first new token lies in front of its sequence's start."""
    check_attention(pv, lens, news, Hq, 1, 64, 16, "bf16", 45, window=window, accumulate=True)
    check_attention(pv, lens, news, Hq, 1, 128, 16, "f16", 46, window=window)


# ---------------------------------------------------------------- threads

@pytest.mark.gpu
def test_threads_on_one_stream(pv):
    """Two threads attend (in parts, with weights) and evict on one stream, over caches of their own, as the scratch
    that they share grows: the same bits as one after the other."""
    import threading

    import torch
    sizes = [([3000, 40], [1, 1]), ([9000, 333, 50], [1, 2, 1]), ([700, 12000], [60, 1]), ([20000], [3])]

    def work(seed, stream):
        out, kept = [], []  # (what the stream's kernels read stays)
        for i, (lens, news) in enumerate(sizes):
            c = Cache(pv, lens, news, 2, 128, 16, "bf16", seed + i, garbage=False)
            q = _dev(np.random.default_rng(seed + 10 + i).standard_normal((sum(news), 8, 128)), "bf16")
            kept.append((c, q))
            torch.cuda.synchronize()
            for _ in range(6):
                o, z = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
                pv.pvmvmd_paged_attention(c.pool, c.batch, q, out=o, lse=z, accumulate=True, stream=stream)
                pv.pvmvmd_kv_evict(c.pool, c.batch, max(lens) - 1 if i % 2 else 10**6, 3, stream=stream)
                out += [o, z]
            out += [c.mass, c.K, c.dlens]
        stream.synchronize()
        return [x.cpu() for x in out]
    alone = [work(s, torch.cuda.Stream()) for s in (51, 71)]
    shared, got = torch.cuda.Stream(), [None, None]

    def go(i, seed):
        got[i] = work(seed, shared)
    threads = [threading.Thread(target=go, args=(i, s)) for i, s in enumerate((51, 71))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert pv.pvmvmd_device_status() == 0
    for a, b in zip(alone, got):
        assert len(a) == len(b) and all(torch.equal(x, y) for x, y in zip(a, b))


# ---------------------------------------------------------------- wide tables

@pytest.mark.gpu
@pytest.mark.parametrize("places", [1 << 14, 1 << 28])
@pytest.mark.parametrize("news", [[1] * 8, [1, 3, 2, 1, 40, 1, 2, 1]])
def test_tables_far_wider_than_what_is_cached(pv, places, news):
    """Room for up to 2^28 keys a sequence, some hundreds of them there: the call has the workspace it needs."""
    import torch
    lens = [200, 17, 333, 90, 400, 1, 64, 129]
    H, G, D, page = 8, 8, 64, 1024
    c = Cache(pv, lens, news, H, D, page, "bf16", 47)
    wide = torch.full((8, places // page), -1, dtype=torch.int32, device="cuda")
    wide[:, :c.table.shape[1]] = c.table
    batch = pv.KvBatch(wide, c.dlens, c.cu, max_new=max(news))
    q = _dev(np.random.default_rng(48).standard_normal((sum(news), H * G, D)), "bf16")
    out, z = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    pv.pvmvmd_paged_attention(c.pool, batch, q, out=out, lse=z, accumulate=True)
    assert pv.pvmvmd_device_status() == 0
    mh = _host(c.mass)
    for b, (L, n) in enumerate(zip(lens, news)):
        r = slice(c.cu_host[b], c.cu_host[b + 1])
        ref = attend_there(_host(q[r]), c.rows(b, "K"), c.rows(b, "V"), np.ones(L, bool), n, D**-0.5)
        check_rows("bf16", _host(out[r]), _host(z[r]), ref)
        got, was = c.masses(b, mh), c.masses(b, c.mass0.astype(np.float64))
        assert (np.abs(got - was - ref[2]) <= ref[2] * (2 * ref[5].max() + 2.0**-18) + 2.0**-22 * (was + ref[2])).all()


@pytest.mark.gpu
def test_a_window_bounds_the_workspace(pv):
    """Few rows with their weights under a window, over a table of 2^20 places: scores of what the window shows."""
    import torch
    L, T, W = 9000, 2, 700
    c = Cache(pv, [L, L - 5], [T, T], 2, 64, 16, "f16", 49)
    wide = torch.full((2, (1 << 20) // 16), -1, dtype=torch.int32, device="cuda")
    wide[:, :c.table.shape[1]] = c.table
    q = _dev(np.random.default_rng(50).standard_normal((2 * T, 8, 64)), "f16")
    res = []
    for table in (c.table, wide):
        c.mass.copy_(torch.from_numpy(c.mass0))
        out, z = torch.empty_like(q), torch.empty(2 * T, 8, device="cuda")
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        free = torch.cuda.mem_get_info()[0]
        pv.pvmvmd_paged_attention(c.pool, pv.KvBatch(table, c.dlens, c.cu, max_new=T), q, out=out, lse=z, window=W,
                                  accumulate=True, stream=s)
        s.synchronize()
        assert free - torch.cuda.mem_get_info()[0] < 64 << 20
        res.append((out, z, c.mass.clone()))
    assert all(torch.equal(x, y) for x, y in zip(*res))
    for b, n in enumerate((L, L - 5)):
        r = slice(b * T, (b + 1) * T)
        check_rows("f16", _host(out[r]), _host(z[r]),
                   attend_there(_host(q[r]), c.rows(b, "K"), c.rows(b, "V"), np.ones(n, bool), T, 64**-0.5, window=W))


# ---------------------------------------------------------------- many heads

@pytest.mark.gpu
@pytest.mark.parametrize("H,T", [(33000, 20), (65535, 1)])
def test_as_many_heads_as_the_header_admits(pv, H, T):
    """A window of one key: every row's output is the value of its own key, and its log sum that key's score."""
    import torch
    D, page, L = 8, 64, 1100
    pages = -(-L // page)
    K = torch.randn(pages, page, H, D, device="cuda").to(torch.bfloat16)
    V = torch.randn(pages, page, H, D, device="cuda").to(torch.bfloat16)
    pool = pv.KvPool(K, V)
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None].contiguous()
    lens = torch.tensor([L], dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    q = torch.randn(T, H, D, device="cuda").to(torch.bfloat16)
    out, z = torch.full_like(q, 7.0), torch.full((T, H), 7.0, device="cuda")
    pv.pvmvmd_paged_attention(pool, pv.KvBatch(table, lens, cu, max_new=T), q, out=out, lse=z, window=1)
    k, v = (x.view(-1, H, D)[L - T:L] for x in (K, V))
    # one key: p = 1, a value of the cache's type comes back as it is
    assert torch.equal(out, v)
    s = (q.double() * k.double()).sum(-1) * D**-0.5
    e = 2.0**-24 * (D + 16) * (q.double() * k.double()).abs().sum(-1) * D**-0.5 + 2.0**-20
    assert ((z.double() - s).abs() <= e + 2.0**-20 * (1 + s.abs())).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T,H,D,inter", [(1, 70000, 2048, False), (1, 66000, 2056, True), (2, 65600, 2048, True)])
def test_rope_of_many_wide_heads(pv, T, H, D, inter):
    import torch
    table = pv.pvmvmd_rope_table(64)
    x = torch.randn(T, H, D, device="cuda").to(torch.bfloat16)
    pos = torch.arange(5, 5 + T, dtype=torch.int32, device="cuda")
    y = pv.pvmvmd_rope(x, pos, table, interleaved=inter)
    assert torch.equal(y[..., 64:], x[..., 64:])
    few = torch.tensor([0, 1, H // 2, H - 2, H - 1], device="cuda")
    assert torch.equal(y[:, few], pv.pvmvmd_rope(x[:, few].contiguous(), pos, table, interleaved=inter))
    a = x[..., :64].float().view(T, H, 32, 2) if inter else x[..., :64].float().view(T, H, 2, 32).transpose(2, 3)
    b = y[..., :64].float().view(T, H, 32, 2) if inter else y[..., :64].float().view(T, H, 2, 32).transpose(2, 3)
    # a rotation keeps a pair's length, but for two roundings to bf16
    assert ((a.norm(dim=-1) - b.norm(dim=-1)).abs() <= 2.0**-8 * b.norm(dim=-1) + 1e-5).all()


# ---------------------------------------------------------------- the example

@pytest.mark.gpu
def test_example_refuses_tokens_beyond_its_cache(pv):
    import torch
    from test_attention_example import _example
    block = _example().AttentionBlock(hidden=64, heads=2, kv_heads=1, dim=32, budget=48, room=60, page=16)
    x = torch.randint(-127, 128, (70, 64), device="cuda")
    block.step(x[:50])
    with pytest.raises(ValueError, match="64 places"):
        block.step(x[:15])
    block.step(x[:14])
    assert block.length == int(block.lens) == 48


# ---------------------------------------------------------------- more candidates than an eviction holds in registers

@pytest.mark.gpu
@pytest.mark.parametrize("lens,H,D,page,budget,recent", [([40000, 33000], 2, 16, 64, 9000, 100),
                                                         ([32769], 1, 8, 7, 32768, 0), ([32768, 32770], 1, 8, 16, 1, 0),
                                                         ([70001, 5], 1, 8, 100, 66000, 40000)])
@pytest.mark.parametrize("where", ["own", "new"])
@pytest.mark.parametrize("values", ["any", "ties", "odd"])
def test_evict_from_long_caches(pv, lens, H, D, page, budget, recent, where, values):
    import torch
    from test_attention import kept_indexes
    need = [-(-min(budget, L) // page) for L in lens]
    c = Cache(pv, lens, [1] * len(lens), H, D, page, "bf16", 61, extra=2 + len(lens) * max(need), garbage=False)
    rng = np.random.default_rng(62)
    m = c.mass0
    if values == "ties":
        m = rng.integers(0, 3, m.shape).astype(np.float32)
    elif values == "odd":
        m = rng.choice(np.array([0.0, -0.0, 1e-45, 3e38, np.inf, -np.inf, np.nan, -1.0], np.float32), m.shape)
    c.mass.copy_(torch.from_numpy(m))
    K0, V0, m0 = _host(c.K), _host(c.V), m.astype(np.float64)
    new_lens = torch.full((len(lens),), -1, dtype=torch.int32, device="cuda")
    table, tab = c.table, c.tab
    if where == "new":
        used = set(c.tab[c.tab >= 0].tolist())
        free = [p for p in range(c.K.shape[0]) if p not in used]
        tab = np.array(free[:len(lens) * max(need)], np.int32).reshape(len(lens), max(need))
        table = _dev(tab, "field")
    pv.pvmvmd_kv_evict(c.pool, c.batch, max(min(budget, L) for L in lens), recent, new_lens=new_lens, new_table=table)
    assert pv.pvmvmd_device_status() == 0
    assert new_lens.tolist() == [min(L, budget) for L in lens]
    Kg, Vg, mg = _host(c.K), _host(c.V), _host(c.mass)
    for b, L in enumerate(lens):
        p, o = c.at(b)
        dp, do = c.at(b, min(L, budget), tab)
        for h in range(H):
            idx = kept_indexes(m0[p, h, o], L, budget, recent)
            assert np.array_equal(Kg[dp, do, h], K0[p[idx], o[idx], h]), (b, h)
            assert np.array_equal(Vg[dp, do, h], V0[p[idx], o[idx], h]), (b, h)
            assert np.array_equal(mg[dp, h, do], m0[p[idx], h, o[idx]], equal_nan=True), (b, h)


# ---------------------------------------------------------------- a captured call with weights

@pytest.mark.gpu
@pytest.mark.parametrize("news", [[1, 1], [40, 40], [2, 300]])
def test_captured_accumulation(pv, news):
    """Rows of few, of chunks and of both with their weights, replayed over new contents and lengths: the same bits as
    the calls."""
    import torch
    c = Cache(pv, [6000, 700], news, 2, 64, 16, "bf16", 63, garbage=False)
    q = _dev(np.random.default_rng(64).standard_normal((sum(news), 8, 64)), "bf16")
    out, z = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    pv.pvmvmd_paged_attention(c.pool, c.batch, q, out=out, lse=z, accumulate=True, stream=s)  # its scratch
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        pv.pvmvmd_paged_attention(c.pool, c.batch, q, out=out, lse=z, accumulate=True)
    for lens in ((6000, 700), (310, 650), (5000, 1), (0, 20)):
        c.dlens.copy_(torch.tensor(lens, dtype=torch.int32))
        q.normal_()
        c.mass.zero_()
        g.replay()
        g.replay()
        got = [out.clone(), z.clone(), c.mass.clone()]
        c.mass.zero_()
        for _ in range(2):
            o2, z2 = torch.empty_like(q), torch.empty_like(z)
            pv.pvmvmd_paged_attention(c.pool, c.batch, q, out=o2, lse=z2, accumulate=True)
        assert all(torch.equal(x, y) for x, y in zip(got, (o2, z2, c.mass)))
    assert pv.pvmvmd_device_status() == 0


# ---------------------------------------------------------------- frequencies that no double holds

def test_turns_refuse_frequencies_that_are_not_finite(pv):
    assert (pv.pvmvmd_rope_turns(128, base=1e-300) >= 0).all()
    for kw in ({"base": 5e-324}, {"base": 1e-320, "scaling": "linear", "factor": 1.0}):
        with pytest.raises(pv.PvmvmdError) as e:
            pv.pvmvmd_rope_turns(1024, **kw)
        assert e.value.status == pv.PVMVMD_E_PARAM
