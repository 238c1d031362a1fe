"""The delegated attention block (examples/client_attention.py) against the same
block in 64 bits: exact integer products, rotary positions, attention over what
the cache holds, eviction by accumulated weight, and the exact product with W_o."""
import importlib.util
import os

import numpy as np
import pytest

from test_attention import attend, centred, rotate, thetas

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("client_attention", os.path.join(ROOT, "examples", "client_attention.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_block_of_a_prompt_and_single_tokens():
    import torch
    ex = _example()
    pv = ex.pv
    block = ex.AttentionBlock(hidden=192, heads=6, kv_heads=2, dim=32, budget=20, recent=4, room=64, seed=3)
    H, D, rng = block.kv_heads, block.dim, np.random.default_rng(4)
    th, pos = thetas(D, base=500000.0), 0
    evicted = 0
    for T in (19, 1, 1, 7, 1, 1, 5, 1):
        x = rng.integers(-127, 128, size=(T, block.hidden), dtype=np.int64)
        before = block.length
        y, q, out = block.step(torch.from_numpy(x).cuda())
        # q: the exact product, scaled, rotated and rounded to bf16 (2^-8), with 2^-18 of the pair for 32 bits
        exact = (x @ block.W["q"].T.astype(np.int64)).reshape(T, block.heads, D) * block.in_scale
        p = np.arange(pos, pos + T)
        pos += T
        exp = rotate(exact, p, th, False)
        mag = np.abs(exp).max(-1, keepdims=True) * 2
        qh = q.double().cpu().numpy()
        assert (np.abs(qh - exp) <= 2.0**-8 * np.abs(exp) + 2.0**-18 * mag).all()
        L = before + T
        if block.length == L:  # nothing was evicted: the cache is what the tokens attended over
            K, V = (t.double().cpu().numpy().reshape(-1, H, D)[:L] for t in (block.pool.K, block.pool.V))
            for name, got in (("k", K[before:]), ("v", V[before:])):
                new = (x @ block.W[name].T.astype(np.int64)).reshape(T, H, D) * block.in_scale
                new = rotate(new, p, th, False) if name == "k" else new
                mag = np.abs(new).max(-1, keepdims=True) * 2
                assert (np.abs(got - new) <= 2.0**-8 * np.abs(new) + 2.0**-18 * mag).all(), name
            o, _, _, pabs, _, e = attend(qh, K, V, T, D**-0.5)
            tol = 2.0**-8 * np.abs(o) + (2.0**-8 + 2 * e[..., None]) * pabs
            assert (np.abs(out.double().cpu().numpy() - o) <= tol * (1 + 2.0**-8)).all()
        else:
            evicted += 1
        # W_o's product of the rounded output, exactly
        o_int = (out.float() * block.out_scale).round().clamp(-1023, 1023).reshape(T, -1).long().cpu().numpy()
        assert np.array_equal(centred(pv.as_u32(y)), (o_int @ block.W["o"].T.astype(np.int64)).astype(np.float64))
        assert int(block.lens) == block.length == (block.budget if L > block.budget + block.recent else L)
    assert evicted >= 2
    assert pv.pvmvmd_device_status() == 0


def test_rejected_product_stops_the_client():
    import torch
    ex = _example()
    block = ex.AttentionBlock(hidden=64, heads=2, kv_heads=1, dim=32, room=32)
    server = ex.pv.pvmvmd_server_mvm_grouped
    x = torch.randint(-127, 128, (2, 64), device="cuda")
    block.step(x)

    def cheat(jobs):
        server(jobs)
        jobs[0][2][0, 0] ^= 1
    ex.pv.pvmvmd_server_mvm_grouped = cheat
    try:
        with pytest.raises(RuntimeError):
            block.step(x)
    finally:
        ex.pv.pvmvmd_server_mvm_grouped = server
