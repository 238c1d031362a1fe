"""The client's steps together, as examples/client_decoder.py runs them between delegated products: every step equals
its definition on what came before it, and the products are the integers' own."""
import os
import subprocess
import sys

import numpy as np
import pytest

import steps_plain as plain

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    import __graft_entry__
    __graft_entry__._load_build_module().build()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import client_decoder
    finally:
        sys.path.pop(0)
    return client_decoder


def _h(t):
    return t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _product(W, x):
    return plain.field(plain.centred(_h(x)) @ W.astype(np.int64).T)


def _weights(norm):
    return _h(norm.weight)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 9])
def test_decoder_is_its_steps(example, T):
    import torch
    model = example.Decoder(layers=2, hidden=128, heads=2, kv_heads=1, dim=64, inner=200, vocabulary=333, seed=T)
    rng = np.random.default_rng(T)
    for tokens in (rng.integers(0, 333, T), rng.integers(0, 333, 1)):
        seen = []
        token = model.step(torch.from_numpy(tokens).cuda(), seen)
        it = iter(seen)
        h = _h(next(it))
        y = None
        for l in range(2):
            x, q, k, v, after = next(it)
            if y is not None:
                h = h + y
            assert np.array_equal(_h(after), h)
            z = plain.norm(h, "rms", _weights(model.norms[2 * l]), eps=1e-5)
            assert np.array_equal(_h(x), plain.field(plain.integers(z, 32.0, 127, False)[0]))
            for name, Y in (("q", q), ("k", k), ("v", v)):
                assert np.array_equal(_h(Y), _product(model.W[l, name], x)), name
            attended, x, step, o = next(it)
            ints, s = plain.integers(_h(attended), 1.0, 127, True)
            assert np.array_equal(_h(x), plain.field(ints)) and np.array_equal(_h(step), s)
            assert np.array_equal(_h(o), _product(model.W[l, "o"], x))
            h = h + plain.read(_h(o), model.scale[l, "o"], s, None, True)
            x, step, gu, after = next(it)
            assert np.array_equal(_h(after), h)
            ints, s = plain.integers(plain.norm(h, "rms", _weights(model.norms[2 * l + 1]), eps=1e-5), 1.0, 127, True)
            assert np.array_equal(_h(x), plain.field(ints)) and np.array_equal(_h(step), s)
            assert np.array_equal(_h(gu), _product(model.W[l, "gate_up"], x))
            g, u = (plain.read(part, model.scale[l, "gate_up"], s, None, True) for part in (_h(gu)[:, :200], _h(gu)[:, 200:]))
            ints, s = plain.integers(plain.act(g, "silu") * u, 1.0, 127, True)
            x, step, down = next(it)
            assert np.array_equal(_h(x), plain.field(ints)) and np.array_equal(_h(step), s)
            assert np.array_equal(_h(down), _product(model.W[l, "down"], x))
            y = plain.read(_h(down), model.scale[l, "down"], s, None, True)
        x, step, logits, word, got, logprob = next(it)
        z = plain.norm((h + y)[-1:], "rms", _weights(model.norms[-1]), eps=1e-5)
        ints, s = plain.integers(z, 1.0, 127, True)
        assert np.array_equal(_h(x), plain.field(ints)) and np.array_equal(_h(step), s)
        assert np.array_equal(_h(logits), _product(model.W[-1, "vocabulary"], x))
        m = plain.multiplier(2.0 * model.scale[-1, "vocabulary"], s[0], 0.8)
        xs = plain.distances(plain.centred(_h(logits)[0]).astype(np.float32), m)
        want, lp = plain.sample(xs, 0.8, 50, float(np.float32(0.95)), 0.0, int(_h(word)[0]))
        assert int(got[0]) == want == int(token[0])
        assert abs(float(logprob[0]) - lp) <= 4 * 2.0**-24 * (1 + abs(lp))
        assert next(it, None) is None


@pytest.mark.gpu
def test_decoder_runs_as_a_program(example):
    cmd = [sys.executable, os.path.join(ROOT, "examples", "client_decoder.py"), "--tokens", "3", "--prompt", "7"]
    runs = [subprocess.run(cmd, capture_output=True, text=True, timeout=300) for _ in range(2)]
    assert all(r.returncode == 0 for r in runs), runs[0].stderr
    assert runs[0].stdout == runs[1].stdout and "prompt of 7" in runs[0].stdout
