"""The binding's native module (csrc/calls.c) between two threads: each call has the
rows of its own tensors, also where both name one batch."""
import ctypes
import os
import subprocess
import threading

import pytest

from test_attention import Fake, pv  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def calls(pv, tmp_path):
    """The module over the stub library, and the stub."""
    import torch
    out = str(tmp_path / "calls_stub.so")
    subprocess.run(["gcc", "-std=gnu11", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "tests", "calls_stub.c"), "-o", out], check=True)
    stub, native = ctypes.CDLL(out), pv._open_calls()
    native.open(stub._handle, torch.bfloat16, torch.float16, torch.float32, torch.int32, None, lambda: 0, None)
    yield native, stub
    pv._open_calls()


@pytest.mark.parametrize("call", ["attend", "append"])
def test_two_threads_with_one_batch(pv, calls, call):
    import torch
    native, stub = calls
    pool = pv.pvmvmd_kv_pool(16, 16, None, 1024, 128, 64, 1024, 128, 64, 4, 8, 2, 64, pv.PVMVMD_BF16)
    batch = pv.pvmvmd_kv_batch(16, 16, 16, 4, 1, 1, 4, 0)
    p, b = ctypes.addressof(pool), ctypes.addressof(batch)
    got = {}

    def go(T):
        q, k = Fake((T, 4, 64), torch.bfloat16), Fake((T, 2, 64), torch.bfloat16)
        got[T] = native.attend(p, b, q, q, None, None, True, 0, False, 0) if call == "attend" else \
            native.append(p, b, 0, None, 1.0, k, k, None, None, 0)
    for _ in range(3):
        stub.stub_reset()
        threads = [threading.Thread(target=go, args=(T,)) for T in (3, 70)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert got == {3: 3, 70: 70}
