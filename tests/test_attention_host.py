"""The host side of the client's attention (csrc/attention_api.cu over launches that only
take time).  A call is several kernels that share a stream's scratch: those of two
threads' calls on one stream must not be enqueued among one another; calls on different
streams need not wait.  And nothing throws where the host's memory is at an end."""
import ctypes
import os
import shutil
import subprocess
import threading

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    out = str(tmp_path_factory.mktemp("attention") / "attention_host.so")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    subprocess.run(["g++", "-std=c++17", "-O1", "-w", "-shared", "-fPIC", "-pthread", "-Wl,-Bsymbolic", "-I",
                    os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2609_10264_gb300", "csrc"), "-I", cuda,
                    "-x", "c++", os.path.join(ROOT, "tests", "attention_host.cpp"), "-o", out], check=True)
    return ctypes.CDLL(out)


@pytest.mark.parametrize("kinds", [("attend", "attend"), ("attend", "evict"), ("evict", "evict")])
@pytest.mark.parametrize("streams", [(1, 1), (0, 0), (1, 2)])
def test_calls_on_one_stream_follow_one_another(lib, kinds, streams):
    import paper_2609_10264_gb300 as pv
    pool = pv.pvmvmd_kv_pool(4096, 8192, 4096, 1024, 64, 64, 1024, 64, 64, 4, 16, 1, 64, pv.PVMVMD_BF16)
    batch = pv.pvmvmd_kv_batch(4096, 4096, None, 4, 2, 2, 4, 0)
    for name in ("pvmvmd_paged_attention", "pvmvmd_kv_evict"):
        f = getattr(lib, name)
        f.restype, f.argtypes = pv.SIGNATURES[name]
    p, b, status = ctypes.byref(pool), ctypes.byref(batch), []

    def go(kind, s):
        if kind == "attend":
            status.append(lib.pvmvmd_paged_attention(p, b, 2, 4096, 64, 64, 1.0, 1, 0, 1, 4096, 64, 64, None, s))
        else:
            status.append(lib.pvmvmd_kv_evict(p, b, 8, 2, 4096, 4, 4, 4096, s))
    lib.host_reset()
    threads = [threading.Thread(target=go, args=(k, s)) for k, s in zip(kinds * 2, streams * 2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert status == [pv.PVMVMD_OK] * 4
    assert all(lib.host_most(s) == 1 for s in streams)
    assert lib.host_most(-1) == len(set(streams))


@pytest.mark.parametrize("what", range(4))
def test_host_memory_at_an_end(lib, what):
    """A status, not an exception, from the calls and from what they and others take scratch from."""
    import paper_2609_10264_gb300 as pv
    pool = pv.pvmvmd_kv_pool(4096, 8192, 4096, 1024, 64, 64, 1024, 64, 64, 4, 16, 1, 64, pv.PVMVMD_BF16)
    batch = pv.pvmvmd_kv_batch(4096, 4096, None, 4, 2, 2, 4, 0)
    lib.host_forget()
    expect = pv.PVMVMD_E_NOMEM if what < 2 else 2  # cudaErrorMemoryAllocation
    assert lib.host_without_memory(what, ctypes.byref(pool), ctypes.byref(batch)) == expect
