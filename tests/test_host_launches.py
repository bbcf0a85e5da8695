"""What the host does around a launch, in a process of its own over a stand-in for the CUDA runtime: which launches would be refused, and what has been
launched when a call ends with an error."""
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)

CALLS = """
import ctypes as C, sys
from concurrent.futures import ThreadPoolExecutor
fake, dll = C.CDLL({fake!r}, mode=C.RTLD_GLOBAL), C.CDLL({lib!r})
sys.path.insert(0, {root!r})
FAKE = 0x7F0000000000                                                  # never dereferenced
class Cache(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("layers", "num_pages", "page_tokens", "kv_heads", "head_dim")] + \\
               [("format", C.c_int32), ("layout", C.c_int32), ("max_seqs", C.c_uint32), ("max_pages", C.c_uint32)] + \\
               [("k", C.c_void_p), ("v", C.c_void_p), ("layer_stride", C.c_int64), ("page_stride", C.c_int64)] + \\
               [(n, C.c_void_p) for n in ("k_scale", "v_scale", "refs", "pages", "length", "status")]
def cache(max_seqs=512, max_pages=16):
    return Cache(2, 100, 32, 4, 128, 0, 0, max_seqs, max_pages, FAKE, FAKE, 100 * 4 * 32 * 128, 4 * 32 * 128, *[FAKE] * 6)
p, u32, size = C.c_void_p, C.c_uint32, C.c_size_t
dll.roomie_kv_workspace_bytes.restype = size
dll.roomie_kv_reorder.argtypes = [p, p, p, u32, p, size, p]
dll.roomie_kv_evict.argtypes = [p, p, u32, p, u32, u32, u32, p, p, size, p]
def reorder(n):
    c = cache()
    return dll.roomie_kv_reorder(C.byref(c), FAKE, FAKE, n, FAKE, 1 << 40, None)
def evict(max_pages):
    c = cache(max_pages=max_pages)
    return dll.roomie_kv_evict(C.byref(c), FAKE, 2, FAKE, 100, 4, 50, FAKE, FAKE, 1 << 40, None)
"""


@pytest.fixture(scope="module")
def python(tmp_path_factory):
    fake = str(tmp_path_factory.mktemp("fake") / "libfakecudart.so")
    import paper_2607_16784_b200.build as build
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    subprocess.run(["gcc", "-shared", "-fPIC", "-O1", "-I", os.path.join(cuda, "include"), os.path.join(HERE, "fake_cudart.c"), "-o", fake, "-lpthread"], check=True)
    head = CALLS.format(fake=fake, lib=build.LIB, root=ROOT)
    import torch
    runtime = os.path.join(os.path.dirname(os.path.dirname(torch.__file__)), "nvidia", "cuda_runtime", "lib")
    env = dict(os.environ, LD_PRELOAD=fake, LD_LIBRARY_PATH=runtime + os.pathsep + os.environ.get("LD_LIBRARY_PATH", ""))

    def run(body):
        got = subprocess.run([sys.executable, "-c", head + body], env=env, capture_output=True, text=True, timeout=120)
        assert got.returncode == 0, got.stdout + got.stderr
    return run


def test_two_threads_with_calls_of_different_size(python):
    """A kernel's limit of shared memory belongs to the process: a small call in one thread must not take it away from the large ones of another."""
    python("""
a, b = ThreadPoolExecutor(1), ThreadPoolExecutor(1)
for big, small, call in ((256, 130, reorder), (8192, 700, evict)):
    for _ in range(2):
        assert a.submit(call, big).result() == 0
        assert b.submit(call, small).result() == 0
    assert a.submit(call, big).result() == 0
assert fake.fake_refused() == 0 and fake.fake_launched() == 20
""")


def test_nothing_is_launched_where_the_second_kernel_cannot_be(python):
    """A plan changes the cache: it is launched when nothing that can refuse the kernel behind it is left."""
    python("""
fake.fake_attributes_fail(1)
for call in (lambda: reorder(256), lambda: reorder(3), lambda: evict(8192), lambda: evict(1)):
    assert call() == -3 and fake.fake_launched() == 0             # ROOMIE_ERR_CUDA
fake.fake_attributes_fail(0)
for n, call in enumerate((lambda: reorder(256), lambda: reorder(3), lambda: evict(8192), lambda: evict(1))):
    assert call() == 0 and fake.fake_launched() == 2 * n + 2
""")
