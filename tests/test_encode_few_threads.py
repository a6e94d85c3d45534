"""Encoding where the system gives it no threads: the calling thread does the work, and nothing ends the process."""
import os
import subprocess
import sys

import numpy as np

import native_host

CHILD = """
import resource, sys
import numpy as np
sys.path.insert(0, {tests!r})
import native_host, ctypes
lib = ctypes.CDLL({lib!r})
p, i64 = ctypes.c_void_p, ctypes.c_int64
lib.usp_test_roundtrip.argtypes = [p, i64, p, i64, i64, i64, p, p, p, p, p]
rng = np.random.default_rng(1)
W = rng.integers(0, 65536, (100, 300)).astype(np.uint16)
mask = (rng.random((100, 300)) < 0.5).astype(np.uint8)
native_host.roundtrip(lib, W[:1], mask[:1])  # everything is loaded
size = int(open("/proc/self/statm").read().split()[0]) * resource.getpagesize()
room = {room} << 20  # a thread's stack takes 8 MB
resource.setrlimit(resource.RLIMIT_AS, (size + room, size + room))
Wo, mo, nnz, _, _ = native_host.roundtrip(lib, W, mask)
assert np.array_equal(Wo, np.where(mask, W, 0)) and np.array_equal(mo, mask) and nnz == mask.sum()
print("encoded")
"""


def test_no_thread_starts(tmp_path):
    native_host.build(str(tmp_path))
    lib = os.path.join(str(tmp_path), "libusp_host_test.so")
    for room in (6, 20):  # none, and one or two of them
        child = CHILD.format(tests=os.path.dirname(os.path.abspath(__file__)), lib=lib, room=room)
        r = subprocess.run(["bash", "-c", 'ulimit -s 8192; exec "$0" -c "$1"', sys.executable, child], capture_output=True,
                           text=True, env={**os.environ, "OPENBLAS_NUM_THREADS": "1"})
        assert r.returncode == 0 and "encoded" in r.stdout, (room, r.returncode, r.stderr[-2000:])


def test_threads_and_rows(tmp_path):
    """Row counts around the number of threads."""
    lib = native_host.build(str(tmp_path))
    rng = np.random.default_rng(2)
    for blocks in (1, 2, 3, (os.cpu_count() or 1), (os.cpu_count() or 1) + 1, 70):
        W = rng.integers(0, 65536, (16 * blocks, 40)).astype(np.uint16)
        mask = (rng.random(W.shape) < 0.5).astype(np.uint8)
        Wo, mo, nnz, _, _ = native_host.roundtrip(lib, W, mask)
        assert np.array_equal(Wo, np.where(mask, W, 0)) and nnz == mask.sum()
