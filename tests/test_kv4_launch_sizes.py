"""Launches of the calls around the 4-bit cache at the sizes that the header allows: work items along a dimension of a grid are fewer than
2^32 (grids of more are refused, and what went out before stays), y and z are at most 65535, and every workgroup that a call needs is
there.  The library runs in a process whose launches are written down instead of going out; no GPU."""
import json
import os
import shutil
import subprocess
import sys

import pytest

from paper_2403_20041_amd import binding, build

RECORDER = r"""
#include <cstddef>
#include <cstdio>
struct Dim { unsigned x, y, z; };
static Dim grid, block;
static size_t shared;
static void* stream;
extern "C" {
unsigned __hipPushCallConfiguration(Dim g, Dim b, size_t s, void* q) { grid = g; block = b; shared = s; stream = q; return 0; }
int __hipPopCallConfiguration(Dim* g, Dim* b, size_t* s, void** q) { *g = grid; *b = block; *s = shared; *q = stream; return 0; }
int hipLaunchKernel(const void*, Dim g, Dim b, void**, size_t s, void*)
{
    std::printf("launch %u %u %u %u %u %u %zu\n", g.x, g.y, g.z, b.x, b.y, b.z, s);
    std::fflush(stdout);
    return 0;
}
int hipGetLastError() { return 0; }
int hipGetDevice(int* d) { *d = 0; return 0; }
int hipFuncSetAttribute(const void*, int, int) { return 0; }
}
"""

CALLER = r"""
import ctypes, json, sys
class Shape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("kv_heads", ctypes.c_int64), ("capacity", ctypes.c_int64), ("dim", ctypes.c_int), ("group", ctypes.c_int)]
class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_ld", ctypes.c_int64), ("row_ld", ctypes.c_int64), ("head_ld", ctypes.c_int64)]
ctypes.CDLL(sys.argv[2], mode=ctypes.RTLD_GLOBAL)     # its definitions come before those of the library's own dependencies
L = ctypes.CDLL(sys.argv[1])
P, FAR, i64, vp, sz = ctypes.c_void_p(0x1000), ctypes.c_void_p(1 << 50), ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t
rows = ctypes.byref(Rows(0x1000, 0, 0, 0))
for call in json.load(sys.stdin):
    s = Shape(*call["shape"])
    for name, value in call.get("knobs", {}).items():
        assert L.e0m4_set_knob(name.encode(), value) == 0
    if call["op"] == "attention":
        rc = L.e0m4_kv4_attention(rows, 0, i64(call["heads"]), i64(call["n"]), P, ctypes.byref(s), P, None, 1, i64(call.get("window", 0)), None,
                                  P if call["weights"] else None, P, P, sz(1 << 62), None)
    elif call["op"] == "append":
        rc = L.e0m4_kv4_append(P, ctypes.byref(s), rows, rows, 0, i64(call["n"]), P, None, None)
    elif call["op"] == "read":
        rc = L.e0m4_kv4_read(P, ctypes.byref(s), P, P, i64(call["n"]), P, P, None)
    else:
        rc = L.e0m4_kv4_evict(P, ctypes.byref(s), P, P, i64(call["n"]), i64(0), FAR, ctypes.byref(s), P, P, P, None)
    for name in call.get("knobs", {}):
        L.e0m4_set_knob(name.encode(), 0)
    print("done", rc, flush=True)
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    """Calls -> [(return code, [(grid, block, bytes of LDS)])]."""
    compiler = shutil.which("g++")
    if compiler is None:
        pytest.skip("needs g++")
    if not os.path.exists(binding.LIB_PATH):
        build.build_library(verbose=False)
    folder = tmp_path_factory.mktemp("launches")
    (folder / "recorder.cpp").write_text(RECORDER)
    (folder / "caller.py").write_text(CALLER)
    library = str(folder / "recorder.so")
    subprocess.run([compiler, "-shared", "-fPIC", "-O1", "-o", library, str(folder / "recorder.cpp")], check=True)

    def go(calls):
        text = subprocess.run([sys.executable, str(folder / "caller.py"), binding.LIB_PATH, library], input=json.dumps(calls), check=True, timeout=120,
                              stdout=subprocess.PIPE, universal_newlines=True).stdout
        out, launches = [], []
        for line in text.splitlines():
            word, *numbers = line.split()
            numbers = [int(n) for n in numbers]
            if word == "launch":
                launches.append((tuple(numbers[:3]), tuple(numbers[3:6]), numbers[6]))
            elif word == "done":
                out.append((numbers[0], launches))
                launches = []
        assert len(out) == len(calls)
        return out

    return go


def workgroups(launch):
    return launch[0][0] * launch[0][1] * launch[0][2]


def fits(launch):
    grid, block, lds = launch
    assert all(1 <= g and g * b < 1 << 32 for g, b in zip(grid, block)), launch
    assert grid[1] <= 65535 and grid[2] <= 65535 and block[0] * block[1] * block[2] <= 1024 and lds <= 160 * 1024, launch


def attention(shape, heads, n, weights=True, **more):
    return dict(op="attention", shape=shape, heads=heads, n=n, weights=weights, **more)


LARGE = [
    attention((32, 1, 1 << 26, 64, 64), 32, 1), attention((32, 1, 1 << 26, 64, 64), 4, 100), attention((32, 1, 1 << 26, 64, 64), 8, 1),
    attention((1, 32, 1 << 26, 64, 64), 1024, 3), attention((64, 64, 1 << 26, 64, 64), 64, 300), attention((64, 64, 1 << 26, 64, 64), 64, 300, False),
    attention((4096, 4096, 1, 64, 64), 4096, 17), attention((4096, 4096, 1, 64, 64), 4096, 200), attention((4096, 4096, 3000, 64, 64), 4096, 80),
    attention((65535, 256, 1, 64, 64), 256, 100), attention((256, 65535, 1, 256, 32), 65535, 100), attention((1, 65535, 1 << 22, 64, 64), 65535, 100),
    attention((1, 1, 1 << 26, 128, 128), 1, 1 << 20), attention((1, 1, 1 << 26, 128, 128), 1024, 4096), attention((1, 4, 1 << 26, 256, 128), 4096, 4096),
    attention((4, 256, 1 << 26, 64, 32), 256 * 1024, 4096), attention((65535, 256, 16384, 64, 64), 256, 100, window=4000),
]


def test_attention(run):
    for call, (rc, launches) in zip(LARGE, run(LARGE)):
        assert rc == 0, call
        for launch in launches:
            fits(launch)
        batch, kv, capacity = call["shape"][:3]
        rows = call["heads"] // kv * call["n"]
        # the attention itself has a workgroup at least for each 256 rows of queries of a head
        assert workgroups(launches[0]) >= batch * kv * ((rows + 255) // 256), call
        if call["weights"] and rows > 16:                                  # ... and the received weights one for each 256 rows of the cache
            assert workgroups(launches[-1]) >= batch * kv * ((capacity + 255) // 256), call


def test_attention_with_kernels_and_chunks_of_choice(run):
    calls = [dict(call, knobs={"kv4_attention": kernel, "kv4_chunk": chunk}) for call in LARGE for kernel in (1, 2, 3) for chunk in (0, 1, 100)]
    refused = 0
    for call, (rc, launches) in zip(calls, run(calls)):
        if rc == -2:                                                       # (tiles of 16 rows of queries times forced chunks)
            assert call["knobs"]["kv4_attention"] == 1 and call["knobs"]["kv4_chunk"] and not launches, call
            refused += 1
            continue
        assert rc == 0 and launches, call
        for launch in launches:
            fits(launch)
    assert refused


def test_zeros_for_a_cache_without_rows(run):
    calls = [attention((4096, 64, 0, 256, 32), 65536, 16), attention((1, 1, 0, 64, 64), 1, 1), attention((2, 2, 0, 64, 64), 8, 1000)]
    for call, (rc, launches) in zip(calls, run(calls)):
        assert rc == 0 and len(launches) == 1, call
        fits(launches[0])


def test_append_read_evict(run):
    calls = [dict(op=op, shape=shape, n=shape[2]) for op in ("append", "read", "evict")
             for shape in ((64, 64, 1 << 26, 64, 64), (65535, 256, 5, 128, 64), (256, 65535, 5, 256, 128), (1, 65535, 1 << 22, 64, 32))]
    for call, (rc, launches) in zip(calls, run(calls)):
        assert rc == 0 and len(launches) == (2 if call["op"] == "evict" else 1), call
        for launch in launches:
            fits(launch)
