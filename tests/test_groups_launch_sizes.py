"""Launches of the operators of rows that choose their weights at the sizes that the header allows: work items along a dimension of a grid are fewer than
2^32, a workgroup fits a compute unit's LDS, and every workgroup that a call needs is there; calls that would not fit are refused before anything
goes out.  The library runs in a process whose launches are written down instead of going out; no GPU."""
import json
import os
import shutil
import subprocess
import sys

import pytest

from paper_2403_20041_amd import binding, build
from test_kv4_launch_sizes import RECORDER, fits, workgroups

CALLER = r"""
import ctypes, json, sys
ctypes.CDLL(sys.argv[2], mode=ctypes.RTLD_GLOBAL)     # its definitions come before those of the library's own dependencies
L = ctypes.CDLL(sys.argv[1])
P, FAR, i64, f32, sz = ctypes.c_void_p(0x1000), ctypes.c_void_p(1 << 50), ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
for call in json.load(sys.stdin):
    g = call.get
    for name, value in g("knobs", {}).items():
        assert L.e0m4_set_knob(name.encode(), value) == 0
    if g("op") == "groups":
        rc = L.e0m4_groups(P, i64(g("rows")), i64(g("groups")), P, None)
    elif g("op") == "route":
        rc = L.e0m4_route(P, 0, i64(g("tokens")), i64(g("groups")), i64(g("groups")), g("k"), 0, 1, f32(1.0), None, P, P, P if g("plan", 1) else None, None)
    elif g("op") == "combine":
        rc = L.e0m4_combine(P, 0, i64(g("N")), P, P, i64(g("tokens")), g("k"), i64(g("groups")), None, FAR, None)
    elif g("op") == "lora":
        rc = L.e0m4_lora(P, i64(g("K")), g("dtype", 0), P, i64(g("rows")), i64(g("groups")), P, P, g("rank"), None, i64(g("N")), i64(g("K")), None, i64(0), FAR,
                         i64(g("N")), P, sz(1 << 62), None)
    else:
        rc = getattr(L, g("op"))(P, i64(g("share", 0)), P, i64(g("rows")), i64(g("groups")), P, i64(g("N")), i64(g("K")), g("group", 128), g("gated", 0), FAR, None)
    for name in g("knobs", {}):
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


def most_tiles(rows, groups, height):
    """The most tiles that rows of so many groups can make: each used group one that is not whole."""
    used = min(rows, groups)
    return used + (rows - used) // height


def test_layouts_and_routes(run):
    calls = [dict(op="groups", rows=rows, groups=groups) for rows in (0, 1, 256, 257, 1024, 1025, 70000, 1 << 24) for groups in (1, 255, 256, 1023)]
    calls += [dict(op="route", tokens=tokens, groups=groups, k=k, plan=plan) for tokens in (1, 33, 300, 1 << 20) for groups, k in ((16, 16), (60, 4), (128, 8), (256, 1), (1023, 16))
              for plan in (0, 1)]
    for call, (rc, launches) in zip(calls, run(calls)):
        assert rc == 0 and launches, call
        for launch in launches:
            fits(launch)
        entries = call["rows"] if call["op"] == "groups" else call["tokens"] * call["k"]
        assert entries <= 1024 or call.get("plan", 1) == 0 or len(launches) == 2, call


@pytest.mark.parametrize("form", range(7))
@pytest.mark.parametrize("op", ["e0m4_matmul_grouped", "e0m8_matmul_grouped", "e0m4_bf16_matmul_grouped"])
def test_products(run, op, form):
    calls = [dict(op=op, rows=rows, groups=groups, N=N, K=K, gated=gated, knobs={"grouped_form": form})
             for rows, groups in ((1, 1), (8, 1023), (3000, 7), (40000, 1023), (1 << 24, 1023)) for N, K in ((64, 128), (1536, 2048), (27392, 4096), (1 << 23, 128))
             for gated in (0, 1)]
    heights, columns = (None, 16, 16, 32, 128, 64, 128), (None, 64, 32, 64, 256, 128, 128)
    refused = 0
    for call, (rc, launches) in zip(calls, run(calls)):
        if rc == -2:
            # (no form that was built has fewer workgroups than the fourth)
            assert not launches and most_tiles(call["rows"], call["groups"], heights[form or 4]) * call["N"] // columns[form or 4] * 512 >= 1 << 32, call
            refused += 1
            continue
        assert rc == 0 and len(launches) == 1, call
        fits(launches[0])
        if form:
            out, each = (call["N"] // 2, columns[form] // 2) if call["gated"] else (call["N"], columns[form])
            assert workgroups(launches[0]) >= most_tiles(call["rows"], call["groups"], heights[form]) * -(-out // each), call
    assert refused


def test_combine_and_adapters(run):
    calls = [dict(op="combine", tokens=tokens, k=k, groups=9, N=N) for tokens, k, N in ((1, 1, 1), (1 << 20, 16, 8), (1 << 20, 16, 33), (1 << 24, 1, 64), (3, 255, 1 << 24))]
    calls += [dict(op="lora", rows=rows, groups=groups, rank=rank, N=N, K=K, dtype=dtype) for rows, groups, K in ((1, 1, 8), (1, 1023, 1 << 20), (1000, 2, 4096), (1 << 20, 1023, 512))
              for rank in (8, 16, 24, 40, 104, 128) for N in (8, 4096, 1 << 20) for dtype in (0, 1)]
    for call, (rc, launches) in zip(calls, run(calls)):
        assert rc == 0 and len(launches) == (2 if call["op"] == "lora" else 1), call
        for launch in launches:
            fits(launch)
        if call["op"] == "lora":
            assert workgroups(launches[0]) >= most_tiles(call["rows"], call["groups"], 32) and workgroups(launches[1]) >= most_tiles(call["rows"], call["groups"], 32)
    (rc, launches), = run([dict(op="combine", tokens=1 << 20, k=1, groups=9, N=1 << 24)])
    assert rc == -2 and not launches
