"""Refusals and sizes of the operators of rows that choose their weights: nothing is enqueued, so no GPU is needed."""
import ctypes
import os

import pytest
import torch

from paper_2403_20041_amd import binding, build

P = ctypes.c_void_p(0x10000)
FAR = ctypes.c_void_p(1 << 40)
ODD = ctypes.c_void_p(0x10008)
NULL, SHAPE, GROUP, ALIGN, WORKSPACE = -1, -2, -3, -4, -5


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(binding.LIB_PATH):
        build.build_library(verbose=False)
    return binding.lib()


def test_sizes(L):
    # offsets, order and place, each in whole fours, and something behind them
    assert L.e0m4_groups_bytes(10, 5) >= 4 * (8 + 12 + 12)
    assert L.e0m4_groups_bytes(0, 1) > 0
    for rows, groups in ((-1, 4), ((1 << 24) + 1, 4), (4, 0), (4, 1024)):
        assert L.e0m4_groups_bytes(rows, groups) == 0
    assert L.e0m4_groups_bytes(1 << 24, 1023) > 2 * (1 << 26)
    assert L.e0m4_lora_workspace_bytes(0, 4, 16, 64, 64) == 0 and L.e0m4_lora_workspace_bytes(4, 4, 12, 64, 64) == 0
    assert L.e0m4_lora_workspace_bytes(5, 4, 16, 64, 64) >= 5 * 16 * 4


def test_groups_refuses(L):
    assert L.e0m4_groups(P, -1, 4, P, None) == SHAPE
    assert L.e0m4_groups(P, 4, 1024, P, None) == SHAPE
    assert L.e0m4_groups(None, 4, 4, P, None) == NULL
    assert L.e0m4_groups(P, 4, 4, None, None) == NULL
    assert L.e0m4_groups(P, 4, 4, ODD, None) == ALIGN
    assert L.e0m4_groups(ctypes.c_void_p(0x10002), 4, 4, P, None) == ALIGN


def test_route_refuses(L):
    def call(logits=P, dtype=0, tokens=4, experts=8, ld=8, k=2, scoring=0, count=None, chosen=P, weights=P, plan=P):
        return L.e0m4_route(logits, dtype, tokens, experts, ld, k, scoring, 1, 1.0, count, chosen, weights, plan, None)

    for bad in (dict(tokens=-1), dict(experts=0), dict(experts=1024), dict(k=0), dict(k=9), dict(k=17, experts=64), dict(dtype=3), dict(scoring=2),
                dict(ld=-1), dict(tokens=(1 << 23) + 1)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(logits=None), dict(chosen=None), dict(weights=None)):
        assert call(**bad) == NULL, bad
    for bad in (dict(logits=ctypes.c_void_p(0x10001)), dict(logits=ctypes.c_void_p(0x10002), dtype=2), dict(plan=ODD), dict(count=ctypes.c_void_p(0x10002))):
        assert call(**bad) == ALIGN, bad
    assert call(tokens=0, plan=None, logits=None, chosen=None, weights=None) == 0


@pytest.mark.parametrize("name,groups", [("e0m4_matmul_grouped", (32, 64, 128)), ("e0m4_bf16_matmul_grouped", (32, 64, 128)), ("e0m8_matmul_grouped", (64, 128))])
def test_products_refuse(L, name, groups):
    def call(X=P, share=0, plan=P, rows=8, number=4, codes=P, N=128, K=256, group=128, epilogue=0, Y=FAR):
        return getattr(L, name)(X, share, plan, rows, number, codes, N, K, group, epilogue, Y, None)

    for bad in (dict(rows=-1), dict(rows=(1 << 24) + 1), dict(number=0), dict(number=1024), dict(share=-1), dict(share=256, rows=512), dict(share=3),
                dict(N=-1), dict(N=(1 << 24) + 1), dict(K=0), dict(K=144), dict(K=1 << 21), dict(epilogue=2), dict(epilogue=1, N=96),
                dict(epilogue=1, N=1 << 24, K=1 << 15), dict(share=2, rows=1 << 20, K=1 << 11)):
        assert call(**bad) == SHAPE, bad
    for group in (0, 16, 32, 64, 128, 256):
        if group not in groups:
            assert call(group=group) == GROUP
    for bad in (dict(X=None), dict(plan=None), dict(codes=None), dict(Y=None)):
        assert call(**bad) == NULL, bad
    for bad in (dict(X=ODD), dict(plan=ODD), dict(codes=ODD), dict(Y=ODD)):
        assert call(**bad) == ALIGN, bad
    assert call(rows=0, X=None, Y=None) == 0 and call(N=0) == 0


@pytest.mark.parametrize("name", ["e0m4_matmul_grouped", "e0m4_bf16_matmul_grouped", "e0m8_matmul_grouped"])
@pytest.mark.parametrize("share,epilogue", [(0, 0), (2, 0), (0, 1)])
def test_products_refuse_results_over_their_rows(L, name, share, epilogue):
    rows, N, K, far = 8, 128, 256, 1 << 40
    x_bytes, y_bytes = (rows // share if share else rows) * K * 2, rows * (N // 2 if epilogue else N) * 2
    for y in (far, far + x_bytes - 16, far - y_bytes + 16):
        assert getattr(L, name)(ctypes.c_void_p(far), share, P, rows, 4, P, N, K, 128, epilogue, ctypes.c_void_p(y), None) == SHAPE, y - far


def test_combine_refuses(L):
    def call(Y=P, dtype=0, N=64, weights=P, plan=P, tokens=4, k=2, groups=8, base=None, out=FAR):
        return L.e0m4_combine(Y, dtype, N, weights, plan, tokens, k, groups, base, out, None)

    far = 1 << 40
    for bad in (dict(dtype=2), dict(N=-1), dict(tokens=-1), dict(k=0), dict(k=256), dict(tokens=1 << 24), dict(groups=0), dict(groups=1024),
                dict(out=ctypes.c_void_p(0x10000 + 16)), dict(base=ctypes.c_void_p(far + 16)), dict(base=ctypes.c_void_p(far - 16))):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(Y=None), dict(weights=None), dict(plan=None), dict(out=None)):
        assert call(**bad) == NULL, bad
    for bad in (dict(Y=ODD), dict(plan=ODD), dict(base=ctypes.c_void_p(far + 8)), dict(out=ctypes.c_void_p(far + 8)), dict(weights=ctypes.c_void_p(0x10002))):
        assert call(**bad) == ALIGN, bad
    assert call(tokens=0, Y=None, out=None) == 0 and call(N=0) == 0


def test_lora_refuses(L):
    def call(X=P, x_ld=256, dtype=0, plan=P, rows=4, adapters=3, A=P, B=P, rank=16, factors=None, N=128, K=256, base=None, base_ld=128, out=FAR, out_ld=128,
             ws=P, ws_bytes=1 << 30):
        return L.e0m4_lora(X, x_ld, dtype, plan, rows, adapters, A, B, rank, factors, N, K, base, base_ld, out, out_ld, ws, ws_bytes, None)

    for bad in (dict(dtype=2), dict(rows=-1), dict(adapters=0), dict(adapters=1024), dict(rank=0), dict(rank=12), dict(rank=136), dict(N=100), dict(N=-8),
                dict(K=0), dict(K=252), dict(x_ld=248), dict(out_ld=120), dict(base=FAR, base_ld=120), dict(base=FAR, base_ld=136, out=FAR),
                dict(rows=1 << 23, x_ld=256), dict(rank=128, N=1 << 23, out_ld=1 << 23)):
        assert call(**bad) == SHAPE, bad
    for bad in (dict(X=None), dict(plan=None), dict(A=None), dict(B=None), dict(out=None), dict(ws=None)):
        assert call(**bad) == NULL, bad
    for bad in (dict(X=ODD), dict(A=ODD), dict(B=ODD), dict(plan=ODD), dict(ws=ODD), dict(x_ld=260), dict(out_ld=132), dict(base=P, base_ld=132),
                dict(factors=ctypes.c_void_p(0x10002))):
        assert call(**bad) == ALIGN, bad
    assert call(ws_bytes=L.e0m4_lora_workspace_bytes(4, 3, 16, 128, 256) - 1) == WORKSPACE
    # results over other rows or columns of base; columns beside each other go on to the next check
    few = dict(ws_bytes=0)
    at = lambda columns: ctypes.c_void_p((1 << 40) + 2 * columns)  # noqa: E731
    for bad in (dict(base=at(8)), dict(base=at(128)), dict(base=at(-8)), dict(base=at(3 * 128 + 120)), dict(base=at(120), base_ld=256, out_ld=256),
                dict(base=at(136), base_ld=256, out_ld=256), dict(base=at(256), base_ld=256, out_ld=256), dict(base=at(128), base_ld=256, out_ld=264)):
        assert call(**bad, **few) == SHAPE, bad
    for good in (dict(base=at(128), base_ld=256, out_ld=256), dict(base=at(-128), base_ld=256, out_ld=256), dict(base=at(4 * 128)), dict(base=at(-4 * 128)),
                 dict(base=at(0)), dict(base=at(128), base_ld=264, out_ld=264)):
        assert call(**good, **few) == WORKSPACE, good
    assert call(rows=0, X=None, ws=None) == 0 and call(N=0) == 0


def test_python_refuses_other_tensors(L):
    """Argument checks of the binding; host tensors are refused before anything looks at a device."""
    plan = binding.E0M4Groups(torch.zeros(1000, dtype=torch.int32), 8, 4)
    x, codes = torch.zeros((8, 256), dtype=torch.float16), torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(ValueError):
        binding.e0m4_matmul_grouped(x, plan, codes, 128, 256, 128)
    with pytest.raises(ValueError):
        binding.e0m4_groups(torch.zeros(8, dtype=torch.int64), 4)
    with pytest.raises(ValueError):
        binding.e0m4_groups(torch.zeros(8, dtype=torch.int32), 4)
    with pytest.raises(TypeError):
        binding.e0m4_route(torch.zeros((4, 8), dtype=torch.float64), 2)
    with pytest.raises(ValueError):
        binding.e0m4_route(torch.zeros((4, 8)), 2)
    with pytest.raises(TypeError):
        binding.e0m4_combine(torch.zeros((8, 64)), torch.zeros((4, 2)), plan)
    with pytest.raises(TypeError):
        binding.e0m4_lora(torch.zeros((4, 64)), plan, torch.zeros((3, 8, 64)), torch.zeros((3, 64, 8)))
    with pytest.raises(ValueError):
        binding.e0m4_groups_alloc(8, 2000, "cpu")
