"""Results over the layout that says where they go, over weights of a sum, over an adapter's B or its sums: refused before anything is enqueued; no GPU."""
import ctypes

import pytest

from test_groups_host_api import SHAPE, WORKSPACE, L  # noqa: F401  (a fixture)

at = ctypes.c_void_p
X, PLAN, Y, MORE = 1 << 40, 1 << 41, 1 << 42, 1 << 43


def ends(begin, size, own):
    """Places of `own` bytes that touch [begin, begin + size) in 16 bytes, and such that do not."""
    return (begin, begin + size - 16, begin - own + 16), (begin + size, begin - own)


@pytest.mark.parametrize("name", ["e0m4_matmul_grouped", "e0m4_bf16_matmul_grouped", "e0m8_matmul_grouped"])
@pytest.mark.parametrize("epilogue", [0, 1])
def test_products(L, name, epilogue):  # noqa: F811
    rows, groups, N, K = 40, 5, 128, 256
    for y in ends(PLAN, L.e0m4_groups_bytes(rows, groups), rows * (N // 2 if epilogue else N) * 2)[0]:
        assert getattr(L, name)(at(X), 0, at(PLAN), rows, groups, at(MORE), N, K, 128, epilogue, at(y), None) == SHAPE


def test_combine(L):  # noqa: F811
    tokens, k, groups, N = 20, 2, 5, 128
    call = lambda out, base=None: L.e0m4_combine(at(Y), 0, N, at(MORE), at(PLAN), tokens, k, groups, base, at(out), None)  # noqa: E731
    own = tokens * N * 2
    for begin, size in ((PLAN, L.e0m4_groups_bytes(tokens * k, groups)), (MORE, tokens * k * 4), (Y, tokens * k * N * 2)):
        for out in ends(begin, size, own)[0]:
            assert call(out) == SHAPE and call(out, at(out)) == SHAPE


@pytest.mark.parametrize("wider", [0, 64])
def test_adapters(L, wider):  # noqa: F811
    rows, adapters, rank, N, K = 20, 3, 16, 128, 256
    B, ws = 1 << 44, 1 << 45
    need, out_ld = L.e0m4_lora_workspace_bytes(rows, adapters, rank, N, K), N + wider
    call = lambda out: L.e0m4_lora(at(X), K, 0, at(PLAN), rows, adapters, at(MORE), at(B), rank, None, N, K, None, 0, at(out), out_ld, at(ws), 0, None)  # noqa: E731
    own = ((rows - 1) * out_ld + N) * 2
    for begin, size in ((PLAN, L.e0m4_groups_bytes(rows, adapters)), (B, adapters * N * rank * 2), (ws, need)):
        bad, good = ends(begin, size, own)
        for out in bad:
            assert call(out) == SHAPE
        for out in good:                                # (goes on to the next check)
            assert call(out) == WORKSPACE
    assert call(X) == WORKSPACE                         # the rows of X are read before any result is written
