"""Checks of the entry points around the key/value cache in E0M4 codes that need no GPU: sizes, and every refusal before anything could
be launched."""
import ctypes
import os

import pytest

from paper_2403_20041_amd import binding, build


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(binding.LIB_PATH):
        build.build_library(verbose=False)
    return binding.lib()


P = 0x1000          # an address that is never used
Shape = binding._KV4Shape


def rows(data=P, batch_ld=0, row_ld=0, head_ld=0):
    return binding._KV4Rows(data, batch_ld, row_ld, head_ld)


def test_sizes(L):
    size = lambda *s: L.e0m4_kv4_bytes(Shape(*s))  # noqa: E731
    for dim in (64, 128, 256):
        for group in (32, 64, 128):
            want = 0 if group > dim else 32 * (dim + 8 * dim // group)           # codes, scales and biases of 32 rows of keys and values
            assert size(1, 1, 1, dim, group) == want
            assert size(3, 5, 65, dim, group) == 3 * 5 * 3 * want
    assert size(0, 1, 1, 64, 64) == size(1, 0, 1, 64, 64) == size(1, 1, 0, 64, 64) == 0
    for bad in ((-1, 1, 1, 64, 64), (1, -1, 1, 64, 64), (1, 1, -1, 64, 64), (1, 1, 1, 96, 32), (1, 1, 1, 64, 48), (1, 1, 1, 64, 128),
                (65536, 1, 1, 64, 64), (1, 65536, 1, 64, 64), (1, 1, (1 << 26) + 1, 64, 64), (65535, 65535, 1 << 26, 64, 64)):
        assert size(*bad) == 0, bad
    assert size(1, 1, 1 << 26, 256, 32) == (1 << 21) * 32 * (256 + 64)


def test_workspace(L):
    ws = lambda s, *a: L.e0m4_kv4_attention_workspace_bytes(Shape(*s), *a)  # noqa: E731
    ok = (2, 4, 5000, 128, 128)
    assert ws(ok, 8, 1, 1) >= ws(ok, 8, 1, 0) >= 0
    assert ws(ok, 8, 0, 1) == 0 and ws((0, 4, 5000, 128, 128), 8, 1, 1) == 0 and ws((2, 4, 0, 128, 128), 8, 1, 1) == 0
    for heads, n in ((7, 1), (0, 1), (-4, 1), (8, -1), (8, (1 << 20) + 1), (4 * 1025, 1), (4096, 1 << 20)):
        assert ws(ok, heads, n, 1) == 0, (heads, n)
    assert ws((2, 4, 5000, 128, 100), 8, 1, 1) == 0


BAD_SHAPES = [((-1, 1, 8, 64, 64), -2), ((1, 1, 8, 80, 16), -2), ((1, 1, 8, 64, 16), -3), ((1, 1, 8, 64, 128), -3),
              ((1 << 20, 1, 8, 64, 64), -2), ((1, 1, 1 << 27, 64, 64), -2)]


def test_append_refusals(L):
    s = Shape(2, 2, 64, 64, 64)
    call = lambda cache=P, shape=s, k=rows(), v=rows(), dtype=0, n=1, starts=P, counts=None: \
        L.e0m4_kv4_append(cache, shape, k, v, dtype, n, starts, counts, None)  # noqa: E731
    for bad, code in BAD_SHAPES:
        assert call(shape=Shape(*bad)) == code
    assert call(shape=None) == -1 and call(cache=None) == -1 and call(starts=None) == -1 and call(k=None) == -1
    assert call(v=rows(data=None)) == -1
    assert call(dtype=2) == -2 and call(n=-1) == -2 and call(n=(1 << 26) + 1) == -2
    assert call(cache=P + 8) == -4 and call(k=rows(P + 2)) == -4 and call(v=rows(row_ld=4)) == -4 and call(k=rows(head_ld=-1)) == -4
    assert call(starts=P + 1) == -4 and call(counts=P + 2) == -4
    assert call(n=0, k=None, cache=None) == 0 and call(shape=Shape(0, 2, 64, 64, 64), cache=None) == 0


def test_read_refusals(L):
    s = Shape(2, 2, 64, 64, 64)
    call = lambda cache=P, shape=s, lengths=P, first=None, n=1, k=P, v=P: L.e0m4_kv4_read(cache, shape, lengths, first, n, k, v, None)  # noqa: E731
    for bad, code in BAD_SHAPES:
        assert call(shape=Shape(*bad)) == code
    assert call(n=-1) == -2 and call(n=(1 << 26) + 1) == -2
    assert call(cache=None) == -1 and call(lengths=None) == -1 and call(k=None) == -1 and call(v=None) == -1
    assert call(cache=P + 4) == -4 and call(lengths=P + 2) == -4 and call(first=P + 1) == -4 and call(k=P + 8) == -4 and call(v=P + 2) == -4
    assert call(n=0, k=None) == 0


def test_attention_refusals(L):
    s = Shape(2, 2, 5000, 64, 64)

    def call(q=rows(), dtype=0, heads=4, n=1, cache=P, shape=s, lengths=P, counts=None, causal=1, window=0, mask=None, weights=None, out=P,
             ws=P, ws_bytes=1 << 40):
        return L.e0m4_kv4_attention(q, dtype, heads, n, cache, shape, lengths, counts, causal, window, mask, weights, out, ws, ws_bytes, None)

    for bad, code in BAD_SHAPES:
        assert call(shape=Shape(*bad)) == code
    for heads, n in ((3, 1), (0, 1), (-2, 1), (2 * 1025, 1), (4, -1), (4, (1 << 20) + 1)):
        assert call(heads=heads, n=n) == -2, (heads, n)
    assert call(dtype=-1) == -2 and call(window=-1) == -2 and call(window=5, causal=0) == -2
    assert call(mask=binding._KV4Mask(P, 0, 0, -1)) == -2
    assert call(q=None) == -1 and call(cache=None) == -1 and call(lengths=None) == -1 and call(out=None) == -1
    assert call(mask=binding._KV4Mask(None, 0, 0, 9)) == -1
    assert call(q=rows(P + 8)) == -4 and call(q=rows(batch_ld=3)) == -4 and call(cache=P + 8) == -4 and call(out=P + 8) == -4
    assert call(lengths=P + 2) == -4 and call(counts=P + 2) == -4 and call(weights=P + 2) == -4
    need = L.e0m4_kv4_attention_workspace_bytes(s, 4, 1, 1)
    assert need > 0
    assert call(weights=P, ws_bytes=need - 1) == -5 and call(weights=P, ws=None) == -1 and call(weights=P, ws=P + 8) == -4
    assert call(n=0, q=None, out=None) == 0 and call(shape=Shape(0, 2, 64, 64, 64), out=None) == 0


def test_evict_refusals(L):
    s, o, far = Shape(2, 2, 64, 64, 64), Shape(2, 2, 40, 64, 64), 0x10000000

    def call(cache=P, shape=s, received=P, lengths=P, budget=40, recent=8, small=far, small_shape=o, kept=P, lengths_out=P, received_out=P):
        return L.e0m4_kv4_evict(cache, shape, received, lengths, budget, recent, small, small_shape, kept, lengths_out, received_out, None)

    for bad, code in BAD_SHAPES:
        assert call(shape=Shape(*bad)) == code and call(small_shape=Shape(*bad)) == code
    for other in ((1, 2, 40, 64, 64), (2, 1, 40, 64, 64), (2, 2, 40, 128, 64), (2, 2, 40, 64, 32)):
        assert call(small_shape=Shape(*other)) == -2
    assert call(budget=0) == -2 and call(budget=41) == -2 and call(recent=-1) == -2 and call(recent=41) == -2
    for name in ("cache", "received", "lengths", "small", "kept", "lengths_out", "received_out"):
        assert call(**{name: None}) == -1, name
        assert call(**{name: P + 2}) == -4, name
    assert call(small=P) == -2 and call(small=P + 16) == -2                    # rows would be overwritten while they are read
    assert call(small=P + L.e0m4_kv4_bytes(s), small_shape=Shape(2, 2, 10, 64, 64), budget=11) == -2
    assert call(shape=Shape(0, 2, 64, 64, 64), small_shape=Shape(0, 2, 40, 64, 64), small=None) == 0


def test_python_arguments():
    torch = pytest.importorskip("torch")
    import paper_2403_20041_amd as e0m4

    shape = e0m4.E0M4KV4Shape(1, 2, 64, 64, 64)
    with pytest.raises(ValueError):
        e0m4.e0m4_kv4_alloc(shape._replace(dim=96), "cpu")
    cache = e0m4.e0m4_kv4_alloc(shape, "cpu")
    assert cache.numel() == e0m4.e0m4_kv4_bytes(shape)
    x, zero = torch.zeros((1, 3, 2, 64), dtype=torch.float16), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):                                            # not on the GPU
        e0m4.e0m4_kv4_append(cache, shape, x, x, zero)
    with pytest.raises(TypeError):
        e0m4.e0m4_kv4_append(cache, shape, x.float(), x.float(), zero)
    with pytest.raises(ValueError):
        e0m4.e0m4_kv4_attention(x, cache, shape, zero)
    with pytest.raises(TypeError):
        e0m4.e0m4_kv4_attention(x.double(), cache, shape, zero)
    with pytest.raises(ValueError):
        e0m4.e0m4_kv4_read(cache, shape, zero, 3)
    with pytest.raises(ValueError):
        e0m4.e0m4_kv4_evict(cache, shape, torch.zeros((1, 2, 64)), zero, 8, 2, cache, shape)


def test_the_largest_caches(L):
    size = lambda *s: L.e0m4_kv4_bytes(Shape(*s))  # noqa: E731
    assert size(4096, 4096, 1, 64, 64) == (1 << 24) * 32 * 72 and size(4097, 4096, 1, 64, 64) == 0
    assert size(64, 64, 1 << 26, 64, 64) == (1 << 12) * (1 << 21) * 32 * 72 and size(64, 65, 1 << 26, 64, 64) == 0
