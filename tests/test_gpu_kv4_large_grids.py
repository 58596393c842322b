"""Launches of attention over the 4-bit cache with more places than a grid's z dimension takes: their runs along x reach every block of
the cache and every block of queries."""
import pytest

torch = pytest.importorskip("torch")

import kv4_plain as plain  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def e0m4():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' elsewhere)")
    import paper_2403_20041_amd as pkg

    pkg.lib()
    return pkg


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def test_received_weights_in_a_cache_of_many_blocks(e0m4, oracle):
    """131072 blocks of 256 rows; the queries see rows at the end."""
    gen = torch.Generator().manual_seed(1)
    dim, group, capacity, n, window = 64, 64, 1 << 25, 100, 30
    shape = e0m4.E0M4KV4Shape(1, 2, capacity, dim, group)
    cache = e0m4.e0m4_kv4_alloc(shape, DEV)
    tail = n + window
    keys, values = (torch.randn((1, tail, 2, dim), generator=gen).half() for _ in range(2))
    e0m4.e0m4_kv4_append(cache, shape, keys.to(DEV), values.to(DEV), ints(capacity - tail))
    q = torch.randn((1, n, 4, dim), generator=gen).half()
    received = torch.zeros((1, 2, capacity), device=DEV)
    out = e0m4.e0m4_kv4_attention(q.to(DEV), cache, shape, ints(capacity), window=window, weights=received)
    look = plain.seen(torch.tensor([tail]), torch.tensor([n]), n, tail, True, window, None)
    want, got, size, reach = plain.attention(q, plain.stored(keys, group, oracle), plain.stored(values, group, oracle), look)
    assert ((out.cpu().double() - want).abs() <= plain.attention_bounds(want, size, reach, dim, tail, torch.float16)).all()
    end = received[..., capacity - tail:].cpu().double()
    assert ((end - got).abs() <= plain.received_bounds(got, reach, dim, 2 * n)).all()
    assert not received[..., :capacity - tail].any()


def test_blocks_of_queries_in_chunks(e0m4, oracle):
    """32768 blocks of 128 rows of queries, three chunks each."""
    gen = torch.Generator(device=DEV).manual_seed(2)
    dim, group, rows, n, share = 64, 32, 150, 4096, 1024
    shape = e0m4.E0M4KV4Shape(1, 1, rows, dim, group)
    cache = e0m4.e0m4_kv4_alloc(shape, DEV)
    keys, values = (torch.randn((1, rows, 1, dim), generator=gen, device=DEV).half() for _ in range(2))
    e0m4.e0m4_kv4_append(cache, shape, keys, values, ints(0))
    q = torch.randn((1, n, share, dim), generator=gen, device=DEV).half()
    e0m4.e0m4_set_knob("kv4_chunk", 1)
    try:
        out = e0m4.e0m4_kv4_attention(q, cache, shape, ints(rows), causal=False)
    finally:
        e0m4.e0m4_set_knob("kv4_chunk", 0)
    k, v = (plain.stored(t.cpu(), group, oracle) for t in (keys, values))
    for tokens in (slice(0, 3), slice(1365, 1368), slice(2047, 2050), slice(n - 3, n)):
        part = q[:, tokens].cpu()
        want, _, size, reach = plain.attention(part, k, v, torch.ones((1, 3, rows), dtype=torch.bool))
        assert ((out[:, tokens].cpu().double() - want).abs() <= plain.attention_bounds(want, size, reach, dim, rows, torch.float16)).all()
    # every block is there: without chunks the same up to the order of the sums
    whole = e0m4.e0m4_kv4_attention(q, cache, shape, ints(rows), causal=False)
    assert (out - whole).abs().amax() <= 2.0 ** -8 and torch.isfinite(out).all()
