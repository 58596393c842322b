"""The key/value cache in E0M4 codes on the GPU: append and read bit for bit against the oracle, attention and the received weights
against the plain form in 64 bits on the same stored values, eviction exactly.  Caches start as bytes of 255 (parameters that are
not numbers), so that a row that was never written shows wherever it is used."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import kv4_plain as plain  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
SHAPES = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128), (256, 32), (256, 64), (256, 128)]


@pytest.fixture(scope="module")
def e0m4():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' elsewhere)")
    import paper_2403_20041_amd as pkg

    pkg.lib()
    return pkg


@pytest.fixture(params=["chosen", "few", "many", "wide"])
def kernels(request, e0m4):
    """The kernel that the library chooses, and each of them on everything."""
    e0m4.e0m4_set_knob("kv4_attention", {"chosen": 0, "few": 1, "many": 2, "wide": 3}[request.param])
    yield request.param
    e0m4.e0m4_set_knob("kv4_attention", 0)


def dirty(e0m4, shape):
    return e0m4.e0m4_kv4_alloc(shape, DEV).fill_(255)


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def rows_of(gen, shape, dtype):
    x = torch.randn(shape, generator=gen)
    x[..., ::7] *= 5
    return x.to(dtype)


def same_bits(a, b):
    return np.array_equal(a.contiguous().view(torch.int16).cpu().numpy(), b.contiguous().view(torch.int16).cpu().numpy())


# ---- append, read ---------------------------------------------------------------------------------


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_appended_rows_read_back_as_the_oracle_has_them(e0m4, oracle, dim, group, dtype):
    gen = torch.Generator().manual_seed(dim + group)
    shape = e0m4.E0M4KV4Shape(3, 2, 100, dim, group)
    cache = dirty(e0m4, shape)
    held = torch.zeros((3, 100, 2, dim), dtype=torch.float16), torch.zeros((3, 100, 2, dim), dtype=torch.float16)
    length = [0, 0, 0]
    # prompts of different lengths, single tokens over a tile's end, a part that starts inside a tile, rows written again
    for starts, counts in (([0, 0, 0], [31, 1, 40]), ([31, 1, 40], [1, 1, 1]), ([32, 2, 41], [1, 0, 1]), ([33, 2, 42], [67, 33, 5]),
                           ([5, 7, 0], [3, 20, 47])):
        n = max(counts)
        k, v = rows_of(gen, (3, n, 2, dim), dtype), rows_of(gen, (3, n, 2, dim), dtype)
        e0m4.e0m4_kv4_append(cache, shape, k.to(DEV), v.to(DEV), ints(*starts), counts=ints(*counts))
        for b in range(3):
            for into, rows in zip(held, (k, v)):
                into[b, starts[b]:starts[b] + counts[b]] = plain.stored(rows[b, :counts[b]], group, oracle)
            length[b] = max(length[b], starts[b] + counts[b])
    got = e0m4.e0m4_kv4_read(cache, shape, ints(*length), 100)
    for g, h in zip(got, held):
        for b in range(3):
            h[b, length[b]:] = 0
        assert same_bits(g, h)
    part = e0m4.e0m4_kv4_read(cache, shape, ints(*length), 41, first=ints(17, 30, -3))
    for g, h in zip(part, held):
        for b, f in enumerate((17, 30, -3)):
            want = torch.zeros((41, 2, dim), dtype=torch.float16)
            for i in range(41):
                if 0 <= f + i < 100:
                    want[i] = h[b, f + i]
            assert same_bits(g[b], want)


def test_append_of_values_at_the_edges(e0m4, oracle):
    shape = e0m4.E0M4KV4Shape(1, 1, 40, 64, 32)
    x = torch.zeros((1, 8, 1, 64), dtype=torch.float16)
    x[0, 0, 0, 3] = float("nan")
    x[0, 0, 0, 4] = 2.0
    x[0, 1, 0, 0], x[0, 1, 0, 1] = float("inf"), float("-inf")
    x[0, 2] = 65504.0
    x[0, 3] = -65504.0
    x[0, 4, 0, ::2] = 6e-8
    x[0, 5] = -0.0
    x[0, 6] = torch.linspace(-3, 5, 64).half()
    x[0, 7] = float("nan")
    for dtype in (torch.float16, torch.bfloat16):
        y = x.to(dtype)
        cache = dirty(e0m4, shape)
        e0m4.e0m4_kv4_append(cache, shape, y.to(DEV), y.to(DEV), ints(20))
        k, v = e0m4.e0m4_kv4_read(cache, shape, ints(28), 8, first=ints(20))
        want = plain.stored(y, 32, oracle)
        assert same_bits(k, want) and same_bits(v, want)
        assert torch.isfinite(k).all()
    # magnitudes beyond fp16's, and far below it
    big = torch.zeros((1, 1, 1, 64), dtype=torch.bfloat16)
    big[0, 0, 0, 0], big[0, 0, 0, 1], big[0, 0, 0, 2] = 3e38, -3e38, 1e-30
    small = torch.full((1, 1, 1, 64), 1e-38).to(torch.bfloat16)
    for y, as_half in ((big, big.float().clamp(-plain.MOST, plain.MOST).half()), (small, torch.zeros((1, 1, 1, 64)).half())):
        cache = dirty(e0m4, shape)
        e0m4.e0m4_kv4_append(cache, shape, y.to(DEV), y.to(DEV), ints(0))
        k, v = e0m4.e0m4_kv4_read(cache, shape, ints(1), 1)
        want = plain.stored(as_half, 32, oracle)
        assert same_bits(k, want) and same_bits(v, want)


def test_append_leaves_out_rows_outside_the_cache(e0m4, oracle):
    gen = torch.Generator().manual_seed(5)
    shape = e0m4.E0M4KV4Shape(4, 1, 50, 64, 64)
    cache = dirty(e0m4, shape)
    k, v = rows_of(gen, (4, 50, 1, 64), torch.float16), rows_of(gen, (4, 50, 1, 64), torch.float16)
    e0m4.e0m4_kv4_append(cache, shape, k.to(DEV), v.to(DEV), ints(0, 0, 0, 0))
    before = cache.clone()
    new = rows_of(gen, (4, 40, 1, 64), torch.float16)
    starts, counts = (-35, 45, 2 ** 31 - 1, -2 ** 31), (40, 99, 40, 40)
    e0m4.e0m4_kv4_append(cache, shape, new.to(DEV), new.to(DEV), ints(*starts), counts=ints(*counts))
    got = e0m4.e0m4_kv4_read(cache, shape, ints(99, 50, 50, 50), 50)
    for g, rows in zip(got, (k, v)):
        want = rows.clone()
        want[0, 0:5] = new[0, 35:40]
        want[1, 45:50] = new[1, 0:5]
        assert same_bits(g, plain.stored(want, 64, oracle))
    assert not torch.equal(before, cache)
    # nothing to do
    e0m4.e0m4_kv4_append(cache, shape, new[:, :0].to(DEV), new[:, :0].to(DEV), ints(0, 0, 0, 0))
    e0m4.e0m4_kv4_append(cache, shape, new.to(DEV), new.to(DEV), ints(0, 0, 0, 0), counts=ints(0, -1, 0, 0))
    again = e0m4.e0m4_kv4_read(cache, shape, ints(50, 50, 50, 50), 50)
    assert same_bits(again[0], got[0]) and same_bits(again[1], got[1])


def test_append_of_strided_and_shared_rows(e0m4, oracle):
    gen = torch.Generator().manual_seed(6)
    shape = e0m4.E0M4KV4Shape(2, 3, 40, 64, 32)
    wide = rows_of(gen, (2, 9, 1000), torch.float16).to(DEV)
    keys = wide[..., 8:8 + 192].view(2, 9, 3, 64)
    values = wide[..., 400:400 + 192].view(2, 9, 3, 64).flip(0)[:1].expand(2, 9, 3, 64)
    cache = dirty(e0m4, shape)
    e0m4.e0m4_kv4_append(cache, shape, keys, values, ints(30, 3))
    k, v = e0m4.e0m4_kv4_read(cache, shape, ints(40, 40), 9, first=ints(30, 3))
    assert same_bits(k, plain.stored(keys.cpu(), 32, oracle)) and same_bits(v, plain.stored(values.cpu(), 32, oracle))
    # heads before rows
    other = rows_of(gen, (2, 3, 9, 64), torch.bfloat16).to(DEV).transpose(1, 2)
    e0m4.e0m4_kv4_append(cache, shape, other, other, ints(1, 2))
    k, v = e0m4.e0m4_kv4_read(cache, shape, ints(40, 40), 9, first=ints(1, 2))
    assert same_bits(k, plain.stored(other.cpu(), 32, oracle)) and same_bits(k, v)


# ---- attention ------------------------------------------------------------------------------------


def check_attention(e0m4, oracle, dim, group, kv, share, n, lengths, counts=None, dtype=torch.float16, causal=True, window=0, mask=None,
                    weights=False, capacity=None, seed=0, strong=1.0):
    gen = torch.Generator().manual_seed(1000 * seed + dim + group + n)
    batch = len(lengths)
    capacity = capacity or max(max(lengths), 1)
    shape = e0m4.E0M4KV4Shape(batch, kv, capacity, dim, group)
    cache = dirty(e0m4, shape)
    rows = max(max(lengths), 1)
    keys, values = rows_of(gen, (batch, rows, kv, dim), dtype), rows_of(gen, (batch, rows, kv, dim), dtype)
    heads = kv * share
    wide = torch.randn((batch, n, (heads + 2) * dim), generator=gen).mul_(strong).to(dtype)
    q = wide[..., dim:dim + heads * dim].view(batch, n, heads, dim)
    length = ints(*lengths)
    e0m4.e0m4_kv4_append(cache, shape, keys.to(DEV), values.to(DEV), ints(*[0] * batch), counts=length)
    k, v = (plain.stored(t, group, oracle) for t in (keys, values))
    for b in range(batch):
        k[b, lengths[b]:], v[b, lengths[b]:] = 0, 0
    got_weights = None
    if weights:
        before = torch.rand((batch, kv, capacity), generator=gen)
        for b in range(batch):
            before[b, :, lengths[b]:] = float("nan")
        got_weights = before.clone().to(DEV)
    qd = wide.to(DEV)[..., dim:dim + heads * dim].view(batch, n, heads, dim)
    m = None if mask is None else mask.to(DEV)
    given = None if counts is None else ints(*counts)
    out = e0m4.e0m4_kv4_attention(qd, cache, shape, length, counts=given, causal=causal, window=window, mask=m, weights=got_weights)
    count = torch.tensor(counts if counts is not None else [n] * batch)
    look = plain.seen(torch.tensor(lengths), count, n, rows, causal, window, mask)
    want, received, size, reach = plain.attention(q, k, v, look)
    bound = plain.attention_bounds(want, size, reach, dim, rows, dtype)
    assert torch.isfinite(out).all()
    over = ((out.cpu().double() - want).abs() - bound).amax()
    assert over <= 0, "outputs off by %g beyond their bound" % over
    nothing = ~look.any(-1)
    assert (out.cpu()[nothing] == 0).all()
    if weights:
        got = got_weights.cpu().double()
        for b in range(batch):
            L = lengths[b]
            assert torch.isnan(got[b, :, L:]).all()                 # what lies behind is not touched
            want_b = before[b, :, :L].double() + received[b, :, :L]
            err = (got[b, :, :L] - want_b).abs()
            assert (err <= plain.received_bounds(received[b, :, :L], reach, dim, n * share) + want_b * 2.0 ** -24).all(), float(err.max())
    # the same again, to the bit
    if weights:
        second = before.clone().to(DEV)
        out2 = e0m4.e0m4_kv4_attention(qd, cache, shape, length, counts=given, causal=causal, window=window, mask=m, weights=second)
        assert torch.equal(second.view(torch.int32), got_weights.view(torch.int32))
    else:
        out2 = e0m4.e0m4_kv4_attention(qd, cache, shape, length, counts=given, causal=causal, window=window, mask=m)
    assert same_bits(out, out2)
    return out


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_single_tokens(e0m4, oracle, kernels, dim, group, dtype):
    check_attention(e0m4, oracle, dim, group, 2, 1, 1, [1, 31, 32, 33, 300], dtype=dtype, weights=True)
    check_attention(e0m4, oracle, dim, group, 1, 16, 1, [700, 5], dtype=dtype)
    check_attention(e0m4, oracle, dim, group, 2, 3, 1, [0, 65, 2000], dtype=dtype, capacity=2050, weights=True)


@pytest.mark.parametrize("dim,group", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_prompts(e0m4, oracle, kernels, dim, group, dtype):
    check_attention(e0m4, oracle, dim, group, 2, 2, 130, [130, 101], counts=[130, 101], dtype=dtype, weights=True)
    check_attention(e0m4, oracle, dim, group, 1, 5, 77, [400, 77, 90], counts=[77, 70, 1], dtype=dtype, weights=True)
    check_attention(e0m4, oracle, dim, group, 1, 1, 300, [300], dtype=dtype)


@pytest.mark.parametrize("n", [2, 3, 8, 15, 16, 17, 31, 33, 48, 63, 64, 65, 100, 128, 129, 200])
def test_numbers_of_new_tokens(e0m4, oracle, kernels, n):
    check_attention(e0m4, oracle, 128, 128, 1, 1, n, [n + 5, n, 333], weights=True, seed=n)
    check_attention(e0m4, oracle, 128, 64, 2, 7, n, [n + 64], dtype=torch.bfloat16, seed=n)


@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 100, 1000])
@pytest.mark.parametrize("n,share", [(1, 4), (9, 4), (150, 2)])
def test_windows(e0m4, oracle, kernels, window, n, share):
    check_attention(e0m4, oracle, 64, 32, 2, share, n, [700, 150, 333], window=window, weights=True, seed=window, counts=[n, n, min(n, 5)])
    check_attention(e0m4, oracle, 128, 128, 1, share, n, [290], window=window, seed=window)


@pytest.mark.parametrize("n,share", [(1, 1), (4, 8), (40, 2), (140, 1)])
def test_every_query_sees_every_row(e0m4, oracle, kernels, n, share):
    check_attention(e0m4, oracle, 128, 64, 2, share, n, [140, 200, 0], counts=[n, max(n - 3, 0), 0], causal=False, weights=True)
    check_attention(e0m4, oracle, 256, 128, 1, share, n, [63], causal=False)


@pytest.mark.parametrize("n,share", [(1, 2), (12, 16), (50, 3), (129, 2)])
@pytest.mark.parametrize("causal", [True, False])
def test_masks(e0m4, oracle, kernels, n, share, causal):
    gen = torch.Generator().manual_seed(n)
    mask = torch.rand((2, n, 300), generator=gen) < 0.3
    mask[0, n // 2] = False                                          # a row with nothing
    mask[1, :, 64:128] = False                                       # whole tiles with nothing
    mask[1, 0, :] = False
    check_attention(e0m4, oracle, 128, 128, 2, share, n, [300, 211], mask=mask, causal=causal, weights=True)
    check_attention(e0m4, oracle, 64, 32, 1, share, n, [300, 211], mask=mask[:1], causal=causal)          # shared by the sequences
    check_attention(e0m4, oracle, 64, 64, 1, share, n, [300, 211], mask=mask[:, :1], causal=causal, dtype=torch.bfloat16)   # by the queries
    check_attention(e0m4, oracle, 128, 32, 1, share, n, [300, 211], mask=mask[..., :190], causal=causal)  # rows beyond the mask
    check_attention(e0m4, oracle, 128, 32, 1, share, n, [300, 211], mask=torch.cat([mask, mask], 2)[..., 301:600][..., ::1], causal=causal)
    check_attention(e0m4, oracle, 128, 64, 1, share, n, [300, 211], mask=torch.zeros((1, 1, 300), dtype=torch.bool), causal=causal)


def test_masks_and_windows_together(e0m4, oracle, kernels):
    gen = torch.Generator().manual_seed(3)
    mask = torch.rand((1, 20, 500), generator=gen) < 0.5
    check_attention(e0m4, oracle, 128, 128, 2, 4, 20, [500, 60], mask=mask, window=37, weights=True)


@pytest.mark.parametrize("strong", [0.0, 1e-3, 30.0])
def test_flat_and_sharp_scores(e0m4, oracle, kernels, strong):
    for n in (1, 90):
        check_attention(e0m4, oracle, 128, 128, 1, 4, n, [1500, 700], strong=strong, weights=True)
        check_attention(e0m4, oracle, 64, 64, 2, 1, n, [1500], strong=strong, dtype=torch.bfloat16)


def test_scores_that_rise_along_the_cache(e0m4, oracle, kernels):
    """The reference of the softmax has to move many times, also far after the first rows."""
    dim, rows = 128, 3000
    shape = e0m4.E0M4KV4Shape(1, 1, rows, dim, 128)
    rise = torch.linspace(0.0, 40.0, rows)[None, :, None, None]
    gen = torch.Generator().manual_seed(2)
    keys = (torch.ones((1, rows, 1, dim)) * rise / dim ** 0.5 + 0.01 * torch.randn((1, rows, 1, dim), generator=gen)).half()
    values = rows_of(gen, (1, rows, 1, dim), torch.float16)
    for n, sign in ((1, 1.0), (1, -1.0), (80, 1.0), (80, -1.0)):
        q = torch.full((1, n, 2, dim), sign).half()
        cache = dirty(e0m4, shape)
        e0m4.e0m4_kv4_append(cache, shape, keys.to(DEV), values.to(DEV), ints(0))
        got = torch.zeros((1, 1, rows), device=DEV)
        out = e0m4.e0m4_kv4_attention(q.to(DEV), cache, shape, ints(rows), weights=got)
        look = plain.seen(torch.tensor([rows]), torch.tensor([n]), n, rows, True, 0, None)
        want, received, size, reach = plain.attention(q, plain.stored(keys, 128, oracle), plain.stored(values, 128, oracle), look)
        assert ((out.cpu().double() - want).abs() <= plain.attention_bounds(want, size, reach, dim, rows, torch.float16)).all()
        assert ((got.cpu().double() - received).abs() <= plain.received_bounds(received, reach, dim, 2 * n)).all()


def test_queries_out_of_the_ordinary(e0m4, oracle, kernels):
    """bfloat16 queries far outside fp16's range; queries that are not finite touch their own row only."""
    dim, rows, kv = 128, 200, 1
    gen = torch.Generator().manual_seed(4)
    shape = e0m4.E0M4KV4Shape(1, kv, rows, dim, 64)
    keys, values = rows_of(gen, (1, rows, kv, dim), torch.bfloat16), rows_of(gen, (1, rows, kv, dim), torch.bfloat16)
    cache = dirty(e0m4, shape)
    e0m4.e0m4_kv4_append(cache, shape, keys.to(DEV), values.to(DEV), ints(0))
    k, v = plain.stored(keys, 64, oracle), plain.stored(values, 64, oracle)
    for n in (4, 70):
        q = torch.randn((1, n, 2, dim), generator=gen).to(torch.bfloat16)
        q[0, 0] *= 1e-30
        q[0, 1, 0] *= 1e4
        q[0, 1, 1, 5] = 1e5
        q[0, 2] *= 1e-39
        look = plain.seen(torch.tensor([rows]), torch.tensor([n]), n, rows, True, 0, None)
        want, _, size, reach = plain.attention(q, k, v, look)
        bound = plain.attention_bounds(want, size, reach, dim, rows, torch.bfloat16)
        out = e0m4.e0m4_kv4_attention(q.to(DEV), cache, shape, ints(rows)).cpu()
        easy = reach[..., 0] < 1e3                                   # (where a score's own error leaves something to compare)
        assert ((out.double() - want).abs() <= bound)[easy].all()
        assert torch.isfinite(out).all()
        bad = q.clone()
        bad[0, 3, 0, 7] = float("nan")
        bad[0, 3, 1, 9] = float("inf")
        out2 = e0m4.e0m4_kv4_attention(bad.to(DEV), cache, shape, ints(rows)).cpu()
        assert torch.isnan(out2[0, 3]).all()
        rest = torch.arange(n) != 3
        assert same_bits(out2[:, rest], out[:, rest])


def test_lengths_and_counts_out_of_range_are_taken_as_the_nearest(e0m4, oracle, kernels):
    gen = torch.Generator().manual_seed(8)
    shape = e0m4.E0M4KV4Shape(4, 1, 70, 64, 64)
    cache = dirty(e0m4, shape)
    keys, values = rows_of(gen, (4, 70, 1, 64), torch.float16), rows_of(gen, (4, 70, 1, 64), torch.float16)
    e0m4.e0m4_kv4_append(cache, shape, keys.to(DEV), values.to(DEV), ints(0, 0, 0, 0))
    q = torch.randn((4, 5, 2, 64), generator=gen).half()
    for n in (5,):
        for causal in (True, False):
            a = e0m4.e0m4_kv4_attention(q.to(DEV), cache, shape, ints(99, -4, 3, 70), counts=ints(9, 2, 5, -1), causal=causal)
            b = e0m4.e0m4_kv4_attention(q.to(DEV), cache, shape, ints(70, 0, 3, 70), counts=ints(5, 2, 5, 0), causal=causal)
            assert same_bits(a, b) and (a[1] == 0).all() and (a[3] == 0).all()
    a = e0m4.e0m4_kv4_attention(q.to(DEV), cache, shape, ints(70, 70, 3, 70))
    assert (a[2, :2] == 0).all() and (a[2, 2:] != 0).any()           # the first of five queries over three rows stand before the first row


def test_long_caches(e0m4, oracle, kernels):
    check_attention(e0m4, oracle, 64, 64, 1, 4, 1, [40000, 7], weights=True)
    check_attention(e0m4, oracle, 128, 128, 1, 8, 3, [20000], dtype=torch.bfloat16)
    check_attention(e0m4, oracle, 64, 32, 1, 1, 70, [9000], weights=True)


def test_offsets_beyond_32_bits(e0m4, oracle, kernels):
    """A cache of more than 4 GiB, rows at its end."""
    gen = torch.Generator().manual_seed(9)
    dim, group, capacity = 256, 32, 14_000_000
    shape = e0m4.E0M4KV4Shape(1, 1, capacity, dim, group)
    assert e0m4.e0m4_kv4_bytes(shape) > 1 << 32
    cache = e0m4.e0m4_kv4_alloc(shape, DEV)
    n, start = 100, capacity - 100
    keys, values = rows_of(gen, (1, n, 1, dim), torch.float16), rows_of(gen, (1, n, 1, dim), torch.float16)
    e0m4.e0m4_kv4_append(cache, shape, keys.to(DEV), values.to(DEV), ints(start))
    k, v = e0m4.e0m4_kv4_read(cache, shape, ints(capacity), n, first=ints(start))
    ks, vs = plain.stored(keys, group, oracle), plain.stored(values, group, oracle)
    assert same_bits(k, ks) and same_bits(v, vs)
    for m in (1, 80):
        q = torch.randn((1, m, 2, dim), generator=gen).half()
        out = e0m4.e0m4_kv4_attention(q.to(DEV), cache, shape, ints(capacity), window=20)
        look = plain.seen(torch.tensor([n]), torch.tensor([m]), m, n, True, 20, None)
        want, _, size, reach = plain.attention(q, ks, vs, look)
        assert ((out.cpu().double() - want).abs() <= plain.attention_bounds(want, size, reach, dim, n, torch.float16)).all()


def test_attention_of_nothing(e0m4, kernels):
    shape = e0m4.E0M4KV4Shape(2, 2, 0, 64, 64)
    cache = e0m4.e0m4_kv4_alloc(shape, DEV)
    out = torch.full((2, 3, 4, 64), 7.0, dtype=torch.float16, device=DEV)
    e0m4.e0m4_kv4_attention(torch.ones_like(out), cache, shape, ints(0, 0), out=out)
    assert (out == 0).all()
    shape = shape._replace(capacity=10)
    cache = dirty(e0m4, shape)
    assert e0m4.e0m4_kv4_attention(out[:, :0], cache, shape, ints(5, 5)).shape == (2, 0, 4, 64)
    w = torch.full((2, 2, 10), 3.0, device=DEV)
    out.fill_(7)
    e0m4.e0m4_kv4_attention(torch.ones_like(out), cache, shape, ints(0, 0), out=out, weights=w)
    assert (out == 0).all() and (w == 3).all()
    k, v = e0m4.e0m4_kv4_read(cache, shape, ints(0, 0), 4)
    assert (k == 0).all() and (v == 0).all() and k.shape == (2, 4, 2, 64)


# ---- eviction -------------------------------------------------------------------------------------


def check_evict(e0m4, oracle, dim, group, kv, lengths, received, budget, recent, small_capacity=None):
    gen = torch.Generator().manual_seed(dim + budget)
    batch, _, capacity = received.shape
    shape = e0m4.E0M4KV4Shape(batch, kv, capacity, dim, group)
    cache = dirty(e0m4, shape)
    keys, values = rows_of(gen, (batch, capacity, kv, dim), torch.float16), rows_of(gen, (batch, capacity, kv, dim), torch.float16)
    e0m4.e0m4_kv4_append(cache, shape, keys.to(DEV), values.to(DEV), ints(*[0] * batch), counts=ints(*lengths))
    small_shape = shape._replace(capacity=small_capacity or budget)
    small = dirty(e0m4, small_shape)
    kept, n, got = e0m4.e0m4_kv4_evict(cache, shape, received.to(DEV), ints(*lengths), budget, recent, small, small_shape)
    want = plain.evict(received, lengths, budget, recent)
    assert torch.equal(kept.cpu(), want)
    assert n.tolist() == [min(max(0, min(x, capacity)), budget) for x in lengths]
    k, v = (t.cpu() for t in e0m4.e0m4_kv4_read(small, small_shape, n, budget))
    ks, vs = plain.stored(keys, group, oracle), plain.stored(values, group, oracle)
    for b in range(batch):
        for h in range(kv):
            stay = want[b, h][want[b, h] >= 0].long()
            m = len(stay)
            assert same_bits(k[b, :m, h], ks[b, stay, h]) and same_bits(v[b, :m, h], vs[b, stay, h])
            assert (k[b, m:] == 0).all() and (v[b, m:] == 0).all()
            assert np.array_equal(got[b, h, :m].cpu().numpy(), received[b, h, stay].numpy(), equal_nan=True)
            assert (got[b, h, m:] == 0).all()


@pytest.mark.parametrize("dim,group", SHAPES)
def test_evict(e0m4, oracle, dim, group):
    gen = torch.Generator().manual_seed(dim * group)
    received = torch.rand((3, 2, 400), generator=gen)
    received[:, :, ::3] = 0                                          # many equal ones
    check_evict(e0m4, oracle, dim, group, 2, [400, 101, 60], received, 100, 17)
    check_evict(e0m4, oracle, dim, group, 2, [399, 0, 350], received, 333, 0, small_capacity=350)


@pytest.mark.parametrize("budget,recent", [(1, 0), (1, 1), (31, 31), (32, 5), (33, 0), (64, 63), (1000, 10), (2999, 300), (3000, 1)])
def test_evict_budgets(e0m4, oracle, budget, recent):
    gen = torch.Generator().manual_seed(budget)
    received = -torch.log(torch.rand((2, 1, 3000), generator=gen))
    check_evict(e0m4, oracle, 64, 64, 1, [3000, 2999], received, budget, recent)


def test_evict_orders_all_numbers(e0m4, oracle):
    gen = torch.Generator().manual_seed(1)
    base = torch.tensor([0.0, -0.0, 1.0, -1.0, float("inf"), float("-inf"), float("nan"), 1e-42, -1e-42, 1e-30, 3e38, 1.0000001])
    received = base[torch.randint(len(base), (1, 4, 500), generator=gen)]
    received[0, 1] = 0.25                                            # all equal: the first ones stay
    received[0, 2] = float("nan")
    received[0, 3] = torch.where(torch.rand(500, generator=gen) < 0.5, 0.0, -0.0)
    for budget in (3, 50, 77, 200, 333, 480):
        check_evict(e0m4, oracle, 64, 32, 4, [500], received, budget, min(budget, 3))


def test_evict_of_long_caches(e0m4, oracle):
    gen = torch.Generator().manual_seed(11)
    received = torch.rand((1, 2, 70000), generator=gen)
    received[0, 1] = (received[0, 1] * 50).floor()
    check_evict(e0m4, oracle, 64, 64, 2, [70000], received, 20001, 100)


# ---- streams and graphs ---------------------------------------------------------------------------


def test_on_another_stream(e0m4, oracle):
    gen = torch.Generator().manual_seed(12)
    shape = e0m4.E0M4KV4Shape(1, 2, 3000, 128, 128)
    keys = rows_of(gen, (1, 3000, 2, 128), torch.float16).to(DEV)
    q = torch.randn((1, 1, 4, 128), generator=gen).half().to(DEV)
    cache = dirty(e0m4, shape)
    e0m4.e0m4_kv4_append(cache, shape, keys, keys, ints(0))
    want = e0m4.e0m4_kv4_attention(q, cache, shape, ints(3000))
    other_cache = dirty(e0m4, shape)
    zero, length = ints(0), ints(3000)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    e0m4.e0m4_kv4_append(other_cache, shape, keys, keys, zero, stream=stream)
    got = e0m4.e0m4_kv4_attention(q, other_cache, shape, length, stream=stream)
    stream.synchronize()
    assert same_bits(got, want)
    raw = torch.cuda.Stream()
    with pytest.raises(ValueError):
        e0m4.e0m4_kv4_attention(q, cache, shape, length, stream=raw.cuda_stream)


def test_in_a_graph(e0m4, oracle):
    """A step (append, tracked attention, eviction) captured once and replayed on other tokens gives what the calls give by themselves."""
    gen = torch.Generator().manual_seed(13)
    shape = e0m4.E0M4KV4Shape(2, 1, 600, 128, 128)
    small_shape = shape._replace(capacity=300)
    rows = rows_of(gen, (2, 500, 1, 128), torch.float16).to(DEV)
    start, one = ints(500, 450), ints(1, 1)
    token = rows[:, :1].clone()
    q = torch.randn((2, 1, 8, 128), generator=gen).half().to(DEV)
    state = {}

    def fresh():
        state["cache"] = dirty(e0m4, shape)
        e0m4.e0m4_kv4_append(state["cache"], shape, rows, rows, ints(0, 0), counts=ints(500, 450))
        state["weights"] = torch.zeros((2, 1, 600), device=DEV)
        state["small"] = dirty(e0m4, small_shape)

    def step(length):
        e0m4.e0m4_kv4_append(state["cache"], shape, token, token, start, counts=one)
        out = e0m4.e0m4_kv4_attention(q, state["cache"], shape, length, weights=state["weights"])
        return (out,) + e0m4.e0m4_kv4_evict(state["cache"], shape, state["weights"], length, 300, 20, state["small"], small_shape)

    fresh()
    length = start + 1
    step(length)
    torch.cuda.synchronize()
    fresh()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(length)
    captured = dict(state)
    for i in range(4):
        token.copy_(rows[:, 7 * i:7 * i + 1])
        q.copy_(torch.randn((2, 1, 8, 128), generator=gen).half())
        captured["weights"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        fresh()
        want = step(length)
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g.view(torch.uint8), w.view(torch.uint8))
        assert torch.equal(captured["weights"], state["weights"])
