"""Attention of few fp16 queries over the 4-bit cache multiplies what the rounding of the softmax weights to fp16 leaves, too: outputs
against the plain form in 64 bits with a bound that has no room for weights of eleven bits, and, on the CPU, that such weights are beyond
it."""
import math

import pytest

torch = pytest.importorskip("torch")

import kv4_plain as plain  # noqa: E402

SHAPES = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128), (256, 32), (256, 64), (256, 128)]
# query heads to one of keys and values, new tokens: up to 8 rows of queries, up to 16, several tiles of 16
ROWS = [(1, 1), (5, 1), (4, 2), (8, 1), (9, 1), (8, 2), (16, 1), (6, 3), (11, 3)]
LENGTHS = (3, 5, 8, 4)


def bounds(out, size, reach, all_values, dim, rows):
    """Bound of the error of each output: its rounding to fp16 (half a step, of the smallest normal number below that); a weight's parts
    of eleven bits each, 2^-22 of it, and half of fp16's smallest step where the parts are subnormal, 2^-25 with a sum of 2^8 at least;
    scores in fp32 as in plain.attention_bounds, for the weight and for the sum; both parts' products and the weights' sum over the
    rows, exp2, the factors of tiles and wavefronts and the quotient in fp32."""
    u = 2.0 ** -24
    score = (dim + 8) * u * reach + 2.0 ** -22
    inner = size * (2.0 ** -22 + 2 * score + (3 * rows + 40) * u) + 2.0 ** -33 * all_values
    return out.abs().clamp(min=torch.finfo(torch.float16).smallest_normal) * torch.finfo(torch.float16).eps / 2 + inner * (1 + 2.0 ** -7)


def inputs(oracle, dim, group, kv, share, n, lengths, seed):
    gen = torch.Generator().manual_seed(seed)
    batch, rows = len(lengths), max(lengths)
    keys, values = (torch.randn((batch, rows, kv, dim), generator=gen).half() for _ in range(2))
    q = (torch.randn((batch, n, kv * share, dim), generator=gen) * 0.1).half()          # (scores of about a tenth: all rows count)
    k, v = (plain.stored(t, group, oracle) for t in (keys, values))
    for b in range(batch):
        k[b, lengths[b]:], v[b, lengths[b]:] = 0, 0
    look = plain.seen(torch.tensor(lengths), torch.tensor([n] * batch), n, rows, True, 0, None)
    want, _, size, reach = plain.attention(q, k, v, look)
    everything = v.double().abs().sum(1).repeat_interleave(share, 1)[:, None].expand(want.shape)
    return keys, values, q, k, v, look, want, bounds(want, size, reach, everything, dim, rows)


def with_rounded_weights(q, k, v, look):
    batch, n, heads, dim = q.shape
    kv = k.shape[2]
    qd = q.double().view(batch, n, kv, heads // kv, dim).permute(0, 2, 3, 1, 4)
    kd, vd = (t.double().permute(0, 2, 1, 3)[:, :, None] for t in (k, v))
    s = (qd @ kd.transpose(-1, -2) * (math.log2(math.e) / math.sqrt(dim))).masked_fill(~look[:, None, None], -math.inf)
    e = torch.exp2(s - s.amax(-1, keepdim=True) + 8)
    out = (e.half().double() @ vd) / e.sum(-1, keepdim=True)
    return out.permute(0, 3, 1, 2, 4).reshape(batch, n, heads, dim).half()


@pytest.mark.parametrize("share,n", ROWS)
@pytest.mark.parametrize("dim,group", SHAPES)
def test_the_bound_has_no_room_for_rounded_weights(oracle, dim, group, share, n):
    _, _, q, k, v, look, want, bound = inputs(oracle, dim, group, 2, share, n, LENGTHS, 100 * dim + 10 * share + n)
    assert look.any(-1).all()
    assert ((want.half().double() - want).abs() <= bound).all()
    assert ((with_rounded_weights(q, k, v, look).double() - want).abs() > bound).any()


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", [0, 1])
@pytest.mark.parametrize("share,n", ROWS)
@pytest.mark.parametrize("dim,group", SHAPES)
def test_few_queries_have_whole_weights(oracle, dim, group, share, n, kernel):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' elsewhere)")
    import paper_2403_20041_amd as e0m4

    for lengths, weights in ((LENGTHS, False), (LENGTHS, True), ((2000, 33), False)):    # one workgroup for all rows, and several
        keys, values, q, _, _, _, want, bound = inputs(oracle, dim, group, 2, share, n, lengths, 100 * dim + 10 * share + n)
        shape = e0m4.E0M4KV4Shape(len(lengths), 2, max(lengths), dim, group)
        cache = e0m4.e0m4_kv4_alloc(shape, "cuda").fill_(255)
        length = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        e0m4.e0m4_kv4_append(cache, shape, keys.cuda(), values.cuda(), torch.zeros_like(length), counts=length)
        received = torch.zeros((len(lengths), 2, max(lengths)), device="cuda") if weights else None
        e0m4.e0m4_set_knob("kv4_attention", kernel)
        try:
            out = e0m4.e0m4_kv4_attention(q.cuda(), cache, shape, length, weights=received)
        finally:
            e0m4.e0m4_set_knob("kv4_attention", 0)
        over = ((out.cpu().double() - want).abs() - bound).amax()
        assert over <= 0, "outputs off by %g beyond their bound" % over
