"""Attention over the 4-bit cache with scores up to the 2^23 that the header allows: the row with the largest score has all the weight."""
import math

import pytest

torch = pytest.importorskip("torch")

import kv4_plain as plain  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("kernel", [0, 1, 2, 3])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows", [40, 700])
def test_scores_far_apart(oracle, rows, dtype, kernel):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' elsewhere)")
    import paper_2403_20041_amd as e0m4

    dim, group = 128, 128
    gen = torch.Generator().manual_seed(rows)
    # rows of one value each, which keeps them apart in four bits; the largest anywhere, and some rise towards it
    level = torch.rand(rows, generator=gen) * 400 - 200
    level[: rows // 2] = torch.linspace(-390, 300, rows // 2)
    level[rows // 3] = 390
    keys = level[None, :, None, None].expand(1, rows, 1, dim).to(dtype).contiguous()
    values = torch.randn((1, rows, 1, dim), generator=gen).to(dtype)
    k, v = plain.stored(keys, group, oracle), plain.stored(values, group, oracle)
    shape = e0m4.E0M4KV4Shape(1, 1, rows, dim, group)
    cache = e0m4.e0m4_kv4_alloc(shape, DEV).fill_(255)
    zero, length = torch.zeros(1, dtype=torch.int32, device=DEV), torch.full((1,), rows, dtype=torch.int32, device=DEV)
    e0m4.e0m4_kv4_append(cache, shape, keys.to(DEV), values.to(DEV), zero)
    for n in (1, 80):
        q = torch.full((1, n, 2, dim), 1800.0)
        q[:, :, 1] = -1800.0                                         # the other head's is the smallest
        scores = q[0, 0, :, :1].double() * k[0, :, 0, 0].double() * (dim / math.sqrt(dim))
        assert 7e6 < scores.abs().max() < 2 ** 23
        first = scores.topk(2).values
        assert (first[:, 0] - first[:, 1] > 1000).all()
        received = torch.zeros((1, 1, rows), device=DEV)
        e0m4.e0m4_set_knob("kv4_attention", kernel)
        try:
            out = e0m4.e0m4_kv4_attention(q.to(dtype).to(DEV), cache, shape, length, causal=False, weights=received)
        finally:
            e0m4.e0m4_set_knob("kv4_attention", 0)
        best = scores.argmax(1)
        want = v[0, best, 0].double()[None, None].expand(1, n, 2, dim)
        # the result's rounding, the weight's to fp16, and some units of fp32 for its sum, quotient and products
        bound = want.abs() * (torch.finfo(dtype).eps / 2 + 2.0 ** -11) * (1 + 2.0 ** -7) + 2.0 ** -25
        assert ((out.cpu().double() - want).abs() <= bound).all()
        got = received[0, 0].cpu()
        others = torch.ones(rows, dtype=torch.bool)
        others[best] = False
        assert torch.isfinite(got).all() and (got[others] == 0).all()
