"""Offsets that pass 32 bits in the operators of rows that choose their weights: outputs, packed weights and gathered rows far into their buffers."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def e0m4():
    import paper_2403_20041_amd as pkg

    pkg.lib()
    return pkg


def weights(e0m4, N, K, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return e0m4.e0m4_quantize((torch.randn((N, K), generator=g, device=DEV) * 0.1).half(), 128)[0]


@pytest.mark.parametrize("form", [1, 4, 5])
def test_outputs_behind_2_to_the_31(e0m4, form):
    rows, N, K = 70001, 32768, 128
    codes = weights(e0m4, N, K, 1).unsqueeze(0)
    x = torch.randn((rows, K), generator=torch.Generator().manual_seed(2)).half().to(DEV)
    plan = e0m4.e0m4_groups(torch.zeros(rows, dtype=torch.int32, device=DEV), 1)
    e0m4.e0m4_set_knob("grouped_form", form)
    try:
        y = e0m4.e0m4_matmul_grouped(x, plan, codes, N, K, 128)
        for part in (slice(0, 40), slice(65530, 65560), slice(rows - 40, rows)):
            few = x[part].contiguous()
            want = e0m4.e0m4_matmul_grouped(few, e0m4.e0m4_groups(torch.zeros(few.shape[0], dtype=torch.int32, device=DEV), 1), codes, N, K, 128)
            assert torch.equal(y[part], want), part
    finally:
        e0m4.e0m4_set_knob("grouped_form", 0)
    # ... read back by the sum over a token's rows
    token = e0m4.e0m4_combine(y, torch.ones((rows, 1), device=DEV), plan)
    assert torch.equal(token[-40:], y[-40:])


@pytest.mark.parametrize("form", [1, 4])
def test_weights_behind_4_GiB(e0m4, form):
    groups, N, K = 150, 16384, 4096
    size = e0m4.e0m4_codes_bytes(N, K, 128)
    assert (groups - 1) * size > 1 << 32
    codes = torch.empty((groups, size), dtype=torch.uint8, device=DEV)
    codes[groups - 1] = weights(e0m4, N, K, 3)
    x = torch.randn((20, K), generator=torch.Generator().manual_seed(4)).half().to(DEV)
    e0m4.e0m4_set_knob("grouped_form", form)
    try:
        far, near = (e0m4.e0m4_matmul_grouped(x, e0m4.e0m4_groups(torch.full((20,), g, dtype=torch.int32, device=DEV), n), c, N, K, 128)
                     for g, n, c in ((groups - 1, groups, codes), (0, 1, codes[groups - 1:].contiguous())))
    finally:
        e0m4.e0m4_set_knob("grouped_form", 0)
    assert torch.equal(far, near)


@pytest.mark.parametrize("form", [1, 4])
def test_gathered_rows_up_to_2_GiB(e0m4, form):
    N, K = 64, 4096
    rows = 0x7fffffff // (2 * K)
    x = torch.zeros((rows, K), dtype=torch.float16, device=DEV)
    x[-30:] = torch.randn((30, K), generator=torch.Generator().manual_seed(5)).half().to(DEV)
    codes = torch.stack([weights(e0m4, N, K, 6), weights(e0m4, N, K, 7)])
    index = torch.full((rows,), -1, dtype=torch.int32, device=DEV)
    index[-30:] = torch.arange(30, dtype=torch.int32, device=DEV) % 2
    index[0] = 1
    plan = e0m4.e0m4_groups(index, 2)
    e0m4.e0m4_set_knob("grouped_form", form)
    try:
        y = e0m4.e0m4_matmul_grouped(x, plan, codes, N, K, 128, share=1)[:31]
        few = e0m4.e0m4_groups(index[-30:].contiguous(), 2)
        want = e0m4.e0m4_matmul_grouped(x[-30:].contiguous(), few, codes, N, K, 128, share=1)
    finally:
        e0m4.e0m4_set_knob("grouped_form", 0)
    assert torch.equal(y[:15], want[:15]) and not y[15].any() and torch.equal(y[16:], want[15:])
    with pytest.raises(e0m4.binding.E0M4Error):         # more than 32-bit offsets reach
        more = torch.zeros((rows + 1, K), dtype=torch.float16, device=DEV)
        e0m4.e0m4_matmul_grouped(more, e0m4.e0m4_groups(torch.zeros(rows + 1, dtype=torch.int32, device=DEV), 2), codes, N, K, 128, share=1)


def test_adapters_of_rows_far_into_their_tensors(e0m4):
    rows, K, N = 70000, 64, 32768
    x = torch.randn((rows, K), generator=torch.Generator().manual_seed(8)).half().to(DEV)
    A = torch.randn((2, 8, K), generator=torch.Generator().manual_seed(9)).half().to(DEV)
    B = torch.randn((2, N, 8), generator=torch.Generator().manual_seed(10)).half().to(DEV)
    index = torch.full((rows,), -1, dtype=torch.int32, device=DEV)
    index[-50:] = torch.arange(50, dtype=torch.int32, device=DEV) % 2
    out = e0m4.e0m4_lora(x, e0m4.e0m4_groups(index, 2), A, B)
    want = e0m4.e0m4_lora(x[-50:].contiguous(), e0m4.e0m4_groups(index[-50:].contiguous(), 2), A, B)
    # (other tiles and K splits, so sums in another order: half a step of the output and as much again)
    assert (out[-50:].float() - want.float()).abs().max() <= 2.0 ** -10 * want.float().abs().max() + 1e-3
    assert not out[:-50].any()
