"""Grouped products: every weight is the one that the dequant entry points give, rounded to 16 bits, in all forms; beyond that there are only sums in
fp32 and the result's rounding."""
import pytest
import torch

import groups_plain as plain
from test_gpu_groups import CASES, DEV, FORMATS, e0m4, gen, make_weights, within  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def call_of(pkg, fmt):
    return {"e0m4": pkg.e0m4_matmul_grouped, "e0m8": pkg.e0m8_matmul_grouped, "bf16": pkg.e0m4_bf16_matmul_grouped}[fmt]


@pytest.mark.parametrize("form", range(1, 7))
@pytest.mark.parametrize("fmt,group,N,K", [("e0m4", 128, 72, 384), ("e0m4", 64, 81, 448), ("e0m4", 32, 300, 160), ("bf16", 128, 72, 384), ("bf16", 64, 81, 448), ("bf16", 32, 300, 160),
                                           ("e0m8", 128, 96, 256), ("e0m8", 64, 301, 320)])
def test_rows_of_one_number_give_the_weights_bit_for_bit(e0m4, fmt, group, N, K, form):  # noqa: F811
    codes, values, _ = make_weights(e0m4, fmt, 2, N, K, group, 5 * N)
    index = torch.arange(2 * K, dtype=torch.int32) // K
    X = torch.eye(K, dtype=FORMATS[fmt]).repeat(2, 1)
    plan = e0m4.e0m4_groups(index.to(DEV), 2)
    e0m4.e0m4_set_knob("grouped_form", form)
    try:
        for share in (0, 1):
            got = call_of(e0m4, fmt)(X.to(DEV), plan, codes, N, K, group, share=share).cpu()
            assert torch.equal(got, torch.cat([values[0].t(), values[1].t()]))
    finally:
        e0m4.e0m4_set_knob("grouped_form", 0)


@pytest.mark.parametrize("form", range(7))
@pytest.mark.parametrize("fmt,group,N,K,sizes,gated", CASES)
def test_nothing_but_sums_in_32_bits(e0m4, fmt, group, N, K, sizes, gated, form):  # noqa: F811
    """Products of 16-bit numbers are exact in fp32; K additions and those of the parts are each off by a step of fp32 (2 U, whether rounded or cut) of what is
    added up; the gated product as in the plain form's bound."""
    groups = len(sizes)
    codes, values, _ = make_weights(e0m4, fmt, groups, N, K, group, N)
    index = torch.cat([torch.full((n,), e, dtype=torch.int32) for e, n in enumerate(sizes)])
    X = torch.randn((len(index), K), generator=gen(N - K)).to(FORMATS[fmt])
    plan = e0m4.e0m4_groups(index.to(DEV), groups)
    w, x = values.double(), X.double()
    a = torch.stack([w[g] @ x[p] for p, g in enumerate(index.tolist())])
    bound = torch.stack([w[g].abs() @ x[p].abs() for p, g in enumerate(index.tolist())]) * (2 * (K + 16) * plain.U)
    if gated:
        gate, up, eg, eu = a[:, :N // 2], a[:, N // 2:], bound[:, :N // 2], bound[:, N // 2:]
        silu = gate * torch.sigmoid(gate)
        # (the slope of silu is at most 1.1; its exponential and quotient are good to 2^-20)
        a = silu * up
        bound = 1.1 * eg * up.abs() + silu.abs() * eu + 1.1 * eg * eu + a.abs() * 2.0 ** -20
    bound = plain.half_step(a.abs() + bound, FORMATS[fmt]) + bound
    e0m4.e0m4_set_knob("grouped_form", form)
    try:
        got = call_of(e0m4, fmt)(X.to(DEV), plan, codes, N, K, group, share=1, epilogue=e0m4.E0M4_EPILOGUE_SWIGLU if gated else e0m4.E0M4_EPILOGUE_NONE)
    finally:
        e0m4.e0m4_set_knob("grouped_form", 0)
    within(got, a, bound)
