"""Low-rank adapters: the sums A x are multiplied with all their 24 bits.  Each case takes what the upper bits give away again, with base or
with another number of the rank, so that what is left is the lower bits alone; every number on the way is a whole number of steps that fp32 holds, so results
are exact."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
FEW, MANY = 5, 70                                       # rows: tiles of 16, whose sums stay in registers, and of 32, whose sums pass through LDS


@pytest.fixture(scope="module")
def e0m4():
    import paper_2403_20041_amd as pkg

    pkg.lib()
    return pkg


def run(e0m4, dtype, rows, rank, x, a, b, scale=1.0):
    """Every row is x (by column), every adapter's rank r has a[r] (by column) and b[r] for all outputs."""
    K, N = 136, 72
    X = torch.zeros((rows, K), dtype=dtype)
    A, B = torch.zeros((1, rank, K), dtype=dtype), torch.zeros((1, N, rank), dtype=dtype)
    for k, v in x.items():
        X[:, k] = v
    for r, columns in a.items():
        for k, v in columns.items():
            A[0, r, k] = v
    for r, v in b.items():
        B[0, :, r] = v
    plan = e0m4.e0m4_groups(torch.zeros(rows, dtype=torch.int32, device=DEV), 1)
    return e0m4.e0m4_lora(X.to(DEV), plan, A.to(DEV), B.to(DEV), factors=torch.tensor([scale], device=DEV)).cpu().double()


@pytest.mark.parametrize("rows", [FEW, MANY])
@pytest.mark.parametrize("rank", [8, 24, 40, 128])
def test_bfloat16(e0m4, rows, rank):
    """A x = 141/256 + 133/2^16 + 9/2^23, 23 bits: three numbers of 8, without the first two."""
    x = {0: 1.0, 50: 2.0 ** -8, 135: 2.0 ** -15}
    a = {0: {0: 141 / 256, 50: 133 / 256, 135: 9 / 256}, rank - 1: {0: 141 / 256, 50: 133 / 256}}
    got = run(e0m4, torch.bfloat16, rows, rank, x, a, {0: 1.0, rank - 1: -1.0})
    assert (got == 9 * 2.0 ** -23).all()


@pytest.mark.parametrize("rows", [FEW, MANY])
@pytest.mark.parametrize("rank", [8, 24, 40, 128])
def test_float16(e0m4, rows, rank):
    """A x = 1501/2^11 + 4095/2^24, 24 bits, of which 4095 are a bit more than two numbers of 11 hold, without all but the last two."""
    x = {0: 1.0, 50: 2.0 ** -11, 135: 2.0 ** -12}
    a = {0: {0: 1501 / 2048, 50: 1023 / 2048, 135: 3 * 2.0 ** -12}, rank - 1: {0: 1501 / 2048, 50: 1023 / 2048}}
    got = run(e0m4, torch.float16, rows, rank, x, a, {0: 1.0, rank - 1: -1.0}, scale=2.0 ** 12)
    assert (got == 3 * 2.0 ** -12).all()


@pytest.mark.parametrize("rows", [FEW, MANY])
@pytest.mark.parametrize("rank", [8, 24, 40, 128])
@pytest.mark.parametrize("least", [-13, -20])
def test_float16_far_below_the_largest_of_its_row(e0m4, rows, rank, least):
    """One number of the rank is a power of two, the others 2^-13 and 2^-20 of it: 1501/2^11 + 1377/2^22 without the first 11 bits.  Steps of 2^-38 of the
    largest are kept, half of one may be lost."""
    x = {0: 1.0, 50: 2.0 ** -11, 135: 2.0 ** 10}
    a = {0: {0: 1501 / 2048, 50: 1377 / 2048}, 3: {135: 2.0 ** (-least - 10)}, rank - 1: {0: 1501 / 2048}}
    got = run(e0m4, torch.float16, rows, rank, x, a, {0: 1.0, rank - 1: -1.0}, scale=2.0 ** 12)
    assert ((got - 1377 * 2.0 ** -10).abs() <= (0.0 if least == -13 else 2.0 ** (-least - 39 + 12))).all()
