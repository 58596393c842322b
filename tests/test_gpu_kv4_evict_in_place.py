"""Eviction through the C entry with the new lengths in the place of the old ones: every head of a sequence has to read the old one."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

import kv4_plain as plain  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("kv", [1, 2, 40, 600])
def test_lengths_in_place(kv):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' elsewhere)")
    import paper_2403_20041_amd as e0m4
    from paper_2403_20041_amd import binding

    gen = torch.Generator().manual_seed(kv)
    batch, capacity, dim, group, budget, recent = 4, 500, 64, 32, 120, 20
    old = [500, 97, 333, 700]
    shape = e0m4.E0M4KV4Shape(batch, kv, capacity, dim, group)
    small_shape = shape._replace(capacity=budget)
    cache, small = e0m4.e0m4_kv4_alloc(shape, DEV), e0m4.e0m4_kv4_alloc(small_shape, DEV)
    rows = torch.randn((batch, capacity, kv, dim), generator=gen).half().to(DEV)
    e0m4.e0m4_kv4_append(cache, shape, rows, rows, torch.zeros(batch, dtype=torch.int32, device=DEV))
    received = torch.rand((batch, kv, capacity), generator=gen)
    received_dev = received.to(DEV)
    want = plain.evict(received, [min(n, capacity) for n in old], budget, recent)
    stream = torch.cuda.current_stream().cuda_stream
    for _ in range(3):
        lengths = torch.tensor(old, dtype=torch.int32, device=DEV)
        kept = torch.empty((batch, kv, budget), dtype=torch.int32, device=DEV)
        received_out = torch.empty((batch, kv, budget), device=DEV)
        rc = binding.lib().e0m4_kv4_evict(cache.data_ptr(), ctypes.byref(binding._KV4Shape(*shape)), received_dev.data_ptr(), lengths.data_ptr(), budget, recent,
                                          small.data_ptr(), ctypes.byref(binding._KV4Shape(*small_shape)), kept.data_ptr(), lengths.data_ptr(),
                                          received_out.data_ptr(), stream)
        assert rc == 0
        assert torch.equal(kept.cpu(), want)
        assert lengths.tolist() == [120, 97, 120, 120]
    there = want >= 0
    picked = torch.where(there, received.gather(-1, want.clamp(min=0).long()), 0.0)
    assert torch.equal(received_out.cpu(), picked)
