"""Adapters beside the attention block's output projection: what e0m4_lora will not take is refused before rows leave the cache or are appended, and adapters that
it cannot read are refused when they are given.  The operators are stand-ins; no GPU."""
import pytest

torch = pytest.importorskip("torch")

from paper_2403_20041_amd import kv4_layer  # noqa: E402
from test_kv4_layer_refusals import calls, full_block  # noqa: E402,F401  (a fixture)


@pytest.fixture
def adapters(monkeypatch, calls):  # noqa: F811
    """lora refuses rows of 2 GiB and more and rows that do not begin at 16 bytes, as the library does."""
    def lora(x, plan, a, b, factors=None, base=None, out=None):
        if x.numel() * 2 >= 1 << 31 or a.data_ptr() % 16 or b.data_ptr() % 16:
            raise kv4_layer.e0m4.E0M4Error(-2, "e0m4_lora")
        calls.append("lora")

    monkeypatch.setattr(kv4_layer.e0m4, "e0m4_lora", lora)
    monkeypatch.setattr(kv4_layer.e0m4, "e0m4_groups", lambda index, groups: calls.append("groups"))
    return calls


def block_with_adapters(most, capacity):
    block = full_block(most, capacity)
    block.gamma = torch.ones(256, dtype=torch.float16)
    block.add_adapters(torch.zeros((3, 16, 256), dtype=torch.float16), torch.zeros((3, 256, 16), dtype=torch.float16))
    return block


@pytest.mark.parametrize("most", [0, 300])
def test_more_tokens_than_the_adapters_take(adapters, most):
    n = 1 << 21                                         # two sequences of 2^21 rows of 512 bytes: 2 GiB (memory that nothing touches)
    block = block_with_adapters(most, capacity=n + 350)
    adapter = torch.tensor([0, -1], dtype=torch.int32)
    received, lengths = block.received, block.lengths
    with pytest.raises(ValueError):
        block(torch.empty((2, n, 256), dtype=torch.float16), adapter=adapter)
    assert not adapters and block.most == most and block.received is received and block.lengths is lengths and lengths.tolist() == [most] * 2


def test_tokens_that_the_adapters_take(adapters):
    block = block_with_adapters(0, 1100)
    block(torch.zeros((2, 20, 256), dtype=torch.float16), adapter=torch.tensor([2, 0], dtype=torch.int32))
    assert adapters == ["matmul", "append", "attention", "matmul", "groups", "lora"] and block.most == 20


def test_adapters_that_do_not_begin_at_16_bytes(adapters):
    block = full_block(0)
    block.gamma = torch.ones(256, dtype=torch.float16)
    a, b = torch.zeros((3, 16, 256), dtype=torch.float16), torch.zeros((3, 256, 16), dtype=torch.float16)
    off = lambda t: torch.zeros(t.numel() + 4, dtype=torch.float16)[4:].view(t.shape)  # noqa: E731
    for bad in ((off(a), b), (a, off(b))):
        with pytest.raises(ValueError):
            block.add_adapters(*bad)
    assert block.adapters is None
    block.add_adapters(a, b)
