"""A layout that nothing has written yet holds no entry."""
import pytest
import torch

from test_gpu_groups import DEV, e0m4, make_weights  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("own_stream", [False, True])
def test_new_layout_has_no_entries(e0m4, own_stream):  # noqa: F811
    rows, groups = 300, 4
    stream = torch.cuda.Stream() if own_stream else None
    with torch.cuda.stream(stream):
        torch.full((1 << 22,), -1, dtype=torch.int32, device=DEV)      # (memory that the allocator may give again)
    plan = e0m4.e0m4_groups_alloc(rows, groups, DEV, stream=stream)
    torch.cuda.synchronize()
    assert plan.offsets.tolist() == [0] * (groups + 1) and not plan.data.any()
    codes = make_weights(e0m4, "e0m4", groups, 64, 128, 128, 3)[0]
    x = torch.ones((rows, 128), dtype=torch.float16, device=DEV)
    for form in range(1, 7):
        out = torch.full((rows, 64), 5.0, dtype=torch.float16, device=DEV)
        e0m4.e0m4_set_knob("grouped_form", form)
        try:
            e0m4.e0m4_matmul_grouped(x, plan, codes, 64, 128, 128, share=1, out=out)
        finally:
            e0m4.e0m4_set_knob("grouped_form", 0)
        assert (out == 5.0).all()
    # ... and takes a layout as any other memory does
    index = torch.arange(rows, dtype=torch.int32, device=DEV) % groups
    assert torch.equal(e0m4.e0m4_groups(index, groups, plan=plan).order, e0m4.e0m4_groups(index, groups).order)


def test_new_layout_is_ready_on_every_stream(e0m4):  # noqa: F811
    """Its zeros are there when the call returns, whatever the stream that was current still has to do: they do not come behind what another stream writes."""
    rows, groups = 300, 4
    index = torch.arange(rows, dtype=torch.int32, device=DEV) % groups
    want = e0m4.e0m4_groups(index, groups)
    a = torch.ones((4096, 4096), device=DEV)
    side = torch.cuda.Stream()
    e0m4.e0m4_groups(index, groups, stream=side)       # (loads the kernel)
    torch.cuda.synchronize()
    for _ in range(40):
        b = a @ a                                       # (some milliseconds)
    plan = e0m4.e0m4_groups_alloc(rows, groups, DEV)
    e0m4.e0m4_groups(index, groups, plan=plan, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(plan.order, want.order) and torch.equal(plan.offsets, want.offsets) and torch.equal(plan.place, want.place)
    del b


def test_new_layout_in_a_captured_graph(e0m4):  # noqa: F811
    rows, groups = 300, 4
    index = torch.arange(rows, dtype=torch.int32, device=DEV) % groups
    e0m4.e0m4_groups(index, groups)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan = e0m4.e0m4_groups_alloc(rows, groups, DEV)
        e0m4.e0m4_groups(index, groups, plan=plan)
    for shift in range(3):
        index.copy_((torch.arange(rows, device=DEV) + shift) % groups)
        want = e0m4.e0m4_groups(index, groups)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(plan.order, want.order) and torch.equal(plan.place, want.place)
