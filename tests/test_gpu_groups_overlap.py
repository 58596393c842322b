"""A layout is not made from an index inside it."""
import pytest
import torch

from test_gpu_groups import DEV, e0m4  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def test_index_inside_its_own_layout_is_refused(e0m4):  # noqa: F811
    plan = e0m4.e0m4_groups_alloc(300, 4, DEV)
    before = plan.data.clone()
    for index in (plan.order, plan.place, plan.data[:300], plan.data[-300:]):
        with pytest.raises(ValueError):
            e0m4.e0m4_groups(index, 4, plan=plan)
    assert torch.equal(plan.data, before)
    other = e0m4.e0m4_groups(plan.order, 4)             # a part of another layout is an index like any
    assert other.offsets.tolist() == [0, 300, 300, 300, 300]
