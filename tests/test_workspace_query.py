"""The workspace query takes every parameter block of the binding, and what is derived from one."""
import pytest

from paper_2603_01875_amd import kdloss as K


def _blocks():
    return [K.make_params(64, 128, 128, 1000), K.make_ce_params(64, 128, 1000), K.make_topk_params(64, 128, 1000, 5)]


@pytest.mark.parametrize("i", range(3))
def test_derived_blocks_are_accepted(i):
    block = _blocks()[i]
    derived = type("Derived", (type(block),), {})
    copy = derived(*[getattr(block, name) for name, _ in block._fields_])
    assert K.kd_loss_workspace_size(copy) == K.kd_loss_workspace_size(block) > 0


def test_anything_else_is_refused_by_name():
    with pytest.raises(TypeError, match="KdLossParams.*got dict"):
        K.kd_loss_workspace_size({})
