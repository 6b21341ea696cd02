"""Calls on caches in 4 bits, rotations and caches without sequences that the runner refuses before anything is allocated or
enqueued (no GPU needed)."""
import pytest

import paper_2607_02612_gb300 as fz
from paper_2607_02612_gb300 import runner


@pytest.mark.parametrize("head_dim", [-64, -1, 0, 1, 16, 33, 48, 63, 65, 80, 129])
def test_packed_caches_of_other_dims_are_refused(head_dim):
    """Two dims share a byte, so that an odd number of them would pass for the even one below."""
    with pytest.raises(fz.FusionError, match="head_dim"):
        runner.device_packed_cache("bf16", 2, 8, 2, 2, head_dim, device="cpu")
    with pytest.raises(fz.FusionError, match="device tensors"):
        runner.device_packed_cache("bf16", 2, 8, 2, 2, 64, device="cpu")


def test_rotation_tables_of_odd_dims_are_refused():
    """A pair has two dims: the table of an odd number had a column fewer and the angles of none that a Rotation takes."""
    for dims in (-16, -1, 0, 1, 17, 33, 65):
        with pytest.raises(fz.FusionError, match="dims"):
            runner.rotation_table(10, dims, device="cpu")
    assert runner.rotation_table(10, 2, device="cpu").shape == (10, 2)
    assert runner.rotation_table(0, 32, device="cpu").shape == (0, 32)
