"""Calls on caches in 4 bits, rotations and caches without sequences that the runner refuses before anything is allocated or
enqueued (no GPU needed)."""
import os
import re
import types

import pytest
import torch

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


def test_samples_for_a_cache_without_sequences_are_refused(monkeypatch):
    """They name no sequence of it: nothing would be written to what the calls return."""
    monkeypatch.setattr(runner, "_enqueue", lambda *args: pytest.fail("enqueued"))
    none = torch.zeros(0, dtype=torch.int32)
    c = types.SimpleNamespace(max_batch=0, kv_heads=2, head_dim=64, heads=4, index=-1, torch_dtype=torch.float32, device="cpu", lengths=none,
                              code=0, _ws=0, ws_bytes=0, c_struct=lambda: None, one_row_each=lambda: rows(0, 0),
                              lib=types.SimpleNamespace(fusion_cache_append_rotated=None, fusion_cache_read=None))
    f, rot = types.SimpleNamespace(status=None), types.SimpleNamespace(table=torch.zeros(9, 64), c_struct=lambda p: None)

    def rows(batch, n):
        return types.SimpleNamespace(max_batch=batch, max_tokens=1, max_rows=n, offsets=torch.zeros(batch + 1, dtype=torch.int32), batch=None,
                                     ids=None, ragged=lambda: None)

    k, q = torch.zeros(3, 2, 64), torch.zeros(3, 7, 64)
    with pytest.raises(fz.FusionError, match="no sequences"):
        runner.Fusion.cache_read(f, c, rows(3, 3))
    for kw in (dict(q=q), dict(q=q, q_out=torch.zeros(3, 7, 64)), {}):
        with pytest.raises(fz.FusionError, match="no sequences"):
            runner.Fusion.cache_append_rotated(f, c, k, k, rot, rows(3, 3), **kw)
    # no samples, as before: nothing to do
    assert runner.Fusion.cache_append_rotated(f, c, k[:0], k[:0], rot, q=q[:0]).shape == (0, 7, 64)
    assert runner.Fusion.cache_append_rotated(f, c, k, k, rot, rows(0, 3), q=q).shape == (3, 7, 64)
    assert [t.shape for t in runner.Fusion.cache_read(f, c, rows(0, 5))] == [(5, 2, 64)] * 2


@pytest.mark.parametrize("name", ["cache_store.cu", "cache_read.cu", "packed_attn.cu", "cache_rows.cuh", "cache_rounds.cuh", "fp4.cuh"])
def test_no_number_of_multiprocessors_in_the_sources(name):
    """How many CTAs a device holds at once is asked of it, not written down (comments may speak of the one that was measured)."""
    text = open(os.path.join(os.path.dirname(fz.__file__), "csrc", name)).read()
    assert not re.findall(r"\b(?:152|148|144|132)\b", re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S))
