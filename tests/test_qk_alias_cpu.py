"""Gradients of norms and rotation that would be written where another workgroup still reads, or where the other weight's sums go: refused on the host (no GPU)."""
import ctypes

import pytest

import paper_2507_17245_amd as da
from test_paged_cpu import P, _qk


@pytest.mark.parametrize("names", [("dq", "q"), ("dq", "k"), ("dq", "dk"), ("dq", "dk_out"), ("dk", "q"), ("dk", "k"), ("dk", "dq_out"), ("dq_weight", "dk_weight")])
def test_tensors_in_one_place_are_refused(names):
    at = dict(zip(("q", "k", "dq_out", "dk_out", "dq", "dk", "dq_weight", "dk_weight"), P))
    p = _qk(workspace=0x100000, workspace_bytes=16)
    call = lambda: da.lib().distr_attn_qk_norm_rope_bwd(*at.values(), ctypes.byref(p))   # noqa: E731
    assert call() == da.DA_ERR_WORKSPACE          # (each in its own place: the next check, of the scratch, is reached)
    at[names[0]] = at[names[1]]
    assert call() == -1
    assert b"alias" in da.lib().distr_attn_last_error()
