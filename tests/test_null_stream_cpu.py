"""What the binding tells the library of the stream in calls around attention: the parameters carry it, the process-wide setting is not touched (no GPU)."""
import ctypes

import pytest
import torch

import paper_2507_17245_amd as da

LEGACY = 1   # hipStreamLegacy


class Recorder:
    """The library, of which the entry points called are written down."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return da.DA_OK
        return call


@pytest.mark.parametrize("current,carried", [(None, LEGACY), (0x1234000, 0x1234000)])
@pytest.mark.parametrize("params,name,n", [(da.DaQk, "distr_attn_qk_norm_rope", 4), (da.DaQk, "distr_attn_qk_norm_rope_bwd", 8),
                                           (da.DaPaged, "distr_attn_cache_append", 4), (da.DaPaged, "distr_attn_paged_fwd", 4)])
def test_parameters_carry_their_stream(params, name, n, current, carried, monkeypatch):
    monkeypatch.setattr(da, "_current_stream", lambda: ctypes.c_void_p(current))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    recorder = Recorder()
    monkeypatch.setattr(da, "_lib", recorder)
    p = params()
    da._fill_workspace(p, None, torch.device("cuda", 0))
    da._run(name, p, *[None] * n)
    assert p.stream == carried and recorder.calls == [name]
