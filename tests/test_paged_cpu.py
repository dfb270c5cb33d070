"""The operators around attention without a GPU: mirrors of the header's structures, and calls that are refused before anything is launched."""
import ctypes
import os
import re

import pytest
import torch

import paper_2507_17245_amd as da

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = [ctypes.c_void_p(0x10000 * (i + 1)) for i in range(8)]   # never dereferenced: every call below fails on the host first


@pytest.mark.parametrize("name,mirror", [("da_rotary", da.DaRotary), ("da_qk", da.DaQk), ("da_paged", da.DaPaged)])
def test_mirrors_follow_the_header(name, mirror):
    header = open(os.path.join(ROOT, "include", "distr_attn.h")).read()
    body = header[:header.index("} %s;" % name)]
    body = re.sub(r"/\*.*?\*/", "", body[body.rindex("typedef struct {"):], flags=re.S).split("{", 1)[1]
    fields = []
    for decl in filter(None, (x.strip() for x in body.split(";"))):
        for part in decl.split(","):
            fields.append(re.search(r"(\w+)\s*(\[\d+\])?\s*$", part.strip()).group(1))
    assert fields == [f[0] for f in mirror._fields_]


def _qk(**kw):
    p = da.DaQk()
    base = dict(B=2, H=4, Hkv=2, N=10, d=64, dtype=da.DA_BF16, norm=1, eps=1e-6, rope=1, rot_dim=64, n_pos=10, cos_table=0x1000, sin_table=0x2000)
    base.update(kw)
    for k, v in base.items():
        if k.endswith("stride"):
            getattr(p, k)[:] = v
        else:
            setattr(p.rotary if hasattr(p.rotary, k) else p, k, v)
    for s, h in (("q_stride", p.H), ("k_stride", p.Hkv), ("q_out_stride", p.H), ("k_out_stride", p.Hkv)):
        if s not in base:
            getattr(p, s)[:] = [h * p.N * p.d, p.N * p.d, p.d]
    return p


QK = [(dict(B=0), -1), (dict(N=0), -1), (dict(Hkv=-1), -1), (dict(d=80), -2), (dict(d=0), -1), (dict(dtype=7), -1), (dict(norm=2), -1), (dict(eps=-1.0), -1),
      (dict(eps=float("nan")), -1), (dict(rope=3), -1), (dict(rot_dim=24), -1), (dict(rot_dim=128), -1), (dict(rot_dim=0), -1), (dict(n_pos=0), -1),
      (dict(cos_table=None), -1), (dict(sin_table=0x2004), -1), (dict(weight_dtype=5), -1), (dict(q_weight=0x1008), -1),
      (dict(q_stride=[2560, 640, 68]), -1), (dict(k_stride=[1280, -640, 64]), -1), (dict(q_out_stride=[2560, 32, 64]), -1), (dict(positions=0x1001), -1),
      (dict(B=1 << 20, N=1 << 20), -2)]


@pytest.mark.parametrize("kw,code", QK)
def test_qk_calls_are_refused(kw, code):
    L, p = da.lib(), _qk(**kw)
    assert L.distr_attn_qk_norm_rope(P[0], P[1], P[2], P[3], ctypes.byref(p)) == code
    if "q_out_stride" not in kw:   # (read by the backward)
        assert L.distr_attn_qk_norm_rope_bwd(P[0], P[1], P[2], P[3], P[4], P[5], None, None, ctypes.byref(p)) == code
        assert da.distr_attn_qk_bwd_workspace_bytes(p) == 0
    assert L.distr_attn_last_error()


def test_qk_pointers():
    L, p, alone, plain = da.lib(), _qk(), _qk(Hkv=0), _qk(norm=0)
    odd = ctypes.c_void_p(0x10008)
    none = None

    def forward(q, k, qo, ko, p=p):
        return L.distr_attn_qk_norm_rope(q, k, qo, ko, ctypes.byref(p))

    def backward(*a, p=p):
        return L.distr_attn_qk_norm_rope_bwd(*a, ctypes.byref(p))
    assert L.distr_attn_qk_norm_rope(P[0], P[1], P[2], P[3], None) == -1
    for a in ((none, P[1], P[2], P[3]), (P[0], none, P[2], P[3]), (P[0], P[1], none, P[3]), (P[0], P[1], P[2], none), (odd, P[1], P[2], P[3]),
              (P[0], P[1], P[2], odd), (P[0], P[1], P[2], P[2]), (P[0], P[1], P[1], P[3]), (P[0], P[1], P[2], P[0])):
        assert forward(*a) == -1
    assert forward(P[0], P[1], P[2], P[3], alone) == -1           # keys without heads
    other = _qk(q_out_stride=[2560, 64, 256])
    assert forward(P[0], P[1], P[0], P[3], other) == -1           # in place, other strides
    assert backward(P[0], P[1], P[2], P[3], P[2], P[5], none, none, p=other) == -1
    for a in ((none, P[1], P[2], P[3], P[4], P[5]), (P[0], none, P[2], P[3], P[4], P[5]), (P[0], P[1], none, P[3], P[4], P[5]), (P[0], P[1], P[2], P[3], none, P[5]),
              (P[0], P[1], P[2], P[3], P[4], P[4]), (P[0], P[1], P[2], P[3], P[0], P[5]), (P[0], P[1], P[2], P[3], P[4], P[2])):
        assert backward(*a, none, none) == -1
    assert backward(P[0], P[1], P[2], P[3], P[4], P[5], P[6], none, p=plain) == -1     # a weight's gradient without a norm
    assert backward(P[0], none, P[2], none, P[4], none, P[6], P[7], p=alone) == -1
    broadcast = _qk(q_stride=[0, 640, 64])
    assert backward(P[0], P[1], P[2], P[3], P[4], P[5], none, none, p=broadcast) == -1   # dq has q's strides: rows in one place
    small = _qk(workspace=0x100000, workspace_bytes=16)
    assert backward(P[0], P[1], P[2], P[3], P[4], P[5], P[6], P[7], p=small) == da.DA_ERR_WORKSPACE
    small.workspace, small.workspace_bytes = 0x100010, 1 << 30
    assert backward(P[0], P[1], P[2], P[3], P[4], P[5], P[6], P[7], p=small) == -1


def _paged(**kw):
    p = da.DaPaged()
    base = dict(H=4, Hkv=2, d=64, dtype=da.DA_BF16, n_seq=3, n_tokens=5, n_pages=9, page_size=16, max_pages=4, page_stride=2048, head_stride=1024,
                row_stride=64, page_table=0x1000, kv_len=0x2000, q_start=0x3000, causal=1)
    strides = dict(q_stride=[256, 64], k_stride=[128, 64], v_stride=[128, 64])
    for k, v in {**base, **strides, **kw}.items():
        if k in strides:
            getattr(p, k)[:] = v
        else:
            setattr(p.rotary if hasattr(p.rotary, k) else p, k, v)
    return p


PAGED = [(dict(H=0), -1), (dict(H=5), -1), (dict(Hkv=0), -1), (dict(d=96), -2), (dict(dtype=2), -1), (dict(n_seq=0), -1), (dict(n_tokens=-1), -1), (dict(n_pages=0), -1),
         (dict(page_size=0), -1), (dict(page_size=24), -2), (dict(max_pages=0), -1), (dict(max_pages=1 << 27), -2), (dict(row_stride=60), -1), (dict(row_stride=32), -1),
         (dict(head_stride=0), -1), (dict(page_stride=-64), -1), (dict(row_stride=1 << 26), -2), (dict(page_table=None), -1), (dict(kv_len=0x2001), -1), (dict(q_start=None), -1),
         (dict(n_tokens=1 << 30), -2)]


@pytest.mark.parametrize("kw,code", PAGED)
def test_paged_calls_are_refused(kw, code):
    L, p = da.lib(), _paged(**kw)
    assert L.distr_attn_paged_fwd(P[0], P[1], P[2], P[3], ctypes.byref(p)) == code
    assert L.distr_attn_cache_append(P[0], P[1], P[2], P[3], ctypes.byref(p)) == code
    assert da.distr_attn_paged_workspace_bytes(p) == 0


def test_paged_pointers():
    L, odd = da.lib(), ctypes.c_void_p(0x10008)

    def attend(a, **kw):
        return L.distr_attn_paged_fwd(*a, ctypes.byref(_paged(**kw)))

    def append(a, **kw):
        return L.distr_attn_cache_append(*a, ctypes.byref(_paged(**kw)))
    good = P[:4]
    for i in range(4):
        for x in (None, odd):
            a = good[:i] + [x] + good[i + 1:]
            assert attend(a) == -1 and append(a) == -1
    assert attend([P[0], P[1], P[2], P[0]]) == -1 and append([P[0], P[1], P[2], P[2]]) == -1 and append([P[0], P[1], P[0], P[3]]) == -1
    assert attend(good, causal=2) == -1 and attend(good, softmax_scale=-1.0) == -1 and attend(good, softmax_scale=float("inf")) == -1
    assert attend(good, q_stride=[252, 64]) == -1 and append(good, k_stride=[128, 60]) == -1 and append(good, v_stride=[-128, 64]) == -1
    assert attend(good, lse_out=0x1002) == -1 and attend(good, workspace=0x1010, workspace_bytes=1 << 30) == -1
    assert append(good, positions=0x1002) == -1 and append(good, rope=1, rot_dim=20) == -1 and append(good, norm=1, eps=-1.0) == -1
    # no new tokens: nothing to do, whatever the tensors are
    assert attend([None] * 4, n_tokens=0) == 0 and append([None] * 4, n_tokens=0) == 0


def test_workspace_does_not_depend_on_lengths():
    want = da.distr_attn_paged_workspace_bytes(_paged())
    assert 0 < want == da.distr_attn_paged_workspace_bytes(_paged(n_seq=1000, max_pages=1 << 16)) <= 128 << 20


def test_binding_wants_gpu_tensors():
    q, k = torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16), torch.zeros(1, 1, 3, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        da.make_qk_params(q, k, q, k, norm=True)
    pages = torch.zeros(4, 1, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        da.make_paged_params(pages, pages, torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), q=q[0].transpose(0, 1))
