"""The cache held in 4 bits without a GPU: its mirror of the header, calls that are refused before anything is launched, the plain implementation."""
import ctypes
import math
import os
import re

import pytest
import torch

import paper_2507_17245_amd as da
from cache4_util import MAGNITUDES, decode, encode

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = [ctypes.c_void_p(0x10000 * (i + 1)) for i in range(8)]   # never dereferenced: every call below fails on the host first


def test_mirror_follows_the_header():
    header = open(os.path.join(ROOT, "include", "distr_attn.h")).read()
    body = header[:header.index("} da_cache4;")]
    body = re.sub(r"/\*.*?\*/", "", body[body.rindex("typedef struct {"):], flags=re.S).split("{", 1)[1]
    fields = [re.search(r"(\w+)\s*(\[\d+\])?\s*$", part.strip()).group(1) for decl in body.split(";") if decl.strip() for part in decl.split(",")]
    assert fields == [f[0] for f in da.DaCache4._fields_]


def _batch(**kw):
    p = da.DaPaged()
    base = dict(H=4, Hkv=2, d=64, dtype=da.DA_BF16, n_seq=2, n_tokens=3, n_pages=8, page_size=16, max_pages=4, page_table=0x1000, kv_len=0x2000,
                q_start=0x3000, causal=1)
    base.update(kw)
    for k, v in base.items():
        if k.endswith("stride"):
            getattr(p, k)[:] = v
        else:
            setattr(p.rotary if hasattr(p.rotary, k) else p, k, v)
    for s, h in (("q_stride", p.H), ("k_stride", p.Hkv), ("v_stride", p.Hkv)):
        if s not in base:
            getattr(p, s)[:] = [h * p.d, p.d]
    return p


def _cache(**kw):
    c = da.DaCache4()
    base = dict(k_codes=0x100000, k_scales=0x200000, v_codes=0x300000, v_scales=0x400000, code_stride=[2 * 16 * 32, 16 * 32, 32], scale_stride=[2 * 16 * 2, 16 * 2, 2])
    base.update(kw)
    for k, v in base.items():
        if k.endswith("stride"):
            getattr(c, k)[:] = v
        else:
            setattr(c, k, v)
    return c


def _all(c, p):
    L = da.lib()
    ref = ctypes.byref(c) if c is not None else None
    return [f(P[0], P[1], ref, ctypes.byref(p)) for f in (L.distr_attn_cache4_append, L.distr_attn_cache4_read, L.distr_attn_paged4_fwd)]


BATCH = [(dict(H=0), -1), (dict(Hkv=0), -1), (dict(H=3), -1), (dict(d=32), -2), (dict(d=96), -2), (dict(d=0), -1), (dict(dtype=9), -1), (dict(n_seq=0), -1),
         (dict(n_tokens=-1), -1), (dict(n_pages=0), -1), (dict(page_size=0), -1), (dict(page_size=24), -2), (dict(max_pages=0), -1),
         (dict(max_pages=1 << 27), -2), (dict(page_table=None), -1), (dict(kv_len=0x2002), -1), (dict(q_start=0x3001), -1),
         (dict(n_tokens=1 << 28, H=64, Hkv=1), -2)]


@pytest.mark.parametrize("kw,code", BATCH)
def test_batches_are_refused(kw, code):
    p = _batch(**kw)
    assert _all(_cache(), p) == [code] * 3
    assert da.distr_attn_paged4_workspace_bytes(p) == 0
    assert da.lib().distr_attn_last_error()


CACHE = [(dict(k_codes=None), -1), (dict(v_scales=None), -1), (dict(k_codes=0x100008), -1), (dict(v_codes=0x300004), -1), (dict(k_scales=0x200002), -1),
         (dict(k_codes=0x300000), -1), (dict(k_scales=0x400000), -1), (dict(v_scales=0x100000), -1), (dict(code_stride=[1024, 512, 24]), -1),
         (dict(code_stride=[1024, 512, 16]), -1), (dict(code_stride=[1024, -512, 32]), -1), (dict(code_stride=[0, 512, 32]), -1),
         (dict(scale_stride=[64, 32, 1]), -1), (dict(scale_stride=[64, 32, 3]), -1), (dict(scale_stride=[64, 0, 2]), -1), (dict(code_stride=[1 << 41, 512, 32]), -1),
         (dict(code_stride=[1 << 30, 1 << 29, 1 << 26]), -2), (dict(scale_stride=[1 << 30, 1 << 29, 1 << 26]), -2)]


@pytest.mark.parametrize("kw,code", CACHE)
def test_caches_are_refused(kw, code):
    assert _all(_cache(**kw), _batch()) == [code] * 3
    assert _all(None, _batch()) == [-1] * 3


def test_strides_of_a_single_entry_do_not_matter():
    one = _batch(n_pages=1, Hkv=1, H=4, n_tokens=0)
    assert _all(_cache(code_stride=[0, 7, 32], scale_stride=[-1, 0, 2]), one) == [0] * 3   # (no tokens: nothing to launch)


def test_pointers_and_options():
    L, c, p = da.lib(), _cache(), _batch()
    odd = ctypes.c_void_p(0x10008)
    at = {name: ctypes.c_void_p(getattr(c, name)) for name in ("k_codes", "k_scales", "v_codes", "v_scales")}
    for f in (L.distr_attn_cache4_append, L.distr_attn_cache4_read, L.distr_attn_paged4_fwd):
        for a, b in ((None, P[1]), (P[0], None), (odd, P[1]), (P[0], odd)):
            assert f(a, b, ctypes.byref(c), ctypes.byref(p)) == -1
        assert f(P[0], P[1], ctypes.byref(c), None) == -1
    for name in at:
        assert L.distr_attn_cache4_append(P[0], at[name], ctypes.byref(c), ctypes.byref(p)) == -1
        assert L.distr_attn_cache4_read(at[name], P[1], ctypes.byref(c), ctypes.byref(p)) == -1
        assert L.distr_attn_paged4_fwd(P[0], at[name], ctypes.byref(c), ctypes.byref(p)) == -1
    assert L.distr_attn_cache4_read(P[0], P[0], ctypes.byref(c), ctypes.byref(p)) == -1
    assert L.distr_attn_paged4_fwd(P[0], P[0], ctypes.byref(c), ctypes.byref(p)) == -1

    def attention(**kw):
        return L.distr_attn_paged4_fwd(P[0], P[1], ctypes.byref(c), ctypes.byref(_batch(**kw)))
    for kw in (dict(causal=2), dict(softmax_scale=-1.0), dict(softmax_scale=math.inf), dict(softmax_scale=math.nan), dict(q_stride=[256, 60]),
               dict(q_stride=[-256, 64]), dict(lse_out=0x10002), dict(workspace=0x10010, workspace_bytes=1 << 30)):
        assert attention(**kw) == -1

    def append(**kw):
        return L.distr_attn_cache4_append(P[0], P[1], ctypes.byref(c), ctypes.byref(_batch(**kw)))
    for kw in (dict(norm=2), dict(norm=1, eps=-1.0), dict(norm=1, k_weight=0x1008), dict(rope=3), dict(rope=1, rot_dim=24, n_pos=1, cos_table=0x1000, sin_table=0x1000),
               dict(rope=1, rot_dim=64, n_pos=0, cos_table=0x1000, sin_table=0x1000), dict(rope=1, rot_dim=64, n_pos=4), dict(positions=0x1002),
               dict(k_stride=[128, 60]), dict(v_stride=[128, -64])):
        assert append(**kw) == -1
    read = _batch(k_stride=[0, 64])   # written: rows in one place
    assert L.distr_attn_cache4_read(P[0], P[1], ctypes.byref(c), ctypes.byref(read)) == -1


def test_nothing_to_do():
    assert _all(_cache(), _batch(n_tokens=0)) == [0] * 3


def test_the_binding_checks_what_it_marshals():
    codes, scales = torch.zeros(4, 2, 16, 32, dtype=torch.uint8), torch.zeros(4, 2, 16, 2, dtype=torch.uint8)
    index = (torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32))
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    good = (codes, scales, codes.clone(), scales.clone())
    for cache in ((codes[..., :16], *good[1:]), (codes, scales[..., :1], codes, scales[..., :1]), (codes.int(), scales, codes.int(), scales),
                  (codes, scales, codes.transpose(1, 2), scales), (codes[..., ::2], scales, codes[..., ::2], scales), (codes[0], scales, codes[0], scales)):
        with pytest.raises((ValueError, TypeError)):
            da.make_paged4_params(cache, *index, q=q)
    for kw in (dict(), dict(q=q[0]), dict(k=q[:, :2]), dict(q=q[..., :32]), dict(k=q, v=q), dict(q=q, k=q[:, :2].float(), v=q[:, :2].float()), dict(q=q)):   # (the last: not on a GPU)
        with pytest.raises((ValueError, TypeError)):
            da.make_paged4_params(good, *index, **kw)


def test_plain_encoding():
    """Ties to the even code, the smallest scale that leaves none beyond 7 times it, limits."""
    x = torch.zeros(9, 32, dtype=torch.float64)
    x[0, :9] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.75])
    x[1, 0], x[2, 0] = 7.0, 7.0 + 1e-12
    x[3, 0], x[4, 0], x[5, 0] = 3.4e38, 1e300, 1e-45
    x[6, 0], x[7, 0], x[8, 0] = math.inf, math.nan, -3.5000001
    codes, scales = encode(x)
    assert scales.squeeze(-1).tolist() == [127, 127, 128, 252, 252, 1, 255, 255, 127]
    assert decode(codes, scales)[0, :9].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, -1.0]
    assert decode(codes, scales)[3, 0] == 6 * 2.0 ** 125 == decode(codes, scales)[4, 0] and (codes[6:8] == 0).all()
    assert decode(codes, scales)[8, 0] == -4.0
    g = torch.Generator().manual_seed(1)
    y = torch.randn(200, 64, generator=g, dtype=torch.float64) * torch.exp(3 * torch.randn(200, 1, generator=g, dtype=torch.float64))
    codes, scales = encode(y)
    step = torch.tensor([2.0 ** (int(e) - 127) for e in scales.flatten()]).view(200, 2, 1).double()
    a = y.unflatten(-1, (2, 32)).abs() / step
    assert (a <= 7).all() and (a.amax(-1) > 3.5).all()
    nearest = (a[..., None] - MAGNITUDES).abs().amin(-1)
    assert torch.equal((decode(codes, scales) - y).abs().unflatten(-1, (2, 32)) / step, nearest)
