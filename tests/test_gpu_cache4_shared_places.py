"""Two tokens appended to one place of a 4-bit cache: what is said to be found there, and nothing beside it."""
import pytest
import torch

import paper_2507_17245_amd as da
from cache4_util import encode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
def test_codes_of_eight_channels_and_scales_come_from_either_token(d, dtype):
    Hkv, page, n = 3, 16, 40
    g = torch.Generator().manual_seed(d)
    x = (torch.randn(2, 2, n, Hkv, d, generator=g) * torch.tensor([1.0, 300.0])[:, None, None, None, None]).to(dtype)   # (k or v of both sequences)
    k, v = (torch.cat((x[0, i], x[1, i])) for i in (0, 1))
    cache = tuple(torch.full((5, Hkv, page, w), 7, dtype=torch.uint8, device="cuda") for w in (d // 2, d // 32) * 2)
    table = torch.tensor([[3, 1, 4], [3, 1, 4]], dtype=torch.int32, device="cuda")   # the same pages
    kv_len, start = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([n, n], [0, n, 2 * n]))
    dk, dv = k.cuda(), v.cuda()
    da.distr_attn_cache4_append(dk, dv, cache, da.make_paged4_params(cache, table, kv_len, start, k=dk, v=dv))
    codes_of = lambda t: t[[3, 1, 4]].transpose(1, 2).reshape(3 * page, Hkv, -1)   # noqa: E731
    for i, rows in enumerate((k, v)):
        (codes, scales), (codes2, scales2) = (encode(rows[at:at + n].double()) for at in (0, n))
        assert (scales != scales2).all()
        got, got_scales = (codes_of(t.cpu()) for t in cache[2 * i:2 * i + 2])
        for mine, one, other, each in ((got, codes, codes2, 4), (got_scales, scales, scales2, 1)):
            mine, one, other = (t.unflatten(-1, (-1, each)) for t in (mine[:n], one, other))
            assert ((mine == one).all(-1) | (mine == other).all(-1)).all()
        assert (got[n:] == 7).all() and (got_scales[n:] == 7).all()
        for t in cache[2 * i:2 * i + 2]:
            assert (t[[0, 2]] == 7).all()
