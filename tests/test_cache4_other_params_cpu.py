"""Parameters made for one kind of paged cache in a call over the other kind: refused with the binding's own error."""
import pytest
import torch

import paper_2507_17245_amd as da


def _params(**layouts):
    p = da.DaPaged()
    p.layouts = layouts
    return p


def test_params_of_the_other_cache_are_refused():
    q, k = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    pages = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    cache = tuple(torch.zeros(4, 2, 16, n, dtype=torch.uint8) for n in (32, 2, 32, 2))
    rows = dict(q=da._layout(q), k=da._layout(k), v=da._layout(k))
    plain, four = _params(pages=da._layout(pages), **rows), _params(cache=da._cache_layout(*cache), **rows)
    for call in (lambda: da.distr_attn_cache_append(k, k.clone(), pages, pages.clone(), four), lambda: da.distr_attn_paged_fwd(q, pages, pages.clone(), q.clone(), four),
                 lambda: da.distr_attn_cache4_append(k, k.clone(), cache, plain), lambda: da.distr_attn_cache4_read(k, k.clone(), cache, plain),
                 lambda: da.distr_attn_paged4_fwd(q, cache, q.clone(), plain)):
        with pytest.raises(ValueError, match="params were made for"):
            call()
