"""The calls over a 4-bit cache with starts, lengths and page tables that make no sense: no access leaves the buffers, as test_gpu_paged_starts.py has it for
the other cache."""
import pytest
import torch

import paper_2507_17245_amd as da
from test_gpu_paged import BF, F
from test_gpu_paged_starts import KINDS, Guarded, _starts

pytestmark = pytest.mark.gpu


class Call:
    def __init__(self, n_seq, n_tokens, H, Hkv, d, dtype, page, max_pages, n_pages=7):
        g = torch.Generator().manual_seed(n_seq + d)
        self.n_pages = n_pages
        self.parts = [Guarded((n_pages, Hkv, page, w), torch.uint8) for w in (d // 2, d // 32) * 2]
        for i, x in enumerate(self.parts):
            x.t.copy_(torch.randint(*((0, 256) if i % 2 == 0 else (120, 128)), x.t.shape, generator=g, dtype=torch.uint8))
        self.cache = tuple(x.t for x in self.parts)
        self.table = torch.randint(0, n_pages, (n_seq, max_pages), generator=g).to(torch.int32).cuda()
        self.kv_len = torch.full((n_seq,), max_pages * page, dtype=torch.int32, device="cuda")
        self.start = torch.zeros(n_seq + 1, dtype=torch.int32, device="cuda")
        self.q = torch.randn(n_tokens, H, d, generator=g).to(dtype).cuda()
        self.kv = torch.randn(n_tokens, 2, Hkv, d, generator=g).to(dtype).cuda()
        self.o, self.lse = Guarded((n_tokens, H, d), dtype), Guarded((n_tokens, H), F)
        self.back = [Guarded((n_tokens, Hkv, d), dtype) for _ in range(2)]
        self.index = (self.table, self.kv_len, self.start)
        self.ws = Guarded((da.distr_attn_paged4_workspace_bytes(da.make_paged4_params(self.cache, *self.index, q=self.q)),), torch.uint8)

    def _held(self):
        torch.cuda.synchronize()
        assert all(x.margins_hold() for x in (*self.parts, self.o, self.lse, self.ws, *self.back))

    def attend(self, start, scratch=None, causal=True):
        self.start.copy_(torch.as_tensor(start, dtype=torch.int32))
        self.ws.t.fill_(255)
        ws = self.ws.t if scratch is None else self.ws.t[:scratch]
        p = da.make_paged4_params(self.cache, *self.index, q=self.q, lse_out=self.lse.t, workspace=ws, causal=causal)
        da.distr_attn_paged4_fwd(self.q, self.cache, self.o.t, p)
        self._held()
        assert scratch is None or (self.ws.t[scratch:] == 255).all()

    def move(self, start):
        self.start.copy_(torch.as_tensor(start, dtype=torch.int32))
        k, v, (k_back, v_back) = self.kv[:, 0], self.kv[:, 1], (x.t for x in self.back)
        da.distr_attn_cache4_append(k, v, self.cache, da.make_paged4_params(self.cache, *self.index, k=k, v=v, norm=True))
        da.distr_attn_cache4_read(k_back, v_back, self.cache, da.make_paged4_params(self.cache, *self.index, k=k_back, v=v_back))
        self._held()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n_seq,n_tokens,H,Hkv,d,page,max_pages", [
    (3, 40, 8, 2, 64, 16, 4), (3, 200, 8, 2, 128, 16, 300), (75, 180, 8, 4, 64, 32, 160), (75, 180, 8, 4, 128, 32, 4),
    (200, 150, 8, 2, 64, 16, 250), (300, 200, 4, 4, 128, 16, 100), (4, 700, 64, 64, 64, 64, 12), (40, 40, 8, 2, 128, 16, 300)])
def test_starts_in_any_order(kind, dtype, n_seq, n_tokens, H, Hkv, d, page, max_pages):
    c = Call(n_seq, n_tokens, H, Hkv, d, dtype, page, max_pages)
    start = _starts(kind, n_seq, n_tokens)
    for length in (max_pages * page, 2 ** 31 - 1, 5, -3):
        c.kv_len.fill_(length)
        c.attend(start)
        c.attend(start, scratch=1 << 20, causal=False)
        c.move(start)
    c.table.copy_(torch.randint(-2 ** 31, 2 ** 31 - 1, c.table.shape).to(torch.int32))
    c.kv_len.fill_(max_pages * page)
    c.attend(start)
    c.move(start)
    # and a batch in order afterwards is as it was
    c.table.copy_(torch.randint(0, c.n_pages, c.table.shape, generator=torch.Generator().manual_seed(1)).to(torch.int32))
    c.attend([n_tokens * i // n_seq for i in range(n_seq + 1)])
    assert c.o.t.isfinite().all() and c.lse.t.isfinite().all()


@pytest.mark.parametrize("n_seq", [64, 65, 4200])
@pytest.mark.parametrize("dtype", [BF, F])
def test_as_many_places_as_ascending_starts_can_make(n_seq, dtype):
    """Full tables and one token a sequence, and all tokens one sequence's: rows are written, all of them."""
    c = Call(n_seq, n_seq, 4, 4, 64, dtype, 16, 70 if n_seq < 4000 else 4)
    for start in (list(range(n_seq + 1)), [0] * n_seq + [n_seq], [0] + [n_seq] * n_seq):
        c.o.t.fill_(float("nan"))
        c.attend(start)
        assert c.o.t.isfinite().all()


def test_more_places_than_32_bits_hold():
    """Every second sequence counts all 4096 tokens against 32768 keys."""
    c = Call(4096, 4096, 32, 8, 64, BF, 64, 512)
    for length in (32768, 30001):
        c.kv_len.fill_(length)
        c.attend(_starts("back and forth", 4096, 4096))
        c.attend(_starts("back and forth", 4096, 4096), scratch=1 << 20)
