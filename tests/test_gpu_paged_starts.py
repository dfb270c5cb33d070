"""Starts, lengths and page tables that make no sense: no access leaves the buffers, whatever the arrays on the device hold. Every tensor that a
call writes lies inside a larger one of a known pattern."""
import pytest
import torch

import paper_2507_17245_amd as da
from test_gpu_paged import BF, F

pytestmark = pytest.mark.gpu
MARGIN = 1 << 20   # bytes in front of and behind each tensor


class Guarded:
    """A tensor between two margins of ones in every bit."""

    def __init__(self, shape, dtype):
        n = torch.empty(0, dtype=dtype).element_size()
        for x in shape:
            n *= x
        self.n = n
        self.room = torch.full((MARGIN + -(-n // 256) * 256 + MARGIN,), 255, dtype=torch.uint8, device="cuda")
        self.t = self.room[MARGIN:MARGIN + n].view(dtype).view(shape)

    def margins_hold(self):
        return bool((self.room[:MARGIN] == 255).all()) and bool((self.room[MARGIN + self.n:] == 255).all())


class Call:
    def __init__(self, n_seq, n_tokens, H, Hkv, d, dtype, page, max_pages, n_pages=7):
        g = torch.Generator().manual_seed(n_seq + d)
        self.n_seq, self.n_tokens = n_seq, n_tokens
        self.pool = Guarded((n_pages, 2, Hkv, page, d), dtype)
        self.pool.t.copy_(torch.randn(self.pool.t.shape, generator=g))
        self.k_pages, self.v_pages = self.pool.t[:, 0], self.pool.t[:, 1]
        self.table = torch.randint(0, n_pages, (n_seq, max_pages), generator=g).to(torch.int32).cuda()
        self.kv_len = torch.full((n_seq,), max_pages * page, dtype=torch.int32, device="cuda")
        self.start = torch.zeros(n_seq + 1, dtype=torch.int32, device="cuda")
        self.q = torch.randn(n_tokens, H, d, generator=g).to(dtype).cuda()
        self.kv = torch.randn(n_tokens, 2, Hkv, d, generator=g).to(dtype).cuda()
        self.o, self.lse = Guarded((n_tokens, H, d), dtype), Guarded((n_tokens, H), F)
        self.cache = (self.k_pages, self.v_pages, self.table, self.kv_len, self.start)
        p = da.make_paged_params(*self.cache, q=self.q)
        self.ws = Guarded((da.distr_attn_paged_workspace_bytes(p),), torch.uint8)

    def attend(self, start, scratch=None, causal=True):
        self.start.copy_(torch.as_tensor(start, dtype=torch.int32))
        self.ws.t.fill_(255)
        ws = self.ws.t if scratch is None else self.ws.t[:scratch]
        p = da.make_paged_params(*self.cache, q=self.q, lse_out=self.lse.t, workspace=ws, causal=causal)
        da.distr_attn_paged_fwd(self.q, self.k_pages, self.v_pages, self.o.t, p)
        torch.cuda.synchronize()
        assert self.o.margins_hold() and self.lse.margins_hold() and self.ws.margins_hold() and self.pool.margins_hold()
        assert scratch is None or (self.ws.t[scratch:] == 255).all()

    def append(self, start):
        self.start.copy_(torch.as_tensor(start, dtype=torch.int32))
        k, v = self.kv[:, 0], self.kv[:, 1]
        da.distr_attn_cache_append(k, v, self.k_pages, self.v_pages, da.make_paged_params(*self.cache, k=k, v=v))
        torch.cuda.synchronize()
        assert self.pool.margins_hold()


def _starts(kind, n_seq, n):
    if kind == "back and forth":
        return [0 if i % 2 == 0 else n for i in range(n_seq + 1)]
    if kind == "descending":
        return [n - n * i // n_seq for i in range(n_seq + 1)]
    if kind == "outside":
        return [(-7, 2 ** 31 - 1, -2 ** 31, n + 3)[i % 4] for i in range(n_seq + 1)]
    g = torch.Generator().manual_seed(n_seq)
    return torch.randint(-n, 2 * n, (n_seq + 1,), generator=g).tolist()


KINDS = ["back and forth", "descending", "outside", "anything"]


def test_more_places_than_32_bits_hold():
    """Every second sequence counts all 4096 tokens against 32768 keys: 4.3e9 places of all kv heads, where ascending starts make 1.9e7."""
    c = Call(4096, 4096, 32, 8, 64, BF, 64, 512)
    start = _starts("back and forth", 4096, 4096)
    for length in (32768, 32768 - 64 * 7, 30001):
        c.kv_len.fill_(length)
        c.attend(start)
        c.attend(start, scratch=1 << 20)
    f = Call(4096, 2048, 8, 8, 64, F, 64, 1024)       # 4096 / 2 * 64 * 2051 * 8 = 2.15e9, of all sequences in LDS' sums
    f.attend(_starts("back and forth", 4096, 2048))
    f = Call(8300, 2048, 8, 8, 64, F, 64, 1024)       # more sequences than those sums are kept of: 4.4e9
    f.attend(_starts("back and forth", 8300, 2048))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n_seq,n_tokens,H,Hkv,d,page,max_pages", [
    (3, 40, 8, 2, 64, 16, 4), (3, 200, 8, 2, 128, 16, 300), (75, 180, 8, 4, 64, 32, 160), (75, 180, 8, 4, 128, 32, 4),
    (200, 150, 8, 2, 64, 16, 250), (300, 200, 4, 4, 128, 16, 100), (4, 700, 64, 64, 64, 64, 12)])
def test_starts_in_any_order(kind, dtype, n_seq, n_tokens, H, Hkv, d, page, max_pages):
    c = Call(n_seq, n_tokens, H, Hkv, d, dtype, page, max_pages)
    start = _starts(kind, n_seq, n_tokens)
    for length in (max_pages * page, 2 ** 31 - 1, 5, -3):
        c.kv_len.fill_(length)
        c.attend(start)
        c.attend(start, scratch=1 << 20, causal=False)
        c.append(start)
    c.table.copy_(torch.randint(-2 ** 31, 2 ** 31 - 1, c.table.shape).to(torch.int32))
    c.kv_len.fill_(max_pages * page)
    c.attend(start)
    c.append(start)
    # and a batch in order afterwards is as it was
    c.table.copy_(torch.randint(0, c.k_pages.shape[0], c.table.shape, generator=torch.Generator().manual_seed(1)).to(torch.int32))
    order = [n_tokens * i // n_seq for i in range(n_seq + 1)]
    c.attend(order)
    assert c.o.t.isfinite().all() and c.lse.t.isfinite().all()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n_seq", [64, 65, 4200])
def test_as_many_places_as_ascending_starts_can_make(n_seq, dtype):
    """Full tables and one token a sequence, and all tokens one sequence's: rows are written, all of them."""
    c = Call(n_seq, n_seq, 4, 4, 64, dtype, 16, 70 if n_seq < 4000 else 4)
    for start in (list(range(n_seq + 1)), [0] * n_seq + [n_seq], [0] + [n_seq] * n_seq):
        c.o.t.fill_(float("nan"))
        c.attend(start)
        assert c.o.t.isfinite().all()
