"""Calls around attention whose parameters were made on the null stream: they go there whatever stream is set for the process, and leave that
setting as it is, also while other threads call on streams of their own."""
import ctypes
import threading

import pytest
import torch

import paper_2507_17245_amd as da
from paged_util import Batch

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
BUSY = 400_000_000   # cycles that a side stream is kept busy for


@pytest.fixture
def side():
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    yield stream
    torch.cuda.synchronize()
    da.lib().distr_attn_set_stream(None)


class Calls:
    """A call of each kind on the current stream, and what they give."""

    def __init__(self):
        g = torch.Generator().manual_seed(0)
        self.b = Batch([300, 40], [2, 1], 4, 2, 64, BF)
        self.x = torch.randn(1, 2, 5, 64, generator=g).to(BF).cuda()
        self.g = torch.randn(1, 2, 5, 64, generator=g).to(BF).cuda()
        self.k = torch.randn(3, 2, 64, generator=g).to(BF).cuda()
        self.turned, self.dx, self.o = torch.empty_like(self.x), torch.empty_like(self.x), torch.empty_like(self.b.dev["q"])
        self.dw = torch.empty(64, device="cuda")
        self.rows = da.make_qk_params(self.x, None, self.turned, None, norm=True)
        self.paged = da.make_paged_params(*self.b.cache(), q=self.b.dev["q"], k=self.k, v=self.k, norm=True)

    def outputs(self):
        return [self.turned, self.dx, self.dw, self.o, self.b.k_pages[int(self.b.table[1, 2])]]

    def clear(self):
        for t in self.outputs():
            t.zero_()

    def run(self):
        da.distr_attn_qk_norm_rope(self.x, None, self.turned, None, self.rows)
        da.distr_attn_qk_norm_rope_bwd(self.x, None, self.g, None, self.dx, None, self.rows, dq_weight=self.dw)
        da.distr_attn_cache_append(self.k, self.k, self.b.k_pages, self.b.v_pages, self.paged)
        da.distr_attn_paged_fwd(self.b.dev["q"], self.b.k_pages, self.b.v_pages, self.o, self.paged)

    def results(self):
        done = torch.cuda.Event()
        done.record()
        done.synchronize()
        return [t.cpu().nan_to_num() for t in self.outputs()]


def test_calls_stay_on_the_null_stream(side):
    c = Calls()
    c.clear()                            # (a page of the cache among them, the same way both times)
    c.run()
    want = c.results()
    c.clear()
    torch.cuda.synchronize()
    da.lib().distr_attn_set_stream(ctypes.c_void_p(side.cuda_stream))
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
    c.run()
    got = c.results()
    busy = not side.query()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    if not busy:
        pytest.skip("the side stream ended first: nothing is shown about where the calls went")


def test_the_stream_that_is_set_stays_set(side):
    c = Calls()
    x = torch.randn(1, 2, 64, 64, device="cuda").to(BF)
    y, want = torch.zeros_like(x), torch.empty_like(x)
    da.distr_attn_exact_fwd(x, x, x, want, 64, 64)
    torch.cuda.synchronize()
    L = da.lib()
    L.distr_attn_set_stream(ctypes.c_void_p(side.cuda_stream))
    c.run()
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
    at = [ctypes.c_void_p(t.data_ptr()) for t in (x, x, x, y)]
    assert L.distr_attn_exact_fwd(*at, 1, 2, 2, 64, 64, 64, 64, 0) == 0      # (a short form, of a program in C)
    early = y.cpu()                                                          # the null stream's copy
    busy = not side.query()
    side.synchronize()
    assert torch.equal(y.cpu(), want.cpu())
    if not busy:
        pytest.skip("the side stream ended first: nothing is shown about where the call went")
    assert (early == 0).all()


def test_short_forms_of_another_thread(side):
    """Each thread's calls follow what it has put on its stream in front of them."""
    c = Calls()
    xs = [torch.randn(1, 2, 64, 64, device="cuda").to(BF) for _ in range(2)]
    want_fwd = []
    for x in xs:
        y = torch.empty_like(x)
        da.distr_attn_exact_fwd(x, x, x, y, 64, 64)
        want_fwd.append(y)
    inputs = [c.x.clone(), c.g.clone()]
    want_rows = []
    for x in inputs:
        c.x.copy_(x)
        c.run()
        want_rows.append([c.turned.clone(), c.dx.clone(), c.dw.clone()])
    torch.cuda.synchronize()
    wrong, device = [], torch.cuda.current_device()

    def short_forms():
        try:
            torch.cuda.set_device(device)
            with torch.cuda.stream(side):
                x, y = torch.empty_like(xs[0]), torch.empty_like(xs[0])
                got = []
                for i in range(200):
                    x.copy_(xs[i % 2])
                    da.distr_attn_exact_fwd(x, x, x, y, 64, 64)
                    got.append(y.clone())
                side.synchronize()
                wrong.extend(("short form", i) for i, t in enumerate(got) if not torch.equal(t, want_fwd[i % 2]))
        except BaseException as e:   # noqa: B036 (shown by the test below)
            wrong.append(e)

    other = threading.Thread(target=short_forms)
    other.start()
    got = []
    for i in range(200):
        c.x.copy_(inputs[i % 2])
        c.run()
        got.append([c.turned.clone(), c.dx.clone(), c.dw.clone()])
    other.join()
    torch.cuda.synchronize()
    for i, three in enumerate(got):
        wrong.extend(("rows", i, j) for j, t in enumerate(three) if not torch.equal(t, want_rows[i % 2][j]))
    assert wrong == []
