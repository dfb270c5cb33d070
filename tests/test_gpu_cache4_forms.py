"""The forms of the calls over a 4-bit cache that their size alone brings in: units that fill the chip, units of 128 rows by workgroups of four waves, calls that
go past the caches, places of more than 2 GB in every kernel. Against 64 bits; codes bit for bit."""
import pytest
import torch

import cache4_util
import paper_2507_17245_amd as da
from cache4_util import Batch4, decode, encode
from paged_util import attend, attention_bounds, normed, tables, turn
from test_gpu_cache4 import BF, F, _attention, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
def test_prompts_that_fill_the_chip(d):
    """Enough units for workgroups of their own: whole prompts, one behind a prefix, a single token and none beside them."""
    lens, new = [1100, 700, 65, 130, 40], [1000, 140, 65, 1, 0]
    b = Batch4(lens, new, 64, 64, d, BF, page=64, order="tokens")
    o, lse = _attention(b)
    _check(b, o, lse, rows_of=[0, 63, 64, 127, 128, 139, 512, 999])
    plain, _ = _attention(b, lse=False)
    assert torch.equal(o.nan_to_num(9.0), plain.nan_to_num(9.0))
    o, lse = _attention(b, causal=False)
    _check(b, o, lse, causal=False, rows_of=[0, 64, 139, 999])
    plain, _ = _attention(b, causal=False, lse=False)
    assert torch.equal(o.nan_to_num(9.0), plain.nan_to_num(9.0))


@pytest.mark.parametrize("n_seq,H,Hkv,d,page,order", [(100, 8, 4, 128, 32, "heads"), (70, 12, 4, 128, 16, "tokens"), (100, 12, 3, 64, 16, "heads"), (140, 4, 2, 64, 48, "tokens")])
@pytest.mark.parametrize("workspace", [True, None, 3 << 20])
@pytest.mark.parametrize("roomy", [0, 5000])
def test_chunks_among_many_sequences(n_seq, H, Hkv, d, page, order, workspace, roomy):
    """Units of 128 rows by workgroups of four waves, whole (narrow tables) and by ranges; chunks, a few tokens, one and none."""
    g = torch.Generator().manual_seed(n_seq + d)
    lens = torch.randint(1, 250, (n_seq,), generator=g).tolist()
    new = [min(int(x), n) for x, n in zip(torch.randint(0, 6, (n_seq,), generator=g), lens)]
    for s, n, fresh in ((3, 900, 200), (40, 300, 300), (69, 1300, 45), (n_seq - 1, 130, 129)):
        lens[s], new[s] = n, fresh
    b = Batch4(lens, new, H, Hkv, d, BF, page=page, order=order, room=roomy // page, pad_front=1, pad_back=2)
    assert b.T > n_seq and n_seq * Hkv > 256
    only, rows = {0, 1, 2, 3, 4, 40, 41, 68, 69, n_seq - 2, n_seq - 1}, [0, 1, 2, 3, 4, 31, 44, 63, 64, 127, 128, 199, 299]
    for causal in (True, False):
        o, lse = _attention(b, causal=causal, workspace=workspace)
        _check(b, o, lse, causal=causal, only=only, rows_of=rows)
        plain, _ = _attention(b, causal=causal, workspace=workspace, lse=False)
        assert torch.equal(o.nan_to_num(9.0), plain.nan_to_num(9.0))
        again, lse2 = _attention(b, causal=causal, workspace=workspace)
        assert torch.equal(o.nan_to_num(9.0), again.nan_to_num(9.0)) and torch.equal(lse.nan_to_num(9.0), lse2.nan_to_num(9.0))


def test_nan_in_a_value_of_a_chunk_among_many_sequences():
    """Workgroups of four waves whose unit is taken again as few rows."""
    n_seq, lens, new = 100, [60] * 100, [1] * 100
    lens[7], new[7] = 400, 90

    def edit(s, which, codes, scales):
        if s == 7 and which == "v":
            scales[2, 399, 1] = 255
    b, clean = (Batch4(lens, new, 8, 4, 128, BF, page=16, edit=e) for e in (edit, None))
    o, lse = _attention(b)
    want = torch.zeros(b.T, 8, 128, dtype=torch.bool)
    want[int(b.start[8]) - 1, 4:6, 32:64] = True
    assert torch.equal(o.isnan(), want)
    whole, _ = _attention(clean)
    _check(clean, torch.where(want, whole, o), lse, only={6, 7, 8}, rows_of=[0, 1, 63, 88, 89])


def _paged_cache(lens, Hkv, d, page, order, g, low=118, high=130):
    """Codes of all kinds, scales 2^(low - 127) .. 2^(high - 128), made on the GPU. -> cache, page table, the pages of each sequence"""
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + 2
    outer = (n_pages, Hkv, page) if order == "heads" else (n_pages, page, Hkv)
    parts = [torch.randint(a, e, (*outer, w), generator=g, device="cuda", dtype=torch.uint8) for w, a, e in ((d // 2, 0, 256), (d // 32, low, high)) * 2]
    ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(need)), -1, dtype=torch.int32, device="cuda")
    for s, n in enumerate(need):
        table[s, :n] = ids[sum(need[:s]):sum(need[:s + 1])]
    return tuple(t if order == "heads" else t.transpose(1, 2) for t in parts), table, need


@pytest.fixture
def on_device(monkeypatch):
    """encode and decode of tensors on the GPU"""
    for name in ("MAGNITUDES", "POWERS", "MIDDLES"):
        monkeypatch.setattr(cache4_util, name, getattr(cache4_util, name).cuda())


@pytest.mark.parametrize("lens,H,Hkv,d,page", [((70001,), 32, 8, 128, 64), ((130001, 3, 61000), 16, 8, 64, 16), ((3700,) * 70, 8, 8, 64, 32), ((3000,) * 40, 16, 8, 128, 16),
                                               ((1250,) * 150, 4, 4, 128, 32), ((1270,) * 260, 8, 4, 64, 16)])
@pytest.mark.parametrize("lse", [True, False])
def test_single_tokens_past_the_caches(lens, H, Hkv, d, page, lse, on_device):
    """More than 64 MB of codes and scales, heads outside: workgroups of eight, four and two waves."""
    tiles = sum(-(-n // 64) for n in lens)
    assert tiles * Hkv * 64 * 2 * (d // 2 + d // 32) > 64 << 20
    n_seq, g = len(lens), torch.Generator(device="cuda").manual_seed(len(lens))
    cache, table, need = _paged_cache(lens, Hkv, d, page, "heads", g)
    kv_len, start = torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.arange(n_seq + 1, dtype=torch.int32, device="cuda")
    q = (0.5 * torch.randn(n_seq, H, d, generator=g, device="cuda")).to(BF)
    o, row = torch.full_like(q, float("nan")), torch.full((n_seq, H), float("nan"), device="cuda") if lse else None
    p = da.make_paged4_params(cache, table, kv_len, start, q=q, lse_out=row)
    ws = torch.empty(da.distr_attn_paged4_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    da.distr_attn_paged4_fwd(q, cache, o, da.make_paged4_params(cache, table, kv_len, start, q=q, lse_out=row, workspace=ws))
    torch.cuda.synchronize()
    for s in sorted({0, min(1, n_seq - 1), min(2, n_seq - 1), n_seq // 2, n_seq - 1}):
        n, at = lens[s], table[s, :need[s]].long()
        want, mean, ln, most = (torch.zeros(*shape, dtype=torch.float64) for shape in ((1, H, d), (1, H, d), (1, H), (1, H)))
        for h in range(Hkv):
            k, v = (decode(cache[i][at, h].reshape(-1, d // 2)[:n], cache[i + 1][at, h].reshape(-1, d // 32)[:n]) for i in (0, 2))
            for j in range(h * H // Hkv, (h + 1) * H // Hkv):
                score = k @ q[s, j].double() * d ** -0.5
                weight = torch.softmax(score, 0)
                want[0, j], mean[0, j], ln[0, j] = weight @ v, weight @ v.abs(), torch.logsumexp(score, 0)
                most[0, j] = (k.abs() @ q[s, j].double().abs()).max() * d ** -0.5
        bound, ln_bound = attention_bounds(want, mean, ln, most, n, d, BF)
        err = (o[s:s + 1].double().cpu() - want).abs()
        assert (err <= bound).all(), (s, float((err / bound).max()))
        assert not lse or ((row[s:s + 1].double().cpu() - ln).abs() <= ln_bound).all(), s
    assert o.isfinite().all()


@pytest.mark.parametrize("new,Hkv,d,page,order,rope", [((5003, 4, 4001), 16, 128, 64, "tokens", "halves"), ((9000, 9001), 16, 64, 16, "heads", "neighbours"),
                                                        ((8300, 33), 16, 128, 48, "heads", "none")])
def test_appends_past_the_caches(new, Hkv, d, page, order, rope, on_device):
    """k and v of more than 64 MB in bf16: every code and scale, and that nothing else is written."""
    T, lens = sum(new), [n + 37 * i for i, n in enumerate(new)]
    assert T * Hkv * d * 4 > 64 << 20
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, 2, Hkv, d, generator=g, device="cuda").to(BF)
    k, v = x[:, 0], x[:, 1]
    cache, table, _ = _paged_cache(lens, Hkv, d, page, order, g, 7, 8)
    before = [t.clone() for t in cache]
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    start = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda")
    norm = {}
    if rope != "none":
        cos, sin = (t.cuda() for t in tables(max(lens), d))
        norm = dict(norm=True, eps=1e-5, k_weight=1 + 0.3 * torch.randn(d, generator=g, device="cuda"), rope=rope, cos=cos, sin=sin)
    da.distr_attn_cache4_append(k, v, cache, da.make_paged4_params(cache, table, kv_len, start, k=k, v=v, **norm))
    torch.cuda.synchronize()
    for s, n in enumerate(new):
        place = torch.arange(lens[s] - n, lens[s], device="cuda")
        at, row, rows = table[s].long()[place // page], place % page, slice(int(start[s]), int(start[s]) + n)
        y = k[rows].double()
        if norm:
            y = normed(y, norm["k_weight"].double(), float(torch.tensor(1e-5, dtype=F)))
            y = turn(y, cos.double()[place][:, None], sin.double()[place][:, None], rope)
        for i, want in ((0, encode(y)), (2, encode(v[rows].double()))):
            for j in (0, 1):
                before[i + j][at, :, row] = want[j]
    assert all(torch.equal(a, e) for a, e in zip(cache, before))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n,Hkv,d,page,order", [((8300, 1), 16, 128, 64, "heads"), ((9000, 9001), 16, 64, 16, "tokens"), ((24001,), 7, 128, 48, "tokens")])
def test_reads_past_the_caches(n, Hkv, d, page, order, dtype, on_device):
    T = sum(n)
    assert T * Hkv * d * 2 * (2 if dtype == BF else 4) > 64 << 20
    g = torch.Generator(device="cuda").manual_seed(T)
    cache, table, need = _paged_cache(n, Hkv, d, page, order, g, 100, 140)
    start = torch.tensor([1 + sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32, device="cuda")
    k, v = (torch.full((T + 2, Hkv, d), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    da.distr_attn_cache4_read(k, v, cache, da.make_paged4_params(cache, table, torch.tensor(n, dtype=torch.int32, device="cuda"), start, k=k, v=v))
    for x, i in ((k, 0), (v, 2)):
        want = torch.full(x.shape, 7.0, dtype=torch.float64, device="cuda")
        for s, m in enumerate(n):
            at, r0 = table[s, :need[s]].long(), int(start[s])
            want[r0:r0 + m] = decode(cache[i][at], cache[i + 1][at]).transpose(1, 2).reshape(-1, Hkv, d)[:m]
        assert torch.equal(x.double(), want)


FAR = [  # sequences, new tokens of each, H, Hkv, d: single tokens by workgroups of eight, four and two waves, units of 128 rows by those of eight and four
    (3, 1, 4, 2, 64), (5, 1, 8, 2, 128), (200, 1, 4, 2, 64), (200, 1, 4, 2, 128), (300, 1, 2, 2, 64), (300, 1, 2, 2, 128),
    (2, 50, 4, 2, 64), (2, 60, 8, 2, 128), (150, 2, 4, 2, 64), (150, 3, 8, 2, 128),
]


@pytest.mark.parametrize("n_seq,new,H,Hkv,d", FAR)
def test_places_of_more_than_two_gigabytes(n_seq, new, H, Hkv, d):
    """Pages 1.5 GB apart, heads 300 MB, rows 1 MB: codes and scales of one buffer of 6 GB. All sequences have the same four pages, each in an order of its own."""
    page, n_pages, g = 16, 4, torch.Generator().manual_seed(n_seq + d)
    store = torch.empty(6 << 30, dtype=torch.uint8, device="cuda")
    part = lambda w, at: torch.as_strided(store, (n_pages, Hkv, page, w), (1536 << 20, 300 << 20, 1 << 20, 1), at)   # noqa: E731
    cache = part(d // 2, 0), part(d // 32, 4096), part(d // 2, 8192), part(d // 32, 16384)
    held = []
    for t in cache:
        x = torch.randint(0, 256, t.shape, generator=g, dtype=torch.uint8) if t.shape[3] == d // 2 else torch.randint(118, 130, t.shape, generator=g, dtype=torch.uint8)
        t.copy_(x.cuda())
        held.append(x)
    pages = [decode(held[i], held[i + 1]) for i in (0, 2)]   # [page, Hkv, row, d]
    lens = torch.randint(new, n_pages * page + 1, (n_seq,), generator=g).tolist()
    lens[0] = n_pages * page
    table = torch.stack([torch.randperm(n_pages, generator=g) for _ in range(n_seq)]).to(torch.int32)
    T = n_seq * new
    start = torch.arange(0, T + 1, new, dtype=torch.int32)
    q = torch.randn(T, H, d, generator=g).to(BF)
    dq, index = q.cuda(), (table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), start.cuda())
    for lse in (True, False):
        o, row = torch.full_like(dq, float("nan")), torch.full((T, H), float("nan"), device="cuda") if lse else None
        da.distr_attn_paged4_fwd(dq, cache, o, da.make_paged4_params(cache, *index, q=dq, lse_out=row))
        torch.cuda.synchronize()
        for s in sorted({0, 1, 2, n_seq // 2, n_seq - 1}):
            if s >= n_seq:
                continue
            k, v = (x[table[s].long()].transpose(0, 1).reshape(Hkv, -1, d)[:, :lens[s]] for x in pages)
            rows = slice(s * new, (s + 1) * new)
            want, mean, ln, most = attend(q[rows].double(), k, v, [lens[s] - new + i for i in range(new)], lens[s], d ** -0.5)
            bound, ln_bound = attention_bounds(want, mean, ln, most, lens[s], d, BF)
            err = (o[rows].cpu().double() - want).abs()
            assert (err <= bound).all(), (s, float((err / bound).max()))
            assert not lse or ((row[rows].cpu().double() - ln).abs() <= ln_bound).all(), s
        assert o.isfinite().all()
