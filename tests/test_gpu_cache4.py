"""A cache held in 4 bits: codes and scales written, values read back, attention over them, against 64 bits. Codes are compared bit for bit."""
import math

import pytest
import torch

import paper_2507_17245_amd as da
from cache4_util import Batch4, decode, encode
from paged_util import attend, attention_bounds, normed, tables, turn

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
ROOMY = [0, 5000]   # tokens that a row of the page table has room for beyond the longest sequence


def _append(b, k, v, **kw):
    """-> the cache on the CPU, as stored"""
    p = da.make_paged4_params(b.cache4, *b.index(), k=k, v=v, **kw)
    da.distr_attn_cache4_append(k, v, b.cache4, p)
    torch.cuda.synchronize()
    return [t.cpu() for t in b.cache4]


def _expected(b, k, v, stored=lambda s, place: True):
    """The cache with rows k, v ([T, Hkv, d] double) in their places."""
    parts = [t.clone() if b.order == "heads" else t.clone().transpose(1, 2) for t in b.cache_cpu]
    enc = [encode(k), encode(v)]
    for row, s, place in b.places():
        if place < 0 or not stored(s, place):
            continue
        at = int(b.table[s, place // b.page]), slice(None), place % b.page
        for i in range(2):
            parts[2 * i][at], parts[2 * i + 1][at] = enc[i][0][row], enc[i][1][row]
    return parts


def _same(got, want):
    for g, w, name in zip(got, want, ("k_codes", "k_scales", "v_codes", "v_scales")):
        wrong = int((g != w).sum())
        assert wrong == 0, (name, g.numel(), (g != w).nonzero()[0].tolist())


def _special(d, dtype):
    """Rows of what a code can go wrong at: ties, limits of a scale, the range's ends, zeros of both signs, infinities, NaN."""
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 6.0, 0.0, -0.0, -0.25, -5.0, 0.5, 4.0, -7.0] * 2)
    g = torch.Generator().manual_seed(3)
    rows = [torch.cat([ties * 2.0 ** e for _ in range(d // 32)]) for e in (0, 1, -1, 7, -20, 100, -100, 119, -126, -130)]
    near = ties * (1 + 2.0 ** -7)
    rows += [near.repeat(d // 32), (ties * (1 - 2.0 ** -7)).repeat(d // 32), torch.zeros(d), -torch.zeros(d)]
    for x in (math.inf, -math.inf, math.nan):
        r = torch.randn(d, generator=g)
        r[3], r[d - 1] = x, x
        rows.append(r)
    rows += [torch.full((d,), torch.finfo(dtype).max), torch.full((d,), -torch.finfo(dtype).max), torch.full((d,), torch.finfo(dtype).tiny),
             torch.full((d,), 1.75), torch.full((d,), 1.7578125), torch.full((d,), 3.3e38)]
    r = torch.full((d,), 1e-30)
    r[5] = 1e30
    rows.append(r)
    return torch.stack(rows).to(dtype)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("order", ["heads", "tokens"])
def test_codes_of_plain_rows(d, dtype, order):
    rows = _special(d, dtype)
    n = rows.shape[0]
    b = Batch4([n + 5, 40], [n, 7], 4, 2, d, dtype, page=16, order=order, stored="old", pad_front=2, pad_back=3)
    k, v = (x.clone() for x in b.raw)
    r0 = int(b.start[0])
    k[r0:r0 + n] = rows[:, None]
    v[r0:r0 + n] = rows.flip(0)[:, None]
    got = _append(b, k.cuda(), v.cuda())
    _same(got, _expected(b, k.double(), v.double()))


FORMS = [  # norm, weight ("", "one", "heads", with the type), rope, rotated channels as a share of d
    (True, "", "none", 0), (True, "one", "halves", 1), (True, "heads", "neighbours", 1), (False, "", "halves", 1), (False, "", "neighbours", 0.5),
    (True, "one", "halves", 0.25), (True, "heads", "halves", 0.75), (True, "", "neighbours", 0.25),
]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", FORMS)
def test_codes_of_normed_and_rotated_rows(form, d, dtype):
    """Keys bit for bit those of the row in 64 bits: a code differs only where 64 bits themselves (their own roundings, 2^-50) leave it open, which
    no row of these comes near."""
    norm, weight, rope, share = form
    lens, new = [700, 3, 260], [650, 3, 1]
    Hkv, eps = 3, 1e-5
    b = Batch4(lens, new, 6, Hkv, d, dtype, page=48, order="tokens", stored="old", seed=d, pad_front=1)
    k = b.raw[0].double() * torch.exp(0.5 * torch.randn(b.T, 1, 1, generator=torch.Generator().manual_seed(5)).double())
    k = k.to(dtype)
    w = None
    if weight:
        w = 1 + 0.3 * torch.randn(*((Hkv, d) if weight == "heads" else (d,)), generator=torch.Generator().manual_seed(6))
        w = w.to(BF if weight == "one" and dtype == BF else F)
    rot = int(d * share)
    c, s = tables(max(lens), rot) if rot else (None, None)
    y = k.double()
    if norm:
        y = normed(y, None if w is None else w.double(), float(torch.tensor(eps, dtype=F)))
    if rot:
        at = torch.zeros(b.T, dtype=torch.long)
        for row, _, place in b.places():
            at[row] = place
        y = turn(y, c.double()[at][:, None], s.double()[at][:, None], rope)
    got = _append(b, k.cuda(), b.raw[1].cuda(), norm=norm, eps=eps, k_weight=None if w is None else w.cuda(), rope=rope, cos=None if c is None else c.cuda(),
                  sin=None if s is None else s.cuda())
    _same(got, _expected(b, y, b.raw[1].double()))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("scale", [1e-18, 1e18, 1e-30, 3e37])
def test_norms_of_rows_whose_squares_leave_the_range(dtype, scale):
    b = Batch4([50], [50], 2, 2, 64, dtype, stored="old")
    k = (b.raw[0].double() * scale).to(dtype)
    k[7] = 0
    for eps in (0.0, 1e-6):
        got = _append(b, k.cuda(), b.raw[1].cuda(), norm=True, eps=eps)
        y = k.double() / (k.double().square().mean(-1, keepdim=True) + float(torch.tensor(eps, dtype=F))).sqrt()
        _same(got, _expected(b, y, b.raw[1].double()))
        b.to_device()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("large", [2.0 ** 25, 2.0 ** 60, 2.0 ** 100])
def test_weights_that_lift_channels_out_of_nowhere(dtype, large):
    """Channels so small that their norm is no full float, and weights that make them count: the codes are still those of the exact row."""
    d, eps = 64, 1e-6
    b = Batch4([50], [50], 2, 2, d, dtype, stored="old")
    k = b.raw[0].double()
    k[..., :32] *= 2.0 ** -95
    k[..., 32:] *= 2.0 ** 50
    k = k.to(dtype)
    w = 1 + 0.3 * torch.randn(d, generator=torch.Generator().manual_seed(6))
    w[:32] *= large
    got = _append(b, k.cuda(), b.raw[1].cuda(), norm=True, eps=eps, k_weight=w.cuda())
    _same(got, _expected(b, normed(k.double(), w.double(), float(torch.tensor(eps, dtype=F))), b.raw[1].double()))


def test_rows_next_to_a_border():
    """Rotations that put thousands of channels within 2^-24 of a border between two codes: 32 bits alone get some of them wrong."""
    d, n = 64, 400
    b = Batch4([n], [n], 2, 2, d, F, stored="old")
    g = torch.Generator().manual_seed(9)
    angle = torch.rand(n, d // 2, generator=g, dtype=torch.float64) * 6.28
    c, s = angle.cos().float(), angle.sin().float()
    borders = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64)
    want = borders[torch.randint(0, 7, (n, 2, d), generator=g)] * torch.where(torch.rand(n, 2, d, generator=g) < 0.5, -1.0, 1.0)
    want[..., 0], want[..., 32] = 5.0, 5.0
    x = turn(want, c.double()[:, None], -s.double()[:, None], "halves")
    k = (x / (c.double().square() + s.double().square()).repeat(1, 2)[:, None]).float()
    y = turn(k.double(), c.double()[:, None], s.double()[:, None], "halves")
    assert ((y - want).abs() <= 2.0 ** -20).all()
    got = _append(b, k.cuda(), b.raw[1].cuda(), rope="halves", cos=c.cuda(), sin=s.cuda())
    _same(got, _expected(b, y, b.raw[1].double()))
    # in 32 bits some of them are on the other side
    a, e = k[..., :32] * c[:, None] - k[..., 32:] * s[:, None], k[..., :32] * s[:, None] + k[..., 32:] * c[:, None]
    assert int((encode(torch.cat((a, e), -1).double())[0] != encode(y)[0]).sum()) > 100


@pytest.mark.parametrize("dtype", [BF, F])
def test_positions_and_strides(dtype):
    """Keys and values as views of one projection, rotations that are not those of the places; a position outside the table makes rotated channels' groups NaN."""
    d, Hkv, n = 128, 2, 30
    b = Batch4([n + 9], [n], 2, Hkv, d, dtype, page=32, order="tokens", stored="old")
    x = torch.randn(n, 2, 3, d, generator=torch.Generator().manual_seed(2)).to(dtype)
    k, v = x[:, :, 0], x[:, :, 2]
    c, s = tables(64, 64)
    at = torch.randint(0, 64, (n,), generator=torch.Generator().manual_seed(3)).to(torch.int32)
    at[4], at[5] = -1, 64
    y = turn(k.double(), c.double()[at.long().clamp(0, 63)][:, None], s.double()[at.long().clamp(0, 63)][:, None], "halves")
    y[4:6, :, :64] = math.nan
    dev = x.cuda()
    got = _append(b, dev[:, :, 0], dev[:, :, 2], rope="halves", cos=c.cuda(), sin=s.cuda(), positions=at.cuda())
    _same(got, _expected(b, y, v.double()))


@pytest.mark.parametrize("dtype", [BF, F])
def test_tokens_without_a_place(dtype):
    """Pages that are none of the cache's, places before the sequence's beginning and behind the table: left out; empty sequences beside full ones."""
    b = Batch4([40, 20, 0, 33, 16], [40, 3, 0, 5, 16], 2, 2, 64, dtype, stored="old", pad_front=2, pad_back=1)
    b.table[0, 1] = -1
    b.table[3, 2] = b.cache_cpu[0].shape[0]
    b.kv_len[4] = 10      # six of its sixteen tokens begin before the sequence
    b.lens[4] = 10
    b.dev["table"], b.dev["kv_len"] = b.table.cuda(), b.kv_len.cuda()
    got = _append(b, b.raw[0].cuda(), b.raw[1].cuda())
    ok = lambda s, place: place >= 0 and not (s == 0 and 16 <= place < 32) and not (s == 3 and place >= 32)   # noqa: E731
    _same(got, _expected(b, b.raw[0].double(), b.raw[1].double(), ok))
    # and back: rows without a place stay
    k, v = (torch.full((b.T, 2, 64), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    da.distr_attn_cache4_read(k, v, b.cache4, da.make_paged4_params(b.cache4, *b.index(), k=k, v=v))
    held = {row: i for i, (row, s, place) in enumerate(b.places()) if ok(s, place)}
    for x, raw in ((k, b.raw[0]), (v, b.raw[1])):
        want = torch.full((b.T, 2, 64), 7.0, dtype=torch.float64)
        rows = list(held)
        want[rows] = decode(*encode(raw.double()))[rows]
        assert torch.equal(x.cpu().double(), want)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("order", ["heads", "tokens"])
def test_every_code_and_scale_is_read(d, dtype, order):
    """All 256 scales, all codes: exact in either type up to its range (bf16 and float share it: 2^128 and more are infinite)."""
    page, n = 16, 256
    b = Batch4([n], [n], 1, 1, d, dtype, page=page, order=order, stored="old")
    g = torch.Generator().manual_seed(4)
    codes = [torch.randint(0, 256, b.cache_cpu[0].shape, generator=g, dtype=torch.uint8) for _ in range(2)]
    scales = [torch.zeros_like(b.cache_cpu[1]) for _ in range(2)]
    view = [t if order == "heads" else t.transpose(1, 2) for t in (*codes, *scales)]
    for i in range(n):
        for j in range(2):
            view[2 + j][b.table[0, i // page], 0, i % page] = torch.tensor([i, 255 - i] * (d // 64), dtype=torch.uint8)
    b.cache_cpu = [codes[0], scales[0], codes[1], scales[1]]
    b.to_device()
    k, v = (torch.empty(n, 3, d, dtype=dtype, device="cuda")[:, 1:2] for _ in range(2))
    da.distr_attn_cache4_read(k, v, b.cache4, da.make_paged4_params(b.cache4, *b.index(), k=k, v=v))
    for j, x in enumerate((k, v)):
        ids = b.table[0].long()
        want = decode(view[j][ids, 0].reshape(-1, d // 2)[:n], view[2 + j][ids, 0].reshape(-1, d // 32)[:n])
        want = torch.where(want.abs() >= 2.0 ** 128, torch.sign(want) * math.inf, want)
        got = x[:, 0].cpu().double()
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0.5, 1.5, -1.5), want.nan_to_num(0.5, 1.5, -1.5))


def _attention(b, causal=True, scale=None, lse=True, workspace=True, q=None):
    """-> o, lse of one call on the batch; o is NaN where nothing is written"""
    q = b.dev["q"] if q is None else q
    o = torch.full((b.T, b.H, b.d), float("nan"), dtype=b.dtype, device="cuda")
    row = torch.full((b.T, b.H), float("nan"), device="cuda") if lse else None
    options = dict(q=q, causal=causal, softmax_scale=0.0 if scale is None else scale, lse_out=row)
    ws = None
    if workspace is not None:
        n = da.distr_attn_paged4_workspace_bytes(da.make_paged4_params(b.cache4, *b.index(), **options))
        ws = torch.full((n if workspace is True else workspace,), 255, dtype=torch.uint8, device="cuda")
    da.distr_attn_paged4_fwd(q, b.cache4, o, da.make_paged4_params(b.cache4, *b.index(), workspace=ws, **options))
    torch.cuda.synchronize()
    return o.cpu(), row.cpu() if lse else None


def _check(b, o, lse, causal=True, scale=None, seen=None, rows_of=None, only=None):
    """Every row of every sequence (rows_of: some of its new tokens; only: some sequences) and that no others were written.

    To attention_bounds comes what floats lose at their lower end: a weight (at most 2^8 and the largest at least 1, whatever the reference) and the
    factors that join a row's parts are off by 2^-126 at most where they fall below it, three of them in a row, so that a row's sum over
    values of any size is off by 2^-124 sum |v| more."""
    scale = b.d ** -0.5 if scale is None else scale
    left = torch.ones(b.T, dtype=torch.bool)
    for s, (n, fresh) in enumerate(zip(b.lens, b.new)):
        r0 = int(b.start[s])
        left[r0:r0 + fresh] = False
        at = list(range(fresh)) if rows_of is None else sorted({i for i in rows_of if i < fresh})
        if not at or (only is not None and s not in only):
            continue
        places = [n - fresh + i if causal else n - 1 for i in at]
        rows = [r0 + i for i in at]
        want, mean, ln, most = attend(b.q[rows].double(), b.keys[s].double(), b.values[s].double(), places, n, scale, None if seen is None else seen[s])
        bound, ln_bound = attention_bounds(want, mean, ln, most, n, b.d, b.dtype)
        bound = bound + 2.0 ** -124 * b.values[s].abs().sum(1).repeat_interleave(b.H // b.Hkv, 0)
        err = (o[rows].double() - want).abs()
        over = float((err / bound).max())
        assert over <= 1, (s, over)
        if lse is not None:
            empty = ln.isinf()
            assert torch.equal(lse[rows].isinf(), empty) and (lse[rows][empty] < 0).all()
            over = float(((lse[rows].double() - ln).abs() / ln_bound)[~empty].max()) if not empty.all() else 0.0
            assert over <= 1, (s, over)
    assert o[left].isnan().all() and (lse is None or lse[left].isnan().all())


RAGGED = [  # lens, new, H, Hkv, d, page, order
    ([1], [1], 1, 1, 64, 16, "heads"),
    ([1, 0, 2], [1, 0, 2], 4, 2, 64, 16, "heads"),
    ([15, 16, 17, 31, 33], [1] * 5, 8, 2, 64, 16, "tokens"),
    ([63, 64, 65, 127, 128, 129], [1, 2, 3, 4, 5, 6], 3, 1, 64, 32, "heads"),
    ([700, 5, 300], [40, 5, 1], 6, 2, 64, 48, "heads"),
    ([1000], [1], 16, 1, 128, 64, "tokens"),
    ([520, 33, 100], [70, 33, 9], 4, 4, 128, 16, "tokens"),
    ([260], [260], 8, 2, 128, 256, "heads"),
    ([2100, 40], [1, 1], 5, 1, 128, 1024, "heads"),
    ([90, 70], [90, 70], 34, 2, 64, 16, "heads"),
    ([400, 380, 200], [150, 1, 200], 8, 2, 64, 64, "tokens"),
    ([130, 64], [1, 1], 20, 1, 128, 16, "heads"),
]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("case", RAGGED)
@pytest.mark.parametrize("roomy", ROOMY)
def test_ragged_batches(case, dtype, roomy):
    lens, new, H, Hkv, d, page, order = case
    b = Batch4(lens, new, H, Hkv, d, dtype, page=page, order=order, pad_front=1, pad_back=2, room=1 + roomy // page)
    some = [0, 1, 2, 3, 7, 8, 15, 16, 30, 31, 32, 33, 63, 64, 69, 127, 128, 129, 149, 199, 259]
    for causal in (True, False):
        o, lse = _attention(b, causal=causal)
        _check(b, o, lse, causal=causal, rows_of=some)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("workspace", [True, None, 256, 300000])
def test_long_rows_with_any_scratch(d, dtype, workspace):
    lens, new = [5000, 3, 1500], [2, 1, 30]
    b = Batch4(lens, new, 8, 2, d, dtype, page=32, scale=3.0)
    o, lse = _attention(b, workspace=workspace)
    _check(b, o, lse, rows_of=[0, 1, 15, 29])
    again, lse2 = _attention(b, workspace=workspace)
    assert torch.equal(o.isnan(), again.isnan()) and torch.equal(o.nan_to_num(), again.nan_to_num()) and torch.equal(lse.nan_to_num(), lse2.nan_to_num())


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [[3, 1], [200, 1]])
def test_without_row_statistics(dtype, d, new):
    b = Batch4([300, 2000], new, 8, 2, d, dtype)
    o, _ = _attention(b)
    plain, _ = _attention(b, lse=False)
    assert torch.equal(o, plain)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n_seq", [63, 64, 65, 300, 4200])
@pytest.mark.parametrize("roomy", ROOMY)
def test_many_sequences(n_seq, dtype, roomy):
    g = torch.Generator().manual_seed(n_seq)
    lens = torch.randint(0, 120 if n_seq < 1000 else 40, (n_seq,), generator=g).tolist()
    new = [min(int(x), n) for x, n in zip(torch.randint(0, 4 if n_seq < 1000 else 2, (n_seq,), generator=g), lens)]
    b = Batch4(lens, new, 4, 2, 64, dtype, pad_back=1, room=roomy // 16 if n_seq < 1000 else 20)
    o, lse = _attention(b)
    _check(b, o, lse, only=set(range(0, n_seq, 1 if n_seq < 100 else n_seq // 60)))


@pytest.mark.parametrize("n_seq,Hkv,d,most", [(7, 5, 64, 300), (70, 8, 64, 300), (203, 3, 128, 90), (403, 1, 64, 60), (90, 16, 128, 200), (40, 8, 128, 3000)])
def test_either_order_of_a_page(n_seq, Hkv, d, most):
    """Where heads' rows lie next to each other their workgroups are dealt out otherwise: the same cache in both orders of a page gives the same results, bit for bit."""
    g = torch.Generator().manual_seed(n_seq)
    lens = torch.randint(0, most, (n_seq,), generator=g).tolist()
    new = [min(n, 1) for n in lens]
    done = []
    for order in ("heads", "tokens"):
        b = Batch4(lens, new, 2 * Hkv, Hkv, d, BF, page=16, order=order, pad_back=1)
        o, lse = _attention(b)
        _check(b, o, lse, only=set(range(0, n_seq, max(1, n_seq // 20))))
        done.append((b, o, lse))
    assert all(torch.equal(x, y) for x, y in zip(done[0][0].values, done[1][0].values))
    assert torch.equal(done[0][1].nan_to_num(9.0), done[1][1].nan_to_num(9.0)) and torch.equal(done[0][2].nan_to_num(9.0), done[1][2].nan_to_num(9.0))


@pytest.mark.parametrize("dtype", [BF, F])
def test_two_streams_at_once(dtype):
    """Appends, reads and attention of two caches on streams of their own without workspaces, call after call: the same as one after the other."""
    batches = [Batch4([3000 + 500 * i, 70], [1, 1 + 40 * i], 8, 2, 64, dtype, seed=i, stored="old", room=300) for i in range(2)]
    torch.cuda.synchronize()

    def run(b):
        k, v = (x.cuda() for x in b.raw)
        back = [torch.zeros_like(k) for _ in range(2)]
        o = torch.zeros(b.T, b.H, b.d, dtype=b.dtype, device="cuda")
        for _ in range(5):
            da.distr_attn_cache4_append(k, v, b.cache4, da.make_paged4_params(b.cache4, *b.index(), k=k, v=v))
            da.distr_attn_cache4_read(*back, b.cache4, da.make_paged4_params(b.cache4, *b.index(), k=back[0], v=back[1]))
            da.distr_attn_paged4_fwd(b.dev["q"], b.cache4, o, da.make_paged4_params(b.cache4, *b.index(), q=b.dev["q"]))
        return [*back, o]

    alone = []
    for b in batches:
        alone.append(run(b))
        torch.cuda.synchronize()
        b.to_device()
    torch.cuda.synchronize()
    streams, both = [torch.cuda.Stream() for _ in batches], []
    for b, stream in zip(batches, streams):
        with torch.cuda.stream(stream):
            both.append(run(b))
    torch.cuda.synchronize()
    for one, other in zip(alone, both):
        assert all(torch.equal(x, y) for x, y in zip(one, other))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 40])
def test_nan_in_keys_and_values(d, dtype, new):
    """A key of NaN reaches the rows that see it, a value's 32 channels of NaN those channels of the rows that see it, and none else."""
    n = 200

    def edit(s, which, codes, scales):
        if which == "k" and s == 0:
            scales[1, n - 3, 0] = 255
        if which == "v":
            scales[0, n - 5, d // 32 - 1] = 255
            scales[1, 77, 0] = 255
    b = Batch4([n, n], [new, new], 4, 2, d, dtype, page=32, edit=edit)
    o, lse = _attention(b)
    for s in range(2):
        for i in range(new):
            place, row = n - new + i, int(b.start[s]) + i
            want = torch.zeros(4, d, dtype=torch.bool)
            if place >= n - 5:
                want[:2, d - 32:] = True
            want[2:, :32] = True
            if s == 0 and place >= n - 3:
                want[2:] = True
            assert torch.equal(o[row].isnan(), want), (s, i)
            assert torch.equal(lse[row].isnan(), torch.tensor([False, False] + [s == 0 and place >= n - 3] * 2))
    clean = Batch4([n, n], [new, new], 4, 2, d, dtype, page=32)
    want, want_lse = _attention(clean)
    # What is no NaN is what it is without it. Rows beside a NaN may be walked otherwise, their sums taken in another order: not the same bits, but
    # within the bounds of the definition, as any order is.
    _check(clean, torch.where(o.isnan(), want, o), torch.where(lse.isnan(), want_lse, lse), rows_of=[0, 1, 20, 36, 37, 38, 39])


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [64, 128])
def test_absent_pages_and_rows_that_see_nothing(d, dtype):
    b = Batch4([300, 100, 40], [3, 100, 2], 4, 2, d, dtype, page=16, room=3)
    seen = [[True] * n for n in b.lens]
    for s, pages in ((0, (0, 5, 18)), (1, (2,)), (2, (0, 1, 2))):
        for at in pages:
            b.table[s, at] = -1 if at % 2 else 1 << 20
            for j in range(at * 16, min(at * 16 + 16, b.lens[s])):
                seen[s][j] = False
    b.dev["table"] = b.table.cuda()
    o, lse = _attention(b)
    _check(b, o, lse, seen=seen)
    assert (o[int(b.start[2]):int(b.start[3])] == 0).all()   # nothing of it is there


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [64, 128])
def test_wide_scores_and_far_scales(d, dtype):
    """Scores of up to some hundreds, rows whose largest comes last, scales from 2^-100 to 2^60 within one tile."""
    def edit(s, which, codes, scales):
        if which == "v":
            scales[:] = torch.tensor([27, 187, 127, 100], dtype=torch.uint8)[torch.arange(scales.shape[1]) % 4][None, :, None]
        else:
            scales[:, -1] += 4
    b = Batch4([150, 900], [20, 1], 4, 2, d, dtype, page=16, scale=8.0, edit=edit)
    o, lse = _attention(b)
    _check(b, o, lse)


@pytest.mark.parametrize("dtype", [BF, F])
def test_scores_far_below_zero(dtype):
    """All scores of a row near -3e4 and beyond -1e30: the row is the softmax of them all the same."""
    for size in (1e3, 1e30):
        b = Batch4([100], [2], 2, 1, 64, dtype, page=16)
        q = b.dev["q"] * 0 + 1.0
        q *= size
        k = -torch.ones(1, 100, 64).double()
        k[0, 50:] = -1.5
        codes, scales = encode(k)
        for j in range(7):
            m = min(16, 100 - 16 * j)
            b.cache4[0][b.table[0, j].item(), :, :m] = codes[:, 16 * j:16 * j + m].cuda()
            b.cache4[1][b.table[0, j].item(), :, :m] = scales[:, 16 * j:16 * j + m].cuda()
        b.keys[0], b.q = decode(codes, scales), q.cpu()
        o, lse = _attention(b, q=q)
        want = b.values[0][0, :50].mean(0)
        err = (o[:, :].double() - want).abs()
        assert (err <= b.values[0][0, :50].abs().mean(0) * (2.0 ** -7 if dtype == BF else 2.0 ** -17) + want.abs() * 2.0 ** -8).all()
        low = -64 * float(q[0, 0, 0]) / 8 + math.log(50)
        assert ((lse.double() - low).abs() <= abs(low) * 2.0 ** -22 + 2.0 ** -17).all()


@pytest.mark.parametrize("dtype", [BF, F])
def test_offsets_past_32_bits(dtype):
    """Pages 1.5 GB apart, heads 300 MB: codes and scales of one buffer, places beyond 4 GB."""
    d, Hkv, page, n_pages = 64, 2, 16, 4
    store = torch.full((6 << 30,), 255, dtype=torch.uint8, device="cuda")
    code = lambda at: torch.as_strided(store, (n_pages, Hkv, page, d // 2), (1536 << 20, 300 << 20, 1 << 20, 1), at)   # noqa: E731
    scale = lambda at: torch.as_strided(store, (n_pages, Hkv, page, d // 32), (1536 << 20, 300 << 20, 1 << 20, 1), at)   # noqa: E731
    b = Batch4([50], [50], 4, Hkv, d, dtype, page=page, stored="old", spare=0)
    b.cache4 = (code(0), scale(4096), code(8192), scale(16384))
    b.cache_cpu = [t.cpu() for t in b.cache4]
    got = _append(b, b.raw[0].cuda(), b.raw[1].cuda())
    _same(got, _expected(b, b.raw[0].double(), b.raw[1].double()))
    o, lse = _attention(b)
    _check(b, o, lse, rows_of=[0, 15, 16, 33, 49])
    k, v = (torch.empty(50, Hkv, d, dtype=dtype, device="cuda") for _ in range(2))
    da.distr_attn_cache4_read(k, v, b.cache4, da.make_paged4_params(b.cache4, *b.index(), k=k, v=v))
    for x, want in ((k, b.keys[0]), (v, b.values[0])):
        assert torch.equal(x.cpu().double(), want.transpose(0, 1))


@pytest.mark.parametrize("dtype", [BF, F])
def test_steps_of_a_program(dtype):
    """A prompt in two chunks, then single tokens: append and attend, as they are used together, the later steps as one captured graph that is replayed
    with eager work between; every step against the definition, and against the same step made eagerly."""
    H, Hkv, d, page, n_seq = 4, 2, 64, 16, 3
    g = torch.Generator().manual_seed(11)
    total = [70, 33, 50]
    q, k, v = ([torch.randn(n, h, d, generator=g).to(dtype) for n in total] for h in (H, Hkv, Hkv))
    c, s = tables(128, d)
    w = (1 + 0.2 * torch.randn(d, generator=g)).to(F)
    eps = float(torch.tensor(1e-6, dtype=F))
    keys = [turn(normed(x.double(), w.double(), eps), c.double()[:n, None], s.double()[:n, None], "halves") for x, n in zip(k, total)]
    keys, values = [decode(*encode(x)) for x in keys], [decode(*encode(x.double())) for x in v]
    n_pages = 16
    cache = tuple(torch.full((n_pages, Hkv, page, x), 255, dtype=torch.uint8, device="cuda") for x in (d // 2, d // 32) * 2)
    table = torch.randperm(n_pages, generator=g)[:15].reshape(3, 5).to(torch.int32).cuda()
    kv_len, start = torch.zeros(n_seq, dtype=torch.int32, device="cuda"), torch.zeros(n_seq + 1, dtype=torch.int32, device="cuda")
    norm = dict(norm=True, eps=1e-6, k_weight=w.cuda(), rope="halves", cos=c.cuda(), sin=s.cuda())

    def buffers(n):
        return [torch.zeros(n, h, d, dtype=dtype, device="cuda") for h in (H, Hkv, Hkv, H)]

    def plans(bq, bk, bv, lse):
        p = da.make_paged4_params(cache, table, kv_len, start, q=bq, lse_out=lse)
        ws = torch.empty(da.distr_attn_paged4_workspace_bytes(p), dtype=torch.uint8, device="cuda")
        return da.make_paged4_params(cache, table, kv_len, start, k=bk, v=bv, **norm), da.make_paged4_params(cache, table, kv_len, start, q=bq, lse_out=lse, workspace=ws)

    def check(done, fresh, o, lse):
        row = 0
        for i in range(n_seq):
            for j in range(fresh[i]):
                n = done[i] + j + 1
                for h in range(H):
                    sc = keys[i][:n, h // 2] @ q[i][n - 1, h].double() / 8
                    want, vv = torch.softmax(sc, 0) @ values[i][:n, h // 2], torch.softmax(sc, 0) @ values[i][:n, h // 2].abs()
                    err = (o[row, h].cpu().double() - want).abs()
                    assert (err <= vv * (2.0 ** -7 if dtype == BF else 2.0 ** -16) + want.abs() * 2.0 ** -8).all(), (i, j, h)
                    assert abs(float(lse[row, h]) - float(torch.logsumexp(sc, 0))) <= 2.0 ** -16
                row += 1

    done = [0, 0, 0]
    for fresh in ([40, 20, 30], [20, 3, 10]):
        bq, bk, bv, o = buffers(sum(fresh))
        lse = torch.zeros(sum(fresh), H, device="cuda")
        for buf, src in ((bq, q), (bk, k), (bv, v)):
            buf.copy_(torch.cat([x[d0:d0 + f] for x, d0, f in zip(src, done, fresh)]))
        kv_len.copy_(torch.tensor([a + f for a, f in zip(done, fresh)], dtype=torch.int32))
        start.copy_(torch.tensor([sum(fresh[:i]) for i in range(4)], dtype=torch.int32))
        pa, pf = plans(bq, bk, bv, lse)
        da.distr_attn_cache4_append(bk, bv, cache, pa)
        da.distr_attn_paged4_fwd(bq, cache, o, pf)
        torch.cuda.synchronize()
        check(done, fresh, o, lse)
        done = [a + f for a, f in zip(done, fresh)]
    bq, bk, bv, o = buffers(3)
    lse = torch.zeros(3, H, device="cuda")
    start.copy_(torch.arange(4, dtype=torch.int32))
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        pa, pf = plans(bq, bk, bv, lse)
        da.distr_attn_cache4_append(bk, bv, cache, pa)
        da.distr_attn_paged4_fwd(bq, cache, o, pf)
    kept = [pa, pf]   # (the graph reads what they hold)
    for step in range(8):
        for buf, src in ((bq, q), (bk, k), (bv, v)):
            buf.copy_(torch.stack([x[d0] for x, d0 in zip(src, done)]))
        kv_len.copy_(torch.tensor([a + 1 for a in done], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        check(done, [1, 1, 1], o, lse)
        o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
        ea, ef = plans(bq, bk, bv, lse2)
        da.distr_attn_cache4_append(bk, bv, cache, ea)
        da.distr_attn_paged4_fwd(bq, cache, o2, ef)
        torch.cuda.synchronize()
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        done = [a + 1 for a in done]
    assert kept


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("Hkv,d,page", [(1, 64, 16), (1, 128, 48), (2, 64, 64), (3, 128, 16), (7, 64, 32), (16, 64, 16), (100, 64, 16)])
def test_reads_of_many_tokens(Hkv, d, page, dtype):
    """Workgroups of several tokens: numbers of heads that divide their rows, that do not, and a single one."""
    n = [70000 // (Hkv * d // 64) // 2, 1, 0, 70000 // (Hkv * d // 64) // 3 + 5]
    g = torch.Generator().manual_seed(Hkv)
    need = [-(-x // page) for x in n]
    n_pages = sum(need) + 2
    table = torch.full((4, max(need)), -1, dtype=torch.int32)
    ids, at = torch.randperm(n_pages, generator=g).to(torch.int32), 0
    for s, m in enumerate(need):
        table[s, :m] = ids[at:at + m]
        at += m
    cache = [torch.randint(0, 256, (n_pages, Hkv, page, d // 2), generator=g, dtype=torch.uint8), torch.randint(100, 140, (n_pages, Hkv, page, d // 32), generator=g, dtype=torch.uint8),
             torch.randint(0, 256, (n_pages, Hkv, page, d // 2), generator=g, dtype=torch.uint8), torch.randint(100, 140, (n_pages, Hkv, page, d // 32), generator=g, dtype=torch.uint8)]
    dev = tuple(t.cuda() for t in cache)
    start = torch.tensor([1 + sum(n[:i]) for i in range(5)], dtype=torch.int32)
    k, v = (torch.full((sum(n) + 2, Hkv, d), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    p = da.make_paged4_params(dev, table.cuda(), torch.tensor(n, dtype=torch.int32).cuda(), start.cuda(), k=k, v=v)
    da.distr_attn_cache4_read(k, v, dev, p)
    for x, codes, scales in ((k, cache[0], cache[1]), (v, cache[2], cache[3])):
        want = torch.full(x.shape, 7.0, dtype=torch.float64)
        for s, m in enumerate(n):
            ids = table[s, :need[s]].long()
            want[start[s]:start[s] + m] = decode(codes[ids], scales[ids]).transpose(1, 2).reshape(-1, Hkv, d)[:m]
        assert torch.equal(x.cpu().double(), want)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [1e3, 1e9, 1e30, -1e9, -1e30])
def test_chunks_of_far_scores(d, dtype, size):
    """Scores of thousands to 1e32 of either sign: the keys of the largest one alone have weight, all of them the same (products and sums of equal numbers are exact)."""
    n, new = 200, 70
    b = Batch4([n, n], [new, new], 4, 2, d, dtype, page=16)
    q = torch.full_like(b.dev["q"], abs(size))
    k = torch.ones(2, n, d).double()
    k[:, 90:] = 0.5 if size > 0 else 1.5
    k *= math.copysign(1.0, size)
    codes, scales = encode(k)
    for s in range(2):
        for j in range(-(-n // 16)):
            m = min(16, n - 16 * j)
            b.cache4[0][b.table[s, j].item(), :, :m] = codes[:, 16 * j:16 * j + m].cuda()
            b.cache4[1][b.table[s, j].item(), :, :m] = scales[:, 16 * j:16 * j + m].cuda()
    o, lse = _attention(b, q=q)
    value = float(q[0, 0, 0])
    low = math.copysign(1.0, size) * d * value / math.sqrt(d)
    for s in range(2):
        v = b.values[s][:, :90]
        want, most = v.mean(1).repeat_interleave(2, 0), v.abs().mean(1).repeat_interleave(2, 0)
        err = (o[s * new:(s + 1) * new].double() - want).abs()
        # (90 equal weights, whatever the parts: the same products in the same order. bf16: rounded once, above and below)
        assert (err <= most * (2.0 ** -7 if dtype == BF else 2.0 ** -17) + want.abs() * 2.0 ** -8).all()
    want = low + math.log(90)
    assert ((lse.double() - want).abs() <= abs(want) * 2.0 ** -21 + 2.0 ** -15).all()
