"""Appending to a paged cache and attention over it against 64 bits: ragged batches, page sizes and orders, empty rows, absent
pages, what lies beside the sequences, streams and graphs."""
import pytest
import torch

import paper_2507_17245_amd as da
from paged_util import HALF_STEP, Batch, attend, attention_bounds, normed, tables, turn, turn_bound

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


# Tokens that a row of the page table has room for beyond the longest sequence: with few the units of a call stay whole, with many they go by ranges.
ROOMY = [0, 5000]


def _attention(b, causal=True, scale=None, lse=True, workspace=True, q=None):
    """-> o, lse of one call on the batch; o is NaN where nothing is written"""
    q = b.dev["q"] if q is None else q
    o = torch.full((b.T, b.H, b.d), float("nan"), dtype=b.dtype, device="cuda")
    row = torch.full((b.T, b.H), float("nan"), device="cuda") if lse else None
    options = dict(q=q, causal=causal, softmax_scale=0.0 if scale is None else scale, lse_out=row)
    ws = None
    if workspace is not None:
        n = da.distr_attn_paged_workspace_bytes(da.make_paged_params(*b.cache(), **options))
        ws = torch.full((n if workspace is True else workspace,), 255, dtype=torch.uint8, device="cuda")
    da.distr_attn_paged_fwd(q, b.k_pages, b.v_pages, o, da.make_paged_params(*b.cache(), workspace=ws, **options))
    torch.cuda.synchronize()
    return o.cpu(), row.cpu() if lse else None


def _check(b, o, lse, causal=True, scale=None, seen=None, rows_of=None, only=None):
    """Every row of every sequence (rows_of: some of its new tokens; only: some sequences) and that no others were written."""
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
        err = (o[rows].double() - want).abs()
        assert (err <= bound).all(), (s, (err / bound).max())
        if lse is not None:
            empty = ln.isinf()
            assert torch.equal(lse[rows].isinf(), empty) and (lse[rows][empty] < 0).all()
            assert ((lse[rows].double() - ln).abs()[~empty] <= ln_bound[~empty]).all()
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
]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("case", RAGGED)
@pytest.mark.parametrize("roomy", ROOMY)
def test_ragged_batches(case, dtype, roomy):
    lens, new, H, Hkv, d, page, order = case
    b = Batch(lens, new, H, Hkv, d, dtype, page=page, order=order, pad_front=1, pad_back=2, room=1 + roomy // page)
    some = [0, 1, 2, 3, 7, 8, 30, 31, 32, 33, 63, 64, 69, 127, 128, 129, 149, 199, 259]
    for causal in (True, False):
        o, lse = _attention(b, causal=causal)
        _check(b, o, lse, causal=causal, rows_of=some)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("workspace", [True, None, 0, 300000])
def test_long_rows_with_any_scratch(d, dtype, workspace):
    """Keys dealt out to many workgroups, to a few, and kept together."""
    lens, new = [5000, 3, 1500], [2, 1, 30]
    b = Batch(lens, new, 8, 2, d, dtype, page=32, scale=3.0)
    if workspace == 0:
        workspace = 256
    o, lse = _attention(b, workspace=workspace)
    _check(b, o, lse, rows_of=[0, 1, 15, 29])
    again, lse2 = _attention(b, workspace=workspace)
    assert torch.equal(o.isnan(), again.isnan()) and torch.equal(o.nan_to_num(), again.nan_to_num()) and torch.equal(lse.nan_to_num(), lse2.nan_to_num())


@pytest.mark.parametrize("dtype", [BF, F])
def test_without_row_statistics(dtype):
    b = Batch([300, 2000], [3, 1], 8, 2, 64, dtype)
    o, lse = _attention(b)
    plain, _ = _attention(b, lse=False)
    assert torch.equal(o, plain)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n_seq", [63, 64, 65, 200])
@pytest.mark.parametrize("roomy", ROOMY)
def test_many_sequences(n_seq, dtype, roomy):
    g = torch.Generator().manual_seed(n_seq)
    lens = torch.randint(0, 120, (n_seq,), generator=g).tolist()
    new = [min(int(x), n) for x, n in zip(torch.randint(0, 4, (n_seq,), generator=g), lens)]
    b = Batch(lens, new, 4, 2, 64, dtype, pad_back=1, room=roomy // 16)
    o, lse = _attention(b)
    _check(b, o, lse)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n_seq", [300, 4096, 4200])
@pytest.mark.parametrize("roomy", ROOMY)
def test_very_many_sequences(n_seq, dtype, roomy):
    """More than a wave's lanes of them, and more than the sums of 64 that a workgroup keeps; with and without ranges."""
    g = torch.Generator().manual_seed(n_seq)
    lens = torch.randint(0, 40, (n_seq,), generator=g).tolist()
    lens[n_seq - 2] = 1500
    new = [min(int(x), n) for x, n in zip(torch.randint(0, 3, (n_seq,), generator=g), lens)]
    new[n_seq - 2], new[70] = 33, 0
    b = Batch(lens, new, 2, 1, 64, dtype, room=roomy // 16)
    only = [0, 1, 63, 64, 65, 69, 70, 71, 127, 128, 255, 256, n_seq - 3, n_seq - 2, n_seq - 1] + list(range(200, 210))
    for workspace in (True, 256):
        o, lse = _attention(b, workspace=workspace)
        _check(b, o, lse, only=only, rows_of=[0, 1, 31, 32])
        assert o.isfinite().all()


@pytest.mark.parametrize("d", [64, 128])
def test_prompts_that_fill_the_chip(d):
    """Enough units for workgroups of their own: whole prompts, one behind a prefix, a single token and none beside them."""
    lens, new = [1100, 700, 65, 130, 40], [1000, 140, 65, 1, 0]
    b = Batch(lens, new, 64, 64, d, BF, page=64, order="tokens")
    o, lse = _attention(b)
    _check(b, o, lse, rows_of=[0, 63, 64, 127, 128, 139, 512, 999])
    o, _ = _attention(b, causal=False, lse=False)
    _check(b, o, None, causal=False, rows_of=[0, 64, 139, 999])


FORMS = [  # sequences, H, Hkv, d, longest, page: kv heads of the sequences beside 256, 512 compute units' worth; ranges and whole units
    (40, 8, 2, 64, 1500, 16, "heads"),
    (9, 32, 1, 128, 2300, 64, "tokens"),
    (100, 8, 4, 64, 1500, 16, "tokens"),
    (70, 12, 4, 128, 900, 16, "heads"),
    (100, 8, 4, 128, 1500, 32, "heads"),
    (150, 8, 4, 64, 1400, 16, "heads"),
    (150, 4, 4, 128, 1400, 16, "tokens"),
    (600, 2, 1, 64, 150, 16, "heads"),
    (300, 64, 2, 64, 100, 16, "heads"),
]


@pytest.mark.parametrize("case", FORMS)
@pytest.mark.parametrize("workspace", [True, None, 4 << 20])
@pytest.mark.parametrize("roomy", ROOMY)
def test_single_tokens_of_many_sequences(case, workspace, roomy):
    """One new token each (none for some): workgroups of eight, four and two waves, many units to a range and many ranges to a unit."""
    n_seq, H, Hkv, d, most, page, order = case
    g = torch.Generator().manual_seed(n_seq + d)
    lens = torch.randint(0, most // 2, (n_seq,), generator=g).tolist()
    lens[1], lens[n_seq // 2], lens[n_seq - 1], lens[3] = most, most - 1, 64, 0
    new = [1 if n else 0 for n in lens]
    new[5] = 0
    b = Batch(lens, new, H, Hkv, d, BF, page=page, order=order, pad_back=1, room=roomy // page)
    assert b.T <= n_seq and H // Hkv <= 32
    only = [0, 1, 2, 3, 4, 5, 6, n_seq // 2, n_seq - 2, n_seq - 1] + list(range(n_seq // 3, n_seq // 3 + 6))
    o, lse = _attention(b, workspace=workspace)
    _check(b, o, lse, only=only)
    assert o[:-1].isfinite().all()
    plain, _ = _attention(b, workspace=workspace, lse=False, causal=False)
    _check(b, plain, None, causal=False, only=only)


@pytest.mark.parametrize("n_seq,Hkv", [(100, 1), (100, 4), (150, 4)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("roomy", ROOMY)
def test_a_prompt_among_places_without_new_tokens(n_seq, Hkv, d, roomy):
    """No more new tokens than sequences, most of them one sequence's: more rows than a unit of single tokens has. A NaN in a value that
    the last token alone sees reaches it alone."""
    lens, new = [30] * n_seq, [0] * n_seq
    lens[7], new[7], lens[50], new[50] = 700, 90, 1300, 1
    H = 3 * Hkv
    b, clean = (Batch(lens, new, H, Hkv, d, BF, page=16, room=roomy // 16) for _ in range(2))
    b.v_pages[int(b.table[7, 699 // 16]), :, 699 % 16, 9] = float("nan")
    for workspace in (True, 256):
        o, lse = _attention(b, workspace=workspace)
        assert o[89, :, 9].isnan().all()
        o[89, :, 9] = _attention(clean, workspace=workspace)[0][89, :, 9]
        assert o.isfinite().all()
        _check(clean, o, lse, only=[7, 50], rows_of=[0, 1, 9, 10, 11, 20, 21, 22, 42, 43, 63, 64, 88, 89])


@pytest.mark.parametrize("workspace", [True, None, 3 << 20])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("roomy", ROOMY)
def test_a_few_tokens_of_many_sequences(workspace, d, roomy):
    """Up to five new tokens each beside a prompt: ranges for two workgroups a compute unit, for one, and what a small scratch has room for."""
    g = torch.Generator().manual_seed(d)
    n_seq, Hkv = 75, 4
    lens = torch.randint(5, 900, (n_seq,), generator=g).tolist()
    new = torch.randint(1, 6, (n_seq,), generator=g).tolist()
    lens[20], new[20], lens[21], lens[74], new[74] = 1500, 150, 1400, 1400, 33
    b = Batch(lens, new, 8, Hkv, d, BF, page=32, order="tokens", room=roomy // 32)
    assert n_seq * Hkv > 256
    o, lse = _attention(b, workspace=workspace)
    only = [0, 1, 19, 20, 21, 22, 40, 63, 64, 65, 73, 74]
    _check(b, o, lse, only=only, rows_of=[0, 1, 2, 3, 4, 31, 32, 63, 64, 149])
    again, lse2 = _attention(b, workspace=workspace)
    assert torch.equal(o, again) and torch.equal(lse, lse2) and o.isfinite().all()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("new", [2, 150])
@pytest.mark.parametrize("roomy", ROOMY)
def test_scores_that_are_no_numbers(new, dtype, roomy):
    """A NaN or an infinity in one query row, and in one key, reaches the rows of its scores and no others."""
    n = new + 90
    b, clean = (Batch([n], [new], 4, 2, 64, dtype, room=roomy // 16) for _ in range(2))
    b.dev["q"][1, 2, 7] = float("nan")
    place = n - 1                                    # a key that the last token alone sees
    b.k_pages[int(b.table[0, place // 16]), 1, place % 16, 3] = float("inf")
    (o, lse), (oc, lc) = _attention(b), _attention(clean)
    odd = torch.zeros(new, 4, dtype=torch.bool)
    odd[1, 2] = True
    # an infinite score: NaN where it is the largest, nothing where the smallest
    high = b.q[-1, 2:].float()[:, 3] > 0
    odd[-1, 2:] |= high
    low = torch.zeros_like(odd)
    low[-1, 2:] = ~high
    low &= ~odd
    assert o[odd].isnan().all() and lse[odd].isnan().all() and o[~odd].isfinite().all() and lse[~odd].isfinite().all()
    same = ~odd & ~low
    _check(clean, oc, lc, rows_of=[0, 1, new // 2, new - 1])
    o[odd | low], lse[odd | low] = oc[odd | low], lc[odd | low]
    _check(clean, o, lse, rows_of=[0, 1, new // 2, new - 1])
    assert same.sum() >= 4 * new - 3


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("new", [1, 40, 200])
@pytest.mark.parametrize("roomy", ROOMY)
def test_rows_that_see_no_key(new, dtype, roomy):
    """More new tokens than the sequence has tokens: the first see nothing. A length of none: no row sees any."""
    lens, fresh = [max(new - 7, 0), 0, 50], [new, 2, 1]
    b = Batch(lens, fresh, 4, 2, 64, dtype, room=2 + roomy // 16)
    o, lse = _attention(b)
    _check(b, o, lse, rows_of=[0, 1, 5, 6, 7, 8, 30, 32, 39, 40, 150, 199])
    assert (o[new:new + 2] == 0).all() and (lse[new:new + 2] == -float("inf")).all()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("new", [1, 140])
@pytest.mark.parametrize("roomy", ROOMY)
def test_pages_that_are_none_of_the_cache(new, dtype, roomy):
    lens = [400, 90, 16]
    b = Batch(lens, [new, 1, 1], 4, 1, 64, dtype, page=16, room=roomy // 16)
    n_pages = b.k_pages.shape[0]
    seen = [[True] * n for n in lens]
    for s, i, value in ((0, 3, -1), (0, 7, n_pages), (0, 24, 2 ** 31 - 1), (1, 0, -2 ** 31), (2, 0, n_pages + 5)):
        b.table[s, i] = value
        for j in range(16 * i, min(16 * i + 16, lens[s])):
            seen[s][j] = False
    b.dev["table"] = b.table.cuda()
    o, lse = _attention(b)
    _check(b, o, lse, seen=seen, rows_of=[0, 1, 63, 100, 139])
    assert (o[-1] == 0).all()


@pytest.mark.parametrize("dtype", [BF, F])
def test_lengths_beyond_the_table_and_starts_out_of_order(dtype):
    """What the arrays on the device hold is not checked: no access leaves the buffers, and sequences that are in order come out right."""
    b = Batch([64, 40], [1, 3], 4, 2, 64, dtype)
    b.dev["kv_len"] = torch.tensor([2 ** 31 - 1, 40], dtype=torch.int32, device="cuda")
    o, _ = _attention(b, causal=False)
    b.dev["kv_len"] = torch.tensor([64, 40], dtype=torch.int32, device="cuda")
    want, _ = _attention(b, causal=False)
    assert torch.equal(o, want)          # (the table has room for 64)
    b.dev["kv_len"] = torch.tensor([-5, 40], dtype=torch.int32, device="cuda")
    o, _ = _attention(b)
    assert (o[0] == 0).all() and torch.equal(o[1:], _attention(Batch([64, 40], [1, 3], 4, 2, 64, dtype))[0][1:])
    b.dev["start"] = torch.tensor([3, -7, 90], dtype=torch.int32, device="cuda")
    _attention(b)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("new", [1, 100, 300])
@pytest.mark.parametrize("roomy", ROOMY)
def test_values_that_later_tokens_alone_see(new, dtype, roomy):
    """An infinity or a NaN in a value (and a key) reaches the rows that see it and no others."""
    b = Batch([new + 70], [new], 4, 2, 64, dtype, room=roomy // 16)
    last, mid = new + 69, 70 + new // 2
    for place, what in ((last, float("nan")), (mid, float("inf"))):
        page, row = int(b.table[0, place // 16]), place % 16
        b.v_pages[page, :, row, 5] = what
        b.values[0][:, place, 5] = what
    o, lse = _attention(b)
    clean = Batch([new + 70], [new], 4, 2, 64, dtype, room=roomy // 16)
    oc, lc = _attention(clean)
    # What they do not reach is what it would be without them, to the bounds of any call (rows with such values may be summed in another order).
    rest = o.clone()
    rest[new // 2 if new > 1 else 0:, :, 5] = oc[new // 2 if new > 1 else 0:, :, 5]
    some = [max(i, 0) for i in (0, 1, new // 2 - 1, new // 2, new - 2, new - 1)]
    _check(clean, oc, lc, rows_of=some)
    _check(clean, rest, lse, rows_of=some)
    assert rest.isfinite().all() and ((rest - oc).abs() <= 4 * HALF_STEP[BF] * (clean.values[0].abs().max())).all()
    assert (o[-1, :, 5].isnan() if new > 1 else o[-1, :, 5] == float("inf")).all()   # (of one token, the second value stands)
    if new > 1:
        assert (o[new // 2:-1, :, 5] == float("inf")).all()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("roomy", ROOMY)
def test_large_scores(dtype, roomy):
    """Scores of thousands: one key takes a row's whole weight."""
    b = Batch([600, 40], [5, 40], 4, 2, 64, dtype, scale=1000.0, room=roomy // 16)
    o, lse = _attention(b)
    _check(b, o, lse)
    o, lse = _attention(b, scale=1e-3)
    _check(b, o, lse, scale=1e-3)


def test_offsets_beyond_32_bits():
    """A cache of 9 GiB whose pages in use lie at its far end."""
    page, Hkv, d, n = 64, 8, 64, 300
    n_pages = (9 << 30) // (2 * page * Hkv * d * 2)
    pool = torch.empty(n_pages, 2, Hkv, page, d, dtype=BF, device="cuda")
    b = Batch([n], [3], 16, Hkv, d, BF, page=page)
    ids = [n_pages - 1 - 3 * i for i in range(-(-n // page))]
    for i, at in enumerate(ids):
        old = int(b.table[0, i])
        pool[at, 0], pool[at, 1] = b.k_pages[old], b.v_pages[old]
    b.k_pages, b.v_pages = pool[:, 0], pool[:, 1]
    b.dev["table"] = torch.tensor([ids], dtype=torch.int32, device="cuda")
    o, lse = _attention(b)
    _check(b, o, lse)
    k, v = (torch.randn(3, Hkv, d, dtype=BF, device="cuda") for _ in (0, 1))
    da.distr_attn_cache_append(k, v, b.k_pages, b.v_pages, da.make_paged_params(*b.cache(), k=k, v=v))
    torch.cuda.synchronize()
    for t in range(3):
        place = n - 3 + t
        assert torch.equal(pool[ids[place // page], 0, :, place % page], k[t]) and torch.equal(pool[ids[place // page], 1, :, place % page], v[t])


def test_strided_queries():
    b = Batch([500, 30], [9, 1], 4, 2, 128, BF)
    o, _ = _attention(b)
    wide = torch.full((b.T, 7, 128 + 8), float("nan"), dtype=BF, device="cuda")
    q = wide[:, 1:5, 8:]
    q.copy_(b.dev["q"])
    assert torch.equal(_attention(b, q=q)[0], o)
    q = b.dev["q"].transpose(0, 1).contiguous().transpose(0, 1)    # [H, T, d] underneath
    assert torch.equal(_attention(b, q=q)[0], o)
    q = b.dev["q"][:, :1].expand(-1, 4, -1)                        # one head for all of them
    assert torch.equal(_attention(b, q=q)[0], _attention(b, q=q.contiguous())[0])


def test_agrees_with_the_contiguous_kernels():
    """One page a sequence is a contiguous cache: the library's exact attention on the same tensors."""
    n, fresh, H, Hkv, d = 512, 200, 8, 2, 64
    b = Batch([n], [fresh], H, Hkv, d, BF, page=512, spare=0)
    o, lse = _attention(b)
    q = b.dev["q"].transpose(0, 1).contiguous()[None]
    k, v = b.k_pages.contiguous(), b.v_pages.contiguous()
    dense, ln = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    da.distr_attn_exact_fwd_ex(q, k, v, dense, da.make_params(q, k, v, Br=64, causal=True, lse_out=ln))
    torch.cuda.synchronize()
    # two roundings of weights and results of magnitude up to 1 at the most
    assert (dense[0].transpose(0, 1).float().cpu() - o.float()).abs().max() <= 4 * 2.0 ** -8 * max(1.0, o.float().abs().max().item())
    assert (ln[0].T.cpu() - lse).abs().max() <= 2.0 ** -8


# ---- appending -----------------------------------------------------------------------------------------

APPEND = [  # lens, new, Hkv, d, dtype, page, order, rope, rot, norm, weight heads, positions
    ([1], [1], 1, 64, BF, 16, "heads", "halves", 64, True, False, False),
    ([5, 40, 16, 17], [1, 1, 1, 1], 8, 64, BF, 16, "heads", "halves", 64, True, False, False),
    ([70, 3, 200], [33, 3, 1], 2, 128, BF, 64, "tokens", "halves", 128, False, False, False),
    ([70, 0, 50, 9], [17, 0, 50, 1], 1, 64, F, 16, "heads", "neighbours", 32, True, True, True),
    ([300], [129], 3, 128, F, 48, "tokens", "halves", 48, True, False, False),
    ([33, 20], [2, 20], 4, 64, BF, 32, "tokens", "none", 0, True, True, False),
    ([33, 20], [2, 20], 4, 128, BF, 32, "heads", "none", 0, False, False, False),
    ([20] * 130, [1] * 130, 1, 64, BF, 16, "heads", "halves", 64, False, False, False),
    ([9] * 90, [i % 3 for i in range(90)], 2, 64, F, 16, "heads", "halves", 64, False, False, True),
]


@pytest.mark.parametrize("case", APPEND)
def test_append(case):
    lens, new, Hkv, d, dtype, page, order, rope, rot, norm, heads, spread = case
    b = Batch(lens, new, Hkv, Hkv, d, dtype, page=page, order=order, stored="old", pad_front=2, pad_back=3)
    g = torch.Generator().manual_seed(1)
    x = torch.randn(b.T, 2, Hkv, d, generator=g).to(dtype)
    k, v = (x.cuda()[:, i] for i in (0, 1))
    w = (1 + 0.3 * torch.randn((Hkv, d) if heads else (d,), generator=g)) if norm else None
    n_pos = max(lens) + 2
    cos, sin = tables(n_pos, rot) if rot else (None, None)
    positions = torch.randint(0, n_pos, (b.T,), generator=g).to(torch.int32) if spread else None
    dev = lambda t: None if t is None else t.cuda()   # noqa: E731
    p = da.make_paged_params(*b.cache(), k=k, v=v, norm=norm, eps=1e-5, k_weight=dev(w), rope=rope, cos=dev(cos), sin=dev(sin), positions=dev(positions))
    da.distr_attn_cache_append(k, v, b.k_pages, b.v_pages, p)
    torch.cuda.synchronize()
    want_k, want_v = (t.double().cpu().clone() for t in (b.pool_cpu[:, 0] if order == "heads" else b.pool_cpu[:, 0].transpose(1, 2),
                                                          b.pool_cpu[:, 1] if order == "heads" else b.pool_cpu[:, 1].transpose(1, 2)))
    bound = torch.zeros_like(want_k)
    for s in range(len(lens)):
        for i in range(new[s]):
            t, place = int(b.start[s]) + i, lens[s] - new[s] + i
            y = x[t, 0].double()
            if norm:
                y = normed(y, w.double(), 1e-5)
            unit = turn_bound(y, rot, rope)
            if rot:
                at = int(positions[t]) if spread else place
                y = turn(y, cos[at].double(), sin[at].double(), rope)
            at = int(b.table[s, place // page])
            want_k[at, :, place % page], want_v[at, :, place % page] = y, x[t, 1].double()
            bound[at, :, place % page] = HALF_STEP[dtype] * 1.01 * y.abs() + 24 * 2.0 ** -24 * unit if norm or rot else 0.0
    got_k, got_v = b.k_pages.double().cpu(), b.v_pages.double().cpu()
    assert torch.equal(got_v.isnan(), want_v.isnan()) and torch.equal(got_v.nan_to_num(), want_v.nan_to_num())
    assert torch.equal(got_k.isnan(), want_k.isnan())
    assert ((got_k - want_k).abs().nan_to_num() <= bound).all()


def test_append_leaves_what_has_no_place():
    """Tokens of negative places, behind the table's end, on pages that are none, and of no sequence are not stored."""
    b = Batch([40, 3, 64, 20], [1, 5, 2, 1], 2, 2, 64, BF, stored="old", pad_front=1, pad_back=1)
    b.dev["kv_len"] = torch.tensor([40, 3, 66, 20], dtype=torch.int32, device="cuda")   # the third: one behind its 64 and the next
    b.table[3, 1] = b.k_pages.shape[0]
    b.table[0, 2] = -3
    b.dev["table"] = b.table.cuda()
    k, v = (torch.randn(b.T, 2, 64, dtype=BF, device="cuda") for _ in (0, 1))
    before = b.k_pages.clone(), b.v_pages.clone()
    da.distr_attn_cache_append(k, v, b.k_pages, b.v_pages, da.make_paged_params(*b.cache(), k=k, v=v))
    torch.cuda.synchronize()
    # the second sequence: places -2, -1, 0, 1, 2
    page = int(b.table[1, 0])
    for new, old, x in ((b.k_pages, before[0], k), (b.v_pages, before[1], v)):
        assert torch.equal(new[page, :, :3], x[4:7].transpose(0, 1))
        changed = (new != old) & ~(new.isnan() & old.isnan())
        changed[page, :, :3] = False
        assert not changed.any()


# ---- together --------------------------------------------------------------------------------------------

class Layer:
    """What a serving program does for a layer in each step: queries normed and rotated, keys on their way into the cache, attention."""

    def __init__(self, b, T, seed=3):
        g = torch.Generator().manual_seed(seed)
        H, Hkv, d = b.H, b.Hkv, b.d
        self.b, self.T = b, T
        self.x = torch.zeros(T, (H + 2 * Hkv) * d, dtype=b.dtype, device="cuda")
        self.qw, self.kw = (1 + 0.2 * torch.randn(d, generator=g) for _ in (0, 1))
        self.cos, self.sin = tables(512, d)
        self.q, self.k, self.v = (t.unflatten(-1, (-1, d)) for t in self.x.split((H * d, Hkv * d, Hkv * d), -1))
        self.positions = torch.zeros(1, T, dtype=torch.int32, device="cuda")
        self.rotated, self.o = (torch.empty(T, H, d, dtype=b.dtype, device="cuda") for _ in (0, 1))
        cos, sin, kw = self.cos.cuda(), self.sin.cuda(), self.kw.cuda()
        self.qk = da.make_qk_params(self.q.transpose(0, 1)[None], None, self.rotated.transpose(0, 1)[None], None, norm=True, eps=1e-6, q_weight=self.qw.cuda(),
                                    rope="halves", cos=cos, sin=sin, positions=self.positions)
        options = dict(q=self.rotated, k=self.k, v=self.v, norm=True, eps=1e-6, k_weight=kw, rope="halves", cos=cos, sin=sin)
        self.ws = torch.empty(da.distr_attn_paged_workspace_bytes(da.make_paged_params(*b.cache(), **options)), dtype=torch.uint8, device="cuda")
        self.paged = da.make_paged_params(*b.cache(), workspace=self.ws, **options)

    def run(self):
        da.distr_attn_qk_norm_rope(self.q.transpose(0, 1)[None], None, self.rotated.transpose(0, 1)[None], None, self.qk)
        da.distr_attn_cache_append(self.k, self.v, self.b.k_pages, self.b.v_pages, self.paged)
        da.distr_attn_paged_fwd(self.rotated, self.b.k_pages, self.b.v_pages, self.o, self.paged)


def _step_reference(layer, history, x, place):
    """Output of a token whose projections are x, at `place`, behind the (k, v) of history, in 64 bits with the cache's roundings."""
    b = layer.b
    H, Hkv, d = b.H, b.Hkv, b.d
    q, k, v = x.double().cpu().split((H * d, Hkv * d, Hkv * d))
    c, s = layer.cos[place].double(), layer.sin[place].double()
    q = turn(normed(q.view(H, d), layer.qw.double(), 1e-6), c, s, "halves").to(b.dtype).double()
    k = turn(normed(k.view(Hkv, d), layer.kw.double(), 1e-6), c, s, "halves").to(b.dtype).double()
    history.append((k, v.view(Hkv, d)))
    ks, vs = (torch.stack([h[i] for h in history], 1) for i in (0, 1))
    return attend(q[None], ks, vs, [place], place + 1, d ** -0.5)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("captured", [False, True])
def test_serving_steps(captured, dtype):
    """Sequences that grow from nothing by a token a step, eager and as one captured step whose lengths change on the device."""
    n_seq, steps = 3, 40
    b = Batch([48, 48, 48], [1, 1, 1], 4, 2, 64, dtype, stored="old")
    b.pool_cpu.fill_(float("nan"))
    b.reset()
    first = torch.tensor([0, 5, 2], dtype=torch.int32)      # (the second and third begin with tokens that no step has stored: absent)
    layer = Layer(b, n_seq)
    g = torch.Generator().manual_seed(9)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        layer = Layer(b, n_seq)
        graph = None
        if captured:
            b.dev["kv_len"].fill_(1)
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                layer.run()
        histories = [[] for _ in range(n_seq)]
        worst = 0.0
        for step in range(steps):
            x = torch.randn(layer.x.shape, generator=g).to(dtype)
            layer.x.copy_(x)
            live = [s for s in range(n_seq) if step >= int(first[s])]
            length = torch.tensor([max(step + 1 - int(first[s]), 0) for s in range(n_seq)], dtype=torch.int32)
            b.dev["kv_len"].copy_(length)
            layer.positions.copy_((length - 1).clamp(min=0)[None])
            graph.replay() if graph is not None else layer.run()
            stream.synchronize()
            for s in range(n_seq):
                if s not in live:
                    assert (layer.o[s] == 0).all()
                    continue
                want, mean, ln, most = _step_reference(layer, histories[s], x[s], int(length[s]) - 1)
                bound, _ = attention_bounds(want, mean, ln, most, int(length[s]), 64, dtype)
                # a score's keys and query may be rounded the other way where float and 64 bits part: two half steps of it
                extra = 2 * 2 * HALF_STEP[dtype] * most.amax() * mean + (2 * 24 * 2.0 ** -24) * most.amax() * mean
                err = (layer.o[s].double().cpu() - want[0]).abs()
                assert (err <= (bound + extra)[0]).all(), (step, s)
                worst = max(worst, err.max().item())
        assert worst > 0


def test_the_null_stream_is_the_null_stream():
    """Calls of the short forms on another stream do not send the null stream's calls there."""
    b = Batch([300], [2], 4, 2, 64, BF)
    want, _ = _attention(b, lse=False)
    p = da.make_paged_params(*b.cache(), q=b.dev["q"])
    x = torch.randn(1, 2, 5, 64, device="cuda", dtype=BF)
    y, rotated = torch.empty_like(x), torch.empty_like(x)
    rows = da.make_qk_params(x, None, rotated, None, norm=True)
    da.distr_attn_qk_norm_rope(x, None, rotated, None, rows)
    expected = rotated.clone()
    o = torch.zeros(b.T, b.H, b.d, dtype=BF, device="cuda")
    rotated.zero_()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        da.distr_attn_exact_fwd(x, x, x, y, 64, 64)
        torch.cuda._sleep(400_000_000)               # the side stream is busy for a while
    da.distr_attn_paged_fwd(b.dev["q"], b.k_pages, b.v_pages, o, p)
    da.distr_attn_qk_norm_rope(x, None, rotated, None, rows)
    done = torch.cuda.Event()
    done.record()
    done.synchronize()
    busy = not side.query()
    got, turned = o.cpu(), rotated.cpu()
    torch.cuda.synchronize()
    if busy:                                         # (else nothing is shown)
        assert torch.equal(got, want) and torch.equal(turned, expected.cpu())


def test_streams_and_their_scratch():
    """Two streams at once, each with the library's buffer or its own: the results of one after the other."""
    batches = [Batch([3000, 700], [1, 2], 8, 2, 64, BF, seed=i) for i in range(2)]
    want = [_attention(b)[0] for b in batches]
    for own in (False, True):
        streams = [torch.cuda.Stream() for _ in batches]
        out = []
        torch.cuda.synchronize()
        for i, (b, st) in enumerate(zip(batches, streams)):
            with torch.cuda.stream(st):
                o = torch.full((b.T, b.H, b.d), float("nan"), dtype=BF, device="cuda")
                p = da.make_paged_params(*b.cache(), q=b.dev["q"])
                ws = torch.empty(da.distr_attn_paged_workspace_bytes(p), dtype=torch.uint8, device="cuda") if own else None
                p = da.make_paged_params(*b.cache(), q=b.dev["q"], workspace=ws)
                out.append((b, st, o, p))
        for _ in range(20):
            for b, st, o, p in out:
                da.distr_attn_paged_fwd(b.dev["q"], b.k_pages, b.v_pages, o, p)
        torch.cuda.synchronize()
        for (b, st, o, p), w in zip(out, want):
            assert torch.equal(o.cpu(), w)


def test_two_captured_graphs_with_a_scratch_each():
    batches = [Batch([2500, 900], [1, 1], 8, 2, 128, BF, seed=i) for i in range(2)]
    want = [_attention(b)[0] for b in batches]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(stream):
        for b in batches:
            o = torch.empty(b.T, b.H, b.d, dtype=BF, device="cuda")
            ws = torch.empty(da.distr_attn_paged_workspace_bytes(da.make_paged_params(*b.cache(), q=b.dev["q"])), dtype=torch.uint8, device="cuda")
            p = da.make_paged_params(*b.cache(), q=b.dev["q"], workspace=ws)
            none = torch.empty(b.T, b.H, b.d, dtype=BF, device="cuda")
            plain = da.make_paged_params(*b.cache(), q=b.dev["q"])      # no scratch under capture: keys stay together
            stream.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                da.distr_attn_paged_fwd(b.dev["q"], b.k_pages, b.v_pages, o, p)
                da.distr_attn_paged_fwd(b.dev["q"], b.k_pages, b.v_pages, none, plain)
            graphs.append((b, g, o, none, ws, p, plain))
        for _ in range(4):
            for (b, g, o, none, *_), w in zip(graphs, want):
                o.fill_(7.0)
                none.fill_(7.0)
                g.replay()
            stream.synchronize()
            for (b, g, o, none, *_), w in zip(graphs, want):
                assert torch.equal(o.cpu(), w)
                _check(b, none.cpu(), None)
            torch.zeros(1000, device="cuda").sum().item()


def test_no_new_tokens():
    b = Batch([40, 20], [0, 0], 4, 2, 64, BF)
    assert _attention(b, lse=False)[0].numel() == 0
    b = Batch([40, 20], [0, 0], 4, 2, 64, BF, pad_back=3)
    assert _attention(b, lse=False)[0].isnan().all()


def test_binding_refusals():
    b = Batch([40, 20], [1, 1], 4, 2, 64, BF)
    c, q = b.cache(), b.dev["q"]
    kv = torch.zeros(2, 2, 64, dtype=BF, device="cuda")
    cases = [(c, {}), (c, dict(k=kv)), ((c[0], c[1][:-1], *c[2:]), dict(q=q)), ((c[0], c[1].contiguous(), *c[2:]), dict(q=q)), ((*c[:2], c[2].long(), *c[3:]), dict(q=q)),
             ((*c[:3], c[3][:1], c[4]), dict(q=q)), ((*c[:4], c[4][:2]), dict(q=q)), ((*c[:3], c[3].cpu(), c[4]), dict(q=q)), (c, dict(q=q[..., :32])), (c, dict(q=q, k=kv[:1], v=kv[:1])),
             (c, dict(k=kv[:, :1], v=kv)), (c, dict(q=q, lse_out=torch.zeros(4, 2, device="cuda"))), (c, dict(k=kv, v=kv, rope="halves")),
             (c, dict(k=kv, v=kv, k_weight=torch.ones(64, device="cuda"))), (c, dict(k=kv, v=kv, positions=torch.zeros(3, dtype=torch.int32, device="cuda")))]
    for args, kw in cases:
        with pytest.raises(ValueError):
            da.make_paged_params(*args, **kw)
    with pytest.raises(TypeError):
        da.make_paged_params(*c, q=q.float())
    p = da.make_paged_params(*c, q=q)
    o = torch.empty_like(q)
    for args in ((q[:1], *c[:2], o), (q, *c[:2], o[:1]), (q, *c[:2], o.float()), (q, c[0], c[1].contiguous(), o), (q, *c[:2], o.transpose(0, 1).contiguous().transpose(0, 1))):
        with pytest.raises(ValueError):
            da.distr_attn_paged_fwd(*args, p)
    with pytest.raises(ValueError):
        da.distr_attn_cache_append(kv, kv, *c[:2], p)
    with pytest.raises(ValueError):
        da.distr_attn_paged_fwd(q, *c[:2], o, da.make_paged_params(*c, k=kv, v=kv))
    with pytest.raises(da.DistrAttnError):
        da.distr_attn_paged_fwd(q, *c[:2], o, da.make_paged_params(*c, q=q, softmax_scale=-1.0))
    torch.cuda.synchronize()
