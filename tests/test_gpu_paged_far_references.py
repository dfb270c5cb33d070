"""Attention over a paged cache where a row first meets scores far below those that count, or has far ones alone: a reference of units of 128 rows is rounded by
more than a weight has room for. As test_gpu_cache4_far_references.py, over keys in 16 and 32 bits."""
import math

import pytest
import torch

from paged_util import Batch
from test_gpu_paged import BF, F, _attention

pytestmark = pytest.mark.gpu
SIZES = [2e8, 1e9, 5e9, 3.3e10, 1e11, 1e13, 1e20]                    # of the queries
LATER = [0.0, 2.0 ** -20, 2.0 ** -21, -(2.0 ** -22), -0.75, 0.5]     # keys behind the first ones, which are `low`


def _store_keys(b, s, k):
    """k [n] as the keys of sequence s, all channels alike"""
    for j in range(-(-k.shape[0] // b.page)):
        m = min(b.page, k.shape[0] - j * b.page)
        b.k_pages[int(b.table[s, j]), :, :m] = k[j * b.page:j * b.page + m, None].to(b.dtype).cuda()


def _compare(b, s, first, causal, sizes=SIZES):
    """Sequence s with its first `first` keys far below the others: rows are the mean of the others' values that they see."""
    n, new, r0, group = b.lens[s], b.new[s], int(b.start[s]), b.H // b.Hkv
    for low in (-1.0, -1.5):
        for later in LATER:
            k = torch.full((n,), later)
            k[:first] = low
            _store_keys(b, s, k)
            for size in sizes:
                b.dev["q"][:] = size
                o, lse = _attention(b, causal=causal)
                ends = [n - new + i + 1 if causal else n for i in range(new)]
                assert min(ends) > first
                v, counts = b.values[s].double(), torch.tensor(ends, dtype=torch.float64) - first
                sums = torch.stack([v[:, first:e].sum(1) for e in ends]), torch.stack([v[:, first:e].abs().sum(1) for e in ends])
                want, most = ((x / counts[:, None, None]).repeat_interleave(group, 1) for x in sums)
                err = (o[r0:r0 + new].double() - want).abs()
                # (equal weights, whatever the parts: the same products in the same order. bf16: rounded once, above and below)
                bound = most * (2.0 ** -7 if b.dtype == BF else 2.0 ** -17) + want.abs() * 2.0 ** -8
                assert (err <= bound).all(), (low, later, size, float((err / bound).max()), int(o[r0:r0 + new].isnan().sum()))
                score = later * b.d * float(b.dev["q"][0, 0, 0]) / math.sqrt(b.d)
                want = score + counts.log()[:, None]
                assert ((lse[r0:r0 + new].double() - want).abs() <= want.abs() * 2.0 ** -21 + 2.0 ** -15).all(), (low, later, size)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("first", [64, 130])
def test_chunks(d, dtype, causal, first):
    """Workgroups of eight waves: a half's first tile, its first two and a part of the third."""
    _compare(Batch([300], [70], 4, 2, d, dtype, page=16), 0, first, causal)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H", [34, 128])
def test_many_heads_to_a_kv_head(d, H):
    """Units of 128 rows that are one token's: every row sees all keys."""
    _compare(Batch([300], [1], H, 1, d, BF, page=32), 0, 64, True)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("room", [0, 300])
def test_a_chunk_among_many_sequences(d, causal, room):
    """Workgroups of four waves, whole units and ranges; beside it sequences with few rows."""
    lens, new = [40] * 140, [1] * 140
    lens[77], new[77] = 300, 70
    _compare(Batch(lens, new, 4, 2, d, BF, page=16, room=room), 77, 64, causal, sizes=SIZES[1:5])


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [64, 128])
def test_single_tokens(d, dtype):
    """Units of few rows: references are unscaled scores."""
    _compare(Batch([300, 20], [1, 1], 8, 2, d, dtype, page=16), 0, 64, True)
