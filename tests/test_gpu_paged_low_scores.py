"""Attention over a paged cache where every score lies far below zero: a part of the keys that a row sees nothing of, or a wave that has none
of its keys, must not count as a score of zero. Every form that a call is launched in, with whole units and with ranges."""
import pytest
import torch

from paged_util import Batch
from test_gpu_paged import BF, F, ROOMY, _attention, _check

pytestmark = pytest.mark.gpu


def _far_below(b, score):
    """Channel 0 of queries and keys adds `score` to every one of the batch's (softmax_scale 1 / 8; both exact in bf16)."""
    b.q[..., 0] = score / 8
    b.dev["q"][..., 0] = score / 8
    b.k_pages[..., 0] = 64.0
    for k in b.keys:
        k[..., 0] = 64.0
    return b


def _compare(b, workspace, only=None, rows_of=None, seen=None):
    for score in (-96.0, -512.0):     # (exp of the first is less than the smallest normal float)
        o, lse = _attention(_far_below(b, score), scale=0.125, workspace=workspace)
        _check(b, o, lse, scale=0.125, only=only, rows_of=rows_of, seen=seen)
        again, lse2 = _attention(b, scale=0.125, workspace=workspace)
        assert torch.equal(o.nan_to_num(), again.nan_to_num()) and torch.equal(lse.nan_to_num(), lse2.nan_to_num())
        assert (lse[~lse.isnan() & ~lse.isinf()] < score / 2).all()


@pytest.mark.parametrize("workspace", [True, None, 3 << 20])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("roomy", ROOMY)
def test_prompts_among_a_few_tokens_of_many_sequences(workspace, d, roomy):
    """Prompts of 321 to 783 tokens from an empty cache among 66 sequences of up to five new ones: ranges for two workgroups a compute unit, whose
    cuts leave parts of a unit's keys that none of its first rows see."""
    g = torch.Generator().manual_seed(0)
    lens = torch.randint(5, 500, (70,), generator=g).tolist()
    new = [min(int(x), n) for x, n in zip(torch.randint(1, 6, (70,), generator=g), lens)]
    for i in (3, 20, 33, 69):
        lens[i] = new[i] = 300 + 7 * i
    b = Batch(lens, new, 8, 4, d, BF, page=32, order="tokens", room=roomy // 32)
    _compare(b, workspace, only=[0, 3, 4, 20, 33, 69], rows_of=[0, 1, 31, 63, 64, 127, 128, 200, 320])


@pytest.mark.parametrize("d", [64, 128])
def test_absent_pages_in_parts_of_many_sequences(d):
    """The same form where the later pages are none of the cache's: parts that no row sees anything of."""
    lens, new = [700] * 70, [2] * 70
    new[9], new[40] = 80, 40
    b = Batch(lens, new, 8, 4, d, BF, page=32, room=ROOMY[1] // 32)
    seen = [[True] * n for n in lens]
    for s in (9, 40, 41):
        b.table[s, 6:] = -1
        for j in range(6 * 32, lens[s]):
            seen[s][j] = False
    b.dev["table"] = b.table.cuda()
    _compare(b, True, only=[8, 9, 40, 41], rows_of=[0, 1, 31, 32, 39, 79], seen=seen)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("roomy", ROOMY)
def test_chunks_of_few_sequences(d, dtype, roomy):
    """Workgroups of eight waves: whole prompts, chunks on a prefix, and units of 32 rows or fewer."""
    lens, new = [600, 300, 200, 90], [150, 300, 9, 1]
    b = Batch(lens, new, 8, 2, d, dtype, page=48, room=roomy // 48, pad_back=1)
    for workspace in (True, 256):
        _compare(b, workspace, rows_of=[0, 1, 8, 31, 63, 127, 128, 149, 299])


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n_seq,H,Hkv", [(5, 8, 2), (100, 8, 4), (300, 2, 2)])
@pytest.mark.parametrize("roomy", ROOMY)
def test_single_tokens(n_seq, H, Hkv, dtype, roomy):
    """Workgroups of eight, four and two waves, most of whose waves have no tile of a short sequence."""
    g = torch.Generator().manual_seed(n_seq)
    lens = torch.randint(1, 300, (n_seq,), generator=g).tolist()
    lens[2] = 1500
    b = Batch(lens, [1] * n_seq, H, Hkv, 64, dtype, room=roomy // 16)
    _compare(b, True, only=[0, 1, 2, 3, 4, n_seq // 2, n_seq - 1])


def test_prompts_that_fill_the_chip():
    """Whole units without ranges."""
    b = Batch([700, 130, 40], [600, 65, 1], 64, 64, 64, BF, page=64)
    _compare(b, True, rows_of=[0, 64, 127, 128, 599])
