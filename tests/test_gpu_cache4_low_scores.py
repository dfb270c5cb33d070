"""Attention over a 4-bit cache where every score lies far below zero: a part of the keys that a row sees nothing of, or a wave that has none of its
keys, must not count as a score of zero. As test_gpu_paged_low_scores.py, whose batches these are."""
import pytest
import torch

from cache4_util import Batch4
from test_gpu_cache4 import BF, F, ROOMY, _attention, _check

pytestmark = pytest.mark.gpu


def _channel0(s, which, codes, scales):
    """Channel 0 of every key is 64, the others of its 32 are 0."""
    if which == "k":
        codes[..., :16], codes[..., 0], scales[..., 0] = 0, 6, 127 + 4


def _compare(b, workspace, only=None, rows_of=None, seen=None):
    for score in (-96.0, -512.0):     # (exp of the first is less than the smallest normal float)
        b.q[..., 0] = score / 8       # (softmax_scale 1 / 8)
        b.dev["q"][..., 0] = score / 8
        o, lse = _attention(b, scale=0.125, workspace=workspace)
        _check(b, o, lse, scale=0.125, only=only, rows_of=rows_of, seen=seen)
        again, lse2 = _attention(b, scale=0.125, workspace=workspace)
        assert torch.equal(o.nan_to_num(), again.nan_to_num()) and torch.equal(lse.nan_to_num(), lse2.nan_to_num())
        assert (lse[~lse.isnan() & ~lse.isinf()] < score / 2).all()


@pytest.mark.parametrize("workspace", [True, None, 3 << 20])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("roomy", ROOMY)
def test_prompts_among_a_few_tokens_of_many_sequences(workspace, d, roomy):
    g = torch.Generator().manual_seed(0)
    lens = torch.randint(5, 500, (70,), generator=g).tolist()
    new = [min(int(x), n) for x, n in zip(torch.randint(1, 6, (70,), generator=g), lens)]
    for i in (3, 20, 33, 69):
        lens[i] = new[i] = 300 + 7 * i
    b = Batch4(lens, new, 8, 4, d, BF, page=32, order="tokens", room=roomy // 32, edit=_channel0)
    _compare(b, workspace, only=[0, 3, 4, 20, 33, 69], rows_of=[0, 1, 31, 63, 64, 127, 128, 200, 320])


@pytest.mark.parametrize("d", [64, 128])
def test_absent_pages_in_parts_of_many_sequences(d):
    lens, new = [700] * 70, [2] * 70
    new[9], new[40] = 80, 40
    b = Batch4(lens, new, 8, 4, d, BF, page=32, room=ROOMY[1] // 32, edit=_channel0)
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
    lens, new = [600, 300, 200, 90], [150, 300, 9, 1]
    b = Batch4(lens, new, 8, 2, d, dtype, page=48, room=roomy // 48, pad_back=1, edit=_channel0)
    for workspace in (True, 256):
        _compare(b, workspace, rows_of=[0, 1, 8, 31, 63, 127, 128, 149, 299])


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n_seq,H,Hkv,d", [(5, 8, 2, 64), (100, 8, 4, 128), (300, 2, 2, 64)])
@pytest.mark.parametrize("roomy", ROOMY)
def test_single_tokens(n_seq, H, Hkv, d, dtype, roomy):
    g = torch.Generator().manual_seed(n_seq)
    lens = torch.randint(1, 300, (n_seq,), generator=g).tolist()
    lens[2] = 1500
    b = Batch4(lens, [1] * n_seq, H, Hkv, d, dtype, room=roomy // 16, edit=_channel0)
    _compare(b, True, only=[0, 1, 2, 3, 4, n_seq // 2, n_seq - 1])


def test_prompts_that_fill_the_chip():
    b = Batch4([700, 130, 40], [600, 65, 1], 64, 64, 64, BF, page=64, edit=_channel0)
    _compare(b, True, rows_of=[0, 64, 127, 128, 599])
