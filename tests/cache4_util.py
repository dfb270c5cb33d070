"""Plain implementation in 64 bits, on the CPU, of a cache held in 4 bits, and batches in one."""
import math

import torch

from paged_util import Batch

MAGNITUDES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
POWERS = torch.tensor([2.0 ** (e - 127) for e in range(255)] + [math.nan], dtype=torch.float64)
MIDDLES = 0.5 * (MAGNITUDES[1:] + MAGNITUDES[:-1])


def encode(x):
    """x [..., d] double -> codes [..., d / 2], scales [..., d / 32], uint8."""
    x = x.unflatten(-1, (-1, 32))
    most = x.abs().amax(-1, keepdim=True)          # (NaN where one is)
    odd = ~(most < math.inf)
    # smallest power that leaves none beyond 7 times it
    e = torch.searchsorted(7.0 * POWERS[1:253].contiguous(), most.nan_to_num(0.0, 0.0).contiguous()).clamp(max=251) + 1
    a = (x.abs() / POWERS[e]).nan_to_num(0.0, 0.0).contiguous()
    below, upto = torch.searchsorted(MIDDLES, a), torch.searchsorted(MIDDLES, a, right=True)   # these differ where a is a middle: the even one
    code = torch.where(below % 2 == 0, below, upto) + 8 * torch.signbit(x)
    code = torch.where(odd, 0, code).flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), torch.where(odd, 255, e).squeeze(-1).to(torch.uint8)


def decode(codes, scales):
    """-> [..., d] double"""
    nibble = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    value = MAGNITUDES[nibble & 7] * (1.0 - 2.0 * (nibble >> 3))
    return (value.unflatten(-1, (-1, 32)) * POWERS[scales.long()][..., None]).flatten(-2)


class Batch4(Batch):
    """Sequences in a paged cache of 4-bit codes. What is not stored is NaN. keys, values: the values that the codes stand for. `raw`: those of the
    new tokens before (T rows, [T, Hkv, d])."""

    def __init__(self, lens, new, H, Hkv, d, dtype, page=16, order="heads", seed=0, stored="all", edit=None, **kw):
        super().__init__(lens, new, H, Hkv, d, dtype, page=page, order=order, seed=seed, stored=stored, **kw)
        n_pages = self.pool_cpu.shape[0]
        outer = (n_pages, Hkv, page) if order == "heads" else (n_pages, page, Hkv)
        self.cache_cpu = [torch.full((*outer, w), 255, dtype=torch.uint8) for w in (d // 2, d // 32) * 2]
        parts = [t if order == "heads" else t.transpose(1, 2) for t in self.cache_cpu]
        self.raw = [torch.zeros(self.T, Hkv, d, dtype=dtype) for _ in range(2)]
        for s, n in enumerate(lens):
            r0 = int(self.start[s])
            for i, rows in enumerate((self.keys, self.values)):
                self.raw[i][r0:r0 + new[s]] = rows[s][:, n - new[s]:].transpose(0, 1)
                codes, scales = encode(rows[s].double())
                if edit is not None:
                    edit(s, "kv"[i], codes, scales)   # [Hkv, n, ..]
                rows[s] = decode(codes, scales)
                have = n if stored == "all" else max(n - new[s], 0)
                for j in range(-(-have // page)):
                    m = min(page, have - j * page)
                    at = self.table[s, j]
                    parts[2 * i][at, :, :m], parts[2 * i + 1][at, :, :m] = codes[:, j * page:j * page + m], scales[:, j * page:j * page + m]
        self.to_device()

    def to_device(self):
        parts = [t.cuda() for t in self.cache_cpu]
        self.cache4 = tuple(t if self.order == "heads" else t.transpose(1, 2) for t in parts)

    def index(self):
        return self.dev["table"], self.dev["kv_len"], self.dev["start"]

    def places(self):
        """(row, sequence, place) of every new token"""
        return [(int(self.start[s]) + i, s, n - fresh + i) for s, (n, fresh) in enumerate(zip(self.lens, self.new)) for i in range(fresh)]
