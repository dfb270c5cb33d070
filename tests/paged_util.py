"""Plain implementations in 64 bits, on the CPU, of the operators around attention, and batches to try them on."""
import numpy as np
import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # of a rounding, relative to the value


def tables(n_pos, rot, base=10000.0):
    rate = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    angle = torch.arange(n_pos, dtype=torch.float64)[:, None] * rate
    return angle.cos().float(), angle.sin().float()


def pair_places(rope, rot):
    j = torch.arange(rot // 2)
    return (j, j + rot // 2) if rope == "halves" else (2 * j, 2 * j + 1)


def turn(x, c, s, rope):
    """x [..., d] double; c, s [..., rot / 2] double"""
    a, b = pair_places(rope, 2 * c.shape[-1])
    y = x.clone()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def turn_bound(x, rot, rope):
    """|a| + |b| of each channel's pair, |x| of the others."""
    y = x.abs().clone()
    if rope != "none":
        a, b = pair_places(rope, rot)
        y[..., a] = y[..., b] = x[..., a].abs() + x[..., b].abs()
    return y


def normed(x, w, eps):
    r = 1.0 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    return x * r * (1.0 if w is None else w)


class Batch:
    """Sequences in a paged cache. lens: tokens with the new ones, new: how many are new. The pool is NaN but for the `stored` tokens of each
    sequence (the older ones; all: with the new ones)."""

    def __init__(self, lens, new, H, Hkv, d, dtype, page=16, order="heads", seed=0, stored="all", spare=3, pad_front=0, pad_back=0, room=0, scale=1.0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.new, self.H, self.Hkv, self.d, self.page, self.dtype = lens, new, H, Hkv, d, page, dtype
        T = sum(new)
        self.T = pad_front + T + pad_back
        need = [-(-n // page) for n in lens]
        n_pages = sum(need) + spare
        self.max_pages = max(max(need), 1) + room
        shape = (n_pages, 2, Hkv, page, d) if order == "heads" else (n_pages, 2, page, Hkv, d)
        pool = torch.full(shape, float("nan"), dtype=dtype)
        kp, vp = (pool[:, i] if order == "heads" else pool[:, i].transpose(1, 2) for i in (0, 1))
        ids = torch.randperm(n_pages, generator=g).to(torch.int32)
        self.table = torch.full((len(lens), self.max_pages), -1, dtype=torch.int32)
        self.keys, self.values = [], []
        at = 0
        for s, n in enumerate(lens):
            self.table[s, :need[s]] = ids[at:at + need[s]]
            at += need[s]
            k, v = (torch.randn(Hkv, n, d, generator=g).to(dtype) for _ in (0, 1))
            self.keys.append(k)
            self.values.append(v)
            have = n if stored == "all" else max(n - new[s], 0)
            for i in range(-(-have // page)):
                m = min(page, have - i * page)
                kp[self.table[s, i], :, :m] = k[:, i * page:i * page + m]
                vp[self.table[s, i], :, :m] = v[:, i * page:i * page + m]
        self.start = torch.tensor([pad_front + sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32)
        self.kv_len = torch.tensor(lens, dtype=torch.int32)
        self.q = (scale * torch.randn(self.T, H, d, generator=g)).to(dtype)
        self.pool_cpu = pool
        self.order = order
        self.reset()

    def reset(self):
        pool = self.pool_cpu.cuda()
        self.k_pages, self.v_pages = (pool[:, i] if self.order == "heads" else pool[:, i].transpose(1, 2) for i in (0, 1))
        self.dev = {"table": self.table.cuda(), "kv_len": self.kv_len.cuda(), "start": self.start.cuda(), "q": self.q.cuda()}

    def cache(self):
        return self.k_pages, self.v_pages, self.dev["table"], self.dev["kv_len"], self.dev["start"]


def attend(q, k, v, places, n_keys, scale, seen=None):
    """q [n, H, d], k, v [Hkv, keys, d] double; row i sees keys up to places[i] (and below n_keys, and of `seen`).
    -> o, sum of weights |v| / sum of weights, lse, bound of |score| sums"""
    H, Hkv = q.shape[1], k.shape[0]
    o, mean, lse, most = (torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64),
                          torch.full(q.shape[:2], -np.inf, dtype=torch.float64), torch.zeros(q.shape[:2], dtype=torch.float64))
    for i in range(q.shape[0]):
        n = min(places[i] + 1, n_keys)
        keys = [j for j in range(n) if seen is None or seen[j]]
        if not keys:
            continue
        for h in range(H):
            kk, vv = k[h // (H // Hkv)][keys], v[h // (H // Hkv)][keys]
            s = kk @ q[i, h] * scale
            lse[i, h] = torch.logsumexp(s, 0)
            p = torch.softmax(s, 0)
            o[i, h], mean[i, h] = p @ vv, p @ vv.abs()
            most[i, h] = (kk.abs() @ q[i, h].abs()).max() * scale
    return o, mean, lse, most


def attention_bounds(o, mean, lse, most, n_keys, d, dtype):
    """How far an output and a row's log-sum-exp may be off: scores summed in float (d terms: d + 8 half steps of the largest sum of
    magnitudes), weights off by that and by the exponential (4 half steps of their argument and result each), their sums (a key in
    eight after the other: chains of n / 8 and 64 more in joining them), bf16: each weight rounded once, above and below; the result rounded once."""
    f = 2.0 ** -24
    score = (d + 8) * f * most + 8 * f * (most + 1)
    weights = 2 * score + (n_keys / 8 + 64) * f
    rounding = 2 * HALF_STEP[torch.bfloat16] if dtype == torch.bfloat16 else 0.0
    return mean * (weights + rounding)[..., None] + HALF_STEP[dtype] * o.abs() * 1.01 + 1e-30, score + (n_keys / 8 + 64) * f + 4 * f * (lse.abs().nan_to_num(posinf=0) + 1)
