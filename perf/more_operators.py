"""A paged cache that holds its keys and values in 4 bits, measured over the range it is used in.

  append4  new keys and values into the cache, keys normed and rotated on the way, and the values that they then stand for
  read4    whole sequences out of the cache
  paged4   attention of new tokens (one for each sequence or chunks of a prompt) over the cache

32 channels of a row share a scale, a power of two; a channel is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times that scale. The scale is
the smallest with which no channel exceeds 7 times it; channels go to the nearest value, ties to the one whose code is even.

Each case is one pass: with `own` through this library's entry points, without it in elementary torch operations.
"""
import math
import random

import torch

own = False

EPS = 1e-6
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---- cases -----------------------------------------------------------------------------------------

def _append(name, dtype, n_seq, new, most, Hkv, d, page, order, rope, norm, len_seed):
    """n_seq sequences of up to `most` tokens with their new ones, up to `new` of them new. order: how a page lies in memory."""
    return {"name": name, "op": "append4", "dtype": dtype, "n_seq": n_seq, "new": new, "most": most, "Hkv": Hkv, "d": d, "page": page,
            "order": order, "rope": rope, "norm": norm, "len_seed": len_seed}


def _read(name, dtype, n_seq, most, Hkv, d, page, order, len_seed):
    """n_seq sequences of up to `most` tokens, all of them read."""
    return {"name": name, "op": "read4", "dtype": dtype, "n_seq": n_seq, "most": most, "Hkv": Hkv, "d": d, "page": page, "order": order,
            "len_seed": len_seed}


def _paged(name, dtype, n_seq, chunks, new, most, H, Hkv, d, page, order, lse, len_seed):
    """n_seq sequences of up to `most` tokens, `chunks` of them with `new` new ones and the others with a single one."""
    return {"name": name, "op": "paged4", "dtype": dtype, "n_seq": n_seq, "chunks": chunks, "new": new, "most": most, "H": H, "Hkv": Hkv,
            "d": d, "page": page, "order": order, "lse": lse, "len_seed": len_seed}


def listed():
    return [
        # One new token for each of 64 sequences of up to 2048: all latency.
        _append("append4_decode", "bf16", 64, 1, 2048, 8, 64, 16, "heads", "halves", True, 1),
        # Prompts of five sequences at once, some with a cached prefix; pages with the tokens outside and the heads inside.
        _append("append4_prompts", "bf16", 5, 4096, 8192, 16, 128, 64, "tokens", "halves", False, 2),
        # A layer kept in float32, an odd number of heads, neighbouring channels as pairs.
        _append("append4_f32", "f32", 3, 700, 1500, 5, 64, 16, "heads", "neighbours", True, 3),
        # The prefix of one short conversation, for a kernel that takes contiguous keys.
        _read("read4_one", "f32", 1, 777, 8, 64, 16, "heads", 4),
        # Four long sequences, as they move to a cache of whole numbers of bytes.
        _read("read4_long", "bf16", 4, 16384, 8, 128, 64, "tokens", 5),
        # A check of a model's block in float32: three short sequences.
        _paged("paged4_f32", "f32", 3, 3, 48, 700, 8, 8, 64, 16, "heads", True, 6),
        # One user's next token after 777.
        _paged("paged4_one", "bf16", 1, 0, 1, 777, 32, 8, 64, 16, "heads", False, 7),
        # A decoding step of 64 sequences of up to 8192 tokens, grouped heads.
        _paged("paged4_decode", "bf16", 64, 0, 1, 8192, 32, 8, 64, 16, "heads", False, 8),
        # A serving step of many sequences of medium length, d = 128.
        _paged("paged4_many", "bf16", 200, 0, 1, 2500, 32, 8, 128, 32, "heads", False, 9),
        # The next token of one very long document, a kv head for each query head, pages with the tokens outside.
        _paged("paged4_long", "bf16", 1, 0, 1, 100003, 16, 16, 128, 128, "tokens", False, 10),
        # A long prompt's last chunk: 2048 tokens on 16384. The most arithmetic.
        _paged("paged4_chunk", "bf16", 1, 1, 2048, 16384, 32, 8, 64, 64, "heads", False, 11),
        # Prompts and decoding in one step: two chunks of 250 tokens beside 14 single tokens, d = 128, grouped heads.
        _paged("paged4_mixed", "bf16", 16, 2, 250, 4096, 32, 8, 128, 32, "heads", True, 12),
    ]


def _spread(rng, lo, hi):
    """An integer of [lo, hi], even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_once(rng):
    op = rng.choice(("append4", "read4", "paged4", "paged4", "paged4", "paged4"))
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    d = rng.choice((64, 128))
    Hkv = rng.choice((1, 2, 4, 5, 8, 16))
    H = Hkv * rng.choice((1, 2, 3, 4, 4, 8))
    page, order, seed = rng.choice((16, 32, 48, 64, 128, 256)), rng.choice(("heads", "tokens")), rng.randrange(1 << 20)
    if op == "append4":
        n_seq = _spread(rng, 1, 128)
        new = 1 if rng.random() < 0.5 else _spread(rng, 2, max(2, 8192 // n_seq))
        return _append("", dtype, n_seq, new, new + _spread(rng, 1, max(1, 65536 // n_seq)), Hkv, d, page, order,
                       rng.choice(("halves", "halves", "neighbours", "none")), rng.random() < 0.6, seed)
    if op == "read4":
        n_seq = _spread(rng, 1, 64)
        return _read("", dtype, n_seq, _spread(rng, 1, 65536 // n_seq), Hkv, d, page, order, seed)
    family = "chunk" if dtype == "f32" else rng.choice(("decode", "decode", "chunk", "mixed"))
    if family == "decode":
        n_seq = _spread(rng, 1, 256)
        return _paged("", dtype, n_seq, 0, 1, _spread(rng, 200, min(131072, 600000 // n_seq)), H, Hkv, d, page, order, rng.random() < 0.3, seed)
    n_seq = rng.choice((1, 1, 2, 3)) if family == "chunk" else rng.randint(2, 16)
    new = _spread(rng, 2, 100 if dtype == "f32" else 2048 // n_seq)
    most = new + _spread(rng, 1, 2000 if dtype == "f32" else 32768 // n_seq)
    return _paged("", dtype, n_seq, n_seq if family == "chunk" else rng.randint(1, n_seq - 1), new, most, H, Hkv, d, page, order, rng.random() < 0.3, seed)


def draw(rng):
    """Another case of the same families: single tokens and prompts, both types, all page orders."""
    most = [work(c) for c in listed()]
    most_bytes, most_flops = max(w["bytes"] for w in most), max(w["flops"] for w in most)
    f32_flops = 3e10   # (float products run at a fifteenth of the rate)
    while True:
        case = _draw_once(rng)
        del case["name"]
        w = work(case)
        paged = case["op"] == "paged4"
        scores = case["n_seq"] * case["H"] * case["new"] * case["most"] if paged else 0            # that the plain form holds
        padded = case["n_seq"] * case["Hkv"] * case["most"] * case["d"] if paged else 0            # and keys
        if w["bytes"] <= most_bytes and w["flops"] <= (most_flops if case["dtype"] == "bf16" else f32_flops) and scores <= 1.1e9 and padded <= 1e9:
            return case


def _lengths(case):
    """(tokens in the cache with the new ones, new ones) of each sequence; the first is the longest there may be."""
    rng = random.Random(case["len_seed"])
    total, fresh = [], []
    for s in range(case["n_seq"]):
        if case["op"] == "append4":
            n = case["new"] if s == 0 or case["new"] == 1 else _spread(rng, 1, case["new"])
        elif case["op"] == "read4":
            n = 1
        else:
            n = case["new"] if s < case["chunks"] else 1
        total.append(case["most"] if s == 0 else max(n, rng.randint(case["most"] // 4, case["most"])))
        fresh.append(total[-1] if case["op"] == "read4" else n)
    return total, fresh


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    d, Hkv = case["d"], case["Hkv"]
    row = d // 2 + d // 32   # bytes of a key or value
    total, fresh = _lengths(case)
    T = sum(fresh)
    if case["op"] == "append4":
        angles = 0 if case["rope"] == "none" else T * d * 4
        return {"bytes": 2 * T * Hkv * (2 * d * size + 2 * row) + angles, "flops": T * Hkv * d * (8 + (3 if angles else 0) + (4 if case["norm"] else 0))}
    if case["op"] == "read4":
        return {"bytes": 2 * T * Hkv * (d * size + row), "flops": 2 * T * Hkv * d}
    pairs = sum(n * (t - n) + n * (n + 1) // 2 for t, n in zip(total, fresh))
    return {"bytes": 2 * T * case["H"] * d * size + 2 * sum(total) * Hkv * row + (4 * T * case["H"] if case["lse"] else 0),
            "flops": 4 * case["H"] * d * pairs}


# ---- inputs ----------------------------------------------------------------------------------------

def _tables(n_pos, rot, dev):
    """cos and sin of position times 10000^(-2 i / rot), float32 [n_pos, rot / 2], the angles in 64 bits."""
    rate = 10000.0 ** (-torch.arange(0, rot, 2, device=dev, dtype=torch.float64) / rot)
    angle = torch.arange(n_pos, device=dev, dtype=torch.float64)[:, None] * rate
    return angle.cos().float(), angle.sin().float()


def _store(case, n_pages, dev, normal):
    """Codes [pages, Hkv, page, d / 2] and scales [pages, Hkv, page, d / 32] of random rows."""
    Hkv, page, d = case["Hkv"], case["page"], case["d"]
    outer = (n_pages, Hkv, page) if case["order"] == "heads" else (n_pages, page, Hkv)
    codes = torch.empty(*outer, d // 2, dtype=torch.uint8, device=dev)
    scales = torch.empty(*outer, d // 32, dtype=torch.uint8, device=dev)
    size = torch.exp(0.3 * normal(d))   # channels of different size
    step = max(1, (1 << 25) // codes[0].numel())
    for at in range(0, n_pages, step):
        part = slice(at, min(at + step, n_pages))
        codes[part], scales[part] = _encode(normal(*codes[part].shape[:3], d) * size)
    return (codes, scales) if case["order"] == "heads" else (codes.transpose(1, 2), scales.transpose(1, 2))


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    s = {"case": case}

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev)

    total, fresh = _lengths(case)
    n_seq, page, Hkv, d = case["n_seq"], case["page"], case["Hkv"], case["d"]
    T, need = sum(fresh), [-(-t // page) for t in total]
    n_pages = sum(need) + 3
    s["fresh"], s["total"], s["T"] = fresh, total, T
    s["k_codes"], s["k_scales"] = _store(case, n_pages, dev, normal)
    s["v_codes"], s["v_scales"] = _store(case, n_pages, dev, normal)
    order = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32).cpu()
    table = torch.full((n_seq, max(need)), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    s["page_table"] = table.to(dev)
    s["kv_len"] = torch.tensor(total, dtype=torch.int32, device=dev)
    starts = [0]
    for n in fresh:
        starts.append(starts[-1] + n)
    s["q_start"] = torch.tensor(starts, dtype=torch.int32, device=dev)
    # (value, code) of a byte's two channels, the first in the low bits
    values = torch.tensor([m * sign for sign in (1.0, -1.0) for m in MAGNITUDES], device=dev)
    byte = torch.arange(256, device=dev)
    s["values"] = torch.stack((values[byte & 15], values[byte >> 4]), -1)
    if case["op"] == "paged4":
        s["q"] = (1.5 * normal(T, case["H"], d)).to(dtype)
        s["o"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(T, case["H"], device=dev) if case["lse"] else None
    else:
        s["k_back"], s["v_back"] = (torch.empty(T, Hkv, d, dtype=dtype, device=dev) for _ in range(2))
    if case["op"] == "append4":
        x = (normal(T, 2 * Hkv * d) * torch.exp(0.3 * normal(2 * Hkv * d))).to(dtype)
        s["k"], s["v"] = (x[:, i * Hkv * d:(i + 1) * Hkv * d].unflatten(-1, (Hkv, d)) for i in (0, 1))
        s["k_weight"] = None
        if case["norm"]:
            w = 1.0 + 0.2 * normal(d)
            s["k_weight"] = w if case["dtype"] == "f32" else w.to(torch.bfloat16)
        s["cos"], s["sin"] = _tables(case["most"], d, dev) if case["rope"] != "none" else (None, None)
    if own:
        _plan(s)
    return s


def _plan(s):
    """What a program that uses the library keeps for a layer: the parameters of its calls, and scratch."""
    import paper_2507_17245_amd as da
    c = s["case"]
    s["cache"] = cache = (s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"])
    at = (s["page_table"], s["kv_len"], s["q_start"])
    if c["op"] == "paged4":
        need = da.distr_attn_paged4_workspace_bytes(da.make_paged4_params(cache, *at, q=s["q"]))
        s["scratch"] = torch.empty(max(256, need), dtype=torch.uint8, device="cuda")
        s["plan"] = da.make_paged4_params(cache, *at, q=s["q"], lse_out=s["lse"], workspace=s["scratch"])
        return
    if c["op"] == "append4":
        s["plan"] = da.make_paged4_params(cache, *at, k=s["k"], v=s["v"], norm=c["norm"], eps=EPS, k_weight=s["k_weight"], rope=c["rope"],
                                          cos=s["cos"], sin=s["sin"])
    s["plan_back"] = da.make_paged4_params(cache, *at, k=s["k_back"], v=s["v_back"])


# ---- one pass --------------------------------------------------------------------------------------

def _run_own(s):
    import paper_2507_17245_amd as da
    c = s["case"]
    if c["op"] == "paged4":
        da.distr_attn_paged4_fwd(s["q"], s["cache"], s["o"], s["plan"])
        return [s["o"], s["lse"]]
    if c["op"] == "append4":
        da.distr_attn_cache4_append(s["k"], s["v"], s["cache"], s["plan"])
    da.distr_attn_cache4_read(s["k_back"], s["v_back"], s["cache"], s["plan_back"])
    return [s["k_back"], s["v_back"]]


def _encode(x):
    """x [..., d] -> codes [..., d / 2], scales [..., d / 32]: see the head of this file."""
    x = x.unflatten(-1, (-1, 32))
    part, up = torch.frexp(x.abs().amax(-1, keepdim=True))   # part * 2^up, part of [0.5, 1)
    up = (up - 3 + (part > 0.875).int()).clamp(min=-126)
    x = torch.ldexp(x, -up)
    a = x.abs()
    step = 0.5 + 0.5 * (a >= 2) + 1.0 * (a >= 4)
    a = (torch.round(a / step) * step).clamp(max=6.0)
    code = (2 * a - (a - 2).clamp(min=0) - 0.5 * (a - 4).clamp(min=0)).to(torch.uint8) + 8 * (x < 0).to(torch.uint8)
    code = code.flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], (up + 127).to(torch.uint8).squeeze(-1)


def _decode(codes, scales, values):
    """float32 [..., d]"""
    scale = (scales.to(torch.int32) << 23).view(torch.float32)
    return (values[codes.to(torch.int32)].flatten(-2).unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2)


def _rotated(x, cos, sin, rope):
    """x [..., d] with its channels rotated, in pairs of a half's channel with the other's or of neighbours."""
    half = cos.shape[-1]
    y = torch.empty_like(x)
    if rope == "halves":
        a, b = x[..., :half], x[..., half:]
        y[..., :half], y[..., half:] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., 0::2], x[..., 1::2]
        y[..., 0::2], y[..., 1::2] = a * cos - b * sin, a * sin + b * cos
    return y


def _places(s):
    """(place in its sequence, page, row in the page) of each new token."""
    start = s["q_start"].long()
    t = torch.arange(s["T"], device=start.device)
    seq = torch.searchsorted(start, t, right=True) - 1
    place = s["kv_len"].long()[seq] - (start[seq + 1] - t)
    return place, s["page_table"].long()[seq, place // s["case"]["page"]], place % s["case"]["page"]


def _run_plain(s):
    c = s["case"]
    dtype = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    if c["op"] != "paged4":
        place, page, row = _places(s)
        if c["op"] == "append4":
            k = s["k"].double()   # (values next to a border between two codes)
            if c["norm"]:
                k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + EPS) * s["k_weight"].double()
            if s["cos"] is not None:
                k = _rotated(k, s["cos"][place][:, None].double(), s["sin"][place][:, None].double(), c["rope"])
            s["k_codes"].transpose(1, 2)[page, row], s["k_scales"].transpose(1, 2)[page, row] = _encode(k)
            s["v_codes"].transpose(1, 2)[page, row], s["v_scales"].transpose(1, 2)[page, row] = _encode(s["v"].float())
        k = _decode(s["k_codes"].transpose(1, 2)[page, row], s["k_scales"].transpose(1, 2)[page, row], s["values"])
        v = _decode(s["v_codes"].transpose(1, 2)[page, row], s["v_scales"].transpose(1, 2)[page, row], s["values"])
        return [k.to(dtype), v.to(dtype)]
    # attention: the sequences padded to the most new tokens and the most pages
    n_seq, new, d, H, Hkv = c["n_seq"], max(s["fresh"]), c["d"], c["H"], c["Hkv"]
    table, kv_len, start = s["page_table"].long().clamp(min=0), s["kv_len"].long(), s["q_start"].long()
    k = _decode(s["k_codes"][table].transpose(1, 2), s["k_scales"][table].transpose(1, 2), s["values"]).reshape(n_seq, Hkv, -1, d)
    v = _decode(s["v_codes"][table].transpose(1, 2), s["v_scales"][table].transpose(1, 2), s["values"]).reshape(n_seq, Hkv, -1, d)
    fresh = start[1:] - start[:-1]
    i = torch.arange(new, device=table.device)
    q = s["q"][(start[:-1, None] + i).clamp(max=s["T"] - 1)].float()                                   # [seq, new, H, d]
    q = q.unflatten(2, (Hkv, H // Hkv)).permute(0, 2, 3, 1, 4).reshape(n_seq, Hkv, -1, d)              # [seq, Hkv, heads x new, d]
    score = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(d)).unflatten(2, (H // Hkv, new))
    place = kv_len[:, None] - fresh[:, None] + i                                                        # of the new tokens
    hidden = torch.arange(k.shape[2], device=table.device) > place[:, :, None].clamp(max=kv_len.max())
    hidden |= torch.arange(k.shape[2], device=table.device) >= kv_len[:, None, None]
    score.masked_fill_(hidden[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(top).exp_()
    weight = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), v).unflatten(2, (H // Hkv, new)) / weight                        # [seq, Hkv, heads, new, d]
    mine = i[None, :] < fresh[:, None]
    o = o.permute(0, 3, 1, 2, 4).reshape(n_seq, new, H, d)[mine].to(dtype)
    if not c["lse"]:
        return [o, None]
    return [o, (top + weight.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(n_seq, new, H)[mine]]


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ---- the definition in 64 bits ---------------------------------------------------------------------

def _stored(x):
    """What the cache holds of x [..., d] (double): the value itself, not its code."""
    groups = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    most = groups.abs().max(-1, keepdim=True).values
    scale = torch.full_like(most, 2.0 ** -126)
    for e in range(-125, 128):
        scale = torch.where(most > 7.0 * 2.0 ** (e - 1), torch.full_like(scale, 2.0 ** e), scale)
    a, kept = groups.abs() / scale, torch.zeros_like(groups)
    for i in range(1, 8):   # past the middle between value i - 1 and value i, or on it and i even
        middle = 0.5 * (MAGNITUDES[i - 1] + MAGNITUDES[i])
        kept = torch.where((a >= middle) if i % 2 == 0 else (a > middle), torch.full_like(kept, MAGNITUDES[i]), kept)
    return (kept * torch.sign(groups) * scale).reshape(x.shape)


def _held(codes, scales):
    """Values [..., d] in 64 bits of codes [..., d / 2] and scales [..., d / 32]."""
    powers = torch.tensor([2.0 ** (i - 127) for i in range(255)] + [math.nan], dtype=torch.float64, device=codes.device)
    magnitude = torch.tensor(MAGNITUDES, dtype=torch.float64, device=codes.device)
    nibble = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    return magnitude[nibble & 7] * torch.where(nibble > 7, -1.0, 1.0).double() * powers[scales.long()].repeat_interleave(32, -1)


def exact(case, seed):
    s = prepare(case, seed)
    total, fresh, page = s["total"], s["fresh"], case["page"]
    if case["op"] != "paged4":
        ks, vs, t = [], [], 0
        for i in range(case["n_seq"]):
            place = torch.arange(total[i] - fresh[i], total[i], device="cuda")
            if case["op"] == "read4":
                ids = s["page_table"][i].long()[place // page]
                k, v = (_held(s[x + "_codes"].permute(0, 2, 1, 3)[ids, place % page], s[x + "_scales"].permute(0, 2, 1, 3)[ids, place % page]) for x in "kv")
            else:
                k = s["k"][t:t + fresh[i]].double()
                if s["k_weight"] is not None:
                    k = k / (k.pow(2).sum(-1, keepdim=True) / case["d"] + EPS).sqrt() * s["k_weight"].double()
                if s["cos"] is not None:
                    turn, half = torch.complex(s["cos"].double()[place], s["sin"].double()[place])[:, None], case["d"] // 2
                    if case["rope"] == "halves":
                        z = torch.complex(k[..., :half], k[..., half:]) * turn
                        k = torch.cat((z.real, z.imag), -1)
                    else:
                        k = torch.view_as_real(torch.view_as_complex(k.unflatten(-1, (half, 2)).contiguous()) * turn).flatten(-2)
                k, v = _stored(k), _stored(s["v"][t:t + fresh[i]].double())
            ks.append(k)
            vs.append(v)
            t += fresh[i]
        return [torch.cat(ks), torch.cat(vs)]
    H, Hkv, d = case["H"], case["Hkv"], case["d"]
    o = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    t = 0
    for i in range(case["n_seq"]):
        n, t1 = total[i], t + fresh[i]
        ids = s["page_table"][i, :-(-n // page)].long()
        sees = torch.arange(n, device="cuda") <= torch.arange(n - fresh[i], n, device="cuda")[:, None]
        for g in range(Hkv):
            k, v = (_held(s[x + "_codes"][ids, g], s[x + "_scales"][ids, g]).reshape(-1, d)[:n] for x in "kv")
            for h in range(g * H // Hkv, (g + 1) * H // Hkv):
                score = (s["q"][t:t1, h].double() @ k.T / math.sqrt(d)).masked_fill(~sees, -math.inf)
                lse[t:t1, h] = torch.logsumexp(score, -1)
                o[t:t1, h] = torch.softmax(score, -1) @ v
        t = t1
    return [o, lse if case["lse"] else None]
