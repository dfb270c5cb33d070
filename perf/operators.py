"""The operators around attention in a language model's layer, measured over the range they are used in.

  qk      norms of queries and keys for each head with the position rotation in the same pass; with its gradient
  append  new keys and values into a paged cache, keys normed and rotated on the way
  paged   attention of new tokens (one for each sequence or chunks of a prompt) over a paged cache

Each case is one pass: with `own` through this library's entry points, without it in elementary torch operations.
"""
import math
import random

import torch

own = False

EPS = 1e-6


# ---- cases -----------------------------------------------------------------------------------------

def _qk(name, kind, dtype, B, H, Hkv, N, d, rope, rot, norm, weights, spread):
    """kind: forward or train (forward and gradient). weights: f32 or bf16, `heads` after it where each head has its own.
    spread: positions come as a tensor (a batch of sequences at different places) instead of one after the other."""
    return {"name": name, "op": "qk", "kind": kind, "dtype": dtype, "B": B, "H": H, "Hkv": Hkv, "N": N, "d": d, "rope": rope,
            "rot": rot, "norm": norm, "weights": weights, "spread": spread}


def _append(name, dtype, n_seq, new, most, Hkv, d, page, order, rope, norm, len_seed):
    """n_seq sequences of up to `most` tokens with their new ones, up to `new` of them new. order: how a page lies in memory."""
    return {"name": name, "op": "append", "dtype": dtype, "n_seq": n_seq, "new": new, "most": most, "Hkv": Hkv, "d": d, "page": page,
            "order": order, "rope": rope, "norm": norm, "len_seed": len_seed}


def _paged(name, dtype, n_seq, chunks, new, most, H, Hkv, d, page, order, lse, len_seed):
    """n_seq sequences of up to `most` tokens, `chunks` of them with `new` new ones and the others with a single one."""
    return {"name": name, "op": "paged", "dtype": dtype, "n_seq": n_seq, "chunks": chunks, "new": new, "most": most, "H": H, "Hkv": Hkv,
            "d": d, "page": page, "order": order, "lse": lse, "len_seed": len_seed}


def listed():
    return [
        # A decoding step of 64 sequences, d = 64 with grouped heads: all latency.
        _qk("qk_decode", "forward", "bf16", 64, 32, 8, 1, 64, "halves", 64, True, "bf16", True),
        # A prompt of 4096 tokens of the same layer, out of one projection for queries, keys and values.
        _qk("qk_prefill", "forward", "bf16", 1, 32, 8, 4096, 64, "halves", 64, True, "bf16", False),
        # A training step on a batch of medium-length sequences, d = 128: the most bytes.
        _qk("qk_train", "train", "bf16", 4, 16, 16, 8192, 128, "halves", 128, True, "f32", False),
        # A layer kept in float32, an odd length, neighbouring channels as pairs, half of them rotated, a weight for each head.
        _qk("qk_train_f32", "train", "f32", 1, 8, 8, 2047, 64, "neighbours", 32, True, "f32 heads", False),
        # One new token for each of 64 sequences of up to 2048.
        _append("append_decode", "bf16", 64, 1, 2048, 8, 64, 16, "heads", "halves", True, 1),
        # Prompts of five sequences at once, some with a cached prefix; pages with the tokens outside and the heads inside.
        _append("append_prompts", "bf16", 5, 4096, 8192, 16, 128, 64, "tokens", "halves", False, 2),
        # A check of a model's block in float32: three short sequences.
        _paged("paged_f32", "f32", 3, 3, 48, 700, 8, 8, 64, 16, "heads", True, 3),
        # One user's next token after 777.
        _paged("paged_one", "bf16", 1, 0, 1, 777, 32, 8, 64, 16, "heads", False, 4),
        # A decoding step of 64 sequences of up to 8192 tokens, grouped heads.
        _paged("paged_decode", "bf16", 64, 0, 1, 8192, 32, 8, 64, 16, "heads", False, 5),
        # The next token of one very long document, d = 128, pages with the tokens outside.
        _paged("paged_long", "bf16", 1, 0, 1, 100003, 16, 16, 128, 128, "tokens", False, 6),
        # A long prompt's last chunk: 2048 tokens on 16384. The most arithmetic.
        _paged("paged_chunk", "bf16", 1, 1, 2048, 16384, 32, 8, 64, 64, "heads", False, 7),
        # Prompts and decoding in one step: two chunks of 250 tokens beside 14 single tokens, d = 128, grouped heads.
        _paged("paged_mixed", "bf16", 16, 2, 250, 4096, 32, 8, 128, 32, "heads", True, 8),
    ]


def _spread(rng, lo, hi):
    """An integer of [lo, hi], even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_once(rng):
    op = rng.choice(("qk", "qk", "append", "paged", "paged", "paged"))
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    d = rng.choice((64, 128))
    Hkv = rng.choice((1, 2, 4, 8, 16))
    H = Hkv * rng.choice((1, 2, 3, 4, 4, 8))
    rope, norm = rng.choice(("halves", "halves", "neighbours", "none")), rng.random() < 0.6
    if op == "qk":
        if rope == "none":
            norm = True
        rot = 0 if rope == "none" else rng.choice((d, d, d // 2, 32))
        weights = rng.choice(("f32", "bf16", "f32 heads")) if dtype == "bf16" else rng.choice(("f32", "f32 heads"))
        if rng.random() < 0.3:
            B, N, kind = _spread(rng, 1, 256), rng.choice((1, 1, 1, 2, 5)), "forward"
        else:
            B, N, kind = rng.choice((1, 1, 2, 4)), _spread(rng, 40, 16384), rng.choice(("forward", "train"))
        return _qk("", kind, dtype, B, H, Hkv, N, d, rope, rot, norm, weights, rng.random() < 0.4)
    page, order, seed = rng.choice((16, 32, 48, 64, 128, 256)), rng.choice(("heads", "tokens")), rng.randrange(1 << 20)
    if op == "append":
        n_seq = _spread(rng, 1, 128)
        new = 1 if rng.random() < 0.5 else _spread(rng, 2, max(2, 8192 // n_seq))
        return _append("", dtype, n_seq, new, new + _spread(rng, 1, max(1, 65536 // n_seq)), Hkv, d, page, order, rope, norm, seed)
    family = "chunk" if dtype == "f32" else rng.choice(("decode", "decode", "chunk", "mixed"))
    if family == "decode":
        n_seq = _spread(rng, 1, 128)
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
        padded = case["n_seq"] * case["H"] * case["new"] * case["most"] if case["op"] == "paged" else 0   # scores that the plain form holds
        if w["bytes"] <= most_bytes and w["flops"] <= (most_flops if case["dtype"] == "bf16" else f32_flops) and padded <= 1.1e9:
            return case


def _lengths(case):
    """(tokens in the cache with the new ones, new ones) of each sequence; the first is the longest there may be."""
    rng = random.Random(case["len_seed"])
    total, fresh = [], []
    for s in range(case["n_seq"]):
        if case["op"] == "append":
            n = case["new"] if s == 0 or case["new"] == 1 else _spread(rng, 1, case["new"])
        else:
            n = case["new"] if s < case["chunks"] else 1
        total.append(case["most"] if s == 0 else max(n, rng.randint(case["most"] // 4, case["most"])))
        fresh.append(n)
    return total, fresh


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    d = case["d"]
    if case["op"] == "qk":
        rows = case["B"] * (case["H"] + case["Hkv"]) * case["N"]
        angles = case["rot"] * 4 * (case["B"] if case["spread"] else 1) * case["N"]
        bytes_, flops = 2 * rows * d * size + angles, rows * (3 * case["rot"] + (4 * d if case["norm"] else 0))
        if case["kind"] == "train":
            bytes_, flops = bytes_ + 3 * rows * d * size + angles, flops + rows * (3 * case["rot"] + (9 * d if case["norm"] else 0))
        return {"bytes": bytes_, "flops": flops}
    total, fresh = _lengths(case)
    T = sum(fresh)
    if case["op"] == "append":
        angles = 0 if case["rope"] == "none" else T * d * 4
        return {"bytes": 4 * T * case["Hkv"] * d * size + angles, "flops": T * case["Hkv"] * d * (3 + (4 if case["norm"] else 0))}
    pairs = sum(n * (t - n) + n * (n + 1) // 2 for t, n in zip(total, fresh))
    return {"bytes": 2 * T * case["H"] * d * size + 2 * sum(total) * case["Hkv"] * d * size + (4 * T * case["H"] if case["lse"] else 0),
            "flops": 4 * case["H"] * d * pairs}


# ---- inputs ----------------------------------------------------------------------------------------

def _tables(n_pos, rot, dev):
    """cos and sin of position times 10000^(-2 i / rot), float32 [n_pos, rot / 2], the angles in 64 bits."""
    rate = 10000.0 ** (-torch.arange(0, rot, 2, device=dev, dtype=torch.float64) / rot)
    angle = torch.arange(n_pos, device=dev, dtype=torch.float64)[:, None] * rate
    return angle.cos().float(), angle.sin().float()


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    s = {"case": case}

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev)

    def weight(heads, kind):
        w = 1.0 + 0.2 * normal(*((heads, case["d"]) if "heads" in kind else (case["d"],)))
        return w.to(torch.bfloat16) if "bf16" in kind else w

    if case["op"] == "qk":
        B, H, Hkv, N, d = (case[x] for x in ("B", "H", "Hkv", "N", "d"))
        # queries and keys as views of one projection [B, N, (H + 2 Hkv) d], channels of different size
        x = (normal(B, N, (H + 2 * Hkv) * d) * torch.exp(0.3 * normal((H + 2 * Hkv) * d))).to(dtype)
        s["q"] = x[..., :H * d].unflatten(-1, (H, d)).transpose(1, 2)
        s["k"] = x[..., H * d:(H + Hkv) * d].unflatten(-1, (Hkv, d)).transpose(1, 2)
        s["q_out"], s["k_out"] = (torch.empty(B, h, N, d, dtype=dtype, device=dev) for h in (H, Hkv))
        s["q_weight"], s["k_weight"] = (weight(h, case["weights"]) if case["norm"] else None for h in (H, Hkv))
        n_pos = N + (1024 if case["spread"] else 0)
        s["cos"], s["sin"] = _tables(n_pos, case["rot"], dev) if case["rot"] else (None, None)
        s["positions"] = None
        if case["spread"] and case["rot"]:
            start = torch.randint(0, 1024, (B, 1), generator=gen, device=dev)
            s["positions"] = (start + torch.arange(N, device=dev)).to(torch.int32)
        if case["kind"] == "train":
            s["dq_out"], s["dk_out"] = (normal(B, h, N, d).to(dtype) for h in (H, Hkv))
            g = torch.empty_like(x)   # the gradient of the projection, in its layout
            s["dq"] = g[..., :H * d].unflatten(-1, (H, d)).transpose(1, 2)
            s["dk"] = g[..., H * d:(H + Hkv) * d].unflatten(-1, (Hkv, d)).transpose(1, 2)
            s["dq_weight"], s["dk_weight"] = (torch.empty(w.shape, device=dev) if w is not None else None for w in (s["q_weight"], s["k_weight"]))
    else:
        total, fresh = _lengths(case)
        n_seq, page, Hkv, d = case["n_seq"], case["page"], case["Hkv"], case["d"]
        T, need = sum(fresh), [-(-t // page) for t in total]
        n_pages = sum(need) + 3
        s["fresh"], s["total"] = fresh, total
        # the pool [pages, 2, ...]: K and V of a page side by side, its heads or its tokens outside
        shape = (n_pages, 2, Hkv, page, d) if case["order"] == "heads" else (n_pages, 2, page, Hkv, d)
        pool = torch.empty(shape, dtype=dtype, device=dev)
        for part in pool.split(max(1, (1 << 26) // pool[0].numel())):
            part.copy_(normal(*part.shape))
        s["k_pages"], s["v_pages"] = (x if case["order"] == "heads" else x.transpose(1, 2) for x in (pool[:, 0], pool[:, 1]))
        order = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32)
        table = torch.full((n_seq, max(need)), -1, dtype=torch.int32, device=dev)
        at = 0
        for i, n in enumerate(need):
            table[i, :n] = order[at:at + n]
            at += n
        s["page_table"] = table
        s["kv_len"] = torch.tensor(total, dtype=torch.int32, device=dev)
        s["q_start"] = torch.tensor([sum(fresh[:i]) for i in range(n_seq + 1)], dtype=torch.int32, device=dev)
        if case["op"] == "append":
            x = (normal(T, 2 * Hkv * d) * torch.exp(0.3 * normal(2 * Hkv * d))).to(dtype)
            s["k"], s["v"] = (x[:, i * Hkv * d:(i + 1) * Hkv * d].unflatten(-1, (Hkv, d)) for i in (0, 1))
            s["k_weight"] = weight(Hkv, "f32" if case["dtype"] == "f32" else "bf16") if case["norm"] else None
            s["cos"], s["sin"] = _tables(case["most"], d, dev) if case["rope"] != "none" else (None, None)
        else:
            s["q"] = (1.5 * normal(T, case["H"], d)).to(dtype)
            s["o"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty(T, case["H"], device=dev) if case["lse"] else None
    if own:
        _plan(s)
    return s


def _plan(s):
    """What a program that uses the library keeps for a layer: the parameters of its calls, and scratch."""
    import paper_2507_17245_amd as da
    c = s["case"]
    if c["op"] == "qk":
        options = dict(norm=c["norm"], eps=EPS, q_weight=s["q_weight"], k_weight=s["k_weight"], rope=c["rope"], cos=s["cos"], sin=s["sin"],
                       positions=s["positions"])
        s["plan"] = da.make_qk_params(s["q"], s["k"], s["q_out"], s["k_out"], **options)
        if c["kind"] == "train":
            s["scratch"] = _scratch(da.distr_attn_qk_bwd_workspace_bytes(s["plan"]))
            s["plan"] = da.make_qk_params(s["q"], s["k"], s["q_out"], s["k_out"], workspace=s["scratch"], **options)
        return
    cache = (s["k_pages"], s["v_pages"], s["page_table"], s["kv_len"], s["q_start"])
    if c["op"] == "append":
        s["plan"] = da.make_paged_params(*cache, k=s["k"], v=s["v"], norm=c["norm"], eps=EPS, k_weight=s["k_weight"], rope=c["rope"],
                                         cos=s["cos"], sin=s["sin"])
    else:
        s["scratch"] = _scratch(da.distr_attn_paged_workspace_bytes(da.make_paged_params(*cache, q=s["q"])))
        s["plan"] = da.make_paged_params(*cache, q=s["q"], lse_out=s["lse"], workspace=s["scratch"])


def _scratch(n):
    return torch.empty(max(256, n), dtype=torch.uint8, device="cuda")


# ---- one pass --------------------------------------------------------------------------------------

def _run_own(s):
    import paper_2507_17245_amd as da
    c = s["case"]
    if c["op"] == "qk":
        da.distr_attn_qk_norm_rope(s["q"], s["k"], s["q_out"], s["k_out"], s["plan"])
        if c["kind"] == "forward":
            return [s["q_out"], s["k_out"]]
        da.distr_attn_qk_norm_rope_bwd(s["q"], s["k"], s["dq_out"], s["dk_out"], s["dq"], s["dk"], s["plan"],
                                       dq_weight=s["dq_weight"], dk_weight=s["dk_weight"])
        return [s["q_out"], s["k_out"], s["dq"], s["dk"], s["dq_weight"], s["dk_weight"]]
    if c["op"] == "append":
        da.distr_attn_cache_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["plan"])
        return [s["k_pages"], s["v_pages"]]
    da.distr_attn_paged_fwd(s["q"], s["k_pages"], s["v_pages"], s["o"], s["plan"])
    return [s["o"], s["lse"]]


def _rotated(x, cos, sin, rope):
    """x [..., d] with its first 2 * cos.shape[-1] channels rotated, in pairs of a half's channel with the other's or of neighbours."""
    if cos is None:
        return x
    half = cos.shape[-1]
    y = x.clone()
    if rope == "halves":
        a, b = x[..., :half], x[..., half:2 * half]
        y[..., :half], y[..., half:2 * half] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * cos - b * sin, a * sin + b * cos
    return y


def _heads_weight(w):
    """[d] or [heads, d] against [B, heads, N, d]"""
    return w.float() if w.dim() == 1 else w.float()[:, None, :]


def _plain_qk(x, w, cos, sin, s):
    c = s["case"]
    x = x.float()
    if c["norm"]:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * _heads_weight(w)
    return _rotated(x, cos, sin, c["rope"])


def _plain_qk_grad(x, w, g, cos, sin, s):
    """(gradient of the input, of the weight)"""
    c = s["case"]
    g = _rotated(g.float(), cos, None if sin is None else -sin, c["rope"])
    if not c["norm"]:
        return g, None
    x = x.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    unit = x * r
    dw = (g * unit).sum((0, 2) if w.dim() == 2 else (0, 1, 2), dtype=torch.float64).float()
    g = g * _heads_weight(w)
    return r * (g - unit * (g * unit).mean(-1, keepdim=True)), dw


def _places(s):
    """(sequence, place in it, page, row in the page) of each new token."""
    start, T = s["q_start"].long(), s["k"].shape[0]
    t = torch.arange(T, device=start.device)
    seq = torch.searchsorted(start, t, right=True) - 1
    place = s["kv_len"].long()[seq] - (start[seq + 1] - t)
    return seq, place, s["page_table"].long()[seq, place // s["case"]["page"]], place % s["case"]["page"]


def _run_plain(s):
    c = s["case"]
    dtype = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    if c["op"] == "qk":
        cos, sin = s["cos"], s["sin"]
        if cos is not None:
            cos, sin = (x[s["positions"].long()][:, None] if s["positions"] is not None else x[:c["N"]] for x in (cos, sin))
        out = [_plain_qk(s[x], s[x + "_weight"], cos, sin, s).to(dtype) for x in ("q", "k")]
        if c["kind"] == "train":
            grads = [_plain_qk_grad(s[x], s[x + "_weight"], s["d" + x + "_out"], cos, sin, s) for x in ("q", "k")]
            out += [g[0].to(dtype) for g in grads] + [g[1] for g in grads]
        return out
    if c["op"] == "append":
        _, place, page, row = _places(s)
        k = s["k"].float()
        if c["norm"]:
            k = k * torch.rsqrt(k.square().mean(-1, keepdim=True) + EPS) * s["k_weight"].float()
        if s["cos"] is not None:
            k = _rotated(k, s["cos"][place][:, None], s["sin"][place][:, None], c["rope"])
        s["k_pages"].transpose(1, 2)[page, row] = k.to(dtype)
        s["v_pages"].transpose(1, 2)[page, row] = s["v"]
        return [s["k_pages"], s["v_pages"]]
    # attention: the sequences padded to the most new tokens and the most pages
    n_seq, new, d, H, Hkv = c["n_seq"], max(s["fresh"]), c["d"], c["H"], c["Hkv"]
    table, kv_len, start = s["page_table"].long().clamp(min=0), s["kv_len"].long(), s["q_start"].long()
    k, v = (x[table].transpose(1, 2).reshape(n_seq, Hkv, -1, d).float() for x in (s["k_pages"], s["v_pages"]))
    fresh = start[1:] - start[:-1]
    i = torch.arange(new, device=table.device)
    q = s["q"][(start[:-1, None] + i.clamp(max=new)).clamp(max=s["q"].shape[0] - 1)].float()             # [seq, new, H, d]
    q = q.unflatten(2, (Hkv, H // Hkv)).permute(0, 2, 3, 1, 4).reshape(n_seq, Hkv, -1, d)              # [seq, Hkv, heads x new, d]
    score = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(d)).unflatten(2, (H // Hkv, new))
    place = kv_len[:, None] - fresh[:, None] + i                                                        # of the new tokens
    hidden = torch.arange(k.shape[2], device=table.device) > place[:, :, None].clamp(max=kv_len.max())
    hidden |= torch.arange(k.shape[2], device=table.device) >= kv_len[:, None, None]
    score.masked_fill_(hidden[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), v).unflatten(2, (H // Hkv, new)) / total                         # [seq, Hkv, heads, new, d]
    mine = i[None, :] < fresh[:, None]
    o = o.permute(0, 3, 1, 2, 4).reshape(n_seq, new, H, d)[mine].to(dtype)
    if not c["lse"]:
        return [o, None]
    return [o, (top + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(n_seq, new, H)[mine]]


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ---- the definition in 64 bits ---------------------------------------------------------------------

def _turned(x, position, s):
    """x [..., d] as complex numbers times (cos + i sin) of each position; position broadcasts against x.shape[:-1]."""
    if s["cos"] is None:
        return x
    half = s["cos"].shape[1]
    turn = torch.complex(s["cos"].double()[position], s["sin"].double()[position])
    if s["case"]["rope"] == "halves":
        z = torch.complex(x[..., :half], x[..., half:2 * half]) * turn
        return torch.cat((z.real, z.imag, x[..., 2 * half:]), -1)
    z = torch.view_as_complex(x[..., :2 * half].unflatten(-1, (half, 2)).contiguous()) * turn
    return torch.cat((torch.view_as_real(z).flatten(-2), x[..., 2 * half:]), -1)


def _normed(x, w):
    if w is None:
        return x
    return x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * w


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "qk":
        position = torch.arange(case["N"], device="cuda").expand(case["B"], -1) if s["positions"] is None else s["positions"].long()
        out = {}
        for x in ("q", "k"):
            leaf, w = s[x].double(), s[x + "_weight"]
            leaves = [leaf] if w is None else [leaf, w.double()]
            train = case["kind"] == "train"
            for t in leaves:
                t.requires_grad_(train)
            y = _normed(leaf, None if w is None else leaves[1].unsqueeze(-2) if w.dim() == 2 else leaves[1])
            y = _turned(y, position[:, None], s)
            out[x] = [y.detach()]
            if train:
                grads = torch.autograd.grad(y, leaves, s["d" + x + "_out"].double())
                out[x] += [grads[0], None if w is None else grads[1]]
            del y
        return [t for pair in zip(out["q"], out["k"]) for t in pair]
    total, fresh, page = s["total"], s["fresh"], case["page"]
    if case["op"] == "append":
        k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
        t = 0
        for i in range(case["n_seq"]):
            place = torch.arange(total[i] - fresh[i], total[i], device="cuda")
            k = _normed(s["k"][t:t + fresh[i]].double(), None if s["k_weight"] is None else s["k_weight"].double())
            k = _turned(k.transpose(0, 1), place, s).transpose(0, 1)
            ids = s["page_table"][i].long()[place // page]
            k_pages.permute(0, 2, 1, 3)[ids, place % page] = k
            v_pages.permute(0, 2, 1, 3)[ids, place % page] = s["v"][t:t + fresh[i]].double()
            t += fresh[i]
        return [k_pages, v_pages]
    H, Hkv, d = case["H"], case["Hkv"], case["d"]
    o = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    t = 0
    for i in range(case["n_seq"]):
        n, t1 = total[i], t + fresh[i]
        ids = s["page_table"][i, :-(-n // page)].long()
        sees = torch.arange(n, device="cuda") <= torch.arange(n - fresh[i], n, device="cuda")[:, None]
        for h in range(H):
            k, v = (x[ids, h * Hkv // H].reshape(-1, d)[:n].double() for x in (s["k_pages"], s["v_pages"]))
            score = (s["q"][t:t1, h].double() @ k.T / math.sqrt(d)).masked_fill(~sees, -math.inf)
            lse[t:t1, h] = torch.logsumexp(score, -1)
            o[t:t1, h] = torch.softmax(score, -1) @ v
        t = t1
    return [o, lse if case["lse"] else None]
