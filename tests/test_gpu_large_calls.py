"""Calls around attention that are large enough for the kernels to go past the caches, to walk the rows several times over, and to take two heads to
a workgroup; against 64 bits on the device."""
import pytest
import torch

import paper_2507_17245_amd as da
from paged_util import HALF_STEP, attention_bounds, normed, tables, turn, turn_bound
from test_gpu_qk_norm_rope import EPS, STEPS

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
STEP = 2.0 ** -24
CUS = 256


def _weight(w):
    return w.double()[:, None, :] if w.dim() == 2 else w.double()


def _chain(rows, heads, d, each):
    """The longest chain of additions of a weight's gradient: a lane's rows (of up to four heads) where workgroups walk them, those of a
    workgroup's lanes, a thread's share of the workgroups' sums, the 32 shares."""
    side = 256 * 16 // d
    chunk = 1 if each else 4
    chunks = sum(-(-h // chunk) for h in heads)
    groups = max(1, 2 * CUS // chunks)          # (at least, where there are as many rows)
    lane = chunk * -(-rows // (side * groups))
    return lane + side + -(-(4 * CUS + chunks) // 32) + 32


ROWS = [  # dtype, B, H, Hkv, N, d, rope, rotated, a weight for each head
    (BF, 2, 16, 16, 5001, 128, "halves", 128, False),        # 164 MB forward, 246 with the gradient
    (BF, 1, 40, 8, 12003, 64, "neighbours", 64, False),      # 147 MB
    (BF, 3, 16, 2, 10007, 64, "halves", 32, True),           # 138 MB, a weight for each head
    (F, 1, 8, 8, 9001, 128, "halves", 128, False),           # float: in the caches' way always
    (BF, 1, 33, 7, 1701, 64, "halves", 64, False),           # two heads to a workgroup, odd numbers of both
    (BF, 1, 5, 3, 9007, 128, "neighbours", 128, True),
    (F, 2, 3, 2, 20011, 64, "neighbours", 64, True),         # one head to a workgroup, many turns of its rows
    (BF, 1, 1, 0, 70001, 64, "halves", 64, False),
]


@pytest.mark.parametrize("case", ROWS)
def test_rows_and_their_gradient(case):
    dtype, B, H, Hkv, N, d, rope, rot, each = case
    g = torch.Generator(device="cuda").manual_seed(N)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    x = normal(B, N, (H + 2 * Hkv) * d).to(dtype)
    grad = torch.full_like(x, float("nan"))
    cos, sin = (t.cuda() for t in tables(N, rot))
    heads = {"q": (H, 0), "k": (Hkv, H)}
    t = {}
    for name, (n, at) in heads.items():
        if n == 0:
            t.update({name + what: None for what in ("", "_out", "_w", "_g", "_d", "_dw")})
            continue
        part = lambda buffer: buffer[..., at * d:(at + n) * d].unflatten(-1, (n, d)).transpose(1, 2)   # noqa: E731
        t[name], t[name + "_d"] = part(x), part(grad)
        t[name + "_out"] = torch.full((B, n, N, d), float("nan"), dtype=dtype, device="cuda")
        t[name + "_g"] = normal(B, n, N, d).to(dtype)
        t[name + "_w"] = 1.0 + 0.3 * normal(*((n, d) if each else (d,)))
        t[name + "_dw"] = torch.full_like(t[name + "_w"], float("nan"))
    p = da.make_qk_params(t["q"], t["k"], t["q_out"], t["k_out"], norm=True, eps=EPS, q_weight=t["q_w"], k_weight=t["k_w"], rope=rope, cos=cos, sin=sin)
    da.distr_attn_qk_norm_rope(t["q"], t["k"], t["q_out"], t["k_out"], p)
    da.distr_attn_qk_norm_rope_bwd(t["q"], t["k"], t["q_g"], t["k_g"], t["q_d"], t["k_d"], p, dq_weight=t["q_dw"], dk_weight=t["k_dw"])
    torch.cuda.synchronize()
    c, s = cos.double(), sin.double()
    for name, (n, _) in heads.items():
        if n == 0:
            continue
        w = _weight(t[name + "_w"])
        dw, dw_size = (torch.zeros_like(t[name + "_dw"], dtype=torch.float64) for _ in (0, 1))
        terms = (0, 2) if each else (0, 1, 2)
        for b in range(B):                                             # (a batch at a time)
            v, dy = t[name][b:b + 1].double(), t[name + "_g"][b:b + 1].double()
            y = normed(v, w, EPS)
            unit_y, want = turn_bound(y, rot, rope), turn(y, c, s, rope)
            err = (t[name + "_out"][b:b + 1].double() - want).abs()
            assert (err <= HALF_STEP[dtype] * 1.01 * want.abs() + STEPS * STEP * unit_y).all(), (name, b)
            size, dy = turn_bound(dy, rot, rope), turn(dy, c, -s, rope)
            r = 1.0 / (v.square().mean(-1, keepdim=True) + EPS).sqrt()
            unit, u = v * r, dy * w
            want = r * (u - unit * (u * unit).mean(-1, keepdim=True))
            # (as for the small calls: u is off by 4 half steps of its pair, unit by STEPS, the mean by both and 20 of its terms' magnitudes)
            bound = 3 * STEPS * STEP * r * w.abs().amax() * (size + unit.abs() * (size * unit.abs()).mean(-1, keepdim=True))
            err = (t[name + "_d"][b:b + 1].double() - want).abs()
            assert (err <= HALF_STEP[dtype] * 1.01 * want.abs() + bound).all(), (name, b)
            dw += (dy * unit).sum(terms)
            dw_size += (size * unit.abs()).sum(terms)
        err = (t[name + "_dw"].double() - dw).abs()
        assert (err <= (_chain(B * N, (H, Hkv), d, each) + 2 * STEPS) * STEP * dw_size).all(), name
    assert grad[..., (H + Hkv) * d:].isnan().all()


@pytest.mark.parametrize("dtype,new,Hkv,d,page,order", [(BF, (5003, 4, 4001), 16, 128, 64, "tokens"), (BF, (17, 9001), 16, 128, 48, "heads"),
                                                        (BF, (9000, 9001), 16, 64, 16, "heads"), (F, (3001, 2000), 16, 128, 64, "heads")])
def test_appends(dtype, new, Hkv, d, page, order):
    """147 to 164 MB, read and written: bf16 past the caches."""
    T, lens = sum(new), [n + 37 * i for i, n in enumerate(new)]
    assert 4 * T * Hkv * d * (2 if dtype == BF else 4) > 128 << 20
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, 2, Hkv, d, generator=g, device="cuda").to(dtype)
    k, v = x[:, 0], x[:, 1]
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + 2
    shape = (n_pages, 2, Hkv, page, d) if order == "heads" else (n_pages, 2, page, Hkv, d)
    pool = torch.full(shape, 7.0, dtype=dtype, device="cuda")
    kp, vp = (pool[:, i] if order == "heads" else pool[:, i].transpose(1, 2) for i in (0, 1))
    ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(new), max(need)), -1, dtype=torch.int32, device="cuda")
    for i, n in enumerate(need):
        table[i, :n] = ids[sum(need[:i]):sum(need[:i + 1])]
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    start = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda")
    w = 1 + 0.3 * torch.randn(d, generator=g, device="cuda")
    cos, sin = (t.cuda() for t in tables(max(lens), d))
    p = da.make_paged_params(kp, vp, table, kv_len, start, k=k, v=v, norm=True, eps=EPS, k_weight=w, rope="halves", cos=cos, sin=sin)
    da.distr_attn_cache_append(k, v, kp, vp, p)
    torch.cuda.synchronize()
    touched = torch.zeros(n_pages, page, dtype=torch.bool, device="cuda")
    for i, n in enumerate(new):
        place = torch.arange(lens[i] - n, lens[i], device="cuda")
        at, row, rows = table[i].long()[place // page], place % page, slice(int(start[i]), int(start[i]) + n)
        touched[at, row] = True
        y = normed(k[rows].double(), w.double(), EPS)
        unit = turn_bound(y, d, "halves")
        y = turn(y, cos.double()[place][:, None], sin.double()[place][:, None], "halves")
        err = (kp[at, :, row].double() - y).abs()
        assert (err <= HALF_STEP[dtype] * 1.01 * y.abs() + STEPS * STEP * unit).all(), i
        assert torch.equal(vp[at, :, row], v[rows]), i
    for t in (kp, vp):
        assert (t.transpose(1, 2)[~touched] == 7.0).all()


@pytest.mark.parametrize("lens,H,Hkv,d,page,order", [((70001,), 16, 8, 128, 64, "heads"), ((90001, 3, 61000), 16, 8, 64, 16, "tokens"),
                                                     ((3700,) * 40, 8, 8, 64, 32, "heads"), ((1200,) * 130, 4, 4, 128, 64, "tokens")])
def test_single_tokens(lens, H, Hkv, d, page, order):
    """More than 256 MB of keys and values: their tiles leave the caches alone. Workgroups of eight, four and two waves."""
    assert 4 * sum(lens) * Hkv * d > 256 << 20
    n_seq, T = len(lens), len(lens)
    g = torch.Generator(device="cuda").manual_seed(T)
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + 2
    shape = (n_pages, 2, Hkv, page, d) if order == "heads" else (n_pages, 2, page, Hkv, d)
    pool = torch.randn(shape, generator=g, device="cuda").to(BF)
    kp, vp = (pool[:, i] if order == "heads" else pool[:, i].transpose(1, 2) for i in (0, 1))
    ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((n_seq, max(need)), -1, dtype=torch.int32, device="cuda")
    for i, n in enumerate(need):
        table[i, :n] = ids[sum(need[:i]):sum(need[:i + 1])]
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    start = torch.arange(n_seq + 1, dtype=torch.int32, device="cuda")
    q = (1.5 * torch.randn(T, H, d, generator=g, device="cuda")).to(BF)
    o, lse = torch.full_like(q, float("nan")), torch.full((T, H), float("nan"), device="cuda")
    p = da.make_paged_params(kp, vp, table, kv_len, start, q=q, lse_out=lse)
    ws = torch.empty(da.distr_attn_paged_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    da.distr_attn_paged_fwd(q, kp, vp, o, da.make_paged_params(kp, vp, table, kv_len, start, q=q, lse_out=lse, workspace=ws))
    torch.cuda.synchronize()
    for i in sorted({0, 1, 2, n_seq // 2, n_seq - 1}):
        if i >= n_seq:
            continue
        n, at = lens[i], table[i, :need[i]].long()
        want, mean, ln, most = (torch.zeros(*s, dtype=torch.float64) for s in ((1, H, d), (1, H, d), (1, H), (1, H)))
        for h in range(H):
            k, v = (t[at, h * Hkv // H].reshape(-1, d)[:n].double() for t in (kp, vp))
            score = k @ q[i, h].double() * d ** -0.5
            weight = torch.softmax(score, 0)
            want[0, h], mean[0, h], ln[0, h] = weight @ v, weight @ v.abs(), torch.logsumexp(score, 0)
            most[0, h] = (k.abs() @ q[i, h].double().abs()).max() * d ** -0.5
        bound, ln_bound = attention_bounds(want, mean, ln, most, n, d, BF)
        assert ((o[i:i + 1].double().cpu() - want).abs() <= bound).all(), i
        assert ((lse[i:i + 1].double().cpu() - ln).abs() <= ln_bound).all(), i
    assert o.isfinite().all()
