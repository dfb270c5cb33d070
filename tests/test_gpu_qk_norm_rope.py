"""Norms and rotation of queries and keys against 64 bits: layouts, pairings, weights, lengths, gradients."""
import pytest
import torch

import paper_2507_17245_amd as da
from paged_util import HALF_STEP, normed, pair_places, tables, turn, turn_bound

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
EPS = 1e-5
# What float arithmetic adds to the result's rounding, in half steps of |a| + |b|: 16 terms of a square sum in a lane, 3 joined, mean
# and eps (together halved by the root), root, reciprocal, two products, two products and a sum of the rotation.
STEPS = 24


def _layouts(kind, B, heads, N, d, dtype, values=None):
    """A [B, heads, N, d] tensor laid out as `kind` says, and the buffer it lies in."""
    if kind == "heads":
        base = torch.full((B, heads, N, d), float("nan"), dtype=dtype, device="cuda")
        t = base
    elif kind == "tokens":           # [B, N, heads, d]
        base = torch.full((B, N, heads, d), float("nan"), dtype=dtype, device="cuda")
        t = base.transpose(1, 2)
    else:                            # part of a wider projection
        base = torch.full((B, N, (heads + 3) * d + 16), float("nan"), dtype=dtype, device="cuda")
        t = base[..., 16:16 + heads * d].unflatten(-1, (heads, d)).transpose(1, 2)
    if values is not None:
        t.copy_(values)
    return t, base


def _reference(x, w, positions, cos, sin, rope, norm):
    """-> result, bound of the float errors in units of a half step"""
    x = x.double().cpu()
    if norm:
        w = None if w is None else (w.double().cpu()[:, None, :] if w.dim() == 2 else w.double().cpu())
        x = normed(x, w, EPS)
    if rope == "none":
        return x, x.abs()
    c, s = (t.double()[positions][:, None] for t in (cos, sin))
    return turn(x, c, s, rope), turn_bound(x, 2 * cos.shape[1], rope)


CASES = [  # dtype, B, H, Hkv, N, d, layout in, layout out, rope, rotated, norm, weights, spread positions
    (BF, 1, 1, 1, 1, 64, "heads", "heads", "halves", 64, True, None, False),
    (BF, 3, 4, 2, 1, 64, "tokens", "heads", "halves", 64, True, "bf16", True),
    (BF, 2, 5, 1, 63, 128, "part", "heads", "halves", 128, True, "f32", False),
    (BF, 1, 6, 3, 65, 64, "part", "tokens", "neighbours", 32, True, "heads", True),
    (BF, 1, 2, 2, 300, 128, "tokens", "part", "halves", 48, False, None, False),
    (BF, 2, 3, 0, 33, 64, "heads", "heads", "neighbours", 64, True, "heads", False),
    (BF, 1, 32, 8, 2050, 64, "part", "heads", "halves", 64, True, "bf16", False),
    (F, 1, 3, 1, 1, 128, "heads", "heads", "halves", 128, True, "f32", True),
    (F, 2, 4, 4, 129, 64, "part", "heads", "neighbours", 64, True, "heads", False),
    (F, 1, 2, 1, 31, 128, "tokens", "tokens", "halves", 16, False, None, True),
    (F, 1, 2, 2, 17, 64, "heads", "part", "none", 0, True, None, False),
    (BF, 1, 2, 1, 17, 128, "tokens", "heads", "none", 0, True, "bf16", False),
]


def _make(case, seed=0):
    dtype, B, H, Hkv, N, d, lin, lout, rope, rot, norm, weights, spread = case
    g = torch.Generator().manual_seed(seed)
    n_pos = N + 7
    cos, sin = tables(n_pos, rot) if rope != "none" else (None, None)
    positions = (torch.randint(0, n_pos, (B, N), generator=g) if spread else torch.arange(N).expand(B, N))
    t = {"positions": positions, "cos": cos, "sin": sin}
    for x, heads in (("q", H), ("k", Hkv)):
        if heads == 0:
            t.update({x: None, x + "_out": None, x + "_base": None, "w" + x: None, "g" + x: None, "d" + x: None, "dw" + x: None})
            continue
        values = (torch.randn(B, heads, N, d, generator=g) * torch.exp(torch.randn(d, generator=g))).to(dtype)
        t[x], _ = _layouts(lin, B, heads, N, d, dtype, values)
        t[x + "_out"], t[x + "_base"] = _layouts(lout, B, heads, N, d, dtype)
        w = None if weights is None else 1.0 + 0.3 * torch.randn((heads, d) if weights == "heads" else (d,), generator=g)
        t["w" + x] = None if w is None else w.to(BF if weights == "bf16" else F).cuda()
        t["g" + x], _ = _layouts(lout, B, heads, N, d, dtype, torch.randn(B, heads, N, d, generator=g).to(dtype))
        t["d" + x], t["d" + x + "_base"] = _layouts(lin, B, heads, N, d, dtype)
        t["dw" + x] = torch.full((heads, d) if weights == "heads" else (d,), float("nan"), device="cuda") if norm else None
    dev = lambda x: None if x is None else x.cuda()   # noqa: E731
    t["params"] = da.make_qk_params(t["q"], t["k"], t["q_out"], t["k_out"], norm=norm, eps=EPS, q_weight=t["wq"], k_weight=t["wk"], rope=rope, cos=dev(cos),
                                    sin=dev(sin), positions=positions.to(torch.int32).cuda() if spread and rope != "none" else None)
    return t


@pytest.mark.parametrize("case", CASES)
def test_forward(case):
    dtype, rope, norm = case[0], case[8], case[10]
    t = _make(case)
    da.distr_attn_qk_norm_rope(t["q"], t["k"], t["q_out"], t["k_out"], t["params"])
    torch.cuda.synchronize()
    for x in ("q", "k"):
        if t[x] is None:
            continue
        want, unit = _reference(t[x], t["w" + x], t["positions"], t["cos"], t["sin"], rope, norm)
        err = (t[x + "_out"].double().cpu() - want).abs()
        assert (err <= HALF_STEP[dtype] * 1.01 * want.abs() + STEPS * 2.0 ** -24 * unit).all(), (x, err.max())
        rows = t[x + "_out"].numel()   # and nothing beside the rows
        assert t[x + "_base"].isnan().sum() == t[x + "_base"].numel() - rows


@pytest.mark.parametrize("case", CASES)
def test_backward(case):
    dtype, B, H, Hkv, N, d, lin, lout, rope, rot, norm, weights, spread = case
    t = _make(case)
    da.distr_attn_qk_norm_rope_bwd(t["q"], t["k"], t["gq"], t["gk"], t["dq"], t["dk"], t["params"], dq_weight=t["dwq"], dk_weight=t["dwk"])
    torch.cuda.synchronize()
    f = 2.0 ** -24
    for x in ("q", "k"):
        if t[x] is None:
            continue
        v, g, w = t[x].double().cpu(), t["g" + x].double().cpu(), t["w" + x]
        w = torch.ones(d, dtype=torch.float64) if w is None else w.double().cpu()
        w = w[:, None, :] if w.dim() == 2 else w
        size = turn_bound(g, rot, rope)
        if rope != "none":
            c, s = (y.double()[t["positions"]][:, None] for y in (t["cos"], t["sin"]))
            g = turn(g, c, -s, rope)
        want, bound = g, STEPS * f * size
        if norm:
            r = 1.0 / (v.square().mean(-1, keepdim=True) + EPS).sqrt()
            unit, u = v * r, g * w
            want = r * (u - unit * (u * unit).mean(-1, keepdim=True))
            # u is off by 4 half steps of its pair, unit by STEPS, the mean by both and 20 of its terms' magnitudes
            bound = 3 * STEPS * f * r * w.abs().amax() * (size + unit.abs() * (size * unit.abs()).mean(-1, keepdim=True))
            terms = (0, 2) if weights == "heads" else (0, 1, 2)
            dw, dw_size = (g * unit).sum(terms), (size * unit.abs()).sum(terms)
            err = (t["dw" + x].double().cpu() - dw).abs()
            # a chain is at most a lane's rows (here 8), 64 of a workgroup, 32 of as many workgroups and those 32
            assert (err <= (136 + 2 * STEPS) * f * dw_size).all(), (x, err.max())
        err = (t["d" + x].double().cpu() - want).abs()
        assert (err <= HALF_STEP[dtype] * 1.01 * want.abs() + bound).all(), (x, err.max())
        assert t["d" + x + "_base"].isnan().sum() == t["d" + x + "_base"].numel() - t["d" + x].numel()


@pytest.mark.parametrize("rope,rot", [("halves", 64), ("neighbours", 32)])
def test_gradient_against_differences(rope, rot):
    case = (F, 2, 2, 1, 9, 64, "heads", "heads", rope, rot, True, "f32", False)
    t = _make(case, seed=5)
    da.distr_attn_qk_norm_rope_bwd(t["q"], t["k"], t["gq"], t["gk"], t["dq"], t["dk"], t["params"], dq_weight=t["dwq"], dk_weight=t["dwk"])
    g = torch.Generator().manual_seed(6)
    for x in ("q", "k"):
        v, gy, w = t[x].double().cpu(), t["g" + x].double().cpu(), t["w" + x].double().cpu()

        def loss(v, w):
            return (_reference(v, w, t["positions"], t["cos"], t["sin"], rope, True)[0] * gy).sum()
        for got, at in ((t["d" + x].double().cpu(), 0), (t["dw" + x].double().cpu(), 1)):
            e, h = torch.randn(got.shape, generator=g, dtype=torch.float64), 1e-4
            ahead, back = ((loss(v + s * h * e, w) if at == 0 else loss(v, w + s * h * e)) for s in (1, -1))
            # central differences of a smooth function: h^2 and 1e-16 / h of its size, beside the gradient's float errors
            assert abs((ahead - back) / (2 * h) - (got * e).sum()) <= 1e-4 * (got.norm() * e.norm() + 1)


def test_in_place_and_without_weight_gradients():
    case = CASES[6]
    t, u = _make(case), _make(case)
    da.distr_attn_qk_norm_rope(t["q"], t["k"], t["q_out"], t["k_out"], t["params"])
    p = da.make_qk_params(u["q"], u["k"], u["q"], u["k"], norm=True, eps=EPS, q_weight=u["wq"], k_weight=u["wk"], rope="halves", cos=t["cos"].cuda(), sin=t["sin"].cuda())
    da.distr_attn_qk_norm_rope(u["q"], u["k"], u["q"], u["k"], p)
    assert torch.equal(u["q"], t["q_out"]) and torch.equal(u["k"], t["k_out"])
    u = _make(case)
    da.distr_attn_qk_norm_rope_bwd(t["q"], t["k"], t["gq"], t["gk"], t["dq"], t["dk"], t["params"], dq_weight=t["dwq"], dk_weight=t["dwk"])
    da.distr_attn_qk_norm_rope_bwd(u["q"], u["k"], u["gq"], u["gk"], u["dq"], u["dk"], u["params"])
    one = torch.full_like(t["dwk"], float("nan"))
    da.distr_attn_qk_norm_rope_bwd(u["q"], u["k"], u["gq"], u["gk"], u["dq"], u["dk"], u["params"], dk_weight=one)
    assert torch.equal(u["dq"], t["dq"]) and torch.equal(u["dk"], t["dk"]) and torch.equal(one, t["dwk"])


def test_gradient_in_place():
    x = torch.randn(2, 3, 40, 64, device="cuda")
    g = torch.randn_like(x)
    p = da.make_qk_params(x, None, g, None, norm=True, eps=EPS)
    dx = torch.empty_like(x)
    da.distr_attn_qk_norm_rope_bwd(x, None, g, None, dx, None, p)
    da.distr_attn_qk_norm_rope_bwd(x, None, g, None, g, None, p)
    assert torch.equal(dx, g)


@pytest.mark.parametrize("rope", ["halves", "neighbours"])
def test_channels_that_are_not_rotated_and_positions_without_a_row(rope):
    """An infinity meets its pair's channel alone; a position outside the tables shows in its rotated channels alone."""
    x = torch.randn(1, 2, 5, 64, device="cuda", dtype=BF)
    x[0, 0, 1, 50] = float("inf")
    x[0, 1, 2, 3] = float("inf")
    cos, sin = (t.cuda() for t in tables(5, 32))
    positions = torch.tensor([[0, 1, 2, 5, -1]], dtype=torch.int32, device="cuda")
    y = torch.empty_like(x)
    da.distr_attn_qk_norm_rope(x, None, y, None, da.make_qk_params(x, None, y, None, rope=rope, cos=cos, sin=sin, positions=positions))
    odd = ~y.isfinite().cpu()
    want = torch.zeros_like(odd)
    want[0, 0, 1, 50] = True
    a, b = pair_places(rope, 32)
    mate = {int(i): int(j) for i, j in zip(torch.cat((a, b)), torch.cat((b, a)))}[3]
    want[0, 1, 2, 3] = want[0, 1, 2, mate] = True
    want[0, :, 3:, :32] = True
    assert torch.equal(odd, want)
    assert torch.equal(y[..., 32:], x[..., 32:])


def test_captured_backward_is_the_eager_one():
    case = (BF, 2, 8, 2, 257, 128, "part", "heads", "halves", 128, True, "f32", False)
    t = _make(case)
    ws = torch.empty(max(256, da.distr_attn_qk_bwd_workspace_bytes(t["params"])), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        p = da.make_qk_params(t["q"], t["k"], t["q_out"], t["k_out"], norm=True, eps=EPS, q_weight=t["wq"], k_weight=t["wk"], rope="halves", cos=t["cos"].cuda(),
                              sin=t["sin"].cuda(), workspace=ws)

        def both():
            da.distr_attn_qk_norm_rope(t["q"], t["k"], t["q_out"], t["k_out"], p)
            da.distr_attn_qk_norm_rope_bwd(t["q"], t["k"], t["gq"], t["gk"], t["dq"], t["dk"], p, dq_weight=t["dwq"], dk_weight=t["dwk"])
            return [t[x].clone() for x in ("q_out", "k_out", "dq", "dk", "dwq", "dwk")]
        graph = torch.cuda.CUDAGraph()
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            captured = both()
        for i in range(4):
            t["q"].mul_(0.5)
            t["gk"].add_(1.0)
            graph.replay()
            for a, b in zip(captured, both()):
                assert torch.equal(a, b), i


def test_binding_refusals():
    x = torch.randn(1, 2, 5, 64, device="cuda", dtype=BF)
    cos, sin = (t.cuda() for t in tables(5, 64))
    y = torch.empty_like(x)
    bad = [dict(q_weight=torch.ones(64, device="cuda")), dict(norm=True, q_weight=torch.ones(3, 64, device="cuda")), dict(norm=True, q_weight=torch.ones(64)),
           dict(rope="halves"), dict(rope="halves", cos=cos, sin=sin[:, :8]), dict(rope="halves", cos=cos.double(), sin=sin), dict(rope="spiral", cos=cos, sin=sin),
           dict(rope="halves", cos=cos, sin=sin, positions=torch.zeros(1, 5, device="cuda", dtype=torch.int64)),
           dict(rope="halves", cos=cos, sin=sin, positions=torch.zeros(1, 4, device="cuda", dtype=torch.int32))]
    for kw in bad:
        with pytest.raises(ValueError):
            da.make_qk_params(x, None, y, None, **kw)
    for args in ((x, x, y, None), (x, None, y[:, :1], None), (x, x[:, :, :4], y, y[:, :, :4]), (x.transpose(2, 3), None, y.transpose(2, 3), None), (x[0], None, y[0], None)):
        with pytest.raises(ValueError):
            da.make_qk_params(*args)
    with pytest.raises(TypeError):
        da.make_qk_params(x, None, y.float(), None)
    p = da.make_qk_params(x, None, y, None, norm=True)
    for args in ((x, x, y, y), (x[:, :, :4], None, y, None), (x, None, y.transpose(1, 2).contiguous().transpose(1, 2), None), (x.float(), None, y, None)):
        with pytest.raises(ValueError):
            da.distr_attn_qk_norm_rope(*args, p)
    with pytest.raises(ValueError):
        da.distr_attn_qk_norm_rope_bwd(x, None, y, None, torch.empty_like(x), None, p, dq_weight=torch.zeros(2, 64, device="cuda"))
    with pytest.raises(ValueError):
        da.distr_attn_qk_norm_rope_bwd(x, None, y, None, torch.empty_like(x), None, p, dk_weight=torch.zeros(64, device="cuda"))
    torch.cuda.synchronize()
