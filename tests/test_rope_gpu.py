"""attn_qk_norm_rope, its gradient and attn_paged_append against plain 64-bit implementations.

Tolerances (u = 2^-24, the unit of fp32; e = eps/2 of the 16-bit type, one rounding on output):
  forward   |err| <= e |y| + 2^-20 (|n_a| + |n_b|): the sum of D squares carries at most 16 u, rsqrt and the products a
            few u each, the turn two products and a sum of the pair: below 2^-20 of the pair's size.
  gradient  the same with the size of its two terms, r |g w| and |x| r^3 mean |g w x|, and 2^-18 for the second sum.
  weights   fp32 sums in a fixed order: a lane adds fewer than 256 values in a row, the rest are trees: 2^-16 sum |g x r|.
Subnormal fp16 results add half of the smallest step, 2^-25.
"""
import pytest
import torch

from paper_2506_12355_b200 import api

pytestmark = pytest.mark.gpu

DT = {"fp16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6


def half_step(dt):
    return torch.finfo(dt).eps / 2


def table(n, R, theta=10000.0):
    f = theta ** (-torch.arange(0, R, 2, dtype=torch.float64) / max(R, 1))
    a = torch.arange(n, dtype=torch.float64)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def pairs(R, inter):
    i = torch.arange(R // 2)
    return (2 * i, 2 * i + 1) if inter else (i, i + R // 2)


def turn(x, tab, R, inter, back=False):
    """x [..., D]; tab [..., R] (cosines, sines of that row)."""
    a, b = pairs(R, inter)
    c, s = tab[..., :R // 2], tab[..., R // 2:]
    s = -s if back else s
    y = x.clone()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def rows64(x, w, tab, R, inter):
    """(y, |n_a| + |n_b|) of rows x [..., D] in 64 bits."""
    x = x.double()
    n = x if w is None else x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * w.double()
    if R == 0:
        return n, n.abs()
    tab = tab.double()
    size = n.abs().clone()
    a, b = pairs(R, inter)
    size[..., a] = n[..., a].abs() + n[..., b].abs()
    size[..., b] = size[..., a]
    return turn(n, tab, R, inter), size


def check_rows(got, want, size, dt, name):
    tol = half_step(dt) * want.abs() + 2.0 ** -20 * size + (2.0 ** -25 if dt == torch.float16 else 0.0)
    bad = (got.double() - want).abs() - tol
    assert not torch.isnan(got).any(), name
    assert bad.max() <= 0, "%s: over the tolerance by %g" % (name, bad.max())


def make(B, S, H, Hkv, D, dt, seed, wdt=None):
    g = torch.Generator().manual_seed(seed)
    qkv = (torch.randn(B, S, H + 2 * Hkv, D, generator=g) * 1.5).to(dt).cuda()
    qw = (1 + 0.2 * torch.randn(D, generator=g)).to(wdt or dt).cuda()
    kw = (1 + 0.2 * torch.randn(D, generator=g)).to(wdt or dt).cuda()
    return qkv[:, :, :H], qkv[:, :, H:H + Hkv], qkv[:, :, H + Hkv:], qw, kw


CASES = [
    # B, S, H, Hkv, D, R, interleaved, type
    (1, 1, 1, 1, 64, 64, False, "fp16"),
    (1, 1, 5, 1, 128, 128, True, "bf16"),
    (2, 37, 4, 2, 64, 32, True, "fp16"),
    (3, 129, 9, 3, 128, 64, False, "bf16"),
    (1, 300, 3, 3, 256, 256, False, "fp16"),
    (2, 65, 17, 1, 256, 16, True, "bf16"),
    (2, 33, 2, 4, 64, 0, False, "bf16"),       # more key heads than query heads, no rotation
    (1, 1000, 33, 8, 128, 128, False, "fp16"),
]


@pytest.mark.parametrize("B,S,H,Hkv,D,R,inter,kind", CASES)
def test_forward(B, S, H, Hkv, D, R, inter, kind):
    dt = DT[kind]
    q, k, v, qw, kw = make(B, S, H, Hkv, D, dt, 1)
    tab = table(S, R) if R else None
    qo, ko, vo = api.attn_qk_norm_rope(q, k, v, qw, kw, tab.cuda() if R else None, eps=EPS, interleaved=inter)
    row = tab[None, :, None] if R else None
    for got, x, w, name in ((qo, q, qw, "q"), (ko, k, kw, "k")):
        want, size = rows64(x.cpu(), w.cpu(), row, R, inter)
        check_rows(got.cpu().transpose(1, 2), want, size, dt, name)
    assert torch.equal(vo.transpose(1, 2), v)
    assert qo.is_contiguous() and api.attn_last_device_status() == 0


@pytest.mark.parametrize("qn,kn", [(True, False), (False, True), (False, False)])
def test_forward_without_norm_fp32_weights_positions(qn, kn):
    B, S, H, Hkv, D, R = 2, 50, 4, 2, 128, 64
    q, k, v, qw, kw = make(B, S, H, Hkv, D, torch.bfloat16, 2, torch.float32)
    qw, kw = qw if qn else None, kw if kn else None
    tab = table(5000, R)
    pos = torch.randint(0, 5000, (B, S), generator=torch.Generator().manual_seed(5), dtype=torch.int32)
    pos[0, 0], pos[1, 3] = 4999, 0
    qo, ko, vo = api.attn_qk_norm_rope(q, k, None, qw, kw, tab.cuda(), pos.cuda(), eps=EPS)
    assert vo is None
    row = tab[pos.long()][:, :, None]
    for got, x, w in ((qo, q, qw), (ko, k, kw)):
        want, size = rows64(x.cpu(), None if w is None else w.cpu(), row, R, False)
        check_rows(got.cpu().transpose(1, 2), want, size, torch.bfloat16, "rows")


def test_broadcast_and_zero_rows():
    # stride 0 over the batch, an all-zero head, and eps that keeps it finite
    D, dt = 64, torch.float16
    q, k, v, qw, kw = make(1, 20, 2, 2, D, dt, 3)
    q = q.clone()
    q[:, 4] = 0
    q, k = q.expand(3, -1, -1, -1), k.expand(3, -1, -1, -1)
    tab = table(20, D)
    qo, ko, _ = api.attn_qk_norm_rope(q, k, None, qw, kw, tab.cuda(), eps=EPS)
    want, size = rows64(q.cpu(), qw.cpu(), tab[None, :, None], D, False)
    check_rows(qo.cpu().transpose(1, 2), want, size, dt, "q")
    assert (qo[:, :, 4] == 0).all() and torch.equal(qo[0], qo[2])


def test_position_out_of_range_is_reported_and_read_nowhere():
    q, k, v, qw, kw = make(1, 8, 2, 1, 64, torch.float16, 4)
    pos = torch.tensor([[0, 1, 2, 16, 3, -1, 4, 2 ** 31 - 1]], dtype=torch.int32).cuda()
    qo, ko, vo = api.attn_qk_norm_rope(q, k, v, qw, kw, table(16, 64).cuda(), pos)
    assert api.attn_last_device_status() == 13 and api.attn_status_string(13) == "ATTN_ERR_DEVICE_INDEX"
    assert api.attn_last_device_status() == 0
    bad = torch.tensor([3, 5, 7]).cuda()
    good = torch.tensor([0, 1, 2, 4, 6]).cuda()
    for x in (qo, ko):
        assert torch.isnan(x[:, :, bad]).all() and not torch.isnan(x[:, :, good]).any()
    assert torch.equal(vo.transpose(1, 2), v)


def grad64(g, x, w, tab, R, inter):
    """(dx, its size, terms of dw) for g [B,S,h,D] in 64 bits."""
    g, x = g.double(), x.double()
    h = turn(g, tab.double(), R, inter, back=True) if R else g
    hsize = g.abs().clone()
    if R:
        a, b = pairs(R, inter)
        hsize[..., a] = g[..., a].abs() + g[..., b].abs()
        hsize[..., b] = hsize[..., a]
    if w is None:
        return h, hsize, None, None
    w = w.double()
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    dx = r * h * w - x * r ** 3 * (h * w * x).mean(-1, keepdim=True)
    size = r * hsize * w.abs() + x.abs() * r ** 3 * (hsize * w.abs() * x.abs()).mean(-1, keepdim=True)
    return dx, size, h * x * r, hsize * x.abs() * r


@pytest.mark.parametrize("B,S,H,Hkv,D,R,inter,kind", CASES)
def test_gradient(B, S, H, Hkv, D, R, inter, kind):
    dt = DT[kind]
    q, k, v, qw, kw = make(B, S, H, Hkv, D, dt, 6)
    g = torch.Generator().manual_seed(7)
    dq, dk, dv = (torch.randn(B, h, S, D, generator=g).to(dt).cuda() for h in (H, Hkv, Hkv))
    tab = table(S, R) if R else None
    # gradients go into one buffer laid out like the projection
    buf = torch.full((B, S, H + 2 * Hkv, D), float("nan"), dtype=dt, device="cuda")
    outs = buf[:, :, :H], buf[:, :, H:H + Hkv], buf[:, :, H + Hkv:]
    res = api.attn_qk_norm_rope_bwd(dq, dk, dv, q, k, qw, kw, tab.cuda() if R else None, eps=EPS, interleaved=inter,
                                    dq_in=outs[0], dk_in=outs[1], dv_in=outs[2])
    row = tab[None, :, None] if R else None
    for got, gw, dy, x, w in ((outs[0], res[3], dq, q, qw), (outs[1], res[4], dk, k, kw)):
        want, size, dw, dwsize = grad64(dy.cpu().transpose(1, 2), x.cpu(), w.cpu(), row, R, inter)
        err = (got.cpu().double() - want).abs()
        tol = half_step(dt) * want.abs() + 2.0 ** -18 * size + (2.0 ** -25 if dt == torch.float16 else 0.0)
        assert (err <= tol).all(), "over by %g" % (err - tol).max()
        werr = (gw.cpu().double() - dw.sum((0, 1, 2))).abs()
        assert (werr <= 2.0 ** -16 * dwsize.sum((0, 1, 2))).all()
    assert torch.equal(outs[2], dv.transpose(1, 2))
    again = api.attn_qk_norm_rope_bwd(dq, dk, dv, q, k, qw, kw, tab.cuda() if R else None, eps=EPS, interleaved=inter)
    assert all(torch.equal(a, b) for a, b in zip(res, again))     # the sums' order is fixed


LONG_CASES = [
    # more than two laps of the gradient kernel's ring of 6 stages per CTA (148 of them), with a last block that is not full
    (2, 2050, 32, 8, 128, 128, False, "bf16", False),      # 8 x 8 tiles of all tensors: 20 per CTA
    (1, 4099, 12, 3, 256, 128, True, "fp16", True),        # heads that do not fill a tile: 17
    (3, 16395, 2, 2, 64, 64, False, "fp16", False),        # tiles of 64 tokens: 15
    (3, 3001, 32, 1, 64, 32, True, "bf16", True),          # q in tiles of 8 tokens, k and v of 128, by turns: 16
    (2, 5003, 1, 9, 128, 64, False, "fp16", True),         # the other way round
]


@pytest.mark.parametrize("B,S,H,Hkv,D,R,inter,kind,given", LONG_CASES)
def test_gradient_of_many_tiles(B, S, H, Hkv, D, R, inter, kind, given):
    """Every stage of the ring is filled, worked on, stored and handed back several times; the walk crosses blocks, tensors and
    sequences.  Tolerances as for the small cases: a lane adds fewer than 256 terms of a weight's sum here as well."""
    dt = DT[kind]
    q, k, v, qw, kw = make(B, S, H, Hkv, D, dt, 16)
    g = torch.Generator().manual_seed(17)
    dq, dk, dv = (torch.randn(B, h, S, D, generator=g).to(dt).cuda() for h in (H, Hkv, Hkv))
    tab = table(S, R).cuda()
    pos = torch.randint(0, S, (B, S), generator=g, dtype=torch.int32).cuda() if given else None
    buf = torch.full((B, S, H + 2 * Hkv, D), float("nan"), dtype=dt, device="cuda")
    outs = buf[:, :, :H], buf[:, :, H:H + Hkv], buf[:, :, H + Hkv:]
    ws = torch.full((api.attn_qk_norm_rope_bwd_workspace_bytes(D),), 255, dtype=torch.uint8, device="cuda")
    res = api.attn_qk_norm_rope_bwd(dq, dk, dv, q, k, qw, kw, tab, pos, eps=EPS, interleaved=inter, dq_in=outs[0], dk_in=outs[1], dv_in=outs[2],
                                    workspace=ws)
    assert api.attn_last_device_status() == 0
    row = tab[pos.long()][:, :, None] if given else tab[None, :, None]
    for got, gw, dy, x, w in ((outs[0], res[3], dq, q, qw), (outs[1], res[4], dk, k, kw)):
        want, size, dw, dwsize = grad64(dy.transpose(1, 2), x, w, row, R, inter)
        err = (got.double() - want).abs()
        tol = half_step(dt) * want.abs() + 2.0 ** -18 * size + (2.0 ** -25 if dt == torch.float16 else 0.0)
        assert (err <= tol).all(), "over by %g" % (err - tol).max()
        werr = (gw.double() - dw.sum((0, 1, 2))).abs()
        assert (werr <= 2.0 ** -16 * dwsize.sum((0, 1, 2))).all()
    assert torch.equal(outs[2], dv.transpose(1, 2))
    again = api.attn_qk_norm_rope_bwd(dq, dk, dv, q, k, qw, kw, tab, pos, eps=EPS, interleaved=inter)
    assert all(torch.equal(a, b) for a, b in zip(res, again))


def test_forward_of_many_tokens():
    dt, B, S, H, Hkv, D = torch.bfloat16, 2, 3001, 16, 4, 128
    q, k, v, qw, kw = make(B, S, H, Hkv, D, dt, 18)
    tab = table(S, D).cuda()
    qo, ko, vo = api.attn_qk_norm_rope(q, k, v, qw, kw, tab, eps=EPS)
    for got, x, w in ((qo, q, qw), (ko, k, kw)):
        want, size = rows64(x, w, tab[None, :, None], D, False)
        check_rows(got.transpose(1, 2), want, size, dt, "rows")
    assert torch.equal(vo.transpose(1, 2), v)


def test_other_input_layouts():
    """Head-major inputs, and rows with room between them."""
    D, R, dt = 128, 64, torch.float16
    g = torch.Generator().manual_seed(15)
    q = torch.randn(2, 5, 40, D, generator=g).to(dt).cuda().transpose(1, 2)                  # [B,S,H,D] over [B,H,S,D]
    k = torch.randn(2, 40, 3, D + 24, generator=g).to(dt).cuda()[..., 8:8 + D]
    qw, kw = (1 + 0.2 * torch.randn(2, D, generator=g)).to(dt).cuda()
    tab = table(40, R)
    qo, ko, _ = api.attn_qk_norm_rope(q, k, None, qw, kw, tab.cuda(), eps=EPS)
    dq, dk = torch.randn(2, 5, 40, D, generator=g).to(dt).cuda(), torch.randn(2, 3, 40, D, generator=g).to(dt).cuda()
    di = torch.empty(2, 5, 40, D, dtype=dt, device="cuda").transpose(1, 2)
    res = api.attn_qk_norm_rope_bwd(dq, dk, None, q, k, qw, kw, tab.cuda(), eps=EPS, dq_in=di)
    for out, x, w, got, dy in ((qo, q, qw, di, dq), (ko, k, kw, res[1], dk)):
        want, size = rows64(x.cpu(), w.cpu(), tab[None, :, None], R, False)
        check_rows(out.cpu().transpose(1, 2), want, size, dt, "rows")
        want, size, _, _ = grad64(dy.cpu().transpose(1, 2), x.cpu(), w.cpu(), tab[None, :, None], R, False)
        assert ((got.cpu().double() - want).abs() <= half_step(dt) * want.abs() + 2.0 ** -18 * size + 2.0 ** -25).all()


def test_gradient_against_differences():
    # central differences of sum(y * g) in 64 bits, at points of the 16-bit grid, against the kernel's gradient
    D, R = 64, 32
    q, k, v, qw, kw = make(1, 3, 2, 1, D, torch.float16, 8, torch.float32)
    tab = table(3, R)
    g = torch.randn(1, 2, 3, D, generator=torch.Generator().manual_seed(9)).half()
    res = api.attn_qk_norm_rope_bwd(g.cuda(), torch.zeros(1, 1, 3, D, dtype=torch.float16, device="cuda"), None, q, k, qw, kw, tab.cuda(), eps=EPS)
    x, w = q.cpu().double(), qw.cpu().double()

    def f(x, w):
        n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * w
        return (turn(n, tab.double()[None, :, None], R, False) * g.double().transpose(1, 2)).sum()
    h = 1e-5
    for (s, hd, d) in [(0, 0, 0), (1, 1, 15), (2, 0, 16), (2, 1, 31), (1, 0, 40), (0, 1, 63)]:
        e = torch.zeros_like(x)
        e[0, s, hd, d] = h
        want = (f(x + e, w) - f(x - e, w)) / (2 * h)
        assert abs(float(res[0][0, s, hd, d]) - float(want)) <= half_step(torch.float16) * abs(float(want)) + 1e-5
    for d in (0, 17, 63):
        e = torch.zeros_like(w)
        e[d] = h
        want = (f(x, w + e) - f(x, w - e)) / (2 * h)
        assert abs(float(res[3][d]) - float(want)) <= 1e-4 * max(1.0, abs(float(want)))


def test_gradient_without_weights_and_empty():
    D = 64
    q, k, v, qw, kw = make(2, 9, 2, 2, D, torch.bfloat16, 10)
    g = torch.randn(2, 2, 9, D, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    tab = table(9, D)
    a = api.attn_qk_norm_rope_bwd(g, g, None, q, k, None, kw, tab.cuda())
    assert a[3] is None and a[2] is None and a[4] is not None
    want, size, _, _ = grad64(g.cpu().transpose(1, 2), q.cpu(), None, tab[None, :, None], D, False)
    check_rows(a[0].cpu(), want, size, torch.bfloat16, "dq")
    e = torch.empty(0, 9, 2, D, dtype=torch.bfloat16, device="cuda")
    ge = torch.empty(0, 2, 9, D, dtype=torch.bfloat16, device="cuda")
    r = api.attn_qk_norm_rope_bwd(ge, ge, ge, e, e, qw, kw, tab.cuda())
    assert (r[3] == 0).all() and (r[4] == 0).all()


def test_gradient_of_broadcast_inputs_and_bad_positions():
    # inputs that stand for every sequence (stride 0), as a tensor map cannot describe them
    D, B, S, R = 128, 3, 21, 64
    q, k, _, qw, kw = make(1, S, 4, 2, D, torch.bfloat16, 12)
    q, k = q.expand(B, -1, -1, -1), k.expand(B, -1, -1, -1)
    g = torch.Generator().manual_seed(13)
    dq, dk = (torch.randn(B, h, S, D, generator=g).bfloat16().cuda() for h in (4, 2))
    tab = table(S, R)
    res = api.attn_qk_norm_rope_bwd(dq, dk, None, q, k, qw, kw, tab.cuda(), eps=EPS)
    for got, gw, dy, x, w in ((res[0], res[3], dq, q, qw), (res[1], res[4], dk, k, kw)):
        want, size, dw, dwsize = grad64(dy.cpu().transpose(1, 2), x.cpu(), w.cpu(), tab[None, :, None], R, False)
        assert ((got.cpu().double() - want).abs() <= half_step(torch.bfloat16) * want.abs() + 2.0 ** -18 * size).all()
        assert ((gw.cpu().double() - dw.sum((0, 1, 2))).abs() <= 2.0 ** -16 * dwsize.sum((0, 1, 2))).all()
    # contiguous ones give the same rows on the other path
    same = api.attn_qk_norm_rope_bwd(dq, dk, None, q.contiguous(), k.contiguous(), qw, kw, tab.cuda(), eps=EPS)
    assert (same[0].float() - res[0].float()).abs().max() <= 2 * half_step(torch.bfloat16) * res[0].float().abs().max()
    for x, y in ((q, k), (q.contiguous(), k.contiguous())):
        pos = torch.arange(S, dtype=torch.int32).repeat(B, 1)
        pos[1, 5], pos[2, 0] = S, -3
        r = api.attn_qk_norm_rope_bwd(dq, dk, None, x, y, qw, kw, tab.cuda(), pos.cuda(), eps=EPS)
        assert api.attn_last_device_status() == 13 and api.attn_last_device_status() == 0
        bad = torch.zeros(B, S, dtype=torch.bool)
        bad[1, 5] = bad[2, 0] = True
        for t in r[:2]:
            nan = torch.isnan(t).flatten(2).cpu()
            assert nan[bad][:, :].any(-1).all() and not nan[~bad].any()
        assert torch.isnan(r[3]).any() and torch.isnan(r[4]).any()


def test_graph_replay_and_second_stream():
    D = 128
    q, k, v, qw, kw = make(1, 70, 4, 2, D, torch.bfloat16, 11)
    tab = table(70, D).cuda()
    want = api.attn_qk_norm_rope(q, k, v, qw, kw, tab)
    g = [torch.randn_like(t) for t in want]
    want_b = api.attn_qk_norm_rope_bwd(*g, q, k, qw, kw, tab)
    ws = torch.empty(api.attn_qk_norm_rope_bwd_workspace_bytes(D), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = api.attn_qk_norm_rope(q, k, v, qw, kw, tab)
        got_b = api.attn_qk_norm_rope_bwd(*g, q, k, qw, kw, tab, workspace=ws)
    for _ in range(3):
        for t in got + got_b:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got + got_b, want + want_b))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = api.attn_qk_norm_rope(q, k, v, qw, kw, tab, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_flag_without_a_truth_value_is_refused():
    q, k, v, qw, kw = make(1, 8, 2, 1, 64, torch.float16, 25)
    tab = table(8, 64).cuda()
    for bad in (torch.tensor([True, False]), torch.zeros(0, 2, dtype=torch.bool)):
        with pytest.raises(RuntimeError):
            api.attn_qk_norm_rope(q, k, v, qw, kw, tab, interleaved=bad)
