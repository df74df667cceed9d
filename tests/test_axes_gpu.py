"""attn_qk_norm_rope_axes, its gradient and attn_paged_append_axes against plain 64-bit implementations; tolerances and helpers are
those of the calls with one axis (test_rope_gpu.py): the arithmetic behind the choice of a pair's position is the same."""
import pytest
import torch

from paper_2506_12355_b200 import api
from test_rope_gpu import DT, EPS, check_rows, grad64, half_step, make, rows64, table

pytestmark = pytest.mark.gpu


def draw_positions(axes, B, S, n, seed):
    pos = torch.randint(0, n, (axes, B, S), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)
    pos[0, 0, 0], pos[-1, -1, -1] = n - 1, 0
    return pos


def rows_of(tab, pos, of):
    """The table row [.., R] that each token turns by: column i from the position on its pair's axis."""
    half, at = tab.shape[1] // 2, pos.long().movedim(0, -1)[..., torch.tensor(list(of))]
    col = torch.arange(half)
    return torch.cat([tab[at, col], tab[at, half + col]], -1)


CASES = [
    # B, S, H, Hkv, D, R, interleaved, type, pairs of each axis, order
    (1, 1, 1, 1, 64, 64, False, "fp16", (32,), "blocks"),
    (1, 1, 5, 1, 128, 128, True, "bf16", (16, 24, 24), "blocks"),
    (2, 37, 4, 2, 64, 32, True, "fp16", (8, 8), "cyclic"),
    (3, 129, 9, 3, 128, 64, False, "bf16", (11, 11, 10), "blocks"),          # runs that end inside a lane's four pairs
    (1, 300, 3, 3, 256, 256, False, "fp16", (32, 32, 32, 32), "cyclic"),
    (2, 65, 17, 1, 256, 16, True, "bf16", (0, 1, 7), "cyclic"),              # an axis that no pair belongs to
    (1, 1000, 33, 8, 128, 128, False, "fp16", (24, 20, 20), "cyclic"),
    (2, 33, 2, 4, 64, 0, False, "bf16", (0, 0), "blocks"),                   # no rotation
]


@pytest.mark.parametrize("B,S,H,Hkv,D,R,inter,kind,sections,order", CASES)
def test_forward(B, S, H, Hkv, D, R, inter, kind, sections, order):
    dt, of = DT[kind], api.rope_pair_axes(sections, order)
    q, k, v, qw, kw = make(B, S, H, Hkv, D, dt, 21)
    tab = table(700, R) if R else None
    pos = draw_positions(len(sections), B, S, 700, 22)
    qo, ko, vo = api.attn_qk_norm_rope_axes(q, k, v, qw, kw, tab.cuda() if R else None, pos.cuda(), of, eps=EPS, interleaved=inter)
    row = rows_of(tab, pos, of)[:, :, None] if R else None
    for got, x, w, name in ((qo, q, qw, "q"), (ko, k, kw, "k")):
        want, size = rows64(x.cpu(), w.cpu(), row, R, inter)
        check_rows(got.cpu().transpose(1, 2), want, size, dt, name)
    assert torch.equal(vo.transpose(1, 2), v) and api.attn_last_device_status() == 0


@pytest.mark.parametrize("B,S,H,Hkv,D,R,inter,kind,sections,order", CASES + [
    # more than two laps of the gradient's ring: 8 x 8 tiles, tiles of more tokens (PACKED), and both by turns
    (2, 2050, 32, 8, 128, 128, False, "bf16", (16, 24, 24), "cyclic"),
    (3, 16395, 2, 2, 64, 64, False, "fp16", (12, 10, 10), "blocks"),
    (3, 3001, 32, 1, 64, 32, True, "bf16", (8, 8), "blocks"),
])
def test_gradient(B, S, H, Hkv, D, R, inter, kind, sections, order):
    dt, of = DT[kind], api.rope_pair_axes(sections, order)
    q, k, v, qw, kw = make(B, S, H, Hkv, D, dt, 23)
    g = torch.Generator().manual_seed(24)
    dq, dk, dv = (torch.randn(B, h, S, D, generator=g).to(dt).cuda() for h in (H, Hkv, Hkv))
    tab = table(700, R) if R else None
    pos = draw_positions(len(sections), B, S, 700, 25)
    buf = torch.full((B, S, H + 2 * Hkv, D), float("nan"), dtype=dt, device="cuda")
    outs = buf[:, :, :H], buf[:, :, H:H + Hkv], buf[:, :, H + Hkv:]
    res = api.attn_qk_norm_rope_axes_bwd(dq, dk, dv, q, k, qw, kw, tab.cuda() if R else None, pos.cuda(), of, eps=EPS, interleaved=inter,
                                         dq_in=outs[0], dk_in=outs[1], dv_in=outs[2])
    row = rows_of(tab, pos, of)[:, :, None] if R else None
    for got, gw, dy, x, w in ((outs[0], res[3], dq, q, qw), (outs[1], res[4], dk, k, kw)):
        want, size, dw, dwsize = grad64(dy.cpu().transpose(1, 2), x.cpu(), w.cpu(), row, R, inter)
        err = (got.cpu().double() - want).abs()
        tol = half_step(dt) * want.abs() + 2.0 ** -18 * size + (2.0 ** -25 if dt == torch.float16 else 0.0)
        assert (err <= tol).all(), "over by %g" % (err - tol).max()
        assert ((gw.cpu().double() - dw.sum((0, 1, 2))).abs() <= 2.0 ** -16 * dwsize.sum((0, 1, 2))).all()
    assert torch.equal(outs[2], dv.transpose(1, 2))
    again = api.attn_qk_norm_rope_axes_bwd(dq, dk, dv, q, k, qw, kw, tab.cuda() if R else None, pos.cuda(), of, eps=EPS, interleaved=inter)
    assert all(torch.equal(a, b) for a, b in zip(res, again))


def test_gradient_of_a_broadcast_input_takes_the_register_form():
    B, S, H, Hkv, D, of = 3, 40, 4, 2, 64, api.rope_pair_axes((12, 10, 10), "cyclic")
    q, k, v, qw, kw = make(1, S, H, Hkv, D, torch.bfloat16, 26)
    g = torch.Generator().manual_seed(27)
    dq, dk, dv = (torch.randn(B, h, S, D, generator=g).bfloat16().cuda() for h in (H, Hkv, Hkv))
    tab, pos = table(90, D).cuda(), draw_positions(3, B, S, 90, 28).cuda()
    wide = [x.expand(B, -1, -1, -1) for x in (q, k)]
    a = api.attn_qk_norm_rope_axes_bwd(dq, dk, dv, *wide, qw, kw, tab, pos, of)
    b = api.attn_qk_norm_rope_axes_bwd(dq, dk, dv, *(x.contiguous() for x in wide), qw, kw, tab, pos, of)
    for x, y in zip(a[:3], b[:3]):     # the same arithmetic per row
        assert (x.double() - y.double()).abs().max() <= torch.finfo(torch.bfloat16).eps * y.double().abs().max()
    for x, y in zip(a[3:], b[3:]):
        assert (x - y).abs().max() <= 2.0 ** -14 * y.abs().max()


def test_one_axis_is_the_plain_call_and_equal_positions_too():
    q, k, v, qw, kw = make(2, 70, 6, 2, 128, torch.bfloat16, 29)
    tab = table(70, 64).cuda()
    plain = api.attn_qk_norm_rope(q, k, v, qw, kw, tab)
    pos = torch.arange(70, dtype=torch.int32).cuda().expand(3, 2, 70).contiguous()
    for n, of in ((1, bytes(32)), (3, api.rope_pair_axes((12, 10, 10), "cyclic")), (3, [0] * 20 + [2] * 12)):
        got = api.attn_qk_norm_rope_axes(q, k, v, qw, kw, tab, pos[:n].contiguous(), of)
        assert all(torch.equal(a, b) for a, b in zip(got, plain))


@pytest.mark.parametrize("sections,order", [((16, 8, 8), "blocks"), ((12, 10, 10), "cyclic")])
def test_position_out_of_range_is_reported_and_read_nowhere(sections, order):
    q, k, v, qw, kw = make(1, 8, 2, 1, 64, torch.float16, 30)
    pos = torch.zeros(3, 1, 8, dtype=torch.int32)
    pos[0, 0, 3], pos[1, 0, 5], pos[2, 0, 7] = 16, -1, 2 ** 31 - 1
    pos, of = pos.cuda(), api.rope_pair_axes(sections, order)
    qo, ko, vo = api.attn_qk_norm_rope_axes(q, k, v, qw, kw, table(16, 64).cuda(), pos, of)
    assert api.attn_last_device_status() == 13 and api.attn_last_device_status() == 0
    bad, good = torch.tensor([3, 5, 7]).cuda(), torch.tensor([0, 1, 2, 4, 6]).cuda()
    for x in (qo, ko):
        assert torch.isnan(x[:, :, bad]).all() and not torch.isnan(x[:, :, good]).any()
    assert torch.equal(vo.transpose(1, 2), v)
    dq, dk, dv = (torch.ones_like(x) for x in (qo, ko, vo))
    dqi, dki, dvi, dqw, dkw = api.attn_qk_norm_rope_axes_bwd(dq, dk, dv, q, k, qw, kw, table(16, 64).cuda(), pos, of)
    assert api.attn_last_device_status() == 13
    for x in (dqi, dki):
        assert torch.isnan(x[:, bad]).all() and not torch.isnan(x[:, good]).any()
    assert torch.isnan(dqw).all() and not torch.isnan(dvi).any()


@pytest.mark.parametrize("new,page,layout,inter", [(1, 16, "head", False), (0, 8, "slot", True), (0, 64, "head", False)])
def test_append(new, page, layout, inter):
    H, Hkv, D, R, dt = 6, 2, 128, 64, torch.float16
    sections, order = (12, 10, 10), "cyclic"
    of = api.rope_pair_axes(sections, order)
    lens = [5, 0, 33, 64, 1, 17]
    news = [min(n, 1) for n in lens] if new else [min(n, m) for n, m in zip(lens, (5, 0, 9, 64, 1, 16))]
    T = len(lens) if new else sum(news) + 7                 # padding behind the last one
    g = torch.Generator().manual_seed(31)
    qkv = (torch.randn(T, H + 2 * Hkv, D, generator=g) * 1.5).to(dt).cuda()
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    qw, kw = ((1 + 0.2 * torch.randn(D, generator=g)).to(dt).cuda() for _ in range(2))
    per = -(-max(lens) // page)
    bt = torch.randperm(len(lens) * per, generator=g).to(torch.int32).view(len(lens), per).cuda()
    shape = (len(lens) * per, Hkv, page, D) if layout == "head" else (len(lens) * per, page, Hkv, D)
    kc, vc = (torch.zeros(shape, dtype=dt, device="cuda") for _ in range(2))
    if layout == "slot":
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    tab, pos = table(700, R), torch.randint(0, 700, (3, T), generator=g, dtype=torch.int32)
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    cu = None if new else torch.tensor(starts, dtype=torch.int32).cuda()
    if not new:
        pos[:, starts[-1]:] = 2 ** 30                       # of padding: not looked at
    qo = torch.full((T, H, D), 7.0, dtype=dt, device="cuda")
    api.attn_paged_append_axes(q, k, v, kc, vc, bt, torch.tensor(lens, dtype=torch.int32).cuda(), pos.cuda(), of, qw, kw, tab.cuda(), cu, EPS, inter, qo)
    assert api.attn_last_device_status() == 0
    t_of, where = [], []
    for b, (n, m) in enumerate(zip(lens, news)):
        for i in range(m):
            t_of.append(b if new else starts[b] + i)
            where.append((int(bt[b, (n - m + i) // page]), (n - m + i) % page))
    t = torch.tensor(t_of)
    row = rows_of(tab, pos[:, t], of)[:, None]
    want, size = rows64(q.cpu()[t], qw.cpu(), row, R, inter)
    check_rows(qo.cpu()[t], want, size, dt, "q")
    want, size = rows64(k.cpu()[t], kw.cpu(), row, R, inter)
    pg, sl = (torch.tensor([w[i] for w in where]) for i in range(2))
    check_rows(kc.cpu()[pg, :, sl], want, size, dt, "k")
    assert torch.equal(vc.cpu()[pg, :, sl], v.cpu()[t])
    rest = torch.ones(T, dtype=torch.bool)
    rest[t] = False
    assert (qo.cpu()[rest] == 7).all()
    assert int((vc.cpu().abs().amax((1, 3)) > 0).sum()) == len(t_of)         # nothing else was written


def test_append_skips_tokens_whose_positions_are_out_of_range():
    g = torch.Generator().manual_seed(32)
    q, k, v = ((torch.randn(4, h, 64, generator=g)).half().cuda() for h in (2, 1, 1))
    kc, vc = (torch.zeros(4, 1, 8, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    bt, lens = torch.arange(4, dtype=torch.int32).view(4, 1).cuda(), torch.full((4,), 3, dtype=torch.int32).cuda()
    pos = torch.tensor([[0, 0, 99, 0], [0, -5, 0, 0]], dtype=torch.int32).cuda()
    qo = torch.zeros(4, 2, 64, dtype=torch.float16, device="cuda")
    api.attn_paged_append_axes(q, k, v, kc, vc, bt, lens, pos, api.rope_pair_axes((16, 16)), None, None, table(20, 64).cuda(), q_out=qo)
    assert api.attn_last_device_status() == 13
    for b in range(4):
        written = b in (0, 3)
        assert bool(kc[b, 0, 2].any()) == written and bool(vc[b, 0, 2].any()) == written and bool(qo[b].any()) == written
    assert not kc[:, :, 3:].any() and not kc[:, :, :2].any()


def test_python_path_and_explicit_stream_agree_with_the_extension(monkeypatch):
    q, k, v, qw, kw = make(2, 30, 4, 2, 64, torch.float16, 33)
    tab, pos, of = table(50, 64).cuda(), draw_positions(2, 2, 30, 50, 34).cuda(), [0] * 16 + [1] * 16
    fast = api.attn_qk_norm_rope_axes(q, k, v, qw, kw, tab, pos, bytes(of))
    gr = [torch.randn_like(x) for x in fast]
    fast_bwd = api.attn_qk_norm_rope_axes_bwd(*gr, q, k, qw, kw, tab, pos, bytes(of))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    on_side = api.attn_qk_norm_rope_axes(q, k, v, qw, kw, tab, pos, bytes(of), stream=side)
    side.synchronize()
    monkeypatch.setattr(api, "_fast", lambda *a: NotImplemented)
    slow = api.attn_qk_norm_rope_axes(q, k, v, qw, kw, tab, pos, of)
    slow_bwd = api.attn_qk_norm_rope_axes_bwd(*gr, q, k, qw, kw, tab, pos, of)
    for a, b in list(zip(fast, slow)) + list(zip(fast, on_side)) + list(zip(fast_bwd, slow_bwd)):
        assert torch.equal(a, b)
