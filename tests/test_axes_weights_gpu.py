"""The calls with several position axes with fp32 weights and without normalisation, and their gradient against differences (tolerances
and helpers: test_rope_gpu.py)."""
import pytest
import torch

from paper_2506_12355_b200 import api
from test_axes_gpu import draw_positions, rows_of
from test_rope_gpu import EPS, check_rows, grad64, half_step, make, rows64, table

pytestmark = pytest.mark.gpu

NORMS = pytest.mark.parametrize("qn,kn", [(True, True), (True, False), (False, True), (False, False)])


@NORMS
@pytest.mark.parametrize("D,R,sections,order,inter,dt", [(128, 64, (12, 10, 10), "cyclic", False, torch.bfloat16), (64, 64, (16, 16), "blocks", True, torch.float16)])
def test_forward_and_gradient(qn, kn, D, R, sections, order, inter, dt):
    B, S, H, Hkv = 2, 50, 6, 2
    of = api.rope_pair_axes(sections, order)
    q, k, v, qw, kw = make(B, S, H, Hkv, D, dt, 41, torch.float32)
    qw, kw = qw if qn else None, kw if kn else None
    tab, pos = table(3000, R), draw_positions(len(sections), B, S, 3000, 42)
    row = rows_of(tab, pos, of)[:, :, None]
    cpu = lambda w: None if w is None else w.cpu()
    qo, ko, vo = api.attn_qk_norm_rope_axes(q, k, None, qw, kw, tab.cuda(), pos.cuda(), of, eps=EPS, interleaved=inter)
    assert vo is None
    for got, x, w, name in ((qo, q, qw, "q"), (ko, k, kw, "k")):
        check_rows(got.cpu().transpose(1, 2), *rows64(x.cpu(), cpu(w), row, R, inter), dt, name)
    g = torch.Generator().manual_seed(43)
    dq, dk = (torch.randn(B, h, S, D, generator=g).to(dt).cuda() for h in (H, Hkv))
    res = api.attn_qk_norm_rope_axes_bwd(dq, dk, None, q, k, qw, kw, tab.cuda(), pos.cuda(), of, eps=EPS, interleaved=inter)
    assert res[2] is None and api.attn_last_device_status() == 0
    for got, gw, dy, x, w in ((res[0], res[3], dq, q, qw), (res[1], res[4], dk, k, kw)):
        want, size, dw, dwsize = grad64(dy.cpu().transpose(1, 2), x.cpu(), cpu(w), row, R, inter)
        tol = half_step(dt) * want.abs() + 2.0 ** -18 * size + (2.0 ** -25 if dt == torch.float16 else 0.0)
        assert ((got.cpu().double() - want).abs() <= tol).all()
        assert (gw is None) == (w is None)
        if w is not None:
            assert gw.dtype == torch.float32 and ((gw.cpu().double() - dw.sum((0, 1, 2))).abs() <= 2.0 ** -16 * dwsize.sum((0, 1, 2))).all()


@NORMS
def test_append(qn, kn):
    n, H, Hkv, D, R, page, dt = 9, 6, 2, 128, 64, 8, torch.bfloat16
    of = api.rope_pair_axes((12, 10, 10), "cyclic")
    q, k, v, qw, kw = (x[0] if x.dim() == 4 else x for x in make(1, n, H, Hkv, D, dt, 44, torch.float32))
    qw, kw = qw if qn else None, kw if kn else None
    kc, vc = (torch.zeros(n, Hkv, page, D, dtype=dt, device="cuda") for _ in range(2))
    bt, lens = torch.arange(n, dtype=torch.int32).view(n, 1).cuda(), torch.full((n,), 5, dtype=torch.int32).cuda()
    tab, pos = table(700, R), draw_positions(3, 1, n, 700, 45)[:, 0].contiguous()
    qo = api.attn_paged_append_axes(q, k, v, kc, vc, bt, lens, pos.cuda(), of, qw, kw, tab.cuda(), eps=EPS)
    assert api.attn_last_device_status() == 0
    row = rows_of(tab, pos, of)[:, None]
    for got, x, w, name in ((qo, q, qw, "q"), (kc[:, :, 4], k, kw, "k")):
        check_rows(got.cpu(), *rows64(x.cpu(), None if w is None else w.cpu(), row, R, False), dt, name)
    assert torch.equal(vc[:, :, 4], v)


@pytest.mark.parametrize("sections,order", [((16, 24, 24), "blocks"), ((22, 21, 21), "cyclic")])
def test_gradient_against_differences(sections, order):
    """Central differences of sum_i dy_i y_i(x), in 64 bits, along directions u in the inputs and the weights: (f(x + h u) - f(x - h u)) / 2 h with
    h = 2^-12 is off by h^2 f''' / 6 (below 2^-24 of the terms' size) and 2^-52 |f| / h; the gradient by its roundings, each half a step of
    a term g_i u_i, and 2^-18 of the terms' size as in grad64."""
    B, S, H, Hkv, D, R, dt = 1, 5, 2, 2, 128, 128, torch.float16
    of = api.rope_pair_axes(sections, order)
    q, k, v, qw, kw = make(B, S, H, Hkv, D, dt, 46, torch.float32)
    tab, pos = table(90, R), draw_positions(3, B, S, 90, 47)
    row = rows_of(tab, pos, of)[:, :, None]
    g = torch.Generator().manual_seed(48)
    dq, dk = (torch.randn(B, h, S, D, generator=g).to(dt).cuda() for h in (H, Hkv))
    res = api.attn_qk_norm_rope_axes_bwd(dq, dk, None, q, k, qw, kw, tab.cuda(), pos.cuda(), of, eps=EPS)
    h = 2.0 ** -12
    for got, gw, dy, x, w in ((res[0], res[3], dq, q, qw), (res[1], res[4], dk, k, kw)):
        x, w, dy = x.cpu().double(), w.cpu().double(), dy.cpu().double().transpose(1, 2)
        f = lambda a, b: float((rows64(a, b, row, R, False)[0] * dy).sum())
        _, size, _, dwsize = grad64(dy, x, w, row, R, False)
        for _ in range(3):
            u, uw = torch.randn(x.shape, generator=g, dtype=torch.float64), torch.randn(D, generator=g, dtype=torch.float64)
            got64, gw64 = got.cpu().double(), gw.cpu().double()
            diff = (f(x + h * u, w) - f(x - h * u, w)) / (2 * h)
            tol = float(((half_step(dt) * got64.abs() + 2.0 ** -18 * size + 2.0 ** -25) * u.abs()).sum()) + 2.0 ** -20 * float((size * u.abs()).sum())
            assert abs(float((got64 * u).sum()) - diff) <= tol
            diff = (f(x, w + h * uw) - f(x, w - h * uw)) / (2 * h)
            assert abs(float((gw64 * uw).sum()) - diff) <= (2.0 ** -16 + 2.0 ** -20) * float((dwsize.sum((0, 1, 2)) * uw.abs()).sum())
