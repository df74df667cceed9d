"""attn_fwd_window and attn_bwd_window against a dense 64-bit implementation.

Tolerances (e = eps/2 of the 16-bit type, all elementwise):
  scores  16-bit products summed in fp32 over D:  ds = D 2^-23 scale max sum_d |q_d k_jd|.
  P       one rounding to 16 bits (e), the polynomial exponential (7.5e-5 < 2^-13) and ds:  dp = e + 2^-12 + 2 ds.
  O       e |O| + dp sum p |v|;  fp16 adds half of its smallest step per key, n 2^-25 max |v| (P is at least that fine).
  LSE     ds + 2^-13 + 2^-20 |LSE|.
  dV      e |dV| + dp' sum_i P |dO|, dp' = dp + the LSE's error;
  dS      P ((dp' + e) |dP - delta| + D 2^-23 sum |dO v| + sum |dO| tolO)   (the last: delta is taken from the rounded O);
  dQ, dK  e |dQ| + scale sum |err dS| |K|, and the same with Q.  fp16 adds 2^-25 per term for small P and dS, and 2^-25 for
          each result: below 2^-14 its values are multiples of 2^-24, so that rounding is off by half of that, whatever e |x| says.
"""
import math

import pytest
import torch

from paper_2506_12355_b200 import api

pytestmark = pytest.mark.gpu

DT = {"fp16": torch.float16, "bf16": torch.bfloat16}


def visible(Sq, Sk, W, sinks, off):
    p = torch.arange(Sq, device="cuda")[:, None] + off
    j = torch.arange(Sk, device="cuda")
    near = j <= p
    return near & ((j > p - W) | (j < sinks)) if W else near


def reference(q, k, v, dout, scale, W, sinks, off):
    """Everything in 64 bits, with the tolerances of the docstring."""
    dt = q.dtype
    e = torch.finfo(dt).eps / 2
    tiny = 2.0 ** -25 if dt == torch.float16 else 0.0
    B, H, Sq, D = q.shape
    Hkv, Sk = k.shape[1], k.shape[2]
    G = H // Hkv
    q, k, v, g = (t.double() for t in (q, k, v, dout))
    kk, vv = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
    vis = visible(Sq, Sk, W, sinks, off)
    x = (q @ kk.transpose(-1, -2) * scale).masked_fill(~vis, -math.inf)
    ds = D * 2.0 ** -23 * scale * ((q.abs() @ kk.abs().transpose(-1, -2)) * vis).amax(-1, keepdim=True)
    lse = torch.logsumexp(x, -1, keepdim=True)
    p = torch.where(vis, torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)), 0.0)
    n = vis.sum(-1)[None, None, :, None]
    o = p @ vv
    dp = e + 2.0 ** -12 + 2 * ds
    tol_o = e * o.abs() + dp * (p @ vv.abs()) + n * tiny * v.abs().max() + tiny
    tol_l = ds + 2.0 ** -13 + 2.0 ** -20 * torch.where(lse == -math.inf, 0.0, lse.abs())
    out = dict(o=(o, tol_o), lse=(lse[..., 0], tol_l[..., 0]))
    dpl = dp + tol_l
    fold = lambda t: t.view(B, Hkv, G, Sk, -1).sum(2)
    dv = fold(p.transpose(-1, -2) @ g)
    seen = vis.double()
    out["dv"] = (dv, e * dv.abs() + fold((dpl * p).transpose(-1, -2) @ g.abs()) + tiny * fold(seen.T @ g.abs()) + tiny)
    dP = g @ vv.transpose(-1, -2)
    delta = (g * o).sum(-1, keepdim=True)
    dS = p * (dP - delta)
    err = p * ((dpl + e) * (dP - delta).abs() + D * 2.0 ** -23 * (g.abs() @ vv.abs().transpose(-1, -2)) + (g.abs() * tol_o).sum(-1, keepdim=True)) + tiny * seen
    dq = scale * dS @ kk
    out["dq"] = (dq, e * dq.abs() + scale * err @ kk.abs() + tiny)
    dk = scale * fold(dS.transpose(-1, -2) @ q)
    out["dk"] = (dk, e * dk.abs() + scale * fold(err.transpose(-1, -2) @ q.abs()) + tiny)
    return out


def inputs(B, H, Hkv, Sq, Sk, D, dt, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(*s, generator=g).to(dt).cuda() for s in ((B, H, Sq, D), (B, Hkv, Sk, D), (B, Hkv, Sk, D), (B, H, Sq, D))]


def check(name, got, want, tol):
    got = got.double()
    empty = want == -math.inf
    assert torch.equal(got == -math.inf, empty), name
    err = (got - want).abs().masked_fill(empty, 0.0)
    assert not torch.isnan(err).any(), name
    over = err - tol
    assert (over <= 0).all(), "%s: over the tolerance by %g (%d values)" % (name, over.max(), (over > 0).sum())


def run(B, H, Hkv, Sq, Sk, D, kind, W, sinks, off, seed=1, scale=None, backward=True, data=None):
    q, k, v, g = data or inputs(B, H, Hkv, Sq, Sk, D, DT[kind], seed)
    scale = float(torch.tensor(1 / math.sqrt(D) if scale is None else scale, dtype=torch.float32))
    ref = reference(q, k, v, g, scale, W, sinks, off)
    o, lse = api.attn_fwd_window(q, k, v, scale, W, sinks, off)
    assert api.attn_last_device_status() == 0
    check("o", o, *ref["o"])
    check("lse", lse, *ref["lse"])
    if not backward:
        return
    grads = api.attn_bwd_window(q, k, v, o, lse, g, scale, W, sinks, off)
    assert api.attn_last_device_status() == 0
    for name, t in zip(("dq", "dk", "dv"), grads):
        check(name, t, *ref[name])
    again = api.attn_bwd_window(q, k, v, o, lse, g, scale, W, sinks, off)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("W,sinks", [(1, 0), (1, 3), (64, 0), (127, 4), (128, 1), (129, 130), (200, 300), (1000, 4), (0, 0), (2 ** 31 - 1, 7)])
def test_window_sizes(D, kind, W, sinks):
    run(1, 2, 1, 700, 700, D, kind, W, sinks, 0)


@pytest.mark.parametrize("Sq,Sk", [(1, 1), (1, 300), (2, 129), (127, 127), (128, 128), (129, 129), (257, 513), (300, 1000), (513, 700), (640, 640)])
@pytest.mark.parametrize("W,sinks", [(100, 2), (256, 140)])
def test_lengths_and_offsets(Sq, Sk, W, sinks):
    run(2, 4, 2, Sq, Sk, 64, "bf16", W, sinks, max(0, Sk - Sq), seed=2)


@pytest.mark.parametrize("W,sinks,off", [(1, 0, 0), (2, 0, 5), (5, 3, 0), (8, 0, 70), (3, 5, 0), (3, 6, 0), (9, 0, 0)])
@pytest.mark.parametrize("D,kind", [(64, "bf16"), (128, "fp16")])
def test_few_keys_per_row(W, sinks, off, D, kind):
    """Rows of up to 8 keys take their row sum of dO o O from the keys, so that dQ and dK carry two roundings, that of dS and their
    own: sqrt(2) u in the 2-norm, where u <= eps / 2 / sqrt(3) is the root mean square of one (values spread over a binade).
    1.5 u leaves room for the exponentials; with the sum taken from the rounded O two-key rows stand at 1.73 u."""
    run(2, 4, 2, 150, 150 + off, D, kind, W, sinks, off, seed=20)
    q, k, v, g = inputs(2, 4, 2, 150, 150 + off, D, DT[kind], 20)
    scale = float(torch.tensor(1 / math.sqrt(D), dtype=torch.float32))
    ref = reference(q, k, v, g, scale, W, sinks, off)
    o, lse = api.attn_fwd_window(q, k, v, scale, W, sinks, off)
    grads = api.attn_bwd_window(q, k, v, o, lse, g, scale, W, sinks, off)
    u = torch.finfo(DT[kind]).eps / 2 / math.sqrt(3)      # root mean square of a rounding, at most
    if W + sinks > 1:
        for name, t in zip(("dq", "dk"), grads):
            err = (t.double() - ref[name][0]).norm() / ref[name][0].norm()
            assert err <= 1.5 * u, (name, float(err / u))


@pytest.mark.parametrize("H,Hkv", [(1, 1), (6, 2), (8, 1), (3, 3)])
def test_head_groups(H, Hkv):
    run(2, H, Hkv, 333, 333, 128, "fp16", 90, 5, 0, seed=3)


@pytest.mark.parametrize("W,sinks,off", [(50, 0, 400), (50, 0, 260), (300, 0, 100), (1, 0, 0), (50, 10, 1000), (64, 129, 5000)])
def test_keys_that_end_before_the_queries(W, sinks, off):
    # queries behind the last key: rows that see part of the keys, only the first ones, or none (O = 0, LSE = -inf, no gradient)
    run(1, 2, 2, 300, 280, 64, "bf16", W, sinks, off, seed=4)


@pytest.mark.parametrize("Sq,Sk,W,off", [(100, 20, 1000, 0), (200, 32, 300, 40), (70, 9, 100, 0), (100, 8, 1000, 3), (90, 33, 64, 0), (10, 10, 50, 0), (3, 25, 100, 12)])
def test_few_keys_for_many_queries(Sq, Sk, W, off):
    # all rows see the same few keys, also those behind the sequence's first rows; nothing is taken from the workspace's old content
    q, k, v, g = inputs(2, 2, 1, Sq, Sk, 128, torch.bfloat16, 6)
    scale = float(torch.tensor(1 / math.sqrt(128), dtype=torch.float32))
    ref = reference(q, k, v, g, scale, W, 0, off)
    o, lse = api.attn_fwd_window(q, k, v, scale, W, 0, off)
    workspace = torch.full((api.attn_bwd_window_workspace_bytes(2, 2, 1, Sq, Sk, 128, W, 0, off),), 255, dtype=torch.uint8, device="cuda")
    grads = api.attn_bwd_window(q, k, v, o, lse, g, scale, W, 0, off, workspace=workspace)
    for name, t in zip(("dq", "dk", "dv"), grads):
        check(name, t, *ref[name])


def test_more_keys_than_positions():
    run(1, 2, 1, 200, 900, 64, "fp16", 64, 3, 100, seed=5)       # keys behind every query: zero gradients


def test_long_rows_and_many_items():
    # more work items than SMs, several rings and items per CTA
    run(2, 16, 4, 2500, 2500, 64, "fp16", 300, 4, 0, seed=6)
    run(1, 24, 8, 2048, 2048, 128, "bf16", 128, 1, 0, seed=7)


@pytest.mark.parametrize("scale", [0.0, 1.0, 4.0])
def test_scales(scale):
    # large scales: the running maximum moves by more than its lag in many steps
    run(1, 2, 1, 400, 400, 64, "fp16", 150, 2, 0, seed=8, scale=scale)


def test_scores_far_below_zero_behind_hidden_tiles():
    # every score is near -1000; rows whose first tiles are hidden must still take their own maximum
    q, k, v, g = inputs(1, 2, 1, 600, 600, 64, torch.bfloat16, 9)
    q, k = (4 + 0.1 * q.float()).bfloat16(), (-4 + 0.1 * k.float()).bfloat16()
    run(1, 2, 1, 600, 600, 64, "bf16", 40, 0, 0, scale=1.0, data=(q, k, v, g))
    run(1, 2, 1, 600, 600, 64, "bf16", 129, 1, 0, scale=1.0, data=(q, k, v, g))


@pytest.mark.parametrize("sinks", [0, 2, 40])
def test_large_values_behind_a_low_first_reference(sinks):
    """The first keys that a row meets score far below the later ones (by 40, 2^57 in the probabilities), and the values are near
    2^100: neither the probabilities nor their sums may carry the whole distance, or the products leave fp32 (2^127)."""
    q, k, v, g = inputs(1, 4, 2, 600, 600, 128, torch.bfloat16, 21)
    q, k = (1 + 0.01 * q.float()).bfloat16(), (1 + 0.01 * k.float()).bfloat16()
    k[:, :, :200] = 0                              # scores 0; all later ones about 128 * 0.3125
    v = (v.float() * 2.0 ** 100).bfloat16()
    run(1, 4, 2, 600, 600, 128, "bf16", 300, sinks, 0, scale=0.3125, backward=False, data=(q, k, v, g))


@pytest.mark.parametrize("W,sinks,off", [(2, 0, 0), (3, 0, 5), (5, 3, 0), (9, 1, 0), (40, 0, 0), (129, 4, 0), (300, 130, 0), (0, 0, 0)])
@pytest.mark.parametrize("D,kind", [(64, "bf16"), (64, "fp16"), (128, "bf16"), (128, "fp16")])
def test_precision_of_the_exponentials(W, sinks, off, D, kind):
    """The window kernels take every exponential from the hardware's exp2 (2^-22), none from the polynomial of the causal kernels
    (2^-13), which would stand in the LSE of rows with few keys as it is.  In units of 2^-24:
      LSE  ex2 4; the reference's product with the scale, once in the exponent and once at the end, 2.4 |m|; the log of the sum 2 |log l|,
           at most 2 (14 ln 2 + ln n); the last addition |LSE|; n additions, in eight chains, n / 8 + 4: below 8 x size for
           size = 10 + |LSE| + largest |score| + ln n, and n / 4.
      O    one rounding of P (e) and one of the result, and the same for the exponentials: dp = e + 2^-21 size + n 2^-26.
    The scores add nothing: q and k are multiples of 1/4 up to 3, so every sum of products is a multiple of 1/16 below 2^11."""
    S = 520
    q, k, v, g = inputs(1, 4, 2, S, S + off, D, DT[kind], 22)
    q, k = ((4 * t.float()).round().clamp(-12, 12).div(4).to(DT[kind]) for t in (q, k))
    scale = float(torch.tensor(1 / math.sqrt(D), dtype=torch.float32))
    o, lse = api.attn_fwd_window(q, k, v, scale, W, sinks, off)
    assert api.attn_last_device_status() == 0
    dt = q.dtype
    e, tiny = torch.finfo(dt).eps / 2, 2.0 ** -25 if dt == torch.float16 else 0.0
    qq, kk, vv = q.double(), k.double().repeat_interleave(2, 1), v.double().repeat_interleave(2, 1)
    vis = visible(S, S + off, W, sinks, off)
    x = (qq @ kk.transpose(-1, -2) * scale).masked_fill(~vis, -math.inf)
    want, n = torch.logsumexp(x, -1, keepdim=True), vis.sum(-1)[None, None, :, None]
    size = 10 + want.abs() + x.masked_fill(~vis, 0.0).abs().amax(-1, keepdim=True) + torch.log(n.double())
    check("lse", lse, want[..., 0], (2.0 ** -21 * size + n * 2.0 ** -26)[..., 0])
    p = torch.softmax(x, -1)
    dp = e + 2.0 ** -21 * size + n * 2.0 ** -26
    check("o", o, p @ vv, e * (p @ vv).abs() + dp * (p @ vv.abs()) + n * tiny * vv.abs().max() + tiny)


@pytest.mark.parametrize("W,sinks", [(2 ** 31 - 1, 0), (2 ** 31 - 1, 5), (1, 7), (0, 0), (2 ** 31 - 500, 2 ** 31 - 1), (2 ** 31 - 400, 33)])
def test_the_last_positions(W, sinks):
    """Queries at the end of the range of positions (2^31 - 1 - 256): nothing in the step lists and masks passes 32 bits."""
    Sq = 300
    run(1, 2, 1, Sq, 200, 64, "bf16", W, sinks, 2 ** 31 - 1 - 256 - Sq, seed=23)


def test_full_window_is_causal_attention():
    """No lower end: the same operator as the causal calls.  Those evaluate part of the exponentials by a polynomial (2^-13), the
    window kernels do not, so the two are compared within the tolerance that allows for it, on either side of the exact value."""
    q, k, v, g = inputs(2, 4, 2, 500, 500, 128, torch.bfloat16, 10)
    scale = float(torch.tensor(0.09, dtype=torch.float32))
    ref = reference(q, k, v, g, scale, 0, 0, 0)
    a, al = api.attn_fwd_gqa(q, k, v, scale, causal=True)
    b, bl = api.attn_fwd_window(q, k, v, scale, 0)
    x = api.attn_bwd(q, k, v, a, al, g, scale, causal=True)
    y = api.attn_bwd_window(q, k, v, b, bl, g, scale, 0)
    for name, s, t in zip(("o", "lse", "dq", "dk", "dv"), (a, al) + x, (b, bl) + y):
        check(name, t, *ref[name])
        check(name, s, *ref[name])
        assert ((s.double() - t.double()).abs() <= 2 * ref[name][1]).all()


def test_chunks_of_a_prompt_equal_the_whole():
    # the rows of a chunk do not depend on the chunk they came in, up to tile order: compare within both tolerances
    q, k, v, g = inputs(1, 4, 2, 700, 700, 64, torch.float16, 11)
    ref = reference(q, k, v, g, 0.125, 150, 3, 0)
    for a, b in ((0, 100), (100, 101), (101, 430), (430, 700)):
        o, lse = api.attn_fwd_window(q[:, :, a:b].contiguous(), k[:, :, :b].contiguous(), v[:, :, :b].contiguous(), 0.125, 150, 3, a)
        check("o", o, ref["o"][0][:, :, a:b], ref["o"][1][:, :, a:b])
        check("lse", lse, ref["lse"][0][:, :, a:b], ref["lse"][1][:, :, a:b])


def test_gradient_against_differences():
    # sum(O * g) differenced in 64 bits along random directions of q, k and v
    q, k, v, g = inputs(1, 2, 1, 150, 150, 64, torch.float16, 12)
    W, sinks, scale = 40, 3, 0.125
    o, lse = api.attn_fwd_window(q, k, v, scale, W, sinks)
    grads = api.attn_bwd_window(q, k, v, o, lse, g, scale, W, sinks)
    ref = reference(q, k, v, g, scale, W, sinks, 0)
    for i, name in enumerate(("dq", "dk", "dv")):
        d = torch.randn((q, k, v)[i].shape, generator=torch.Generator().manual_seed(i), dtype=torch.float64).cuda()
        h = 1e-4
        hi, lo = [t.double() for t in (q, k, v)], [t.double() for t in (q, k, v)]
        hi[i], lo[i] = hi[i] + h * d, lo[i] - h * d

        def value(ts):
            vis = visible(150, 150, W, sinks, 0)
            qq, kk, vv = ts[0], ts[1].repeat_interleave(2, 1), ts[2].repeat_interleave(2, 1)
            x = (qq @ kk.transpose(-1, -2) * scale).masked_fill(~vis, -math.inf)
            return float(((torch.softmax(x, -1) @ vv) * g.double()).sum())
        want = (value(hi) - value(lo)) / (2 * h)
        got = float((grads[i].double() * d).sum())
        slack = float((ref[name][1] * d.abs()).sum())
        assert abs(got - want) <= slack + 1e-5 * abs(want)


def test_graph_and_second_stream():
    q, k, v, g = inputs(1, 8, 2, 1500, 1500, 64, torch.bfloat16, 13)
    args = (0.125, 200, 4, 0)
    o, lse = api.attn_fwd_window(q, k, v, *args)
    want = api.attn_bwd_window(q, k, v, o, lse, g, *args)
    ws = torch.empty(api.attn_bwd_window_workspace_bytes(1, 8, 2, 1500, 1500, 64, 200, 4), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o2, lse2 = api.attn_fwd_window(q, k, v, *args)
        got = api.attn_bwd_window(q, k, v, o2, lse2, g, *args, workspace=ws)
    side = torch.cuda.Stream()
    for _ in range(3):
        graph.replay()
        o3, lse3 = api.attn_fwd_window(q, k, v, *args, stream=side)
        eager = api.attn_bwd_window(q, k, v, o, lse, g, *args, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(o, o2) and torch.equal(o, o3) and torch.equal(lse, lse3)
        assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, got, eager))
    assert api.attn_last_device_status() == 0


def test_training_step_from_projection_to_weight_gradients():
    """norm + rotation -> window attention -> both gradients, as a layer runs them, against autograd in 64 bits."""
    B, S, H, Hkv, D, W, sinks, dt = 2, 200, 4, 2, 64, 48, 2, torch.float16
    gen = torch.Generator().manual_seed(14)
    qkv = torch.randn(B, S, H + 2 * Hkv, D, generator=gen).to(dt).cuda()
    qw, kw = (1 + 0.2 * torch.randn(2, D, generator=gen)).to(dt).cuda()
    f = 1e4 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    a = torch.arange(S, dtype=torch.float64)[:, None] * f
    tab = torch.cat([a.cos(), a.sin()], 1).float().cuda()
    parts = lambda x: (x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:])
    q, k, v = api.attn_qk_norm_rope(*parts(qkv), qw, kw, tab)
    o, lse = api.attn_fwd_window(q, k, v, 0.125, W, sinks)
    g = torch.randn(B, H, S, D, generator=gen).to(dt).cuda()
    dq, dk, dv = api.attn_bwd_window(q, k, v, o, lse, g, 0.125, W, sinks)
    out = torch.empty_like(qkv)
    di = parts(out)
    _, _, _, dqw, dkw = api.attn_qk_norm_rope_bwd(dq, dk, dv, *parts(qkv)[:2], qw, kw, tab, dq_in=di[0], dk_in=di[1], dv_in=di[2])

    x = qkv.double().requires_grad_()
    w = [qw.double().requires_grad_(), kw.double().requires_grad_()]

    def rows(t, w):
        n = t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6) * w
        c, s = tab.double()[None, :, None, :D // 2], tab.double()[None, :, None, D // 2:]
        return torch.cat([n[..., :D // 2] * c - n[..., D // 2:] * s, n[..., D // 2:] * c + n[..., :D // 2] * s], -1).transpose(1, 2)
    xq, xk, xv = parts(x)
    kk, vv = rows(xk, w[1]).repeat_interleave(2, 1), xv.transpose(1, 2).repeat_interleave(2, 1)
    sc = (rows(xq, w[0]) @ kk.transpose(-1, -2) * 0.125).masked_fill(~visible(S, S, W, sinks, 0), -math.inf)
    (torch.softmax(sc, -1) @ vv * g.double()).sum().backward()
    # 16-bit roundings of q, k, v, o, P, dS, dq, dk in a row: each 2^-11 relative at most, incoherent over hundreds of terms
    for got, want in ((out, x.grad), (dqw, w[0].grad), (dkw, w[1].grad)):
        assert float((got.double() - want).norm() / want.norm()) <= 8 * 2.0 ** -11
