"""attn_paged_append and attn_paged_decode against plain 64-bit implementations, and the two together.

Tolerances of the decode (u = 2^-24, e = eps/2 of the 16-bit type):
  scores      exact products of 16-bit values summed in fp32 over D: |ds| <= D 2^-23 scale max_j sum_d |q_d k_jd|.
  O           |err| <= e |O| + (2 |ds| + 2^-15 + n 2^-26) sum_j p_j |v_j|: each probability is off by |ds| and exp2's 2^-22,
              in numerator and denominator; it is fed in two 16-bit parts (2^-16 for bf16); n additions in fp32, 16 at a time.
              fp16: parts below its smallest step add n 2^-31 max |v|.  Subnormal results: 2^-25.
  LSE         |err| <= |ds| + 2^-20 max(1, |LSE|) + n 2^-28.
"""
import math

import pytest
import torch

from paper_2506_12355_b200 import api
from test_rope_gpu import DT, EPS, check_rows, half_step, rows64, table

pytestmark = pytest.mark.gpu


def make_cache(lens, Hkv, D, page, dt, layout, seed, spare=2, dead=float("nan")):
    """Caches whose live slots hold normal values and every other slot `dead`; a shuffled block table, -1 where unused."""
    g = torch.Generator().manual_seed(seed)
    per = max(1, -(-max(lens) // page)) if lens else 1
    used = sum(-(-n // page) for n in lens)
    order = torch.randperm(used + spare, generator=g).to(torch.int32)
    tab = torch.full((len(lens), per), -1, dtype=torch.int32)
    shape = {"head": (used + spare, Hkv, page, D), "slot": (used + spare, page, Hkv, D), "both": (used + spare, 2, Hkv, page, D)}[layout]
    if layout == "both":
        buf = torch.full(shape, dead, dtype=dt)
        kc, vc = buf[:, 0], buf[:, 1]
    else:
        kc, vc = torch.full(shape, dead, dtype=dt), torch.full(shape, dead, dtype=dt)
        if layout == "slot":
            kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    ks, vs, at = [], [], 0
    for b, n in enumerate(lens):
        m = -(-n // page)
        tab[b, :m] = order[at:at + m]
        at += m
        k, v = torch.randn(n, Hkv, D, generator=g).to(dt), torch.randn(n, Hkv, D, generator=g).to(dt)
        j = torch.arange(n)
        kc[tab[b].long()[j // page], :, j % page] = k
        vc[tab[b].long()[j // page], :, j % page] = v
        ks.append(k)
        vs.append(v)
    if layout == "slot":   # keep the strides on the device
        dev = lambda t: t.transpose(1, 2).contiguous().cuda().transpose(1, 2)
        return dev(kc), dev(vc), tab, ks, vs
    if layout == "both":
        d = buf.cuda()
        return d[:, 0], d[:, 1], tab, ks, vs
    return kc.cuda(), vc.cuda(), tab, ks, vs


def decode64(q, k, v, scale, window, sinks):
    """One sequence: q [H,D], k, v [n,Hkv,D] -> O, sum p|v|, score error, LSE, n."""
    H, D = q.shape
    n, Hkv, _ = k.shape
    j = torch.arange(n)
    if window:
        j = j[(j >= n - window) | (j < sinks)]
    q = q.double().view(Hkv, H // Hkv, D)
    k, v = k[j].double(), v[j].double()
    x = torch.einsum("gid,jgd->gij", q, k) * scale
    ds = D * 2.0 ** -23 * scale * torch.einsum("gid,jgd->gij", q.abs(), k.abs()).amax(-1, keepdim=True)
    p = torch.softmax(x, -1)
    o, av = torch.einsum("gij,jgd->gid", p, v), torch.einsum("gij,jgd->gid", p, v.abs())
    return o.reshape(H, D), av.reshape(H, D), ds.reshape(H, 1), torch.logsumexp(x, -1).reshape(H), len(j), v.abs().max()


def check_decode(o, lse, q, ks, vs, scale, window, sinks, dt):
    o, lse, q = o.cpu(), lse.cpu(), q.cpu()
    for b in range(q.shape[0]):
        if ks[b].shape[0] == 0:
            assert (o[b] == 0).all() and (lse[b] == -math.inf).all()
            continue
        want, av, ds, wl, n, vmax = decode64(q[b], ks[b], vs[b], scale, window, sinks)
        tol = half_step(dt) * want.abs() + (2 * ds + 2.0 ** -15 + n * 2.0 ** -26) * av
        if dt == torch.float16:
            tol = tol + n * 2.0 ** -31 * vmax + 2.0 ** -25
        err = (o[b].double() - want).abs()
        assert (err <= tol).all(), "sequence %d: over by %g" % (b, (err - tol).max())
        lerr = (lse[b].double() - wl).abs()
        assert (lerr <= ds[:, 0] + 2.0 ** -20 * wl.abs().clamp(min=1) + n * 2.0 ** -28).all(), "sequence %d" % b


def run_decode(lens, H, Hkv, D, page, kind, layout, window=0, sinks=0, seed=1, scale=None):
    dt = DT[kind]
    kc, vc, tab, ks, vs = make_cache(lens, Hkv, D, page, dt, layout, seed)
    q = torch.randn(len(lens), H, D, generator=torch.Generator().manual_seed(seed + 100)).to(dt).cuda()
    scale = 1 / math.sqrt(D) if scale is None else scale
    # pages that hold hidden keys only need no entry
    if window:
        for b, n in enumerate(lens):
            for j in range(tab.shape[1]):
                keys = range(j * page, min(n, (j + 1) * page))
                if not any(x >= n - window or x < sinks for x in keys):
                    tab[b, j] = -1
    lens_t = torch.tensor(lens, dtype=torch.int32).cuda()
    o, lse = api.attn_paged_decode(q, kc, vc, tab.cuda(), lens_t, scale, window, sinks)
    assert api.attn_last_device_status() == 0
    check_decode(o, lse, q, ks, vs, scale, window, sinks, dt)
    o2, lse2 = api.attn_paged_decode(q, kc, vc, tab.cuda(), lens_t, scale, window, sinks)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


EDGES = [0, 1, 15, 16, 17, 0, 127, 128, 129, 1000, 0]


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("H,Hkv", [(2, 2), (8, 2), (8, 1), (12, 1), (16, 1), (40, 2)])
def test_decode_head_layouts(D, kind, H, Hkv):
    run_decode(EDGES, H, Hkv, D, 16, kind, "head")


@pytest.mark.parametrize("page", [1, 2, 8, 32, 256])
@pytest.mark.parametrize("layout", ["head", "slot", "both"])
def test_decode_pages_and_layouts(page, layout):
    run_decode(EDGES, 4, 2, 64, page, "bf16", layout, seed=3)


@pytest.mark.parametrize("lens", [[1], [0, 0, 0], [5000], [1, 30000], [3] * 700, list(range(0, 520, 2))])
def test_decode_length_mixes(lens):
    run_decode(lens, 4, 2, 128 if sum(lens) < 20000 else 64, 16, "fp16", "slot", seed=4)


@pytest.mark.parametrize("H,Hkv,D,kind", [(8, 8, 64, "fp16"), (32, 8, 128, "bf16"), (48, 16, 64, "bf16"), (64, 4, 128, "fp16"),
                                          (160, 8, 128, "bf16"), (8, 4, 256, "fp16"), (24, 24, 128, "fp16"), (6, 6, 64, "bf16")])
@pytest.mark.parametrize("window,sinks", [(0, 0), (700, 5)])
def test_decode_long_lists(H, Hkv, D, kind, window, sinks):
    """Enough tiles that the warps of a CTA take different heads: all of them where 8 (D = 256: 4) divide the heads, some or none."""
    g = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 2000, (24,), generator=g).tolist() + [1, 16, 0, 2500]
    run_decode(lens, H, Hkv, D, 16, kind, "slot", window, sinks, seed=13)


def test_decode_padded_and_interleaved_caches():
    """Views of larger buffers: padded pages, K and V side by side in one row, a head axis outside the pages."""
    dt, D, Hkv, page, lens = torch.float16, 64, 3, 8, [77, 5, 300]
    kc, vc, tab, ks, vs = make_cache(lens, Hkv, D, page, dt, "head", 14)
    q = torch.randn(3, 6, D, generator=torch.Generator().manual_seed(4)).to(dt).cuda()
    tab, len_t, n = tab.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), kc.shape[0]
    nan = lambda *s: torch.full(s, float("nan"), dtype=dt, device="cuda")
    padded = nan(n, Hkv, page + 3, D + 8)[:, :, :page, :D], nan(n, Hkv + 1, page, D)[:, :Hkv]
    side = nan(n, page, Hkv, 2 * D).transpose(1, 2)
    heads_first = nan(Hkv, n, page, D).transpose(0, 1), nan(Hkv, page, n, D).permute(2, 0, 1, 3)
    for k, v in (padded, (side[..., :D], side[..., D:]), heads_first):
        k.copy_(kc)
        v.copy_(vc)
        o, lse = api.attn_paged_decode(q, k, v, tab, len_t, 0.125)
        check_decode(o, lse, q, ks, vs, 0.125, 0, 0, dt)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (100, 0), (100, 33), (130, 200), (999, 1), (100000, 4)])
@pytest.mark.parametrize("H,Hkv", [(4, 2), (12, 1)])
def test_decode_window(window, sinks, H, Hkv):
    run_decode(EDGES + [2000], H, Hkv, 64, 16, "bf16", "head", window, sinks, seed=5)


@pytest.mark.parametrize("lens", [[1], [0], [16], [129], [1000], [4096], [0, 5], [300, 2000]])
@pytest.mark.parametrize("H,Hkv,D", [(2, 1, 64), (8, 8, 128), (20, 1, 64), (24, 2, 256), (12, 4, 128)])
def test_decode_few_pairs(lens, H, Hkv, D):
    """One or two sequences: few pairs of a sequence and a head, which clusters of CTAs take."""
    run_decode(lens, H, Hkv, D, 16, "bf16", "slot", seed=6)
    run_decode(lens, H, Hkv, D, 64, "fp16", "head", window=70, sinks=5, seed=7)


@pytest.mark.parametrize("n", [3, 4, 7, 8, 15, 18, 19])
@pytest.mark.parametrize("Hkv,group,D", [(8, 4, 128), (8, 2, 64), (4, 12, 128), (2, 20, 256)])
def test_decode_some_pairs(n, Hkv, group, D):
    """Every size of cluster, and the shapes on both sides of the last one."""
    lens = [(0, 1, 500, 129, 16, 333, 512)[i % 7] for i in range(n)]
    run_decode(lens, Hkv * group, Hkv, D, 16, "bf16", "head", seed=8)
    run_decode(lens, Hkv * group, Hkv, D, 32, "fp16", "slot", window=200, sinks=3, seed=9)


@pytest.mark.parametrize("lens", [[1000], [700, 3, 0]])
def test_decode_through_a_view_of_a_wide_table(lens):
    """The form of the call follows from the table's width: the whole table (a list of tiles) and a view of its first columns
    (clusters), on which the rows stand further apart than they are wide."""
    D, dt, page = 128, torch.bfloat16, 16
    kc, vc, tab, ks, vs = make_cache(lens, 4, D, page, dt, "head", 15)
    wide = torch.full((len(lens), 2048), -1, dtype=torch.int32)
    wide[:, :tab.shape[1]] = tab
    wide, len_t = wide.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    q = torch.randn(len(lens), 8, D, generator=torch.Generator().manual_seed(5)).to(dt).cuda()
    for t in (wide, wide[:, :tab.shape[1]]):
        o, lse = api.attn_paged_decode(q, kc, vc, t, len_t, 0.09)
        assert api.attn_last_device_status() == 0
        check_decode(o, lse, q, ks, vs, 0.09, 0, 0, dt)


def test_decode_few_long_sequences():
    run_decode([14000, 9000], 8, 8, 128, 64, "bf16", "head", seed=10)


def test_decode_zero_scale_and_large_scores():
    run_decode([1, 50, 400], 4, 2, 128, 16, "bf16", "head", scale=0.0, seed=6)
    run_decode([1, 50, 3000], 4, 2, 128, 16, "fp16", "head", scale=3.0, seed=7)    # scores of a hundred and more: the maximum moves
    # scores that grow along the keys, so that every chunk overtakes the reference maximum
    D, n, dt = 64, 700, torch.bfloat16
    kc, vc, tab, ks, vs = make_cache([n], 1, D, 16, dt, "head", 8, dead=0.0)
    ramp = torch.linspace(-40, 40, n)[:, None, None].expand(n, 1, D).to(dt)
    j = torch.arange(n)
    kc[tab[0].long()[j // 16].cuda(), :, (j % 16).cuda()] = ramp.cuda()
    q = torch.ones(1, 2, D, dtype=dt).cuda()
    o, lse = api.attn_paged_decode(q, kc, vc, tab.cuda(), torch.tensor([n], dtype=torch.int32).cuda(), 0.5)
    check_decode(o, lse, q, [ramp], vs, 0.5, 0, 0, dt)


def test_decode_bad_pages_and_lengths_are_reported():
    D, page, dt = 64, 16, torch.float16
    kc, vc, tab, ks, vs = make_cache([64, 64, 40], 2, D, page, dt, "head", 9)
    q = torch.randn(3, 4, D, generator=torch.Generator().manual_seed(1)).to(dt).cuda()
    bad = tab.clone()
    bad[0, 1] = kc.shape[0]          # one page out of range: its keys count as hidden
    bad[1, :] = -7                   # no valid page at all
    o, lse = api.attn_paged_decode(q, kc, vc, bad.cuda(), torch.tensor([64, 64, 40], dtype=torch.int32).cuda(), 0.125)
    assert api.attn_last_device_status() == 13 and api.attn_last_device_status() == 0
    keep = torch.cat([torch.arange(16), torch.arange(32, 64)])
    check_decode(o[:1], lse[:1], q[:1], [ks[0][keep]], [vs[0][keep]], 0.125, 0, 0, dt)
    assert (o[1] == 0).all() and (lse[1] == -math.inf).all()
    check_decode(o[2:], lse[2:], q[2:], ks[2:], vs[2:], 0.125, 0, 0, dt)
    # lengths beyond the table are cut to it, negative ones are 0
    o, lse = api.attn_paged_decode(q, kc, vc, tab.cuda(), torch.tensor([2 ** 31 - 1, -5, 40], dtype=torch.int32).cuda(), 0.125)
    assert api.attn_last_device_status() == 13
    check_decode(o[:1], lse[:1], q[:1], ks[:1], vs[:1], 0.125, 0, 0, dt)
    assert (o[1] == 0).all() and (lse[1] == -math.inf).all()


def test_decode_offsets_beyond_32_bits():
    D, page, Hkv, dt = 128, 64, 8, torch.bfloat16
    pages = (2 ** 32) // (page * Hkv * D * 2) * 2 + 40          # more than 2^32 elements
    kc = torch.zeros(pages, Hkv, page, D, dtype=dt, device="cuda")
    n = 200
    g = torch.Generator().manual_seed(10)
    k, v = torch.randn(n, Hkv, D, generator=g).to(dt), torch.randn(n, Hkv, D, generator=g).to(dt)
    tab = torch.tensor([[pages - 1, 3, pages - 30, pages // 2 + 9]], dtype=torch.int32)
    vc = torch.zeros_like(kc)
    j = torch.arange(n)
    kc[tab[0].long()[j // page].cuda(), :, (j % page).cuda()] = k.cuda()
    vc[tab[0].long()[j // page].cuda(), :, (j % page).cuda()] = v.cuda()
    q = torch.randn(1, 32, D, generator=g).to(dt).cuda()
    o, lse = api.attn_paged_decode(q, kc, vc, tab.cuda(), torch.tensor([n], dtype=torch.int32).cuda(), 0.09)
    check_decode(o, lse, q, [k], [v], 0.09, 0, 0, dt)
    # and the append at such an offset
    api.attn_paged_append(None, k[:1].cuda(), v[:1].cuda(), kc, vc, tab[:, :1].contiguous().cuda(), torch.tensor([7], dtype=torch.int32).cuda())
    assert torch.equal(kc[pages - 1, :, 6].cpu(), k[0]) and torch.equal(vc[pages - 1, :, 6].cpu(), v[0])


@pytest.mark.parametrize("times", [1, 9])      # few pairs (clusters), many (a list of tiles, two kernels)
def test_decode_graph_with_new_lengths_and_two_streams(times):
    D, page, dt, lens = 128, 16, torch.bfloat16, [300, 5, 0, 900] * times
    kc, vc, tab, ks, vs = make_cache([900] * len(lens), 2, D, page, dt, "head", 11)
    q = torch.randn(len(lens), 8, D, generator=torch.Generator().manual_seed(2)).to(dt).cuda()
    tab, len_t = tab.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    ws = [torch.empty(api.attn_paged_decode_workspace_bytes(8, 2, D), dtype=torch.uint8, device="cuda") for _ in range(2)]
    api.attn_paged_decode(q, kc, vc, tab, len_t, 0.1, workspace=ws[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = api.attn_paged_decode(q, kc, vc, tab, len_t, 0.1, workspace=ws[0])
    side = torch.cuda.Stream()
    for new in ([300, 5, 0, 900], [1, 900, 899, 17], [0, 0, 0, 0], [900, 900, 900, 900]):
        new = new * times
        len_t.copy_(torch.tensor(new, dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        o2, lse2 = api.attn_paged_decode(q, kc, vc, tab, len_t, 0.1, workspace=ws[1], stream=side)   # beside the replay
        torch.cuda.synchronize()
        check_decode(o, lse, q, [k[:n] for k, n in zip(ks, new)], [v[:n] for v, n in zip(vs, new)], 0.1, 0, 0, dt)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_decode_nan_in_a_visible_key_reaches_its_row_only():
    D, dt = 64, torch.float16
    kc, vc, tab, ks, vs = make_cache([100, 100], 1, D, 16, dt, "head", 12, dead=0.0)
    kc[tab[0, 2].item(), 0, 5, 3] = float("nan")
    q = torch.randn(2, 2, D, generator=torch.Generator().manual_seed(3)).to(dt).cuda()
    o, lse = api.attn_paged_decode(q, kc, vc, tab.cuda(), torch.tensor([100, 100], dtype=torch.int32).cuda(), 0.125)
    assert torch.isnan(o[0]).all() and torch.isnan(lse[0]).all()
    check_decode(o[1:], lse[1:], q[1:], ks[1:], vs[1:], 0.125, 0, 0, dt)


# ------------------------------------------------------------------ append

@pytest.mark.parametrize("D,R,inter,kind,page,layout", [(64, 64, False, "fp16", 16, "head"), (128, 64, True, "bf16", 8, "slot"),
                                                       (256, 256, False, "bf16", 1, "both"), (128, 0, False, "fp16", 128, "head")])
def test_append_ragged(D, R, inter, kind, page, layout):
    dt, H, Hkv = DT[kind], 6, 2
    lens, new = [40, 0, 7, 130, 9, 1], [3, 0, 7, 100, 0, 1]
    kc, vc, tab, ks, vs = make_cache(lens, Hkv, D, page, dt, layout, 20, dead=0.5)
    kc0, vc0 = kc.cpu().clone(), vc.cpu().clone()
    T = sum(new)
    pad = T + 9
    g = torch.Generator().manual_seed(21)
    qkv = torch.randn(pad, H + 2 * Hkv, D, generator=g).to(dt).cuda()
    qw, kw = (1 + 0.2 * torch.randn(2, D, generator=g)).to(dt).cuda()
    rt = table(256, R) if R else None
    q_out = torch.full((pad, H, D), 0.25, dtype=dt, device="cuda")
    cu = torch.tensor([0] + list(torch.tensor(new).cumsum(0)), dtype=torch.int32).cuda()
    lens_t = torch.tensor(lens, dtype=torch.int32).cuda()
    api.attn_paged_append(qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:], kc, vc, tab.cuda(), lens_t, qw, kw, rt.cuda() if R else None,
                          cu_seqlens=cu, eps=EPS, interleaved=inter, q_out=q_out)
    assert api.attn_last_device_status() == 0
    got_q, got_k, got_v, x = q_out.cpu(), kc.cpu(), vc.cpu(), qkv.cpu()
    at = 0
    for b, (n, m) in enumerate(zip(lens, new)):
        pos = torch.arange(n - m, n)
        rows = rt[pos][:, None] if R else None
        t = slice(at, at + m)
        want, size = rows64(x[t, :H], qw.cpu(), rows, R, inter)
        if m:
            check_rows(got_q[t], want, size, dt, "q")
            want, size = rows64(x[t, H:H + Hkv], kw.cpu(), rows, R, inter)
            p = tab[b].long()[pos // page]
            check_rows(got_k[p, :, pos % page], want, size, dt, "k")
            assert torch.equal(got_v[p, :, pos % page], x[t, H + Hkv:])
            got_k[p, :, pos % page] = kc0[p, :, pos % page]
            got_v[p, :, pos % page] = vc0[p, :, pos % page]
        at += m
    assert (got_q[T:] == 0.25).all()                                  # padding rows stay
    assert torch.equal(got_k, kc0) and torch.equal(got_v, vc0)        # and so does every other slot


@pytest.mark.parametrize("first", [1, 5, 13])
def test_append_tokens_before_the_first_sequence_are_padding(first):
    """A slice of a larger batch's cu_seqlens beside the whole projection: the tokens in front of it belong to no sequence here."""
    D, dt, page, H, Hkv = 64, torch.float16, 16, 4, 2
    lens, new = [100, 3, 20], [10, 3, 4]
    kc, vc, tab, ks, vs = make_cache(lens, Hkv, D, page, dt, "head", 23, dead=0.5)
    kc0, vc0 = kc.cpu().clone(), vc.cpu().clone()
    cu = torch.tensor([first, first + 10, first + 13, first + 17], dtype=torch.int32)
    T = int(cu[-1]) + 6
    qkv = torch.randn(T, H + 2 * Hkv, D, generator=torch.Generator().manual_seed(24)).to(dt).cuda()
    q_out = torch.full((T, H, D), 0.25, dtype=dt, device="cuda")
    api.attn_paged_append(qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:], kc, vc, tab.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
                          cu_seqlens=cu.cuda(), q_out=q_out)
    assert api.attn_last_device_status() == 0
    want_k, want_v, x = kc0.clone(), vc0.clone(), qkv.cpu()
    want_q = torch.full((T, H, D), 0.25, dtype=dt)
    for b, (n, m) in enumerate(zip(lens, new)):
        pos, t = torch.arange(n - m, n), slice(int(cu[b]), int(cu[b + 1]))
        p = tab[b].long()[pos // page]
        want_q[t], want_k[p, :, pos % page], want_v[p, :, pos % page] = x[t, :H], x[t, H:H + Hkv], x[t, H + Hkv:]
    assert torch.equal(q_out.cpu(), want_q) and torch.equal(kc.cpu(), want_k) and torch.equal(vc.cpu(), want_v)


def test_append_reports_and_skips_bad_entries():
    D, dt, page = 64, torch.float16, 16
    kc, vc, tab, ks, vs = make_cache([20, 20, 20, 20], 1, D, page, dt, "head", 22, dead=0.0)
    kc0 = kc.clone()
    k = torch.ones(4, 1, D, dtype=dt, device="cuda")
    t = tab.clone()
    t[1, 1] = kc.shape[0]
    lens = torch.tensor([0, 20, 2 ** 31 - 1, 33], dtype=torch.int32).cuda()      # padding, bad page, two beyond the table
    api.attn_paged_append(None, k, k, kc, vc, t.cuda(), lens)
    assert api.attn_last_device_status() == 13
    assert torch.equal(kc, kc0)
    api.attn_paged_append(None, k, k, kc, vc, tab.cuda(), torch.tensor([20, 20, 20, 20], dtype=torch.int32).cuda(), cos_sin=table(10, 64).cuda())
    assert api.attn_last_device_status() == 13 and torch.equal(kc, kc0)          # beyond the rotation table


def test_serving_steps_match_attention_over_the_same_tokens():
    """A prompt and then single tokens through append and decode, against the dense calls of the library on the same projection."""
    D, H, Hkv, page, dt = 128, 8, 2, 16, torch.bfloat16
    prompts, steps = [37, 120], 5
    B, total = 2, [p + steps for p in prompts]
    g = torch.Generator().manual_seed(30)
    qkv = [torch.randn(1, n, H + 2 * Hkv, D, generator=g).to(dt).cuda() for n in total]
    qw, kw = (1 + 0.2 * torch.randn(2, D, generator=g)).to(dt).cuda()
    rt, scale = table(256, D).cuda(), 1 / math.sqrt(D)
    tab = torch.randperm(2 * 9, generator=g).to(torch.int32).view(2, 9).cuda()
    kc = torch.full((18, Hkv, page, D), float("nan"), dtype=dt, device="cuda")
    vc = torch.full_like(kc, float("nan"))
    split = lambda x: (x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:])
    first = torch.cat([x[0, :p] for x, p in zip(qkv, prompts)])
    cu = torch.tensor([0, prompts[0], sum(prompts)], dtype=torch.int32).cuda()
    lens = torch.tensor(prompts, dtype=torch.int32).cuda()
    api.attn_paged_append(*split(first), kc, vc, tab, lens, qw, kw, rt, cu_seqlens=cu)
    for i in range(steps):
        lens += 1
        x = torch.stack([y[0, p + i] for y, p in zip(qkv, prompts)])
        q = api.attn_paged_append(*split(x), kc, vc, tab, lens, qw, kw, rt)
        o, lse = api.attn_paged_decode(q, kc, vc, tab, lens, scale)
        for b in range(B):
            n = prompts[b] + i + 1
            y = qkv[b][:, :n]
            dq, dk, dv = api.attn_qk_norm_rope(y[:, :, :H], y[:, :, H:H + Hkv], y[:, :, H + Hkv:], qw, kw, rt)
            assert torch.equal(dq[0, :, -1], q[b])
            want, wl = api.attn_fwd_gqa(dq, dk, dv, scale, causal=True)
            # the dense call rounds P to bf16 (2^-9 of each term at most, |v| < 5) on top of both calls' rounding of O
            assert (want[0, :, -1].float() - o[b].float()).abs().max() <= 2 * 2.0 ** -8 * 5
            assert (wl[0, :, -1] - lse[b]).abs().max() <= 1e-3
    assert api.attn_last_device_status() == 0


def test_both_ways_of_marshalling_agree():
    """Without an explicit stream a plain call is marshalled by the extension, with one by Python: same results, same refusals."""
    D, dt = 64, torch.bfloat16
    kc, vc, tab, ks, vs = make_cache([70, 33], 2, D, 16, dt, "slot", 40, dead=0.0)
    tab, lens = tab.cuda(), torch.tensor([70, 33], dtype=torch.int32).cuda()
    q = torch.randn(2, 8, D, generator=torch.Generator().manual_seed(1)).to(dt).cuda()
    here = torch.cuda.current_stream()
    for extra in ({}, dict(window=20, sinks=3)):
        a = api.attn_paged_decode(q, kc, vc, tab, lens, 0.125, **extra)
        b = api.attn_paged_decode(q, kc, vc, tab, lens, 0.125, stream=here, **extra)
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    for s in (None, here):
        with pytest.raises(api.AttnError) as err:
            api.attn_paged_decode(q, kc, vc, tab, lens, float("nan"), stream=s)
        assert err.value.status == 6
        with pytest.raises(ValueError):
            api.attn_paged_decode(q, kc, vc, tab[:1], lens, 0.125, stream=s)
        with pytest.raises(TypeError):
            api.attn_paged_decode(q, kc, vc, tab, lens.long(), 0.125, stream=s)
        with pytest.raises(ValueError):
            api.attn_paged_decode(q, kc.cpu(), vc, tab, lens, 0.125, stream=s)
    # outputs given by the caller, one of the wrong shape
    o, lse = torch.empty_like(q), torch.empty(2, 8, device="cuda")
    r = api.attn_paged_decode(q, kc, vc, tab, lens, 0.125, out=o, lse=lse)
    assert r[0].data_ptr() == o.data_ptr() and r[1].data_ptr() == lse.data_ptr()
    with pytest.raises(ValueError):
        api.attn_paged_decode(q, kc, vc, tab, lens, 0.125, out=o[:, :4])


def test_serving_step_as_one_graph():
    """Lengths advanced, tokens appended and attended in one captured graph, replayed step after step, against eager calls."""
    D, H, Hkv, page, dt, steps = 64, 8, 2, 16, torch.float16, 40
    lens0, g = [1, 15, 200, 63], torch.Generator().manual_seed(50)
    B, per = len(lens0), 16
    tab = torch.randperm(B * per, generator=g).to(torch.int32).view(B, per).cuda()
    rt = table(per * page, D).cuda()
    qw, kw = (1 + 0.2 * torch.randn(2, D, generator=g)).to(dt).cuda()
    start = torch.randn(B * per, Hkv, page, D, generator=g).to(dt).cuda()
    tokens = torch.randn(steps, B, H + 2 * Hkv, D, generator=g).to(dt).cuda()
    ws = torch.empty(api.attn_paged_decode_workspace_bytes(H, Hkv, D), dtype=torch.uint8, device="cuda")

    def step(x, kc, vc, lens):
        lens += 1
        q = api.attn_paged_append(x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:], kc, vc, tab, lens, qw, kw, rt)
        return api.attn_paged_decode(q, kc, vc, tab, lens, 0.125, window=100, sinks=3, workspace=ws)
    kc, vc, lens = start.clone(), start.clone(), torch.tensor(lens0, dtype=torch.int32).cuda()
    want = [step(x, kc, vc, lens) for x in tokens]
    kc2, vc2, lens2, x2 = start.clone(), start.clone(), torch.tensor(lens0, dtype=torch.int32).cuda(), torch.empty_like(tokens[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = step(x2, kc2, vc2, lens2)
    for x, (wo, wl) in zip(tokens, want):
        x2.copy_(x)
        graph.replay()
        assert torch.equal(o, wo) and torch.equal(lse, wl)
    assert torch.equal(kc, kc2) and torch.equal(vc, vc2) and lens2.tolist() == [n + steps for n in lens0]
    assert api.attn_last_device_status() == 0


@pytest.mark.parametrize("times", [1, 12])      # clusters, a list of tiles
def test_decode_of_sequences_that_share_pages(times):
    """A common beginning is held once: several sequences name the same pages, some the same ones altogether."""
    D, dt, page, n = 64, torch.bfloat16, 16, 150
    kc, vc, tab, ks, vs = make_cache([n], 2, D, page, dt, "head", 51)
    lens = [150, 33, 150, 96] * times
    q = torch.randn(len(lens), 6, D, generator=torch.Generator().manual_seed(6)).to(dt).cuda()
    o, lse = api.attn_paged_decode(q, kc, vc, tab.expand(len(lens), -1).contiguous().cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), 0.125)
    check_decode(o, lse, q, [ks[0][:m] for m in lens], [vs[0][:m] for m in lens], 0.125, 0, 0, dt)
    # the rows of the block table may be one and the same (stride 0)
    o2, lse2 = api.attn_paged_decode(q, kc, vc, tab.cuda().expand(len(lens), -1), torch.tensor(lens, dtype=torch.int32).cuda(), 0.125)
    assert torch.equal(o, o2) and torch.equal(lse, lse2) and api.attn_last_device_status() == 0
