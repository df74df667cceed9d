"""attn_paged_prefill and attn_paged_prefix_decode against plain 64-bit implementations, alone and as a serving step uses them.

Tolerances (u = 2^-24, e = eps/2 of the 16-bit type): those of the decode (test_paged_gpu.py), and for P, which is rounded to the
16-bit type before its product, e sum_j p_j |v_j|; in fp16 a P below 2^-14 (the largest of a row is at least 1 where the row
sum is taken, so that sum is at least 1) is off by at most 2^-25: n 2^-25 max |v|.
"""
import math

import pytest
import torch

from paper_2506_12355_b200 import api
from test_paged_gpu import check_decode, make_cache
from test_rope_gpu import DT, EPS, check_rows, half_step, rows64, table

pytestmark = pytest.mark.gpu


def bounds(want, av, ds, n, vmax, dt):
    e = half_step(dt)
    tol = e * want.abs() + (e + 2 * ds + 2.0 ** -15 + n * 2.0 ** -26) * av
    return tol + n * 2.0 ** -25 * vmax + 2.0 ** -25 if dt == torch.float16 else tol


def check_prefill(o, lse, q, k, v, scale, dt, name=""):
    """One sequence: o, q [n,H,D], lse [n,H], k, v [len,Hkv,D]."""
    n, H, D = q.shape
    length, Hkv, _ = k.shape
    q, k, v, o, lse = (x.cuda().double() for x in (q, k, v, o, lse))
    for i in range(0, n, 128):
        rows = slice(i, min(n, i + 128))
        qq = q[rows].view(-1, Hkv, H // Hkv, D)
        pos = torch.arange(length - n, length, device="cuda")[rows]
        seen = (torch.arange(length, device="cuda") <= pos[:, None])[:, None, None]
        x = (torch.einsum("tgid,jgd->tgij", qq, k) * scale).masked_fill(~seen, -math.inf)
        ds = D * 2.0 ** -23 * scale * torch.einsum("tgid,jgd->tgij", qq.abs(), k.abs()).masked_fill(~seen, 0).amax(-1, keepdim=True)
        p = torch.softmax(x, -1)
        want, av = torch.einsum("tgij,jgd->tgid", p, v), torch.einsum("tgij,jgd->tgid", p, v.abs())
        cnt = (pos + 1).double()[:, None, None, None]
        err = (o[rows].view(want.shape) - want).abs()
        tol = bounds(want, av, ds, cnt, v.abs().max(), dt)
        assert (err <= tol).all(), "%s tokens %d..: O over by %g" % (name, i, (err - tol).max())
        wl = torch.logsumexp(x, -1)
        lerr = (lse[rows].view(wl.shape) - wl).abs()
        assert (lerr <= ds[..., 0] + 2.0 ** -20 * wl.abs().clamp(min=1) + cnt[..., 0] * 2.0 ** -28).all(), "%s tokens %d..: LSE" % (name, i)


def run_prefill(lens, news, H, Hkv, D, page, kind, layout, seed=1, scale=None, before=0, behind=5, grow=0.0):
    dt = DT[kind]
    kc, vc, tab, ks, vs = make_cache(lens, Hkv, D, page, dt, layout, seed)
    if grow:     # keys that get longer along the sequence: the running maximum keeps growing
        for b, n in enumerate(lens):
            f = (1 + grow * torch.arange(n) / max(1, n)).view(-1, 1, 1)
            ks[b] = (ks[b].float() * f).to(dt)
            j = torch.arange(n)
            kc[tab[b].long()[j // page].cuda(), :, (j % page).cuda()] = ks[b].cuda()
    starts = [before]
    for n in news:
        starts.append(starts[-1] + n)
    T = starts[-1] + behind
    q = torch.randn(T, H, D, generator=torch.Generator().manual_seed(seed + 100)).to(dt).cuda()
    scale = 1 / math.sqrt(D) if scale is None else scale
    out, lse = torch.full((T, H, D), 7.0, dtype=dt, device="cuda"), torch.full((T, H), 7.0, device="cuda")
    args = (q, kc, vc, tab.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), torch.tensor(starts, dtype=torch.int32).cuda(), scale)
    api.attn_paged_prefill(*args, out=out, lse=lse)
    assert api.attn_last_device_status() == 0
    live = torch.zeros(T, dtype=torch.bool)
    for b, (n, length) in enumerate(zip(news, lens)):
        if n and length:
            rows = slice(starts[b], starts[b] + n)
            live[rows] = True
            check_prefill(out[rows], lse[rows], q[rows], ks[b], vs[b], scale, dt, "sequence %d" % b)
    assert (out.cpu()[~live] == 7).all() and (lse.cpu()[~live] == 7).all()
    again, lse2 = api.attn_paged_prefill(*args)
    live = live.cuda()
    assert torch.equal(again[live], out[live]) and torch.equal(lse2[live], lse[live])


LENS = [0, 1, 15, 128, 129, 0, 300, 77, 1000]
NEWS = [0, 1, 15, 128, 1, 0, 299, 13, 64]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("H,Hkv", [(2, 2), (8, 2), (3, 1), (12, 1), (40, 2), (128, 1), (7, 7)])
def test_prefill_head_layouts(D, kind, H, Hkv):
    run_prefill(LENS, NEWS, H, Hkv, D, 16, kind, "head", before=3)


@pytest.mark.parametrize("page", [1, 2, 8, 32, 128, 512])
@pytest.mark.parametrize("layout", ["head", "slot", "both"])
def test_prefill_pages_and_layouts(page, layout):
    run_prefill(LENS, NEWS, 4, 2, 64 if page < 32 else 128, page, "bf16", layout, seed=3)


@pytest.mark.parametrize("lens,news", [
    ([1], [1]), ([5000], [1]), ([5000], [300]), ([2049], [2049]),           # few lists: cut into many parts
    ([3] * 700, [1, 2, 3] * 233 + [1]),                                     # more sequences than lanes
    (list(range(1, 400, 3)), list(range(1, 400, 3))),
    ([4000, 1, 1, 1], [1, 1, 1, 1]), ([600] * 30, [520] * 30),
])
def test_prefill_length_mixes(lens, news):
    run_prefill(lens, news, 4, 2, 128 if sum(lens) < 15000 else 64, 16, "fp16", "slot", seed=4)


@pytest.mark.parametrize("scale,grow", [(0.0, 0.0), (1.0, 0.0), (0.3, 20.0), (1e-3, 0.0)])
@pytest.mark.parametrize("kind", ["fp16", "bf16"])
def test_prefill_scales(scale, grow, kind):
    run_prefill([700, 300], [200, 300], 8, 2, 128, 16, kind, "head", seed=5, scale=scale, grow=grow)


def test_prefill_bad_pages_lengths_and_lists():
    D, page, dt = 64, 16, torch.float16
    lens = [200, 64, 40]
    kc, vc, tab, ks, vs = make_cache(lens, 2, D, page, dt, "head", 9)
    q = torch.randn(60, 4, D, generator=torch.Generator().manual_seed(1)).to(dt).cuda()
    cu = torch.tensor([0, 20, 40, 60], dtype=torch.int32).cuda()

    def call(table_, lens_, cu_=cu):
        out, lse = torch.full((60, 4, D), 7.0, dtype=dt, device="cuda"), torch.full((60, 4), 7.0, device="cuda")
        api.attn_paged_prefill(q, kc, vc, table_.cuda(), torch.tensor(lens_, dtype=torch.int32).cuda(), cu_, 0.125, out, lse)
        return out, lse, api.attn_last_device_status()
    bad = tab.clone()
    bad[0, 0] = kc.shape[0]          # the first 16 keys of sequence 0 and 16 in the middle count as hidden
    bad[0, 5] = -3
    bad[1, :] = -7                   # no valid page at all
    o, lse, status = call(bad, lens)
    assert status == 13
    keep = torch.tensor([j for j in range(200) if j // 16 not in (0, 5)])
    check_prefill(o[:20], lse[:20], q[:20], ks[0][keep], vs[0][keep], 0.125, dt)
    assert (o[20:40] == 0).all() and (lse[20:40] == -math.inf).all()
    check_prefill(o[40:], lse[40:], q[40:], ks[2], vs[2], 0.125, dt)
    # a length beyond the table is cut to it; one below 0 is padding; a token in front of the first key sees nothing
    o, lse, status = call(tab, [2 ** 31 - 1, -5, 12])
    assert status == 13
    full = tab.shape[1] * page
    assert full == 208 and (o[20:40] == 7).all() and (lse[20:40] == 7).all()
    assert (o[40:48] == 0).all() and (lse[40:48] == -math.inf).all()
    check_prefill(o[48:], lse[48:], q[48:], ks[2][:12], vs[2][:12], 0.125, dt)
    # lists that run backwards or past the tokens are cut
    for cu_ in ([0, 40, 20, 60], [-4, 20, 40, 99], [50, 10, 10, 10]):
        o, lse, status = call(tab, lens, torch.tensor(cu_, dtype=torch.int32).cuda())
        assert o.shape == q.shape


def test_prefill_of_a_cache_above_4_gigaelements():
    D, page, Hkv, dt = 128, 64, 8, torch.bfloat16
    pages = (2 ** 32) // (page * Hkv * D) + 40
    kc, vc = (torch.zeros(pages, Hkv, page, D, dtype=dt, device="cuda") for _ in range(2))
    g = torch.Generator().manual_seed(8)
    n = 200
    k, v = torch.randn(n, Hkv, D, generator=g).to(dt), torch.randn(n, Hkv, D, generator=g).to(dt)
    tab = torch.tensor([[pages - 1, 3, pages - 30, pages // 2 + 9]], dtype=torch.int32)
    j = torch.arange(n)
    kc[tab[0].long()[j // page].cuda(), :, (j % page).cuda()] = k.cuda()
    vc[tab[0].long()[j // page].cuda(), :, (j % page).cuda()] = v.cuda()
    q = torch.randn(70, 16, D, generator=g).to(dt).cuda()
    cu, lens = torch.tensor([0, 70], dtype=torch.int32).cuda(), torch.tensor([n], dtype=torch.int32).cuda()
    o, lse = api.attn_paged_prefill(q, kc, vc, tab.cuda(), lens, cu, 0.09)
    check_prefill(o, lse, q, k, v, 0.09, dt)
    o, lse = api.attn_paged_prefix_decode(q[-1:], kc, vc, wide(tab, page, Hkv, D).cuda(), lens, torch.tensor([0, 1], dtype=torch.int32).cuda(),
                                          torch.tensor([150], dtype=torch.int32).cuda(), 0.09)
    check_prefill(o, lse, q[-1:], k, v, 0.09, dt)


# ------------------------------------------------------------------ shared prefixes

def wide(tab, page, Hkv, D):
    """The table with as many columns of no page as it takes for the call to share prefixes: below 128 MB of keys and values that it
    could stand for, all is read for every sequence (attn_paged_decode)."""
    columns = -(-2 ** 27 // (tab.shape[0] * page * Hkv * D * 4))
    return torch.cat([tab, torch.full((tab.shape[0], columns), -1, dtype=torch.int32)], 1)


def make_shared(lens, starts, prefix, Hkv, D, page, dt, layout, seed):
    """make_cache with the first prefix[g] keys of the sequences of group g in common: whole pages shared, the rest copied."""
    kc, vc, tab, ks, vs = make_cache(lens, Hkv, D, page, dt, layout, seed)
    for g, n in enumerate(prefix):
        first = starts[g]
        for b in range(starts[g], starts[g + 1]):
            m = min(n, lens[first], lens[b])
            ks[b][:m], vs[b][:m] = ks[first][:m], vs[first][:m]
            tab[b, :m // page] = tab[first, :m // page]
            j = torch.arange(m // page * page, m)
            if len(j):
                at, slot = tab[b].long()[j // page].cuda(), (j % page).cuda()
                kc[at, :, slot], vc[at, :, slot] = ks[b][j].cuda(), vs[b][j].cuda()
    return kc, vc, tab, ks, vs


def check_prefix(o, lse, q, ks, vs, scale, dt):
    for b in range(q.shape[0]):
        if ks[b].shape[0] == 0:
            assert (o[b] == 0).all() and (lse[b] == -math.inf).all()
        else:
            check_prefill(o[b:b + 1], lse[b:b + 1], q[b:b + 1], ks[b], vs[b], scale, dt, "sequence %d" % b)


def run_prefix(lens, starts, prefix, H, Hkv, D, page, kind, layout="head", seed=1, scale=None):
    dt = DT[kind]
    kc, vc, tab, ks, vs = make_shared(lens, starts, prefix, Hkv, D, page, dt, layout, seed)
    q = torch.randn(len(lens), H, D, generator=torch.Generator().manual_seed(seed + 100)).to(dt).cuda()
    scale = 1 / math.sqrt(D) if scale is None else scale
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    args = (q, kc, vc, wide(tab, page, Hkv, D).cuda(), i32(lens), i32(starts), i32(prefix), scale)
    o, lse = api.attn_paged_prefix_decode(*args)
    assert api.attn_last_device_status() == 0
    check_prefix(o, lse, q, ks, vs, scale, dt)
    o2, lse2 = api.attn_paged_prefix_decode(*args)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("H,Hkv", [(2, 2), (8, 2), (3, 1), (12, 1), (40, 2), (128, 1), (7, 7)])
def test_prefix_head_layouts(D, kind, H, Hkv):
    run_prefix([300, 257, 600, 256, 700, 20, 90, 64], [0, 4, 8], [256, 20], H, Hkv, D, 16, kind)


@pytest.mark.parametrize("page", [1, 2, 8, 32, 128, 512])
@pytest.mark.parametrize("layout", ["head", "slot", "both"])
def test_prefix_pages_and_layouts(page, layout):
    run_prefix([300, 400, 290, 1000, 513], [0, 3, 5], [277, 513], 4, 2, 64, page, "bf16", layout, seed=3)


@pytest.mark.parametrize("lens,starts,prefix", [
    ([1], [0, 1], [1]),
    ([130], [0, 1], [0]),                                          # nothing in common
    ([5, 5], [0, 2], [5]),                                         # everything in common
    ([3000] * 3 + [40], [0, 3], [2990]),                           # a sequence behind the last group
    ([40, 3000, 3000], [1, 3], [10 ** 9]),                         # one in front; a prefix beyond the sequences
    ([500, 0, 100, 499, 0], [0, 5], [400]),                        # padding rows, a sequence shorter than the prefix
    ([0, 300, 300], [0, 3], [200]),                                # the first sequence is padding: nothing is taken as common
    ([200] * 6, [0, 0, 2, 2, 6, 6], [9, 150, 9, 128, 9]),          # empty groups
    ([1030 + b % 7 for b in range(150)], [0, 150], [1024]),        # more rows than one list holds
    ([70 + b % 40 for b in range(120)], list(range(0, 121, 3)), [64] * 40),
    ([300 + b for b in range(90)], list(range(91)), [290] * 90),   # a group per sequence, more of them than lanes
    ([0, 0], [0, 2], [100]),
])
def test_prefix_groups(lens, starts, prefix):
    run_prefix(lens, starts, prefix, 8, 2, 128, 16, "bf16", seed=4)
    run_prefix(lens, starts, prefix, 4, 4, 64, 8, "fp16", "slot", seed=5)


@pytest.mark.parametrize("H,Hkv,D,kind", [(8, 2, 128, "bf16"), (4, 2, 64, "fp16")])
@pytest.mark.parametrize("singles", [70, 1100])
def test_prefix_of_many_groups(H, Hkv, D, kind, singles):
    """Groups of one sequence and short prefixes of few, which are read for each sequence, among groups of many that are not; groups
    whose sequences have no keys of their own."""
    lens, starts, prefix = [], [0], []
    for x in range(singles):
        size, common = (1, 20) if x % 23 else ((3, 33) if x % 2 else (40, 250))
        lens += [common + (x + 7 * y) % 30 for y in range(size)]
        starts.append(len(lens))
        prefix.append(common)
    lens += [300] * 100 + [290 + y for y in range(20)]
    starts += [starts[-1] + 100, starts[-1] + 120]
    prefix += [300, 290]
    run_prefix(lens, starts, prefix, H, Hkv, D, 16, kind, seed=7)


@pytest.mark.parametrize("scale", [0.0, 1.0])
def test_prefix_scales(scale):
    run_prefix([400, 300, 290], [0, 3], [280], 8, 2, 128, 16, "fp16", scale=scale, seed=6)


def test_prefix_bad_pages_lengths_and_groups():
    D, page, dt = 64, 16, torch.float16
    lens = [200, 300, 250]
    kc, vc, tab, ks, vs = make_shared(lens, [0, 3], [160], 2, D, page, dt, "head", 9)
    tab = wide(tab, page, 2, D)
    q = torch.randn(3, 4, D, generator=torch.Generator().manual_seed(1)).to(dt).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    bad = tab.clone()
    bad[:, 3], bad[1, 12] = kc.shape[0], -1
    o, lse = api.attn_paged_prefix_decode(q, kc, vc, bad.cuda(), i32(lens), i32([0, 3]), i32([160]), 0.125)
    assert api.attn_last_device_status() == 13
    for b, n in enumerate(lens):
        keep = torch.tensor([j for j in range(n) if j // 16 != 3 and not (b == 1 and j // 16 == 12)])
        check_prefill(o[b:b + 1], lse[b:b + 1], q[b:b + 1], ks[b][keep], vs[b][keep], 0.125, dt)
    o, lse = api.attn_paged_prefix_decode(q, kc, vc, tab.cuda(), i32([2 ** 31 - 1, -5, 250]), i32([0, 3]), i32([160]), 0.125)
    assert api.attn_last_device_status() == 13 and (o[1] == 0).all() and (lse[1] == -math.inf).all()
    check_prefill(o[2:], lse[2:], q[2:], ks[2], vs[2], 0.125, dt)
    # groups that run backwards or past the batch, prefixes below 0: no access out of range
    for starts, prefix in (([0, 3, 1], [160, 160]), ([-5, 2, 99], [160, 160]), ([3, 0, 3], [-1, 2 ** 31 - 1]), ([7, 9], [5])):
        o, lse = api.attn_paged_prefix_decode(q, kc, vc, tab.cuda(), i32(lens), i32(starts), i32(prefix), 0.125)
        api.attn_last_device_status()
        assert o.shape == q.shape


def test_prefix_without_groups_is_the_decode():
    kc, vc, tab, ks, vs = make_cache([300, 0, 77], 2, 64, 16, torch.float16, "head", 12)
    q = torch.randn(3, 8, 64, generator=torch.Generator().manual_seed(2)).half().cuda()
    lens = torch.tensor([300, 0, 77], dtype=torch.int32).cuda()
    none = torch.zeros(0, dtype=torch.int32).cuda()
    b = api.attn_paged_decode(q, kc, vc, tab.cuda(), lens, 0.125)
    a = api.attn_paged_prefix_decode(q, kc, vc, tab.cuda(), lens, torch.zeros(1, dtype=torch.int32).cuda(), none, 0.125)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # few keys in all: nothing is shared either
    a = api.attn_paged_prefix_decode(q, kc, vc, tab.cuda(), lens, torch.tensor([0, 1], dtype=torch.int32).cuda(),
                                     torch.tensor([200], dtype=torch.int32).cuda(), 0.125)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ------------------------------------------------------------------ as they are used

def test_captured_calls_replayed_with_other_lengths_beside_eager_ones():
    D, page, dt, Hkv, H = 128, 16, torch.bfloat16, 2, 8
    lens, starts, prefix = [600, 700, 650, 900], [0, 3, 4], [512, 100]
    kc, vc, tab, ks, vs = make_shared(lens, starts, prefix, Hkv, D, page, dt, "head", 20)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    lens_t, starts_t, prefix_t, cu, table_ = i32(lens), i32(starts), i32(prefix), i32([0, 40, 80, 120, 160]), wide(tab, page, Hkv, D).cuda()
    g = torch.Generator().manual_seed(21)
    q, qp = torch.randn(4, H, D, generator=g).to(dt).cuda(), torch.randn(160, H, D, generator=g).to(dt).cuda()
    ws = torch.empty(api.attn_paged_prefix_decode_workspace_bytes(4, H, Hkv, D), dtype=torch.uint8, device="cuda")
    ws_p = torch.empty(api.attn_paged_prefill_workspace_bytes(D), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        api.attn_paged_prefix_decode(q, kc, vc, table_, lens_t, starts_t, prefix_t, 0.09, workspace=ws)
        api.attn_paged_prefill(qp, kc, vc, table_, lens_t, cu, 0.09, workspace=ws_p)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        op, lp = api.attn_paged_prefill(qp, kc, vc, table_, lens_t, cu, 0.09, workspace=ws_p)
        o, lse = api.attn_paged_prefix_decode(q, kc, vc, table_, lens_t, starts_t, prefix_t, 0.09, workspace=ws)
    for new_lens, new_prefix, new_cu in ((lens, prefix, [0, 40, 80, 120, 160]), ([600, 560, 0, 313], [77, 300], [0, 1, 100, 100, 160])):
        lens_t.copy_(i32(new_lens))
        prefix_t.copy_(i32(new_prefix))
        cu.copy_(i32(new_cu))
        graph.replay()
        with torch.cuda.stream(side):       # beside the replay, with workspaces of their own
            side_o, _ = api.attn_paged_prefix_decode(q, kc, vc, table_, lens_t, starts_t, prefix_t, 0.09)
            side_p, _ = api.attn_paged_prefill(qp, kc, vc, table_, lens_t, cu, 0.09)
        torch.cuda.synchronize()
        assert torch.equal(side_o, o)
        check_prefix(o, lse, q, [k[:n] for k, n in zip(ks, new_lens)], [v[:n] for v, n in zip(vs, new_lens)], 0.09, dt)
        for b, n in enumerate(new_lens):
            rows = slice(new_cu[b], new_cu[b + 1])
            if n and new_cu[b + 1] > new_cu[b]:
                assert torch.equal(side_p[rows], op[rows])
                check_prefill(op[rows], lp[rows], qp[rows], ks[b][:n], vs[b][:n], 0.09, dt)
    assert api.attn_last_device_status() == 0


def test_serving_step_with_images_behind_a_shared_instruction():
    """An instruction appended once, questions with pictures in them appended behind it with three position axes and attended to, then
    a token each: append, prefill and prefix decode over one cache."""
    D, page, dt, Hkv, H, R = 128, 16, torch.bfloat16, 2, 8, 128
    of = api.rope_pair_axes((16, 24, 24), "blocks")
    scale, shared, asks = 1 / math.sqrt(D), 80, [37, 5, 130]
    tab64 = table(1000, R)
    g = torch.Generator().manual_seed(30)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    kc, vc = (torch.full((60, Hkv, page, D), float("nan"), dtype=dt, device="cuda") for _ in range(2))
    order = torch.randperm(60, generator=g).to(torch.int32)
    bt = torch.full((3, 14), -1, dtype=torch.int32)
    bt[:, :5] = order[:5]                                                   # 80 tokens in 5 shared pages
    for b in range(3):
        bt[b, 5:14] = order[5 + 9 * b:14 + 9 * b]
    bt = wide(bt, page, Hkv, D).cuda()
    qw, kw = ((1 + 0.2 * torch.randn(D, generator=g)).to(dt).cuda() for _ in range(2))
    made_k, made_v, made_q = [], [], []

    def append(n, pos, lens, cu, table_):
        x = (torch.randn(n, H + 2 * Hkv, D, generator=g) * 1.5).to(dt).cuda()
        q = api.attn_paged_append_axes(x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:], kc, vc, table_, i32(lens), pos.to(torch.int32).cuda(), of, qw, kw,
                                       tab64.cuda(), None if cu is None else i32(cu), EPS)
        at = pos.long().T[:, torch.tensor(list(of))]
        col = torch.arange(R // 2)
        row = torch.cat([tab64[at, col], tab64[at, R // 2 + col]], -1)[:, None]
        want_k, size = rows64(x[:, H:H + Hkv].cpu(), kw.cpu(), row, R, False)
        made_k.append((want_k, size))
        made_v.append(x[:, H + Hkv:].cpu())
        want_q, size = rows64(x[:, :H].cpu(), qw.cpu(), row, R, False)
        check_rows(q.cpu(), want_q, size, dt, "q")
        return q

    text = lambda n, at: torch.arange(at, at + n).expand(3, -1)
    append(shared, text(shared, 0), [shared], [0, shared], bt[:1])
    ends = [0, 37, 42, 172]
    pos = torch.cat([torch.stack([torch.full((n,), shared), shared + torch.arange(n) // 7, shared + torch.arange(n) % 7]) for n in asks], 1)
    lens = [shared + n for n in asks]
    q = append(172, pos, lens, ends, bt)
    o, lse = api.attn_paged_prefill(q, kc, vc, bt, i32(lens), i32(ends), scale)
    # the cache's own rows are what attention reads: their values were checked against the definition above
    def rows(b, n):
        j = torch.arange(n, device="cuda")
        return kc[bt[b].long()[j // page], :, j % page].cpu(), vc[bt[b].long()[j // page], :, j % page].cpu()
    for b, n in enumerate(lens):
        k, v = rows(b, n)
        check_rows(k[shared:], made_k[1][0][ends[b]:ends[b + 1]], made_k[1][1][ends[b]:ends[b + 1]], dt, "k")
        check_rows(k[:shared], *made_k[0], dt, "k")
        assert torch.equal(v, torch.cat([made_v[0], made_v[1][ends[b]:ends[b + 1]]]))
        check_prefill(o[ends[b]:ends[b + 1]], lse[ends[b]:ends[b + 1]], q[ends[b]:ends[b + 1]], k, v, scale, dt)
    for step in range(2):
        lens = [n + 1 for n in lens]
        q = append(3, torch.tensor([[200 + step] * 3] * 3), lens, None, bt)
        o, lse = api.attn_paged_prefix_decode(q, kc, vc, bt, i32(lens), i32([0, 3]), i32([shared]), scale)
        kv = [rows(b, n) for b, n in enumerate(lens)]
        check_prefix(o, lse, q, [k for k, _ in kv], [v for _, v in kv], scale, dt)
    assert api.attn_last_device_status() == 0
