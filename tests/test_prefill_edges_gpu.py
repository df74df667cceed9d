"""attn_paged_prefill and attn_paged_prefix_decode at the edges of what their arguments may hold."""
import math

import pytest
import torch

from paper_2506_12355_b200 import api
from test_paged_gpu import make_cache
from test_prefill_gpu import check_prefill, make_shared, wide
from test_rope_gpu import DT

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,new,length", [(300, 60, 70), (2, 300, 2000), (1, 40, 5000)])       # whole lists; cut ones, of two tiles and of one
def test_a_visible_key_that_is_no_number_shows_in_o_and_lse(kind, D, n, new, length):
    """A NaN in one K row of one K/V head: NaN in O and LSE of the rows that see it, whether one CTA has their list to itself or several;
    all other rows as if it were not there."""
    H, Hkv, page, dt = 4, 2, 16, DT[kind]
    kc, vc, tab, ks, vs = make_cache([length] * n, Hkv, D, page, dt, "head", 41)
    j = length - new // 2
    kc[tab[:, j // page].long().cuda(), 1, j % page, 3] = math.nan
    q = torch.randn(n * new, H, D, generator=torch.Generator().manual_seed(42)).to(dt).cuda()
    cu = i32([new * b for b in range(n + 1)])
    o, lse = api.attn_paged_prefill(q, kc, vc, tab.cuda(), i32([length] * n), cu, D ** -0.5)
    assert api.attn_last_device_status() == 0
    o, lse = o.view(n, new, H, D), lse.view(n, new, H)
    first = j - (length - new)                        # token that sees the key first
    assert torch.isnan(o[:, first:, 2:]).all() and torch.isnan(lse[:, first:, 2:]).all()
    for b in range(0, n, 50):
        rows = q.view(n, new, H, D)[b]
        check_prefill(o[b, :, :2], lse[b, :, :2], rows[:, :2], ks[b][:, :1], vs[b][:, :1], D ** -0.5, dt)
        check_prefill(o[b, :first], lse[b, :first], rows[:first], ks[b][:j], vs[b][:j], D ** -0.5, dt)


@pytest.mark.parametrize("n", [5, 90])
def test_a_common_key_that_is_no_number_shows_in_o_and_lse(n):
    D, H, Hkv, page, dt, lens = 128, 8, 2, 16, torch.bfloat16, [300 + b % 7 for b in range(n)]
    kc, vc, tab, ks, vs = make_shared(lens, [0, n], [280], Hkv, D, page, dt, "head", 43)
    kc[int(tab[0, 3]), 1, 5, 7] = math.nan
    q = torch.randn(n, H, D, generator=torch.Generator().manual_seed(44)).to(dt).cuda()
    o, lse = api.attn_paged_prefix_decode(q, kc, vc, wide(tab, page, Hkv, D).cuda(), i32(lens), i32([0, n]), i32([280]), D ** -0.5)
    assert api.attn_last_device_status() == 0
    assert torch.isnan(o[:, 4:]).all() and torch.isnan(lse[:, 4:]).all()
    for b in range(n):
        check_prefill(o[b:b + 1, :4], lse[b:b + 1, :4], q[b:b + 1, :4], ks[b][:, :1], vs[b][:, :1], D ** -0.5, dt)
