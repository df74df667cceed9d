"""Which common keys attn_paged_prefix_decode reads once.  The copies differ here (which no caller may do), to show whose are read."""
import math

import pytest
import torch

from paper_2506_12355_b200 import api
from test_paged_gpu import check_decode
from test_prefill_gpu import wide

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("common,shared", [(16, False), (400, True)])
def test_a_group_of_more_blocks_than_ctas(common, shared):
    """One group, 20 blocks of 32 sequences for each of 8 K/V heads: 160 lists.  16 common keys are read for every sequence (a list takes
    longer than they do), 400 once."""
    n, H, Hkv, D, page, own, dt = 640, 64, 8, 128, 16, 3, torch.bfloat16
    g = torch.Generator().manual_seed(3)
    used = common // page
    per = used if not shared else 1                   # a sequence's pages of the prefix (shared: one, of NaN); then one with its own keys
    kc, vc = (torch.randn(n * (per + 1) + used, Hkv, page, D, generator=g).to(dt) for _ in range(2))
    tab = torch.empty(n, used + 1, dtype=torch.int32)
    first = torch.arange(n, dtype=torch.int32) * (per + 1)
    tab[:, used] = first + per
    if shared:
        kc[first.long()], vc[first.long()] = math.nan, math.nan
        tab[:, :used] = first[:, None]
        tab[0, :used] = torch.arange(used) + n * (per + 1)
    else:
        tab[:, :used] = first[:, None] + torch.arange(used)
    ks, vs = [], []
    for b in range(n):
        rows = torch.cat([tab[0 if shared else b, :used], tab[b, used:]]).long()
        for cache, to in ((kc, ks), (vc, vs)):
            to.append(cache[rows].transpose(1, 2).reshape(-1, Hkv, D)[:common + own])
    q = torch.randn(n, H, D, generator=g).to(dt).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    o, lse = api.attn_paged_prefix_decode(q, kc.cuda(), vc.cuda(), wide(tab, page, Hkv, D).cuda(), i32([common + own] * n), i32([0, n]),
                                          i32([common]), D ** -0.5)
    assert api.attn_last_device_status() == 0
    check_decode(o, lse, q, ks, vs, D ** -0.5, 0, 0, dt)
