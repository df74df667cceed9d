"""attn_paged_prefix_decode to the tolerances of attn_paged_decode (test_paged_gpu.py): P goes into its product in two 16-bit parts
whichever kernel a key is read by.  Common keys only, so that nothing else adds to the error; even scores, so that many keys count and
their values cancel: a P rounded once is off by up to half_step(dt) sum_j p_j |v_j| there, 2^-9 (bf16) or 2^-12 (fp16) for the 2^-15 and
2 |ds| (2^-16 with these queries) that are allowed."""
import math

import pytest
import torch

from paper_2506_12355_b200 import api
from test_paged_gpu import check_decode
from test_prefill_gpu import make_shared, wide
from test_rope_gpu import DT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [9, 70, 300])              # lists of one tile of queries, of two, several
@pytest.mark.parametrize("common", [12, 500])            # one step, several
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", ["fp16", "bf16"])
def test_common_keys_are_as_exact_as_others(n, common, D, kind):
    H, Hkv, page, dt = 8, 2, 16, DT[kind]
    lens = [common - (b % 5 if common > 100 else 0) for b in range(n)]
    lens[0] = common
    kc, vc, tab, ks, vs = make_shared(lens, [0, n], [common], Hkv, D, page, dt, "head", 31)
    q = (0.25 * torch.randn(n, H, D, generator=torch.Generator().manual_seed(32))).to(dt).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    o, lse = api.attn_paged_prefix_decode(q, kc, vc, wide(tab, page, Hkv, D).cuda(), i32(lens), i32([0, n]), i32([common]), D ** -0.5)
    assert api.attn_last_device_status() == 0
    check_decode(o, lse, q, ks, vs, D ** -0.5, 0, 0, dt)


@pytest.mark.parametrize("n,H,Hkv", [(3, 4, 2), (320, 128, 16)])         # a list cut into its steps, each CTA with a largest P of its own; whole lists
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", ["fp16", "bf16"])
def test_many_small_probabilities(n, H, Hkv, D, kind):
    """One key that takes nearly everything and has no value, 4000 others of 2^-18 of it, all with the value 1.  A fp16 P of that size without a
    scale of its own lies half way between two multiples of 2^-24, and 4000 equal errors of 2^-25 are a hundredth of O."""
    page, dt, common = 16, DT[kind], 4001
    pages = -(-common // page)
    k, v = torch.zeros(pages * page, Hkv, D), torch.ones(pages * page, Hkv, D)
    k[0, :, 0], v[0] = 8, 0
    kc, vc = (x.to(dt).view(pages, page, Hkv, D).transpose(1, 2).contiguous().cuda() for x in (k, v))
    q = torch.zeros(n, H, D, dtype=dt)
    q[:, :, 0] = 1
    scale = (18 - math.log2(1 + 2.0 ** -7)) * math.log(2) / 8        # 8 scale = ln(2^18 / (1 + 2^-7))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    tab = wide(torch.arange(pages, dtype=torch.int32).expand(n, -1), page, Hkv, D).cuda()
    o, lse = api.attn_paged_prefix_decode(q.cuda(), kc, vc, tab, i32([common] * n), i32([0, n]), i32([common]), scale)
    assert api.attn_last_device_status() == 0
    some = list(range(0, n, 33))                                     # of every block of rows, whole and cut
    check_decode(o[some], lse[some], q[some], [k[:common].to(dt)] * len(some), [v[:common].to(dt)] * len(some), scale, 0, 0, dt)
