"""attn_paged_prefix_decode to the tolerances of attn_paged_decode (test_paged_gpu.py): P goes into its product in two 16-bit parts
whichever kernel a key is read by.  Common keys only, so that nothing else adds to the error; even scores, so that many keys count and
their values cancel: a P rounded once is off by up to half_step(dt) sum_j p_j |v_j| there, 2^-9 (bf16) or 2^-12 (fp16) for the 2^-15 and
2 |ds| (2^-16 with these queries) that are allowed."""
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
