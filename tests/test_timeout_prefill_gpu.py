"""The bounded waits of attn_paged_prefill and attn_paged_prefix_decode, made to run out in the form of
tests/test_timeout_operators_gpu.py (waits of 1 ms, one ring group's copies left out in every CTA)."""
import ctypes

import pytest
import torch

from paper_2506_12355_b200 import api
from test_paged_gpu import make_cache
from test_prefill_gpu import wide
from test_timeout_operators_gpu import lib  # noqa: F401

pytestmark = pytest.mark.gpu


def check(lib, call, outputs, skip):
    stream = torch.cuda.current_stream().cuda_stream
    lib.attn_test_skip_group.restype = None
    lib.attn_test_skip_group.argtypes = [ctypes.c_int]

    def run():
        for t in outputs:
            t.zero_()
        assert call(stream) == 0
        return lib.attn_last_device_status(stream)          # synchronises
    assert run() == 0
    before = [t.clone() for t in outputs]
    lib.attn_test_skip_group(skip)
    assert run() == 9
    assert lib.attn_last_device_status(stream) == 0
    assert run() == 0
    assert all(torch.equal(a, b) for a, b in zip(outputs, before))


@pytest.mark.parametrize("skip", [0, 1, 4])
@pytest.mark.parametrize("D,n,new,page", [(128, 3, 400, 16), (64, 40, 30, 16), (64, 3, 400, 1)])      # lists of two tiles, of one; small boxes
def test_prefill(lib, D, n, new, page, skip):
    H, Hkv, dt, length = 16, 4, torch.bfloat16, 3000
    kc, vc, tab, _, _ = make_cache([length] * n, Hkv, D, page, dt, "head", 60, dead=0.0)
    tab, lens = tab.cuda(), torch.full((n,), length, dtype=torch.int32, device="cuda")
    cu = (torch.arange(n + 1, dtype=torch.int32) * new).cuda()
    q = torch.randn(n * new, H, D, generator=torch.Generator().manual_seed(7)).to(dt).cuda()
    o, lse = torch.empty_like(q), torch.empty(n * new, H, device="cuda")
    ws = torch.empty(api.attn_paged_prefill_workspace_bytes(D), dtype=torch.uint8, device="cuda")
    strides = (ctypes.c_longlong * 6)(*kc.stride()[:3], *vc.stride()[:3])
    check(lib, lambda stream: lib.attn_paged_prefill(q.data_ptr(), kc.data_ptr(), vc.data_ptr(), strides, kc.shape[0], page, tab.data_ptr(), tab.stride(0),
                                                     tab.shape[1], lens.data_ptr(), cu.data_ptr(), o.data_ptr(), lse.data_ptr(), n, n * new, H, Hkv, D,
                                                     0.09, 1, ws.data_ptr(), ws.numel(), stream), (o, lse), skip)


@pytest.mark.parametrize("skip", [0, 1, 4])
@pytest.mark.parametrize("D,n", [(128, 24), (64, 80)])          # lists of one tile, of two
def test_prefix_decode(lib, D, n, skip):
    H, Hkv, dt, length, page = 16, 4, torch.bfloat16, 20100, 16
    kc, vc, tab, _, _ = make_cache([length], Hkv, D, page, dt, "head", 61, dead=0.0)
    tab = wide(tab.expand(n, -1), page, Hkv, D).cuda()          # one sequence's pages for all: what lies in them does not matter here
    lens = torch.full((n,), length, dtype=torch.int32, device="cuda")
    starts, prefix = torch.tensor([0, n], dtype=torch.int32).cuda(), torch.tensor([20000], dtype=torch.int32).cuda()
    q = torch.randn(n, H, D, generator=torch.Generator().manual_seed(7)).to(dt).cuda()
    o, lse = torch.empty_like(q), torch.empty(n, H, device="cuda")
    ws = torch.empty(api.attn_paged_prefix_decode_workspace_bytes(n, H, Hkv, D), dtype=torch.uint8, device="cuda")
    strides = (ctypes.c_longlong * 6)(*kc.stride()[:3], *vc.stride()[:3])
    check(lib, lambda stream: lib.attn_paged_prefix_decode(q.data_ptr(), kc.data_ptr(), vc.data_ptr(), strides, kc.shape[0], page, tab.data_ptr(),
                                                           tab.stride(0), tab.shape[1], lens.data_ptr(), starts.data_ptr(), prefix.data_ptr(), 1,
                                                           o.data_ptr(), lse.data_ptr(), n, H, Hkv, D, 0.09, 1, ws.data_ptr(), ws.numel(), stream),
          (o, lse), skip)
