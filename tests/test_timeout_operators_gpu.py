"""The bounded waits of the decode kernel and of the rotation's gradient, made to run out in the form of tests/test_timeout_gpu.py:
the test build limits waits to 1 ms and leaves out one step's copies.  Every role falls through to the normal end, nothing more is
asked for, the CTA stays until the copies under way have had time to arrive, the status is reported once, and the same call right
afterwards gives the bits of the call before."""
import ctypes

import pytest
import torch

from paper_2506_12355_b200 import api, build
from test_paged_gpu import make_cache
from test_rope_gpu import make, table

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    lib, package = ctypes.CDLL(build.build_wait_test()), api.load()
    for name in api.EXPORTS:
        getattr(lib, name).restype, getattr(lib, name).argtypes = getattr(package, name).restype, getattr(package, name).argtypes
    lib.attn_test_skip_step.restype = None
    lib.attn_test_skip_step.argtypes = [ctypes.c_int]
    return lib


def check(lib, call, outputs, skip):
    stream = torch.cuda.current_stream().cuda_stream

    def run():
        for t in outputs:
            t.zero_()
        assert call(stream) == 0
        return lib.attn_last_device_status(stream)          # synchronises
    assert run() == 0
    before = [t.clone() for t in outputs]
    lib.attn_test_skip_step(skip)
    assert run() == 9
    assert lib.attn_last_device_status(stream) == 0
    assert run() == 0
    assert all(torch.equal(a, b) for a, b in zip(outputs, before))


@pytest.mark.parametrize("skip", [0, 1, 4])
@pytest.mark.parametrize("n,length,page", [(1, 8000, 16), (20, 3000, 16), (20, 3000, 1)])     # clusters of 8, a list of tiles; many small boxes
def test_decode(lib, n, length, page, skip):
    D, H, Hkv, dt = 128, 16, 4, torch.bfloat16
    kc, vc, tab, _, _ = make_cache([length] * n, Hkv, D, page, dt, "head", 60, dead=0.0)
    tab, lens = tab.cuda(), torch.full((n,), length, dtype=torch.int32, device="cuda")
    q = torch.randn(n, H, D, generator=torch.Generator().manual_seed(7)).to(dt).cuda()
    o, lse = torch.empty_like(q), torch.empty(n, H, device="cuda")
    ws = torch.empty(api.attn_paged_decode_workspace_bytes(H, Hkv, D), dtype=torch.uint8, device="cuda")
    strides = (ctypes.c_longlong * 6)(*kc.stride()[:3], *vc.stride()[:3])
    check(lib, lambda stream: lib.attn_paged_decode(q.data_ptr(), kc.data_ptr(), vc.data_ptr(), strides, kc.shape[0], page, tab.data_ptr(), tab.stride(0),
                                                    tab.shape[1], lens.data_ptr(), o.data_ptr(), lse.data_ptr(), n, H, Hkv, D, 0.09, 0, 0, 1,
                                                    ws.data_ptr(), ws.numel(), stream), (o, lse), skip)


@pytest.mark.parametrize("skip", [0, 3, 11])
@pytest.mark.parametrize("B,S,H,Hkv,D", [(2, 2050, 32, 8, 128), (3, 16395, 2, 2, 64)])        # tiles of 8 tokens, of 64
def test_gradient_of_the_rotation(lib, B, S, H, Hkv, D, skip):
    q, k, v, qw, kw = make(B, S, H, Hkv, D, torch.bfloat16, 61)
    g = torch.Generator().manual_seed(62)
    dq, dk, dv = (torch.randn(B, h, S, D, generator=g).bfloat16().cuda() for h in (H, Hkv, Hkv))
    tab = table(S, D).cuda()
    out = [torch.empty(B, S, h, D, dtype=torch.bfloat16, device="cuda") for h in (H, Hkv, Hkv)] + [torch.empty(D, device="cuda") for _ in range(2)]
    ws = torch.empty(api.attn_qk_norm_rope_bwd_workspace_bytes(D), dtype=torch.uint8, device="cuda")
    ins = (ctypes.c_longlong * 6)(*q.stride()[:3], *k.stride()[:3])
    outs = (ctypes.c_longlong * 9)(*(s for t in out[:3] for s in t.stride()[:3]))
    check(lib, lambda stream: lib.attn_qk_norm_rope_bwd(dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), q.data_ptr(), k.data_ptr(), ins, qw.data_ptr(), kw.data_ptr(),
                                                        0, tab.data_ptr(), S, D, 0, None, 1e-6, *(t.data_ptr() for t in out[:3]), outs, out[3].data_ptr(),
                                                        out[4].data_ptr(), B, S, H, Hkv, D, 1, ws.data_ptr(), ws.numel(), stream), out, skip)
