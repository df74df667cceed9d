"""Refusals of attn_paged_prefill and attn_paged_prefix_decode, decided on the host (CPU only)."""
import pytest
import torch

from paper_2506_12355_b200 import api, build
from test_abi import no_device
from test_cache_abi import ll


@pytest.fixture(scope="module")
def lib():
    build.build()
    return api.load()


CS = (2048, 1024, 64, 2048, 1024, 64)


def test_validation(lib):
    def f(q=0x1000, kc=0x5000, vc=0x6000, cs=CS, pages=4, page=16, bt=0x700, mp=4, lens=0x800, cu=0x900, o=0x2000, lse=0x3000, n=3, T=9, H=4, Hkv=2,
          D=64, scale=0.1, dtype=0, ws=0x10000, ws_n=1 << 28):
        return lib.attn_paged_prefill(q, kc, vc, ll(*cs), pages, page, bt, 4, mp, lens, cu, o, lse, n, T, H, Hkv, D, scale, dtype, ws, ws_n, None)

    def g(q=0x1000, kc=0x5000, vc=0x6000, cs=CS, pages=4, page=16, bt=0x700, mp=4, lens=0x800, cu=0x900, o=0x2000, lse=0x3000, n=2, T=9, H=4, Hkv=2,
          D=64, scale=0.1, dtype=0, ws=0x10000, ws_n=1 << 28, pl=0xa00):
        return lib.attn_paged_prefix_decode(q, kc, vc, ll(*cs), pages, page, bt, 4, mp, lens, cu, pl, n, o, lse, T, H, Hkv, D, scale, dtype, ws, ws_n, None)
    for call in (f, g):
        for name in ("q", "kc", "vc", "bt", "lens", "cu", "o", "lse"):
            assert call(**{name: None}) == 1, name
        assert call(n=-1) == 2 and call(T=-1) == 2 and call(Hkv=3) == 2 and call(Hkv=0) == 2 and call(H=258) == 2 and call(page=12) == 2 and call(mp=-1) == 2
        assert call(T=2 ** 30) == 2                                           # more rows than 32 bits count
        for D in (0, 96, 256):
            assert call(D=D) == 3
        assert call(dtype=2) == 4 and call(q=0x1008) == 5 and call(lse=0x3002) == 5 and call(cu=0x902) == 5
        assert call(cs=(2048, 1024, 60) * 2) == 5 and call(cs=(0, 1024, 64) * 2) == 2
        assert call(scale=float("inf")) == 6 and call(scale=-1.0) == 6
        assert call(ws=None) == 10 and call(ws=0x10010) == 10 and call(ws_n=1000) == 10
        assert call(T=0) == 0 and call(H=0, Hkv=0) == 0
        if no_device():
            assert call() in (7, 8) and call(H=256, D=128) in (7, 8)
    assert f(pages=0, kc=None, vc=None) == 2 and f(mp=0) == 2 and f(n=0) == 0
    assert g(pl=None) == 1 and g(pl=0xa02) == 5
    if no_device():
        assert g(n=0, cu=None, pl=None) in (7, 8)


def test_workspaces(lib):
    up = lambda n: (n + 255) // 256 * 256
    # two partial results of 256 rows per SM, and what the joining kernels read beside them
    assert lib.attn_paged_prefill_workspace_bytes(128) == 2 * 148 * 256 * 130 * 4 + up(148 * 20) and lib.attn_paged_prefill_workspace_bytes(64) == 2 * 148 * 256 * 66 * 4 + up(148 * 20)
    assert lib.attn_paged_prefill_workspace_bytes(256) == 0
    b = lib.attn_paged_prefix_decode_workspace_bytes
    rows, plan, prefix_plan = up(64 * 32 * 130 * 4), up(65 * 16), up(65 * 32)
    assert b(64, 32, 8, 128) == lib.attn_paged_decode_workspace_bytes(32, 8, 128) + 2 * rows + plan + prefix_plan + 2 * 148 * 256 * 130 * 4
    assert b(-1, 32, 8, 128) == 0 and b(4, 3, 2, 64) == 0 and b(4, 4, 2, 256) == 0


def test_binding_refuses_wrong_tensors():
    q = torch.zeros(3, 4, 64, dtype=torch.float16)
    c = torch.zeros(4, 2, 16, 64, dtype=torch.float16)
    bt, lens = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        api.attn_paged_prefill(q, c, c, bt, lens, torch.zeros(4, dtype=torch.int32), 0.1)          # not on a GPU
    with pytest.raises(ValueError):
        api.attn_paged_prefill(q[0], c, c, bt, lens, torch.zeros(4, dtype=torch.int32), 0.1)
    with pytest.raises(TypeError):
        api.attn_paged_prefix_decode(q.float(), c, c, bt, lens, torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 0.1)
    with pytest.raises(ValueError):
        api.attn_paged_prefix_decode(q, c, c, bt, lens, torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 0.1)
