"""Refusals of the calls with several position axes, decided on the host, and rope_pair_axes (CPU only)."""
import pytest
import torch

from paper_2506_12355_b200 import api, build
from test_abi import no_device
from test_cache_abi import ll


@pytest.fixture(scope="module")
def lib():
    build.build()
    return api.load()


OF = bytes([0] * 8 + [1] * 12 + [2] * 12)


def test_rope_axes_validation(lib):
    def f(q=0x1000, tab=0x400, n=128, R=64, pos=0x700, axes=3, of=OF, S=128, B=1, D=64, eps=1e-6):
        st = ll(*([64 * 128, 64, 64] * 3))
        return lib.attn_qk_norm_rope_axes(q, 0x2000, 0x3000, st, 0x100, 0x200, 0, tab, n, R, 0, pos, axes, of, eps, 0x4000, 0x5000, 0x6000, B, S, 4,
                                          2, D, 0, None)

    def b(q=0x1000, tab=0x400, n=128, R=64, pos=0x700, axes=3, of=OF, S=128, B=1, D=64, eps=1e-6, ws=0x10000):
        st = ll(*([64 * 128, 64, 64] * 3))
        return lib.attn_qk_norm_rope_axes_bwd(0x1000, 0x2000, 0x3000, q, 0x8000, st, 0x100, 0x200, 0, tab, n, R, 0, pos, axes, of, eps, 0x4000, 0x5000,
                                              0x6000, st, 0x500, 0x600, B, S, 4, 2, D, 0, ws, 1 << 22, None)

    def a(q=0x1000, tab=0x400, n=128, R=64, pos=0x700, axes=3, of=OF, S=3, D=64, eps=1e-6):
        st, cs = ll(512, 64, 512, 64, 512, 64), ll(2048, 1024, 64, 2048, 1024, 64)
        return lib.attn_paged_append_axes(q, 0x2000, 0x3000, st, None, None, 0, tab, n, R, 0, pos, axes, of, eps, 0x4000, 0x5000, 0x6000, cs, 4, 16,
                                          0x700, 4, 4, 0x800, None, S, S, 4, 2, D, 0, None)
    for call in (f, b, a):
        assert call(pos=None) == 1 and call(of=None) == 1 and call(tab=None) == 1 and call(q=None) == 1
        for axes in (0, -1, 2, 5):                          # 2: pairs of an axis that is not there
            assert call(axes=axes) == 2, axes
        assert call(R=24) == 2 and call(n=0) == 2 and call(D=96) == 3
        assert call(pos=0x702) == 5 and call(eps=-1.0) == 6
        if no_device():
            assert call() in (7, 8) and call(axes=4) in (7, 8) and call(R=0, of=None, tab=None, n=0) in (7, 8)
    assert f(S=0, pos=None) == 0 and a(S=0, pos=None) == 0
    if no_device():
        assert f(S=500) in (7, 8)                           # positions are given, so the table may be shorter than the sequence
    assert b(ws=None) == 10


def test_pair_axes():
    assert api.rope_pair_axes((2, 1, 3)) == bytes([0, 0, 1, 2, 2, 2])
    assert api.rope_pair_axes((4, 2, 1), "cyclic") == bytes([0, 1, 2, 0, 1, 0, 0])
    assert api.rope_pair_axes((0, 2), "cyclic") == bytes([1, 1]) and api.rope_pair_axes((3,)) == bytes(3)
    for sections in ((), (1, 1, 1, 1, 1), (4, -1)):
        with pytest.raises(ValueError):
            api.rope_pair_axes(sections)
    with pytest.raises(ValueError):
        api.rope_pair_axes((1, 1), "other")


def test_binding_refuses_wrong_positions():
    pos, tokens, dev = torch.zeros(2, 1, 8, dtype=torch.int32), (1, 8), torch.device("cpu")
    assert api._where(pos, [0] * 4 + [1] * 4, 16, tokens, dev) == (pos.data_ptr(), 2, bytes([0] * 4 + [1] * 4))
    for bad, of in ((None, bytes(8)), (pos[0], bytes(8)), (pos, bytes(7)), (pos, bytes([2] * 8)), (torch.zeros(5, 1, 8, dtype=torch.int32), bytes(8)),
                    (pos[:, :, :7], bytes(8)), (torch.zeros(8, 1, 2, dtype=torch.int32).permute(2, 1, 0), bytes(8))):
        with pytest.raises(ValueError):
            api._where(bad, of, 16, tokens, dev)
    with pytest.raises(TypeError):
        api._where(pos.long(), bytes(8), 16, tokens, dev)
    with pytest.raises(TypeError):
        api._where(pos, 8, 16, tokens, dev)
    x, w = torch.zeros(1, 8, 4, 64, dtype=torch.float16), torch.ones(64, dtype=torch.float16)
    with pytest.raises(ValueError):
        api.attn_qk_norm_rope_axes(x, x, x, w, w, torch.zeros(8, 64), pos, None)
    with pytest.raises(ValueError):
        api.attn_qk_norm_rope_axes(x, x, x, w, w, torch.zeros(8, 64), pos, bytes(32))      # not on a GPU
