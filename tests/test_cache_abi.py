"""Refusals of the normalisation/rotation and paged-cache entry points: decided on the host, before a device is looked at (the
pointers are fake), and the checks of the Python binding (CPU only)."""
import ctypes

import pytest
import torch

from paper_2506_12355_b200 import api, build
from test_abi import no_device


@pytest.fixture(scope="module")
def lib():
    build.build()
    return api.load()


def ll(*v):
    return (ctypes.c_longlong * len(v))(*v)


def test_norm_rope_validation(lib):
    def f(q=0x1000, k=0x2000, v=0x3000, st=None, qw=0x100, kw=0x200, f32=0, tab=0x400, n=128, R=64, inter=0, pos=None, eps=1e-6, qo=0x4000,
          ko=0x5000, vo=0x6000, B=1, S=128, H=4, Hkv=2, D=64, dtype=0):
        st = ll(*([64 * 128, 64, 64] * 3)) if st is None else st
        return lib.attn_qk_norm_rope(q, k, v, st, qw, kw, f32, tab, n, R, inter, pos, eps, qo, ko, vo, B, S, H, Hkv, D, dtype, None)
    for name in ("q", "k", "qo", "ko", "tab", "v", "vo"):
        assert f(**{name: None}) == 1, name
    for name in ("B", "S", "H", "Hkv"):
        assert f(**{name: -1}) == 2
    for R in (-16, 8, 20, 80):
        assert f(R=R) == 2
    assert f(S=129) == 2 and f(n=0) == 2                # positions beyond the table
    for D in (0, 32, 96, 512):
        assert f(D=D) == 3
    assert f(dtype=2) == 4
    for name in ("q", "k", "v", "qo", "ko", "vo", "qw", "kw", "tab"):
        assert f(**{name: 0x1008}) == 5, name
    assert f(pos=0x1002) == 5
    assert f(st=ll(8192, 64, 4, *([8192, 64, 64] * 2))) == 5
    assert f(eps=-1.0) == 6 and f(eps=float("nan")) == 6
    assert f(B=0) == 0 and f(S=0) == 0 and f(H=0, Hkv=0) == 0
    if no_device():
        assert f() in (7, 8) and f(v=None, vo=None) in (7, 8) and f(R=0, tab=None, n=0) in (7, 8) and f(qw=None, kw=None) in (7, 8)


def test_norm_rope_bwd_validation(lib):
    assert lib.attn_qk_norm_rope_bwd_workspace_bytes(64) == 148 * 2 * 64 * 4 and lib.attn_qk_norm_rope_bwd_workspace_bytes(96) == 0

    def f(dq=0x1000, dk=0x2000, dv=0x3000, q=0x7000, k=0x8000, qw=0x100, kw=0x200, tab=0x400, n=128, R=64, eps=1e-6, dqi=0x4000, dki=0x5000,
          dvi=0x6000, out=None, dqw=0x500, dkw=0x600, B=1, S=128, H=4, Hkv=2, D=64, dtype=0, ws=0x10000, ws_n=1 << 22):
        out = ll(*([64 * 128, 64, 64] * 3)) if out is None else out
        return lib.attn_qk_norm_rope_bwd(dq, dk, dv, q, k, ll(*([8192, 64, 64] * 2)), qw, kw, 0, tab, n, R, 0, None, eps, dqi, dki, dvi, out, dqw,
                                         dkw, B, S, H, Hkv, D, dtype, ws, ws_n, None)
    for name in ("dq", "dk", "dv", "q", "k", "dqi", "dki", "dvi", "dqw", "dkw", "tab"):
        assert f(**{name: None}) == 1, name
    assert f(B=-1) == 2 and f(R=24) == 2 and f(S=200) == 2 and f(D=96) == 3 and f(dtype=5) == 4
    assert f(dqi=0x4008) == 5 and f(dqw=0x502) == 5 and f(eps=float("inf")) == 6
    assert f(out=ll(8192, 0, 64, *([8192, 64, 64] * 2))) == 2             # gradient rows on top of each other
    assert f(ws=None) == 10 and f(ws=0x10010) == 10 and f(ws_n=1000) == 10
    if no_device():
        assert f() in (7, 8) and f(qw=None, q=None, dqw=None) in (7, 8) and f(dv=None, dvi=None) in (7, 8)


def test_window_validation(lib):
    def f(q=0x1000, k=0x2000, v=0x3000, o=0x4000, lse=0x5000, B=1, H=4, Hkv=2, Sq=128, Sk=256, D=128, scale=0.1, W=16, sinks=2, off=0, dtype=1):
        return lib.attn_fwd_window(q, k, v, o, lse, B, H, Hkv, Sq, Sk, D, scale, W, sinks, off, dtype, None)

    def b(q=0x1000, k=0x2000, v=0x3000, o=0x4000, lse=0x5000, B=1, H=4, Hkv=2, Sq=128, Sk=256, D=128, scale=0.1, W=16, sinks=2, off=0, dtype=1,
          dout=0x6000, dq=0x7000, dk=0x8000, dv=0x9000, ws=0x10000, ws_n=1 << 28):
        return lib.attn_bwd_window(q, k, v, o, lse, dout, dq, dk, dv, B, H, Hkv, Sq, Sk, D, scale, W, sinks, off, dtype, ws, ws_n, None)
    for call in (f, b):
        for name in ("q", "k", "v", "o", "lse"):
            assert call(**{name: None}) == 1, name
        assert call(W=-1) == 2 and call(sinks=-1) == 2 and call(off=-1) == 2 and call(off=2 ** 31 - 300) == 2
        assert call(B=-1) == 2 and call(Hkv=3) == 2
        for D in (256, 96, 0):
            assert call(D=D) == 3
        assert call(dtype=2) == 4 and call(q=0x1008) == 5 and call(scale=float("nan")) == 6
        if no_device():
            assert call() in (7, 8) and call(W=0) in (7, 8) and call(W=2 ** 31 - 1, sinks=2 ** 31 - 1) in (7, 8)
    assert f(Sq=0) == 0 and b(Sq=0, Sk=0) == 0
    for name in ("dout", "dq", "dk", "dv"):
        assert b(**{name: None}) == 1
    assert b(ws=None) == 10 and b(ws_n=64) == 10
    # partial sums of the first keys' gradients: none without such keys, and bounded when all keys are first keys
    plain = lib.attn_bwd_workspace_bytes(1, 32, 16384)
    assert lib.attn_bwd_window_workspace_bytes(1, 32, 8, 16384, 16384, 128, 1024, 0, 0) == plain
    assert 0 < lib.attn_bwd_window_workspace_bytes(1, 32, 8, 16384, 16384, 128, 1024, 4, 0) - plain < 200 << 20
    for s in (128, 500, 2000, 5000, 16384, 2 ** 31 - 1):
        assert lib.attn_bwd_window_workspace_bytes(1, 32, 8, 16384, 16384, 128, 64, s, 0) - plain < 200 << 20
    assert lib.attn_bwd_window_workspace_bytes(1, 2, 2, 100, 100, 64, 10, 0, 0) >= lib.attn_bwd_workspace_bytes(1, 2, 100)
    assert lib.attn_bwd_window_workspace_bytes(-1, 2, 2, 100, 100, 64, 10, 0, 0) == 0


def test_append_validation(lib):
    def f(q=0x1000, k=0x2000, v=0x3000, st=None, tab=None, n=0, R=0, eps=1e-6, qo=0x4000, kc=0x5000, vc=0x6000, cs=None, pages=4, page=16,
          bt=0x700, ts=4, mp=4, lens=0x800, cu=None, seqs=3, tokens=3, H=4, Hkv=2, D=64, dtype=0):
        st = ll(64 * 8, 64, 64 * 8, 64, 64 * 8, 64) if st is None else st
        cs = ll(2048, 1024, 64, 2048, 1024, 64) if cs is None else cs
        return lib.attn_paged_append(q, k, v, st, None, None, 0, tab, n, R, 0, eps, qo, kc, vc, cs, pages, page, bt, ts, mp, lens, cu, seqs, tokens,
                                     H, Hkv, D, dtype, None)
    for name in ("q", "k", "v", "qo", "kc", "vc", "bt", "lens"):
        assert f(**{name: None}) == 1, name
    assert f(tokens=4) == 2 and f(seqs=-1) == 2 and f(tokens=-1) == 2
    for page in (0, 3, 24, -16):
        assert f(page=page) == 2
    assert f(mp=1 << 27, page=16) == 2 and f(pages=-1) == 2
    assert f(R=64) == 2 and f(R=64, n=5) == 1
    assert f(D=80) == 3 and f(dtype=2) == 4
    assert f(kc=0x5008) == 5 and f(cs=ll(2048, 1024, 60, 2048, 1024, 64)) == 5 and f(st=ll(512, 64, 512, 63, 512, 64)) == 5 and f(lens=0x802) == 5
    assert f(cs=ll(0, 1024, 64, 2048, 1024, 64)) == 2                     # pages on top of each other
    assert f(eps=-1.0) == 6
    assert f(tokens=0, seqs=0) == 0
    if no_device():
        assert f() in (7, 8) and f(q=None, qo=None) in (7, 8) and f(cu=0x900, tokens=9) in (7, 8)


def test_decode_validation(lib):
    ws_bytes = lib.attn_paged_decode_workspace_bytes
    # two partial results per SM, each of as many heads as a tile covers (a power of two that divides them, at most 8)
    assert ws_bytes(8, 2, 128) == (2 * 148 * 2 * 8 * 130 * 4 + 255) // 256 * 256
    assert ws_bytes(40, 2, 64) == (2 * 148 * 4 * 16 * 66 * 4 + 255) // 256 * 256 and ws_bytes(3, 2, 64) == 0 and ws_bytes(2, 2, 96) == 0
    assert ws_bytes(64, 64, 64) == (2 * 148 * 8 * 8 * 66 * 4 + 255) // 256 * 256

    def f(q=0x1000, kc=0x5000, vc=0x6000, cs=None, pages=4, page=16, bt=0x700, ts=4, mp=4, lens=0x800, o=0x2000, lse=0x3000, B=3, H=4, Hkv=2, D=64,
          scale=0.1, window=0, sinks=0, dtype=0, ws=0x10000, ws_n=1 << 24):
        cs = ll(2048, 1024, 64, 2048, 1024, 64) if cs is None else cs
        return lib.attn_paged_decode(q, kc, vc, cs, pages, page, bt, ts, mp, lens, o, lse, B, H, Hkv, D, scale, window, sinks, dtype, ws, ws_n, None)
    for name in ("q", "kc", "vc", "bt", "lens", "o", "lse"):
        assert f(**{name: None}) == 1, name
    assert f(B=-1) == 2 and f(Hkv=3) == 2 and f(window=-1) == 2 and f(sinks=-1) == 2 and f(page=12) == 2 and f(mp=-1) == 2
    assert f(D=96) == 3 and f(dtype=2) == 4 and f(q=0x1008) == 5 and f(lse=0x3002) == 5
    for cs in (ll(0, 1024, 64, 2048, 1024, 64), ll(2048, 1024, 64, 2048, 0, 64), ll(2048, -1024, 64, 2048, 1024, 64), ll(1 << 39, 1024, 64, 2048, 1024, 64)):
        assert f(cs=cs) == 2                                              # strides that the copies cannot take
    assert f(scale=float("nan")) == 6 and f(scale=-1.0) == 6
    assert f(ws=None) == 10 and f(ws=0x10010) == 10 and f(ws_n=100) == 10
    assert f(B=0) == 0 and f(H=0, Hkv=0) == 0
    if no_device():
        assert f() in (7, 8) and f(pages=0, kc=None, vc=None) in (7, 8)


def test_binding_refuses_wrong_tensors():
    x = torch.zeros(1, 8, 4, 64, dtype=torch.float16)
    w = torch.ones(64, dtype=torch.float16)
    tab = torch.zeros(8, 64)
    with pytest.raises(ValueError):
        api.attn_qk_norm_rope(x[0], x, x, w, w, tab)
    with pytest.raises(ValueError):
        api.attn_qk_norm_rope(x, x[:, :4], x, w, w, tab)
    with pytest.raises(TypeError):
        api.attn_qk_norm_rope(x.float(), x, x, w, w, tab)
    with pytest.raises(ValueError):
        api.attn_qk_norm_rope(x, x, x, w, w, tab)                    # not on a GPU
    c = torch.zeros(4, 2, 16, 64, dtype=torch.float16)
    bt, lens = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        api.attn_paged_decode(torch.zeros(3, 4, 64, dtype=torch.float16), c, c, bt, lens, 0.1)
    with pytest.raises(ValueError):
        api.attn_paged_append(None, torch.zeros(3, 2, 64, dtype=torch.float16), torch.zeros(3, 2, 64, dtype=torch.float16), c, c, bt, lens)


def test_extension_is_built_and_refuses_what_is_not_plain():
    build.build()
    b = api._bind()
    assert b is not None
    x = torch.zeros(1, 8, 4, 64, dtype=torch.float16)
    # CPU tensors, wrong argument counts and wrong types go back to the Python path, which reports them
    assert b.attn_fwd_window(x, x, x, 0.1, 4, 0, 0, None, None) is NotImplemented
    assert b.attn_fwd_window(x, x, x) is NotImplemented
    assert b.attn_paged_decode(1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11) is NotImplemented
    with pytest.raises(ValueError):
        b.bind([1, 2])
