"""The calls with several position axes, of prompts over pages and of shared prefixes on explicit streams, other devices and given
workspaces, on the host with the stand-ins of test_streams_cpu.py."""
import pytest
import torch

from paper_2506_12355_b200 import api
from test_streams_cpu import D, F16, F32, H, HKV, I32, PAGE, PAGES, B, S, Stream, Tensor, world  # noqa: F401


def calls(device=0, ws=None):
    def t(*shape, dtype=F16):
        return Tensor(shape, dtype, device)
    w, tab, of, pos = t(D), t(S, D, dtype=F32), bytes(D // 2), t(2, B, S, dtype=I32)
    qt, kt = t(B, S, H, D), t(B, S, HKV, D)
    kc, table, lens = t(PAGES, HKV, PAGE, D), t(B, 3, dtype=I32), t(B, dtype=I32)
    return dict(
        attn_qk_norm_rope_axes=lambda s: api.attn_qk_norm_rope_axes(qt, kt, kt, w, w, tab, pos, of, stream=s),
        attn_qk_norm_rope_axes_bwd=lambda s: api.attn_qk_norm_rope_axes_bwd(t(B, H, S, D), t(B, HKV, S, D), t(B, HKV, S, D), qt, kt, w, w, tab, pos, of,
                                                                            workspace=ws, stream=s),
        attn_paged_append_axes=lambda s: api.attn_paged_append_axes(t(B, H, D), t(B, HKV, D), t(B, HKV, D), kc, kc, table, lens, t(2, B, dtype=I32), of,
                                                                    cos_sin=tab, stream=s),
        attn_paged_prefill=lambda s: api.attn_paged_prefill(t(7, H, D), kc, kc, table, lens, t(B + 1, dtype=I32), 0.1, workspace=ws, stream=s),
        attn_paged_prefix_decode=lambda s: api.attn_paged_prefix_decode(t(B, H, D), kc, kc, table, lens, t(2, dtype=I32), t(1, dtype=I32), 0.1, workspace=ws,
                                                                        stream=s),
    )


NAMES = sorted(calls())


@pytest.mark.parametrize("name", NAMES)
def test_allocations_belong_to_the_streams_pool(world, name):
    side = Stream(77)
    calls()[name](side)
    assert world.launches == [(name, 77)] and world.made and all(t.stream is side for t in world.made)
    assert world.now.cuda_stream == 0
    calls()[name](None)
    assert world.launches[1:] == [(name, 0)]


@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_another_device(world, name):
    side = Stream(78, 1)
    calls(1)[name](side)
    assert world.launches == [(name, 78)] and all(t.stream is side and t.device.index == 1 for t in world.made)
    with pytest.raises(ValueError):
        calls(1)[name](Stream(79, 0))
    assert len(world.launches) == 1


@pytest.mark.parametrize("name", ["attn_qk_norm_rope_axes_bwd", "attn_paged_prefill", "attn_paged_prefix_decode"])
def test_a_workspace_lies_on_the_calls_device(world, name):
    for bad in (Tensor((8192,), torch.uint8, torch.device("cpu")), Tensor((8192,), torch.uint8, 1), Tensor((8192,), torch.uint8, 0, dense=False)):
        with pytest.raises(ValueError):
            calls(ws=bad)[name](None)
    assert not world.launches


def test_lists_of_another_device_are_refused(world):
    def t(*shape, dtype=F16, device=0):
        return Tensor(shape, dtype, device)
    kc, table, lens, q = t(PAGES, HKV, PAGE, D), t(B, 3, dtype=I32), t(B, dtype=I32), t(B, H, D)
    two, far = t(2, dtype=I32), lambda n: t(n, dtype=I32, device=1)
    for call in (lambda: api.attn_paged_prefill(q, kc, kc, table, lens, far(B + 1), 0.1),
                 lambda: api.attn_paged_prefix_decode(q, kc, kc, table, lens, far(2), t(1, dtype=I32), 0.1),
                 lambda: api.attn_paged_prefix_decode(q, kc, kc, table, lens, two, far(1), 0.1)):
        with pytest.raises(ValueError):
            call()
    assert not world.launches
