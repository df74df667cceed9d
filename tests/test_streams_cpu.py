"""Calls with an explicit stream, on the host: what such a call allocates has to belong to that stream, whatever torch's current one
is.  A block taken from the current stream's pool and dropped at return may be handed out again while the kernels on the other
stream still use it.  A GPU can only show this by losing the race, so the tensors, the streams and the library are stand-ins here."""
import contextlib
import types

import pytest
import torch

from paper_2506_12355_b200 import api


class Tensor:
    """What the binding asks of a tensor."""
    next_address = 1 << 20

    def __init__(self, shape, dtype, device=0, stream=None, dense=True):
        self.shape, self.dtype, self.stream, self.dense = torch.Size(shape), dtype, stream, dense
        self.device = torch.device("cuda", device) if isinstance(device, int) else device
        self.address = Tensor.next_address
        Tensor.next_address += 1 << 20

    is_cuda = property(lambda t: t.device.type == "cuda")

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return self.device.index

    def stride(self, axis=None):
        s, n = [], 1
        for x in reversed(self.shape):
            s.insert(0, n)
            n *= x
        return tuple(s) if axis is None else s[axis]

    def is_contiguous(self):
        return self.dense

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def data_ptr(self):
        return self.address


class Stream:
    def __init__(self, handle, device=0):
        self.cuda_stream, self.device = handle, torch.device("cuda", device)


class World:
    """Stand-ins for torch (allocations and streams) and for the library (launches)."""

    def __init__(self):
        self.now, self.made, self.launches = Stream(0), [], []
        world = self

        @contextlib.contextmanager
        def stream(s):
            before, world.now = world.now, s
            try:
                yield
            finally:
                world.now = before

        @contextlib.contextmanager
        def device(d):
            before, index = world.now, torch.device(d).index
            if index != before.device.index:
                world.now = Stream(0, index)
            try:
                yield
            finally:
                world.now = before

        def external(handle, device=None):
            assert handle != 0          # (torch makes a new stream of that)
            return Stream(handle, torch.device(device).index)

        def empty(shape, dtype=None, device=None):
            t = Tensor((shape,) if isinstance(shape, int) else shape, dtype, device, world.now)
            world.made.append(t)
            return t

        cuda = types.SimpleNamespace(Stream=Stream, ExternalStream=external, stream=stream, device=device, current_stream=lambda: world.now,
                                     current_device=lambda: world.now.device.index, default_stream=lambda d: Stream(0, torch.device(d).index))
        self.torch = types.SimpleNamespace(cuda=cuda, empty=empty, empty_like=lambda t: empty(t.shape, t.dtype, t.device), float16=torch.float16,
                                           bfloat16=torch.bfloat16, float32=torch.float32, int32=torch.int32, uint8=torch.uint8, float8_e4m3fn=torch.float8_e4m3fn,
                                           device=torch.device, Tensor=torch.Tensor)

    def __getattr__(self, name):      # the library's functions
        if name.endswith("_bytes"):
            return lambda *args: 4096
        return lambda *args: self.launches.append((name, args[-1])) or 0


@pytest.fixture
def world(monkeypatch):
    w = World()
    monkeypatch.setattr(api, "torch", w.torch)
    monkeypatch.setattr(api, "_lib", w)
    monkeypatch.setattr(api, "_binding_module", None)
    monkeypatch.setattr(api, "_raw_stream", None)
    monkeypatch.setattr(api, "_set_stream", None)
    return w


F16, F32, I32 = torch.float16, torch.float32, torch.int32
B, H, HKV, S, D, PAGES, PAGE = 2, 4, 2, 40, 64, 9, 16


def calls(device=0):
    """name -> a call of every entry point that allocates, taking the stream."""
    def t(*shape, dtype=F16):
        return Tensor(shape, dtype, device)
    q, k, v = t(B, H, S, D), t(B, HKV, S, D), t(B, HKV, S, D)
    o, lse = t(B, H, S, D), t(B, H, S, dtype=F32)
    qt, kt, vt, w = t(B, S, H, D), t(B, S, HKV, D), t(B, S, HKV, D), t(D)
    tab = t(S, D, dtype=F32)
    kc, vc = t(PAGES, HKV, PAGE, D), t(PAGES, HKV, PAGE, D)
    table, lens = t(B, 3, dtype=I32), t(B, dtype=I32)
    b8 = lambda *shape: t(*shape, dtype=torch.uint8)
    return dict(
        attn_fwd=lambda s: api.attn_fwd(q, t(B, H, S, D), t(B, H, S, D), 0.1, stream=s),
        attn_fwd_simt=lambda s: api.attn_fwd_simt(q, t(B, H, S, D), t(B, H, S, D), 0.1, stream=s),
        attn_fwd_gqa=lambda s: api.attn_fwd_gqa(q, k, v, 0.1, stream=s),
        attn_fwd_partial=lambda s: api.attn_fwd_partial(q, k, v, 0.1, False, 0, stream=s),
        attn_combine=lambda s: api.attn_combine(t(3, B, H, S, D), t(3, B, H, S, dtype=F32), stream=s),
        attn_fwd_qkv_dims=lambda s: api.attn_fwd_qkv_dims(q, k, v, 0.1, stream=s),
        attn_fwd_splitkv=lambda s: api.attn_fwd_splitkv(q, k, v, 0.1, False, 2, stream=s),
        attn_fwd_fp8=lambda s: api.attn_fwd_fp8(b8(B, H, S, 128), b8(B, HKV, S, 128), b8(B, HKV, S, 128), 0.1, stream=s),
        attn_bwd=lambda s: api.attn_bwd(q, k, v, o, lse, o, 0.1, stream=s),
        attn_fwd_window=lambda s: api.attn_fwd_window(q, k, v, 0.1, 8, 1, stream=s),
        attn_bwd_window=lambda s: api.attn_bwd_window(q, k, v, o, lse, o, 0.1, 8, 1, stream=s),
        attn_qk_norm_rope=lambda s: api.attn_qk_norm_rope(qt, kt, vt, w, w, tab, stream=s),
        attn_qk_norm_rope_bwd=lambda s: api.attn_qk_norm_rope_bwd(o, t(B, HKV, S, D), t(B, HKV, S, D), qt, kt, w, w, tab, stream=s),
        attn_paged_append=lambda s: api.attn_paged_append(t(B, H, D), t(B, HKV, D), t(B, HKV, D), kc, vc, table, lens, stream=s),
        attn_paged_decode=lambda s: api.attn_paged_decode(t(B, H, D), kc, vc, table, lens, 0.1, stream=s),
    )


NAMES = sorted(calls())


@pytest.mark.parametrize("name", NAMES)
def test_allocations_belong_to_the_streams_pool(world, name):
    side = Stream(77)
    calls()[name](side)
    assert world.launches == [(name, 77)]
    assert world.made and all(t.stream is side for t in world.made)
    assert world.now.cuda_stream == 0                   # the caller's current stream is as it was


@pytest.mark.parametrize("name", NAMES)
def test_without_a_stream_the_current_one_is_taken(world, name):
    calls()[name](None)
    assert world.launches == [(name, 0)] and all(t.stream is world.now for t in world.made)


@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_another_device(world, name):
    side = Stream(78, 1)
    calls(1)[name](side)
    assert world.launches == [(name, 78)] and all(t.stream is side and t.device.index == 1 for t in world.made)
    calls(1)[name](None)
    assert world.launches[1:] == [(name, 0)]
    with pytest.raises(ValueError):                     # a stream of another device than the tensors'
        calls(1)[name](Stream(79, 0))
    assert len(world.launches) == 2


@pytest.mark.parametrize("handle", [0, 80])
def test_a_handle_of_another_library_is_wrapped(world, handle):
    for device in (0, 1):
        calls(device)["attn_paged_decode"](types.SimpleNamespace(cuda_stream=handle))
        assert world.launches.pop() == ("attn_paged_decode", handle)
        assert all(t.stream.cuda_stream == handle and t.stream.device.index == t.device.index for t in world.made)


def workspace_calls():
    """name -> a call of every entry point that takes a workspace, taking that."""
    def t(*shape, dtype=F16):
        return Tensor(shape, dtype)
    q, k, v = t(B, H, S, D), t(B, HKV, S, D), t(B, HKV, S, D)
    lse, w, tab = t(B, H, S, dtype=F32), t(D), t(S, D, dtype=F32)
    qt, kt = t(B, S, H, D), t(B, S, HKV, D)
    kc, table, lens = t(PAGES, HKV, PAGE, D), t(B, 3, dtype=I32), t(B, dtype=I32)
    return dict(
        attn_fwd_splitkv=lambda x, **s: api.attn_fwd_splitkv(q, k, v, 0.1, False, 2, workspace=x, **s),
        attn_bwd=lambda x, **s: api.attn_bwd(q, k, v, q, lse, q, 0.1, workspace=x, **s),
        attn_bwd_window=lambda x, **s: api.attn_bwd_window(q, k, v, q, lse, q, 0.1, 8, 1, workspace=x, **s),
        attn_qk_norm_rope_bwd=lambda x, **s: api.attn_qk_norm_rope_bwd(q, k, v, qt, kt, w, w, tab, workspace=x, **s),
        attn_paged_decode=lambda x, **s: api.attn_paged_decode(t(B, H, D), kc, kc, table, lens, 0.1, workspace=x, **s),
    )


@pytest.mark.parametrize("name", sorted(workspace_calls()))
def test_a_workspace_lies_on_the_calls_device(world, name):
    """Its address goes to the kernels as it is: host memory, another GPU's, or a view with gaps is refused before a launch."""
    call = workspace_calls()[name]
    for bad in (Tensor((8192,), torch.uint8, torch.device("cpu")), Tensor((8192,), torch.uint8, 1), Tensor((8192,), torch.uint8, 0, dense=False)):
        for stream in (None, Stream(81)):
            with pytest.raises(ValueError):
                call(bad, stream=stream)
    assert not world.launches
    call(Tensor((8192,), torch.uint8))
    assert [n for n, _ in world.launches] == [name]


def test_a_workspace_of_another_type_counts_in_bytes(world, monkeypatch):
    seen = []
    world.attn_bwd = lambda *args: seen.append(args[-2]) or 0
    workspace_calls()["attn_bwd"](Tensor((2048,), F32))
    assert seen == [8192]


def test_inputs_of_two_devices_are_refused(world):
    """One call reads memory of one GPU: a tensor of another would reach the kernels as an address that they may not read."""
    def t(*shape, dtype=F16, device=0):
        return Tensor(shape, dtype, device)
    q, k = t(B, H, S, D), t(B, HKV, S, D)
    lse, far_q, far_k, far_lse = t(B, H, S, dtype=F32), t(B, H, S, D, device=1), t(B, HKV, S, D, device=1), t(B, H, S, dtype=F32, device=1)
    b8, far_b8 = t(B, H, S, 128, dtype=torch.uint8), t(B, H, S, 128, dtype=torch.uint8, device=1)
    for call in (lambda: api.attn_fwd(q, far_q, q, 0.1), lambda: api.attn_fwd(q, q, far_q, 0.1), lambda: api.attn_fwd_simt(far_q, q, q, 0.1),
                 lambda: api.attn_fwd_gqa(q, far_k, k, 0.1), lambda: api.attn_fwd_partial(q, k, far_k, 0.1, False, 0),
                 lambda: api.attn_fwd_qkv_dims(q, k, far_k, 0.1), lambda: api.attn_fwd_splitkv(q, far_k, far_k, 0.1, False, 2),
                 lambda: api.attn_fwd_fp8(b8, far_b8, b8, 0.1), lambda: api.attn_combine(t(3, B, H, S, D), t(3, B, H, S, dtype=F32, device=1)),
                 lambda: api.attn_fwd_window(q, far_k, k, 0.1, 8), lambda: api.attn_fwd_window(q, k, far_k, 0.1, 8),
                 lambda: api.attn_bwd_window(q, k, far_k, q, lse, q, 0.1, 8), lambda: api.attn_bwd_window(q, k, k, far_q, lse, q, 0.1, 8),
                 lambda: api.attn_bwd(q, far_k, k, q, lse, q, 0.1), lambda: api.attn_bwd(q, k, k, far_q, lse, q, 0.1),
                 lambda: api.attn_bwd(q, k, k, q, far_lse, q, 0.1), lambda: api.attn_bwd(q, k, k, q, lse, far_q, 0.1)):
        with pytest.raises(ValueError):
            call()
    assert not world.launches
