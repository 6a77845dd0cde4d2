"""What the Python entry points of the decoding operators pass to the C calls, and
what they refuse, with stand-ins for device tensors: nothing is enqueued."""
import contextlib

import numpy as np
import pytest
import torch

from paper_2605_31598_gb300 import qcache, rotary


class OnDevice:
    """A CPU tensor that says it is on a CUDA device."""
    is_cuda = True

    def __init__(self, x, device=0):
        self.x, self.index = x, device

    def get_device(self):
        return self.index

    def __getattr__(self, name):
        return getattr(self.x, name)


class MropeCall:
    """Stands for the C call of ``mrope``; keeps the fields of its arguments."""
    NAMES = ("tokens", "hq", "hk", "d", "axes", "pairs", "adjacent", "transpose", "scale", "freq", "axis", "positions",
             "position_stride", "q", "k", "q_out", "k_out", "q_stride", "k_stride", "q_out_stride", "k_out_stride")

    def __init__(self, monkeypatch):
        self.args = None
        monkeypatch.setattr(rotary, "_call", lambda: (lambda args, stream: 0, self.pack))
        monkeypatch.setattr(rotary, "raw_stream", lambda stream, x: 0)

    def pack(self, *fields):
        self.args = dict(zip(self.NAMES, fields))


def turn(positions, tokens, **kw):
    q = OnDevice(torch.zeros((tokens, 2, 64), dtype=torch.bfloat16))
    freq, axis = rotary.mrope_frequencies((8, 12, 12)[:positions.shape[0]], 1e4)
    return rotary.mrope(q, None, OnDevice(positions), freq, axis, q_out=q, **kw)


@pytest.mark.parametrize("positions", [
    torch.arange(40, 47, dtype=torch.int32).expand(3, 7),                       # text: one row for all axes
    torch.tensor([9], dtype=torch.int32).expand(3, 1),
    torch.arange(40, 52, dtype=torch.int32).expand(3, 12)[:, 2:9],              # a slice of such a row
    torch.arange(60, dtype=torch.int32).view(3, 20)[:, 4:11],
    torch.arange(60, dtype=torch.int32).view(3, 20)[1:2, 4:11],
    torch.arange(9, dtype=torch.int32)[:, None][3:6],                           # a column
    torch.arange(30, dtype=torch.int32).as_strided((3, 10), (8, 1)),            # wider than the call's tokens and its stride
    torch.arange(7, dtype=torch.int32).as_strided((1, 7), (3, 1)),              # one axis: any stride
], ids=str)
def test_mrope_reads_the_positions_it_was_given(monkeypatch, positions):
    """The kernel reads element axis * position_stride + token behind the pointer."""
    call, tokens = MropeCall(monkeypatch), min(7, positions.shape[1])
    turn(positions, tokens)
    assert call.args["positions"] == positions.data_ptr() and call.args["axes"] == positions.shape[0]
    held = np.frombuffer(bytes(positions.untyped_storage()), np.int32)[positions.storage_offset():]
    at = np.arange(positions.shape[0])[:, None] * call.args["position_stride"] + np.arange(tokens)
    assert at.max() < len(held)
    assert np.array_equal(held[at], positions[:, :tokens].numpy())


@pytest.mark.parametrize("positions", [
    torch.arange(9, dtype=torch.int32).as_strided((3, 7), (1, 1)),   # overlapping windows
    torch.arange(21, dtype=torch.int32).view(7, 3).T,                # a token's positions side by side
    torch.arange(18, dtype=torch.int32).view(3, 6),                  # fewer than the tokens
    torch.arange(21).view(3, 7),
], ids=["overlapping", "transposed", "few", "int64"])
def test_mrope_refuses_positions_it_cannot_read(monkeypatch, positions):
    call = MropeCall(monkeypatch)
    with pytest.raises(ValueError, match="positions"):
        turn(positions, 7)
    assert call.args is None


@pytest.mark.parametrize("stride", [-1, 1, 6])
def test_the_c_call_refuses_other_strides(stride):
    from paper_2605_31598_gb300 import build_ext, statekv

    build_ext.build()
    fake = 1 << 20  # aligned, never touched
    freq, axis = rotary.mrope_frequencies((16, 16), 1e4)
    args = statekv.statekv_mrope_args(7, 4, 2, 64, 2, 32, 0, 0, 1.0, freq.data_ptr(), axis.data_ptr(), fake, stride,
                                      fake, fake, fake, fake, 256, 128, 256, 128)
    assert statekv.statekv_mrope(args, 0) == 1


def cache_of_stand_ins(monkeypatch, capturing=False):
    """A QCache without buffers, whose calls need 100 bytes of workspace for a token and
    1000 for more; memory comes from the CPU."""
    c = qcache.QCache.__new__(qcache.QCache)
    c.shape, c.device, c._sizes, c._outgrown = (2, 3, 4, 128), 0, {}, []
    c.workspace = torch.zeros(100, dtype=torch.uint8)
    monkeypatch.setattr(c, "workspace_bytes", lambda n, hq, sc, lc: 100 if n == 1 else 1000, raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: None)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda x, s: None)
    return c


def test_a_workspace_that_was_handed_out_stays(monkeypatch):
    """A captured call holds its address: a larger call must not give the memory back."""
    c = cache_of_stand_ins(monkeypatch)
    q = torch.zeros(1)
    at = c._own_workspace((2, 3, 1, 28), q, None).data_ptr()
    large = c._own_workspace((2, 3, 9, 28), q, None)
    assert large.numel() == 1000 and not large.any()
    assert [x.data_ptr() for x in c._outgrown] == [at]
    assert c._own_workspace((2, 3, 9, 28), q, None) is large and c._own_workspace((2, 3, 1, 28), q, None) is large
    assert len(c._outgrown) == 1  # and no more of them, however often calls alternate


def test_a_capture_makes_no_workspace_for_later_calls(monkeypatch):
    """What a capture zeroes is zero at a replay only, so no eager call may take it."""
    c = cache_of_stand_ins(monkeypatch, capturing=True)
    q, small = torch.zeros(1), c.workspace
    assert c._own_workspace((2, 3, 1, 28), q, None) is small
    large = c._own_workspace((2, 3, 9, 28), q, None)
    assert large.numel() == 1000 and not large[:4096].any()
    assert c.workspace is small and not c._outgrown
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    eager = c._own_workspace((2, 3, 9, 28), q, None)
    assert eager is c.workspace and eager is not large and not eager.any()


class CacheCalls:
    """The C calls of a cache of stand-ins; counts what gets that far."""

    def __init__(self, monkeypatch, device=0, current=0):
        self.cache, self.device, self.calls = cache_of_stand_ins(monkeypatch), device, 0
        c = self.cache
        c.device, c._at = device, 0
        c._append = c._attend = self.call
        c._pack_append = c._pack_attend = lambda *fields: fields
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current, raising=False)
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 0, raising=False)

    def call(self, *args):
        self.calls += 1
        return 0

    def tensors(self, elsewhere=None):
        """A call's tensors on the cache's device, but for one."""
        def on(name, x):
            return OnDevice(x, self.device + (name == elsewhere))

        rows = {x: on(x, torch.zeros((2, 3, 5, h, 128), dtype=torch.bfloat16))
                for x, h in (("q", 28), ("out", 28), ("k", 4), ("v", 4))}
        units = {x: on(x, torch.zeros((2, 3), dtype=torch.int32)) for x in ("start", "first")}
        return dict(rows, **units, lse=on("lse", torch.zeros((2, 3, 5, 28))),
                    workspace=on("workspace", torch.zeros(2000, dtype=torch.uint8)))

    def append(self, t, **kw):
        return self.cache.append(t["k"], t["v"], t["start"], **kw)

    def attend(self, t, **kw):
        return self.cache.attend(t["q"], t["start"], t["out"], lse=t["lse"], first=t["first"], workspace=t["workspace"], **kw)


class OtherStream:
    device_index, cuda_stream = 1, 0


def test_a_cache_takes_tensors_of_its_device_only(monkeypatch):
    c = CacheCalls(monkeypatch)
    assert c.append(c.tensors()) == 0 and c.attend(c.tensors()) == 0 and c.calls == 2
    for call, names in ((c.append, ("k", "v", "start")), (c.attend, ("q", "out", "lse", "start", "first", "workspace"))):
        for name in names:
            with pytest.raises(ValueError, match="device"):
                call(c.tensors(elsewhere=name))
        with pytest.raises(ValueError, match="device"):
            call(c.tensors(), stream=OtherStream)
    assert c.calls == 2


def test_the_device_of_a_cache_has_to_be_current(monkeypatch):
    c = CacheCalls(monkeypatch, device=1, current=0)
    for call in (c.append, c.attend):
        with pytest.raises(ValueError, match="current"):
            call(c.tensors())
    assert c.calls == 0
    # nor is a cache made there: kernels are prepared, and the workspace sized, for the current device
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(qcache, "statekv_qcache_init", lambda c: pytest.fail("a cache elsewhere was prepared"))
    shapes = {"codes": ((1, 1, 1, 16, 64), torch.uint8), "scale": ((1, 1, 1, 1), torch.float32),
              "tail": ((1, 1, 1, 16, 64), torch.bfloat16)}
    for devices in ({}, {"k_codes": 0, "v_codes": 0}):  # all on device 1, and some
        buffers = {x: OnDevice(torch.zeros(shapes[x[2:]][0], dtype=shapes[x[2:]][1]), devices.get(x, 1)) for x in qcache.BUFFERS}
        with pytest.raises(ValueError, match="device"):
            qcache.QCache(1, 1, 1, 64, 16, block_tokens=16, tensors=buffers)


@pytest.mark.parametrize("devices,stream", [
    (dict(q=1), None), (dict(k=1), None), (dict(positions=1), None), (dict(q_out=1), None), (dict(k_out=1), None),
    (dict(q=1, k=1, positions=1, q_out=1, k_out=1), None),  # together, but elsewhere than the launch
    (dict(), OtherStream),
])
def test_mrope_takes_tensors_of_the_current_device_only(monkeypatch, devices, stream):
    called = []
    monkeypatch.setattr(rotary, "_call", lambda: (lambda args, stream: called.append(args) or 0, lambda *fields: fields))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 0, raising=False)
    freq, axis = rotary.mrope_frequencies((8, 12, 12), 1e4)

    def call(devices, stream):
        t = {x: OnDevice(torch.zeros((7, 2, 64), dtype=torch.bfloat16), devices.get(x, 0)) for x in ("q", "k", "q_out", "k_out")}
        at = OnDevice(torch.zeros((3, 7), dtype=torch.int32), devices.get("positions", 0))
        rotary.mrope(t["q"], t["k"], at, freq, axis, q_out=t["q_out"], k_out=t["k_out"], stream=stream)

    call({}, None)
    assert len(called) == 1
    with pytest.raises(ValueError, match="device"):
        call(devices, stream)
    assert len(called) == 1
