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
    c.shape, c._sizes, c._outgrown = (2, 3, 4, 128), {}, []
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
