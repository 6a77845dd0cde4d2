"""A K/V cache held in 8 bits: its buffers, its append and the attention over it
(argument marshalling for the ``statekv_qcache_*`` calls)."""
from __future__ import annotations

import ctypes

import torch

from .statekv import (STATUS_NAMES, check, packed_call, raw_stream, statekv_qcache, statekv_qcache_append_args,
                      statekv_qcache_attend_args, statekv_qcache_init, statekv_qcache_sync,
                      statekv_qcache_workspace_bytes)

COUNTER_BYTES = 4096  # of a workspace, zero before its first use
BUFFERS = ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail")


class QCache:
    """Owns (or, with ``tensors``, borrows) the buffers of a cache of
    [num_streams][num_layers] units, and a workspace for the attention.

    ``start`` arguments are int32 device tensors [num_streams][num_layers]: the
    rows that each unit held before the step, -1 for a slot without a request.
    ``append`` and ``attend`` of one step take the same ``start``; the caller
    advances it after the step's last layer (``start += n``)."""

    def __init__(self, num_streams: int, num_layers: int, num_kv_heads: int, head_dim: int,
                 capacity: int, *, block_tokens: int = 64, device="cuda", tensors=None):
        """``capacity`` rows per head (a multiple of ``block_tokens``).  ``tensors``:
        the buffers by name (k_codes, v_codes uint8 or float8_e4m3fn
        [S][L][H][capacity][d], k_scale, v_scale fp32 [S][L][H][capacity /
        block_tokens], k_tail, v_tail bf16 [S][L][H][block_tokens][d]); made here
        if None."""
        S, L, H, d, b = num_streams, num_layers, num_kv_heads, head_dim, block_tokens
        if b < 1 or capacity < 1 or capacity % b:
            raise ValueError("capacity: a positive multiple of block_tokens")
        shapes = {"codes": (S, L, H, capacity, d), "scale": (S, L, H, capacity // b),
                  "tail": (S, L, H, b, d)}
        types = {"codes": (torch.uint8, torch.float8_e4m3fn), "scale": (torch.float32,),
                 "tail": (torch.bfloat16,)}
        if tensors is None:
            tensors = {x: torch.zeros(shapes[x[2:]], dtype=types[x[2:]][0], device=device)
                       for x in BUFFERS}
        self.device = tensors[BUFFERS[0]].get_device()
        if self.device < 0 or self.device != torch.cuda.current_device():
            raise ValueError("the cache's device has to be the current one (torch.cuda.device)")
        for x in BUFFERS:
            t = tensors[x]
            if t.shape != shapes[x[2:]] or t.dtype not in types[x[2:]] or not t.is_contiguous() or \
                    t.get_device() != self.device:
                raise ValueError(f"{x}: a contiguous {types[x[2:]][0]} tensor {shapes[x[2:]]} on the cache's device")
            setattr(self, x, t)
        self.shape = (S, L, H, d)
        self.capacity, self.block_tokens = capacity, b
        self.status = torch.zeros(1, dtype=torch.int32, device=self.k_codes.device)
        self.c = statekv_qcache(S, L, H, d, b, capacity,
                                *(getattr(self, x).data_ptr() for x in BUFFERS),
                                self.status.data_ptr())
        check(statekv_qcache_init(self.c), "statekv_qcache_init")
        # enough for a few query rows per KV head; the attention of more makes a larger one
        self.workspace = torch.zeros(self.workspace_bytes(1, H), dtype=torch.uint8,
                                     device=self.k_codes.device)
        self._outgrown = []
        self._sizes = {}
        self._at = ctypes.addressof(self.c)
        self._append, self._pack_append = packed_call("statekv_qcache_append", statekv_qcache_append_args, "5i3P6q")
        self._attend, self._pack_attend = packed_call("statekv_qcache_attend", statekv_qcache_attend_args, "7if6PN")
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream().synchronize()  # what is zeroed here is zero for calls on any stream

    def _range(self, stream_begin, stream_count, layer_begin, layer_count):
        S, L = self.shape[:2]
        return (stream_begin, S - stream_begin if stream_count is None else stream_count,
                layer_begin, L - layer_begin if layer_count is None else layer_count)

    def _units(self, x, name):
        if x.dtype != torch.int32 or x.shape != self.shape[:2] or not x.is_contiguous() or \
                x.get_device() != self.device:
            raise ValueError(f"{name}: a contiguous int32 tensor {self.shape[:2]} on the cache's device")
        return x.data_ptr()

    def append(self, k, v, start, *, stream_begin=0, stream_count=None, layer_begin=0,
               layer_count=None, stream=None) -> int:
        """Enqueue k, v (bf16 [S_cnt][L_cnt][n][H][d] each, elements of a row
        contiguous, units evenly spaced, any other strides) behind the ``start``
        rows of each unit.  Returns the C status."""
        r = self._range(stream_begin, stream_count, layer_begin, layer_count)
        n = k.shape[2]
        args = self._pack_append(*r, n, self._units(start, "start"), k.data_ptr(), v.data_ptr(),
                                 *self._strides(k, r, n, "k"), *self._strides(v, r, n, "v"))
        return self._append(self._at, args, raw_stream(stream, k))

    def _strides(self, x, r, n, name):
        """Elements between units, tokens and heads of rows to append (0 where there is
        one only: its stride may be anything)."""
        st = x.stride()
        if x.shape != (r[1], r[3], n, self.shape[2], self.shape[3]) or x.dtype != torch.bfloat16 or \
                st[4] != 1 or x.get_device() != self.device or (r[1] > 1 and r[3] > 1 and st[0] != r[3] * st[1]):
            raise ValueError(f"{name}: a bf16 tensor [streams][layers][n][heads][d] on the cache's device, its "
                             "rows contiguous and its units evenly spaced")
        return (st[1] if r[3] > 1 else st[0] if r[1] > 1 else 0, st[2] if n > 1 else 0,
                st[3] if self.shape[2] > 1 else 0)

    def workspace_bytes(self, num_tokens: int, num_q_heads: int, stream_count=None, layer_count=None) -> int:
        _, sc, _, lc = self._range(0, stream_count, 0, layer_count)
        return statekv_qcache_workspace_bytes(self.c, sc, lc, num_tokens, num_q_heads)

    def _own_workspace(self, key, q, stream):
        need = self._sizes.get(key)
        if need is None:
            need = self._sizes[key] = self.workspace_bytes(key[2], key[3], key[0], key[1])
        if self.workspace.numel() < need:
            with torch.cuda.stream(stream or torch.cuda.current_stream()):
                if torch.cuda.is_current_stream_capturing():
                    # memory of the graph, zeroed at each replay only: this call's and no other's
                    ws = torch.empty(need, dtype=torch.uint8, device=q.device)
                    ws[:COUNTER_BYTES].zero_()
                    return ws
                # graphs captured with the smaller one may replay at any time, so it stays (there are
                # two sizes: of calls for the few-row kernel alone, and of the others)
                self._outgrown.append(self.workspace)
                self.workspace = torch.zeros(need, dtype=torch.uint8, device=q.device)
        return self.workspace

    def attend(self, q, start, out, *, lse=None, first=None, causal=True, softmax_scale=0.0,
               stream_begin=0, stream_count=None, layer_begin=0, layer_count=None, workspace=None,
               stream=None) -> int:
        """Enqueue the attention of q (bf16 [S_cnt][L_cnt][n][Hq][d]) over the
        cache into ``out`` (like q) and ``lse`` (fp32 [S_cnt][L_cnt][n][Hq], may be
        None).  ``first``: int32 [S][L], first visible row of each unit.
        ``workspace``: a uint8 device tensor of ``workspace_bytes``, zero before its
        first use; by default the cache's own, which calls on one stream share (calls
        that may overlap bring their own).  A captured call that needs a larger one than
        the cache has by then takes it from the graph's memory, with a node that zeroes
        its counters: a call of its size beforehand, or ``workspace``, saves that.
        Returns the C status."""
        r = self._range(stream_begin, stream_count, layer_begin, layer_count)
        shape = q.shape
        S, L, n, Hq, d = shape
        if (q.dtype != torch.bfloat16 or out.dtype != torch.bfloat16 or out.shape != shape
                or not q.is_contiguous() or not out.is_contiguous() or S != r[1] or L != r[3]
                or d != self.shape[3] or q.get_device() != self.device or out.get_device() != self.device):
            raise ValueError("q, out: contiguous bf16 tensors [streams][layers][n][heads][d] on the cache's device")
        if lse is not None and (lse.dtype != torch.float32 or lse.shape != shape[:4]
                                or not lse.is_contiguous() or lse.get_device() != self.device):
            raise ValueError("lse: a contiguous fp32 tensor [streams][layers][n][heads] on the cache's device")
        handle = raw_stream(stream, q)
        ws = self._own_workspace((S, L, n, Hq), q, stream) if workspace is None else workspace
        if ws.dtype != torch.uint8 or not ws.is_contiguous() or ws.get_device() != self.device:
            raise ValueError("workspace: a contiguous uint8 tensor on the cache's device")
        args = self._pack_attend(
            *r, n, Hq, causal, softmax_scale, self._units(start, "start"),
            0 if first is None else self._units(first, "first"), q.data_ptr(), out.data_ptr(),
            0 if lse is None else lse.data_ptr(), ws.data_ptr(), ws.numel())
        return self._attend(self._at, args, handle)

    def sync(self, stream=None) -> int:
        """Synchronise and return what the kernels recorded (statekv_qcache_sync).
        After an expired wait the cache's own workspaces are made usable again, for that
        stream's next calls."""
        status = statekv_qcache_sync(self.c, raw_stream(stream, self.status))
        if STATUS_NAMES.get(status) == "STATEKV_ERR_DEVICE_TIMEOUT":
            with torch.cuda.stream(stream or torch.cuda.current_stream()):
                for ws in (self.workspace, *self._outgrown):
                    ws[:COUNTER_BYTES].zero_()
        return status
