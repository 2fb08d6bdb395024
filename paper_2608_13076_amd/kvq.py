"""K/V caches in 4 bits (``spade_kvq_*`` of include/spade.h).

``QuantCache`` owns the buffers of one cache -- the codes, the lengths, the
attention's workspace and an error word -- and marshals its calls: ``append``
new rows (head norms, rotation, quantisation), ``attend`` over the cache,
``evict`` positions by accumulated attention weight and ``read`` rows back.
Every call runs on the current stream of the cache's device.
"""

from __future__ import annotations

import ctypes
import math
from typing import Optional, Tuple

import torch

from . import spade
from .spade import BF16, F32, KVQShape, _check, load_library

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}


def rope_table(n: int, head_dim: int, theta: float = 10000.0, device="cuda:0") -> torch.Tensor:
    """float32 [n][head_dim / 2][2]: cosine and sine of pos theta^(-2 i /
    head_dim), the angles in double."""
    pos = torch.arange(n, dtype=torch.float64, device=device)[:, None]
    inv = float(theta) ** (-2.0 * torch.arange(head_dim // 2, dtype=torch.float64, device=device) / head_dim)
    return torch.stack([torch.cos(pos * inv), torch.sin(pos * inv)], -1).float().contiguous()


class QuantCache:
    """A 4-bit K/V cache of ``n_layers`` layers and ``batch`` requests.

    ``lens`` (int32 [batch], on the device) counts the positions each request
    holds; ``append`` and ``attend`` leave it alone, so a program adds the rows
    it keeps itself (``cache.lens += n``).  ``max_rows``: most rows per request
    of an ``attend`` call.  ``attend`` calls share one workspace, so those on
    different streams have to be ordered by the program.  No call records a
    gradient: outputs do not require one, whatever the inputs do."""

    def __init__(self, n_layers: int, batch: int, n_heads: int, n_kv_heads: int, head_dim: int, max_len: int,
                 max_rows: int = 16, device="cuda:0"):
        self.lib = load_library()
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.shape = KVQShape(n_layers, batch, n_heads, n_kv_heads, head_dim, max_len)
        self.n_layers, self.batch, self.n_heads, self.n_kv_heads = n_layers, batch, n_heads, n_kv_heads
        self.head_dim, self.max_len, self.max_rows = head_dim, max_len, max_rows
        self._sp = ctypes.byref(self.shape)
        nbytes = self.lib.spade_kvq_bytes(self._sp)
        ws = self.lib.spade_kvq_workspace_bytes(self._sp, max_rows)
        if nbytes == 0 or ws == 0:
            raise spade.SpadeError(-1, "cache shape: " + self.lib.spade_last_error().decode())
        with torch.cuda.device(self.device):
            self.buf = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            self.workspace = torch.empty(ws, dtype=torch.uint8, device=self.device)
            self.lens = torch.zeros(batch, dtype=torch.int32, device=self.device)
            self.err = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._wshape = (batch, n_kv_heads, max_len)
        # (a call costs the host about as much as a short one costs the GPU)
        self._index = self.device.index
        self._at_buf, self._at_ws, self._at_err = self.buf.data_ptr(), self.workspace.data_ptr(), self.err.data_ptr()
        self._ws_bytes, self._scale = ws, 1.0 / math.sqrt(head_dim)

    def _call(self, fn, *args) -> None:
        """fn(shape, *args, stream) with the cache's device current, on its
        current stream."""
        i = self._index
        # (the handle of torch.cuda.current_stream(i), without building the object)
        stream = torch._C._cuda_getCurrentRawStream(i)
        if torch.cuda.current_device() == i:
            status = fn(self._sp, *args, stream)
        else:
            with torch.cuda.device(i):
                status = fn(self._sp, *args, stream)
        if status:
            _check(status)

    def _arg(self, t: Optional[torch.Tensor], dtype, shape: tuple, name: str):
        """Address of a contiguous tensor of this dtype and shape on the cache's device."""
        if t is None:
            return None
        if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != self._index:
            raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {shape} on {self.device}")
        return t.data_ptr()

    def _rows(self, t: torch.Tensor, shape: tuple, dtype, name: str):
        """(address, ld) of rows [B, R, heads, head_dim]: contiguous heads, the
        rows of all requests one stride apart."""
        if t.dtype is not dtype or t.shape != shape or t.get_device() != self._index:
            raise ValueError(f"{name}: expected {dtype} {list(shape)} on {self.device}")
        B, R, heads, hd = shape
        if t.is_contiguous():
            return t.data_ptr(), heads * hd
        sb, sr, sh, sf = t.stride()
        ld = sr if R > 1 else (sb if B > 1 else heads * hd)
        if sf != 1 or (heads > 1 and sh != hd) or (R > 1 and B > 1 and sb != R * sr):
            raise ValueError(f"{name}: heads must be contiguous and rows one stride apart")
        return t.data_ptr(), ld

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, q: Optional[torch.Tensor] = None,
               gain_q: Optional[torch.Tensor] = None, gain_k: Optional[torch.Tensor] = None, eps: float = 1e-5,
               rope: Optional[torch.Tensor] = None, pos: Optional[torch.Tensor] = None,
               rows: Optional[torch.Tensor] = None, weights: Optional[torch.Tensor] = None,
               q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """Store rows k, v [B, R, n_kv_heads, head_dim] as positions lens[b] ..
        lens[b] + R - 1 and return the queries q [B, R, n_heads, head_dim]
        (q_out where given), normed and rotated like the keys.  ``weights``: the
        layer's running weights [batch, n_kv_heads, max_len], zeroed for the new
        positions.  See spade_kvq_append."""
        dt, shape, hd, arg = k.dtype, k.shape, self.head_dim, self._arg
        if dt not in _DTYPES or len(shape) != 4:
            raise ValueError("k: float32 or bfloat16 [B, R, n_kv_heads, head_dim]")
        B, R = shape[0], shape[1]
        shape = (B, R, self.n_kv_heads, hd)
        kp, kld = self._rows(k, shape, dt, "k")
        vp, vld = self._rows(v, shape, dt, "v")
        qp, qld, op, old = None, 0, None, 0
        if q is not None:
            shape = (B, R, self.n_heads, hd)
            qp, qld = self._rows(q, shape, dt, "q")
            if q_out is None:
                q_out = q.new_empty(shape)
            op, old = self._rows(q_out, shape, dt, "q_out")
        elif q_out is not None:
            raise ValueError("q_out without q")
        f32, i32 = torch.float32, torch.int32
        n_rope = 0 if rope is None else rope.shape[0]
        self._call(
            self.lib.spade_kvq_append, layer, self._at_buf, B, R, _DTYPES[dt], qp, qld, kp, kld, vp, vld,
            arg(gain_q, f32, (hd,), "gain_q"), arg(gain_k, f32, (hd,), "gain_k"), eps,
            arg(rope, f32, (n_rope, hd // 2, 2), "rope"), n_rope, arg(pos, i32, (B,), "pos"),
            arg(self.lens, i32, (self.batch,), "lens"), arg(rows, i32, (B,), "rows"), op, old,
            arg(weights, f32, self._wshape, "weights"), self._at_err)
        return q_out

    def attend(self, layer: int, q: torch.Tensor, out: Optional[torch.Tensor] = None, scale: Optional[float] = None,
               rows: Optional[torch.Tensor] = None, max_keys: int = 0, weights: Optional[torch.Tensor] = None,
               weights_out: Optional[torch.Tensor] = None, weight_rows: int = 0) -> torch.Tensor:
        """Causal attention of q [B, R, n_heads, head_dim], whose rows ``append``
        has stored, over the layer; returns out (same shape and dtype).  scale:
        1 / sqrt(head_dim) unless given.  max_keys: the host's bound of lens +
        the rows in use (0: max_len; at least R without ``rows``).  weights_out = weights + the probabilities of the
        first weight_rows rows, both [batch, n_kv_heads, max_len] (may be one
        tensor).  See spade_kvq_attend."""
        dt, shape, arg = q.dtype, q.shape, self._arg
        if dt not in _DTYPES or len(shape) != 4:
            raise ValueError("q: float32 or bfloat16 [B, R, n_heads, head_dim]")
        B, R = shape[0], shape[1]
        shape = (B, R, self.n_heads, self.head_dim)
        qp, qld = self._rows(q, shape, dt, "q")
        if out is None:
            out = q.new_empty(shape)
        op, old = self._rows(out, shape, dt, "out")
        f32, i32 = torch.float32, torch.int32
        self._call(
            self.lib.spade_kvq_attend, layer, self._at_buf, B, R, _DTYPES[dt], qp, qld,
            self._scale if scale is None else scale, arg(self.lens, i32, (self.batch,), "lens"),
            arg(rows, i32, (B,), "rows"), max_keys, op, old, arg(weights, f32, self._wshape, "weights"),
            arg(weights_out, f32, self._wshape, "weights_out"), weight_rows, self._at_ws, self._ws_bytes, self._at_err)
        return out

    def read(self, layer: int, n: int, start: Optional[torch.Tensor] = None, rows: Optional[torch.Tensor] = None,
             dtype: torch.dtype = torch.float32) -> Tuple[torch.Tensor, torch.Tensor]:
        """Keys and values [batch, n, n_kv_heads, head_dim] of positions start[b]
        (0) .. + n - 1 as they are held; zeros past rows[b].  See spade_kvq_read."""
        if dtype not in _DTYPES:
            raise ValueError("dtype: float32 or bfloat16")
        shape = (self.batch, n, self.n_kv_heads, self.head_dim)
        k = self.buf.new_empty(shape, dtype=dtype)
        v = k.new_empty(shape)
        i32, one = torch.int32, (self.batch,)
        self._call(
            self.lib.spade_kvq_read, layer, self._at_buf, self.batch, n, self._arg(start, i32, one, "start"),
            self._arg(rows, i32, one, "rows"), _DTYPES[dtype], k.data_ptr(), v.data_ptr())
        return k, v

    def evict(self, weights: torch.Tensor, budget: int, recent: int, kept: Optional[torch.Tensor] = None,
              into: Optional["QuantCache"] = None, weights_out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Keep, per layer, request and K/V head, the last ``recent`` positions
        and the heaviest others, ``budget`` in all; in place, or into another
        cache of the same layers and heads, whose lens become the new ones.
        weights [n_layers, batch, n_kv_heads, max_len]; weights_out likewise
        with the other cache's sizes (may be weights in place).  Returns kept
        int32 [n_layers, batch, n_kv_heads, budget].  See spade_kvq_evict."""
        dst = self if into is None else into
        if dst.device != self.device:
            raise ValueError("the caches are on different devices")
        i32, f32 = torch.int32, torch.float32
        kshape = (self.n_layers, self.batch, self.n_kv_heads, budget)
        if kept is None:
            kept = torch.empty(tuple(max(int(x), 0) for x in kshape), dtype=i32, device=self.device)
        self._call(
            self.lib.spade_kvq_evict, self._at_buf, dst._sp, dst._at_buf, self.batch, budget, recent,
            self._arg(weights, f32, (self.n_layers,) + self._wshape, "weights"),
            dst._arg(weights_out, f32, (dst.n_layers,) + dst._wshape, "weights_out"),
            self._arg(self.lens, i32, (self.batch,), "lens"), dst._arg(dst.lens, i32, (dst.batch,), "lens"),
            self._arg(kept, i32, kshape, "kept"))
        return kept

    def device_error(self) -> int:
        """Read and clear the error word (synchronises)."""
        v = int(self.err.item())
        self.err.zero_()
        return v
