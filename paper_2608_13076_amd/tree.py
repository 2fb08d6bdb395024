"""Trees of drafts (``spade_tree_*`` of include/spade.h).

``TreeCache`` owns the buffers of one bfloat16 K/V cache -- keys and values, the
lengths, the attention's workspace and an error word -- or works on a model's
(``TreeCache.over``), and marshals its calls: ``append`` the rows of a tree
(rotated by position), ``attend`` to the context and the ancestors, ``commit`` the
path that the drawn tokens follow, and ``read`` rows back.  ``rotary_frequencies``
gives the angles of a rotation, also scaled for contexts longer than a model was
trained on.  Every call runs on the current stream of the cache's device.
"""

from __future__ import annotations

import ctypes
import math
import threading
from typing import Optional, Tuple

import torch

from . import spade
from .spade import BF16, F32, RotaryArgs, TreeShape, _check, load_library

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}


def rotary_frequencies(rot_dim: int, theta: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0,
                       trained: int = 8192, slow: float = 1.0, fast: float = 32.0,
                       device="cuda:0") -> Tuple[torch.Tensor, float]:
    """Angle per position of the pairs of ``rot_dim`` features (float64
    [rot_dim / 2]) and the rotated features' amplitude.  ``scaling`` for contexts
    ``factor`` times longer than the ``trained`` positions:

    None      theta^(-2 j / rot_dim)
    "linear"  every frequency divided by factor
    "base"    theta times factor^(rot_dim / (rot_dim - 2)): the fastest pair
              stays, the slowest is divided by factor
    "bands"   by the turns that a pair makes in ``trained`` positions: at least
              ``fast`` stay, at most ``slow`` are divided, in between a straight
              line over the turns
    "ramp"    as "bands", with the line over the pairs' numbers (its ends rounded
              outwards to whole ones and kept within 0 and rot_dim - 1: behind
              the last pair where that turns more than ``slow`` times) and the
              amplitude 0.1 log(factor) + 1
    """
    if rot_dim < 2 or rot_dim % 2 or not theta > 0 or not factor > 0:
        raise ValueError("rot_dim must be even, theta and factor positive")
    n = rot_dim // 2
    j = torch.arange(n, dtype=torch.float64, device=device)
    if scaling == "base":
        theta = theta * factor ** (rot_dim / max(rot_dim - 2, 1))
    f = float(theta) ** (-2.0 * j / rot_dim)
    if scaling in (None, "base"):
        return f, 1.0
    if scaling == "linear":
        return f / factor, 1.0
    if scaling not in ("bands", "ramp"):
        raise ValueError(f"scaling: unknown {scaling!r}")
    if not fast > slow > 0 or trained < 1:
        raise ValueError("0 < slow < fast and trained >= 1 required")
    if scaling == "ramp" and not theta > 1:
        raise ValueError("a ramp's frequencies must fall from pair to pair: theta above 1 required")
    if scaling == "bands":
        keep = ((trained * f / (2.0 * math.pi) - slow) / (fast - slow)).clamp(0.0, 1.0)
        return f * keep + f / factor * (1.0 - keep), 1.0

    def pair(turns: float) -> float:  # the (fractional) pair that makes so many
        return n * math.log(trained / (2.0 * math.pi * turns)) / math.log(theta)

    lo, hi = max(math.floor(pair(fast)), 0), min(math.ceil(pair(slow)), rot_dim - 1)
    keep = 1.0 - ((j - lo) / max(hi - lo, 1e-3)).clamp(0.0, 1.0)
    return f * keep + f / factor * (1.0 - keep), (0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0)


class Rotary:
    """A rotation of queries and keys: ``freq`` float64 [rot_dim / 2] on the
    device, of the first rot_dim features (the whole head or a part of it), pairs
    j and j + rot_dim / 2, or 2 j and 2 j + 1 (``interleaved``)."""

    def __init__(self, freq: torch.Tensor, interleaved: bool = False, amplitude: float = 1.0):
        if freq.dtype is not torch.float64 or freq.dim() != 1 or not freq.is_contiguous():
            raise ValueError("freq: expected a contiguous float64 vector")
        self.freq, self.device = freq, freq.device
        self.rot_dim, self.interleaved, self.amplitude = 2 * freq.numel(), bool(interleaved), float(amplitude)
        self._args = RotaryArgs(freq.data_ptr(), self.rot_dim, int(self.interleaved), self.amplitude)
        self._ref = ctypes.byref(self._args)


class TreeCache:
    """A bfloat16 K/V cache of ``n_layers`` layers and ``batch`` requests.

    ``lens`` (int32 [batch], on the device) counts the positions each request
    holds; only ``commit`` changes it (a program that appends a prompt adds its
    rows itself: ``cache.lens += n``).  ``max_rows``: most rows per request of an
    ``attend`` call.  ``attend`` calls share one workspace, so those on different
    streams have to be ordered by the program; threads may call at once on one stream
    (a call's kernels are launched together).  No call records a gradient."""

    def __init__(self, n_layers: int, batch: int, n_heads: int, n_kv_heads: int, head_dim: int, max_len: int,
                 max_rows: int = 64, device="cuda:0", buf: Optional[torch.Tensor] = None,
                 lens: Optional[torch.Tensor] = None):
        self.lib = load_library()
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.shape = TreeShape(n_layers, batch, n_heads, n_kv_heads, head_dim, max_len)
        self.n_layers, self.batch, self.n_heads, self.n_kv_heads = n_layers, batch, n_heads, n_kv_heads
        self.head_dim, self.max_len, self.max_rows = head_dim, max_len, max_rows
        self._sp = ctypes.byref(self.shape)
        nbytes = self.lib.spade_tree_bytes(self._sp)
        ws = self.lib.spade_tree_workspace_bytes(self._sp, max_rows)
        if nbytes == 0 or ws == 0:
            raise spade.SpadeError(-1, "cache shape: " + self.lib.spade_last_error().decode())
        self._index = self.device.index
        if buf is not None and (buf.dtype is not torch.uint8 or buf.numel() < nbytes or not buf.is_contiguous()
                                or buf.get_device() != self._index):
            raise ValueError(f"buf: expected at least {nbytes} contiguous bytes on {self.device}")
        with torch.cuda.device(self.device):
            self.buf = torch.empty(nbytes, dtype=torch.uint8, device=self.device) if buf is None else buf
            self.workspace = torch.empty(ws, dtype=torch.uint8, device=self.device)
            self.lens = torch.zeros(batch, dtype=torch.int32, device=self.device) if lens is None else lens
            self.err = torch.zeros(1, dtype=torch.int32, device=self.device)
        # (a call costs the host about as much as a short one costs the GPU)
        self._at_buf, self._at_ws, self._at_err = self.buf.data_ptr(), self.workspace.data_ptr(), self.err.data_ptr()
        self._ws_bytes, self._scale = ws, 1.0 / math.sqrt(head_dim)
        self._launch = threading.Lock()  # (the library's calls leave the interpreter's lock)

    @classmethod
    def over(cls, kv: spade.KVCache, max_rows: int = 64) -> "TreeCache":
        """The cache of a model with a bfloat16 cache: its buffer and lengths.
        What ``commit`` adds to the lengths the model's own calls learn from
        ``kv.set_state``."""
        s = kv.model.shape
        if s.kv_dtype != "bf16":
            raise ValueError("the model's cache is not bfloat16")
        return cls(s.n_layers, kv.max_batch, s.n_heads, getattr(s, "n_kv_heads", 0) or s.n_heads, s.head_dim, kv.max_len,
                   max_rows=max_rows, device=kv.model.device, buf=kv.buf, lens=kv.lens)

    def _call(self, fn, *args) -> None:
        """fn(shape, *args, stream) with the cache's device current, on its
        current stream."""
        i = self._index
        # (the handle of torch.cuda.current_stream(i), without building the object)
        stream = torch._C._cuda_getCurrentRawStream(i)
        with self._launch:
            if torch.cuda.current_device() == i:
                status = fn(self._sp, *args, stream)
            else:
                with torch.cuda.device(i):
                    status = fn(self._sp, *args, stream)
        if status:
            _check(status)

    def _arg(self, t: Optional[torch.Tensor], shape: tuple, name: str):
        """Address of a contiguous int32 tensor of this shape on the cache's device."""
        if t is None:
            return None
        if t.dtype is not torch.int32 or t.shape != shape or not t.is_contiguous() or t.get_device() != self._index:
            raise ValueError(f"{name}: expected a contiguous torch.int32 tensor of shape {shape} on {self.device}")
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
               rope: Optional[Rotary] = None, depth: Optional[torch.Tensor] = None,
               pos: Optional[torch.Tensor] = None, rows: Optional[torch.Tensor] = None,
               q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """Store rows k, v [B, R, n_kv_heads, head_dim] as positions lens[b] ..
        lens[b] + R - 1 and return the queries q [B, R, n_heads, head_dim] (q_out
        where given); queries and keys rotated by ``rope`` at position pos[b]
        (lens[b]) + depth[b, i] (i).  See spade_tree_append."""
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
        if rope is not None and rope.device != self.device:
            raise ValueError(f"rope: expected frequencies on {self.device}")
        self._call(
            self.lib.spade_tree_append, layer, self._at_buf, B, R, _DTYPES[dt], qp, qld, kp, kld, vp, vld,
            None if rope is None else rope._ref, arg(pos, (B,), "pos"), arg(depth, (B, R), "depth"),
            arg(self.lens, (self.batch,), "lens"), arg(rows, (B,), "rows"), op, old, self._at_err)
        return q_out

    def attend(self, layer: int, q: torch.Tensor, parents: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None, scale: Optional[float] = None,
               rows: Optional[torch.Tensor] = None, max_keys: int = 0) -> torch.Tensor:
        """Attention of q [B, R, n_heads, head_dim], whose rows ``append`` has
        stored, to the context, their ancestors (parents int32 [B, R]; None: a
        chain) and themselves; returns out (same shape and dtype).  scale: 1 /
        sqrt(head_dim) unless given.  max_keys: the host's bound of lens + the rows
        in use (0: max_len; at least R without ``rows``).  See spade_tree_attend."""
        dt, shape, arg = q.dtype, q.shape, self._arg
        if dt not in _DTYPES or len(shape) != 4:
            raise ValueError("q: float32 or bfloat16 [B, R, n_heads, head_dim]")
        B, R = shape[0], shape[1]
        shape = (B, R, self.n_heads, self.head_dim)
        qp, qld = self._rows(q, shape, dt, "q")
        if out is None:
            out = q.new_empty(shape)
        op, old = self._rows(out, shape, dt, "out")
        self._call(
            self.lib.spade_tree_attend, layer, self._at_buf, B, R, _DTYPES[dt], qp, qld,
            self._scale if scale is None else scale, arg(parents, (B, R), "parents"),
            arg(self.lens, (self.batch,), "lens"), arg(rows, (B,), "rows"), max_keys, op, old, self._at_ws,
            self._ws_bytes, self._at_err)
        return out

    def read(self, layer: int, n: int, start: Optional[torch.Tensor] = None, rows: Optional[torch.Tensor] = None,
             dtype: torch.dtype = torch.bfloat16) -> Tuple[torch.Tensor, torch.Tensor]:
        """Keys and values [batch, n, n_kv_heads, head_dim] of positions start[b]
        (0) .. + n - 1; zeros past rows[b].  See spade_tree_read."""
        if dtype not in _DTYPES:
            raise ValueError("dtype: float32 or bfloat16")
        shape = (self.batch, n, self.n_kv_heads, self.head_dim)
        k = self.buf.new_empty(shape, dtype=dtype)
        v = k.new_empty(shape)
        one = (self.batch,)
        self._call(self.lib.spade_tree_read, layer, self._at_buf, self.batch, n, self._arg(start, one, "start"),
                   self._arg(rows, one, "rows"), _DTYPES[dtype], k.data_ptr(), v.data_ptr())
        return k, v

    def commit(self, tokens: torch.Tensor, parents: Optional[torch.Tensor], next_tokens: torch.Tensor,
               rows: Optional[torch.Tensor] = None, lens_out: Optional[torch.Tensor] = None
               ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        """Walk the tree of tokens [B, R] along next_tokens [B, R] (what was drawn
        for every row), close the path's rows up and add them to the lengths
        (lens_out where given).  Returns int32 (accepted drafts [B], path [B, R],
        correction [B]).  See spade_tree_commit."""
        if tokens.dim() != 2:
            raise ValueError("tokens: int32 [B, R]")
        B, R = tokens.shape
        arg, one, all_ = self._arg, (B,), (B, R)
        tp = arg(tokens, all_, "tokens")
        n, path, corr = tokens.new_empty(B), tokens.new_empty(all_), tokens.new_empty(B)
        lens = arg(self.lens, (self.batch,), "lens")
        self._call(
            self.lib.spade_tree_commit, self._at_buf, B, R, tp, arg(parents, all_, "parents"),
            arg(next_tokens, all_, "next_tokens"), arg(rows, one, "rows"), lens,
            lens if lens_out is None else arg(lens_out, (self.batch,), "lens_out"), n.data_ptr(), path.data_ptr(),
            corr.data_ptr(), self._at_err)
        return n, path, corr

    def device_error(self) -> int:
        """Read and clear the error word (synchronises)."""
        v = int(self.err.item())
        self.err.zero_()
        return v
