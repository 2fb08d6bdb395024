"""Filtered sampling (``spade_sample`` of include/spade.h).

``Sampler`` owns the workspace and error word of calls of up to ``max_rows`` rows
and draws a token per row of logits: temperature, top-k, top-p and min-p, each one
value for all or one per request, from given uniforms.  Calls run on the current
stream of its device.
"""

from __future__ import annotations

import ctypes
import threading
from typing import Optional, Tuple, Union

import torch

from . import spade
from .spade import BF16, F32, SamplingArgs, _check, load_library

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}
_Float = Union[float, torch.Tensor]
_Int = Union[int, torch.Tensor]


class Sampler:
    """Draws for up to ``max_rows`` rows of up to ``vocab`` tokens.  Calls share one
    workspace, so those on different streams have to be ordered by the program; threads
    may call at once on one stream (a call's kernels are launched together)."""

    def __init__(self, max_rows: int, vocab: int, device="cuda:0"):
        self.lib = load_library()
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.max_rows, self.vocab = max_rows, vocab
        nbytes = self.lib.spade_sample_workspace_bytes(max_rows, vocab)
        if nbytes == 0:
            raise spade.SpadeError(-1, "sampler: " + self.lib.spade_last_error().decode())
        with torch.cuda.device(self.device):
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            self.err = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._index, self._bytes = self.device.index, nbytes
        self._at_ws, self._at_err = self.workspace.data_ptr(), self.err.data_ptr()
        self._launch = threading.Lock()  # (the library's calls leave the interpreter's lock)

    def _arg(self, t: Optional[torch.Tensor], dtype, shape: tuple, name: str):
        if t is None:
            return None
        if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != self._index:
            raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {shape} on {self.device}")
        return t.data_ptr()

    def draw(self, logits: torch.Tensor, uniforms: torch.Tensor, temperature: _Float = 1.0, top_k: _Int = 0,
             top_p: _Float = 1.0, min_p: _Float = 0.0, probs: Optional[torch.Tensor] = None,
             tokens: Optional[torch.Tensor] = None, chosen: Optional[torch.Tensor] = None
             ) -> Tuple[torch.Tensor, torch.Tensor]:
        """A token per row of logits [rows, V] (float32 or bfloat16, rows one stride
        apart) from uniforms float32 [rows]: (tokens int32 [rows], their
        probabilities float32 [rows]).  A parameter is a number or a tensor
        [requests] (float32; top_k int32), whose requests have rows / requests rows
        each.  probs: float32 [rows, V], gets the whole distributions (may be the
        logits).  See spade_sample."""
        dt = logits.dtype
        if dt not in _DTYPES or logits.dim() != 2 or logits.get_device() != self._index:
            raise ValueError(f"logits: expected float32 or bfloat16 [rows, V] on {self.device}")
        rows, V = logits.shape
        sr, sv = logits.stride()
        if sv != 1 and V > 1:
            raise ValueError("logits: rows must be contiguous")
        if rows > self.max_rows or V > self.vocab:
            raise ValueError(f"the sampler holds {self.max_rows} rows of {self.vocab} tokens")
        f32, i32, arg = torch.float32, torch.int32, self._arg
        all_ = SamplingArgs(1.0, 0, 1.0, 0.0)
        n, at = None, [None] * 4
        for j, (p, t, name) in enumerate(((temperature, f32, "temperature"), (top_k, i32, "top_k"), (top_p, f32, "top_p"),
                                          (min_p, f32, "min_p"))):
            if isinstance(p, torch.Tensor):
                # (of no requests it has no address, which the library takes as not given)
                if p.numel() != n and (n is not None or p.numel() == 0):
                    raise ValueError(f"{name}: expected {n or 'one or more'} requests")
                n = p.numel()
                at[j] = arg(p, t, (n,), name)
            elif j == 0:
                all_.temperature = p
            elif j == 1:
                all_.top_k = min(max(p, 0), V)  # (the struct's field would take the low 32 bits)
            elif j == 2:
                all_.top_p = p
            else:
                all_.min_p = p
        if n is not None and rows % n:
            raise ValueError(f"{rows} rows do not divide into {n} requests")
        one = (rows,)
        if tokens is None:
            tokens = uniforms.new_empty(one, dtype=i32)
        if chosen is None:
            chosen = uniforms.new_empty(one)
        args = (rows, V, _DTYPES[dt], logits.data_ptr(), sr if rows > 1 else V, rows // n if n else max(rows, 1),
                ctypes.byref(all_), *at, arg(uniforms, f32, one, "uniforms"), arg(tokens, i32, one, "tokens"),
                arg(chosen, f32, one, "chosen"), arg(probs, f32, (rows, V), "probs"), self._at_ws, self._bytes,
                self._at_err)
        i = self._index
        stream = torch._C._cuda_getCurrentRawStream(i)
        with self._launch:
            if torch.cuda.current_device() == i:
                status = self.lib.spade_sample(*args, stream)
            else:
                with torch.cuda.device(i):
                    status = self.lib.spade_sample(*args, stream)
        if status:
            _check(status)
        return tokens, chosen

    def device_error(self) -> int:
        """Read and clear the error word (synchronises)."""
        v = int(self.err.item())
        self.err.zero_()
        return v
