"""One MLP block with weights and activations in 4-bit floating point, between two attention blocks, as it is served:

    residual += gate * attention's output;   h = norm(residual), modulated, rotated and quantised        (one launch)
    hidden = gelu(h W_gate) * (h W_up)                                                                   (one launch)
    out = hidden W_down, hidden rotated and quantised ahead of it                                        (two launches)
    residual += gate * out;   next = norm(residual), modulated                                           (one launch)

``next`` is what the following layer's fused Q/K/V linear takes.  Every step of the computation is a libqvla call on the current
stream; this file only places buffers, all of them made at construction: a call allocates nothing and can be captured in a CUDA
graph.  Calls share the buffers and the outputs: they run one after the other, also where they are made on different streams.
"""

from __future__ import annotations

import torch

from . import qvla as Q

_TORCH = {Q.F16: torch.float16, Q.BF16: torch.bfloat16, Q.F32: torch.float32}


class Fp4Mlp:
    """``gate_up``: a gated Fp4Layer; ``down``: an Fp4Layer with K = gate_up.N and N = gate_up.K, of one 16-bit type.  ``before``
    and ``after``: the BlockNorm on either side, of that type.  Up to ``max_tokens`` tokens a call; the residual is kept in
    ``residual_dtype`` (the layers' type, or F32).  Layers, norms, residual and branch lie on one device, the current one in every
    call."""

    def __init__(self, gate_up: Q.Fp4Layer, down: Q.Fp4Layer, before: Q.BlockNorm, after: Q.BlockNorm, max_tokens: int,
                 residual_dtype: int | None = None, device=None):
        if not gate_up.gated or down.gated or down.K != gate_up.N or down.N != gate_up.K:
            raise ValueError("the layers' widths do not match: a gated layer and one back to its input's width are wanted")
        dt = gate_up.ydt
        if not dt == gate_up.xdt == down.xdt == down.ydt == before.dt == after.dt or dt == Q.F32:
            raise ValueError("the layers and norms must share one 16-bit type")
        residual_dtype = dt if residual_dtype is None else residual_dtype
        if residual_dtype not in (dt, Q.F32):
            raise ValueError("the residual is kept in the layers' type or in float32")
        if max_tokens < 1:
            raise ValueError("max_tokens must be positive")
        self.gate_up, self.down, self.before, self.after = gate_up, down, before, after
        self.dt, self.rdt, self.max_tokens, self.width = dt, residual_dtype, max_tokens, gate_up.K

        def empty(n, dtype):
            return torch.empty(n, dtype=dtype, device="cuda" if device is None else device)

        k, t = self.width, _TORCH[dt]
        self.codes = empty((max_tokens, k // 2), torch.uint8)
        self.scales = empty(Q.qvla_fp4_scale_bytes(gate_up.fmt, max_tokens, k), torch.uint8)
        self.row_scales = empty(max_tokens, torch.float32)
        self.hidden, self.out, self.next = empty((max_tokens, gate_up.N), t), empty((max_tokens, k), t), empty((max_tokens, k), t)
        self.work = empty(Q.qvla_fp4_linear_workspace_bytes(down, max_tokens), torch.uint8)
        self.device = self.codes.device  # with its index
        # The stream of the latest call.  The buffers are the allocator's memory of this one, which its earlier work may still use.
        self._last = torch.cuda.current_stream(self.device) if self.codes.is_cuda else None
        self._tokens = {}  # that each norm's conditioning reaches over
        for name, norm in (("before", before), ("after", after)):
            conditioned = norm.struct.mod_rows > 0 and norm.tensors[-1] is None
            self._tokens[name] = norm.struct.mod_rows * norm.struct.mod_tokens if conditioned else norm.tokens
            if any(t is not None and t.device != self.device for t in norm.tensors):
                raise ValueError(f"the tensors of `{name}` must lie on {self.device}")
            if any(t is not None and t.shape[-1] != k for t in norm.tensors[:-1]):  # (wider ones would be cut, silently)
                raise ValueError(f"the vectors of `{name}` must have the layers' {k} channels")

    def _stream(self) -> torch.cuda.Stream:
        """The current stream, behind the block's construction and latest call.  (What a graph is captured from, or replayed
        beside, is ordered by the one who replays it, and the block has to outlive the replays.)"""
        stream = torch.cuda.current_stream(self.device)
        if torch.cuda.is_current_stream_capturing():
            return stream
        if stream != self._last:
            stream.wait_stream(self._last)
            for t in (self.codes, self.scales, self.row_scales, self.hidden, self.out, self.next, self.work):
                t.record_stream(stream)
            self._last = stream
        return stream

    def _check(self, residual, branch) -> int:
        """The library takes addresses and sizes on trust: an input of other sizes would be read past its end, one of another GPU
        through an address that means nothing on this one."""
        m = residual.shape[0]
        if m > self.max_tokens:
            raise ValueError(f"{m} tokens are more than {self.max_tokens}")
        for name, tokens in self._tokens.items():  # (the call itself would say so, of `after` when the residual has changed)
            if m > tokens:
                raise ValueError(f"{m} tokens are more than the {tokens} of the conditioning of `{name}`")
        for name, x, dtype in (("residual", residual, _TORCH[self.rdt]), ("branch", branch, _TORCH[self.dt])):
            if tuple(x.shape) != (m, self.width) or x.dtype != dtype or not x.is_contiguous():
                raise ValueError(f"{name} must be contiguous {dtype} [{m}, {self.width}]")
            if x.device != self.device:
                raise ValueError(f"{name} must lie on {self.device}")
        if self.codes.is_cuda and torch.cuda.current_device() != self.device.index:  # the kernels run there
            raise ValueError(f"the current device must be {self.device}")
        return m

    def __call__(self, residual: torch.Tensor, branch: torch.Tensor) -> torch.Tensor:
        """residual [m, K], updated in place by `branch` (attention's output, [m, K]) and by the MLP's; returns the next block's
        input [m, K], which the next call overwrites."""
        m = self._check(residual, branch)
        st, k = self._stream(), self.width
        up, down = self.gate_up, self.down
        Q.qvla_block_norm_fp4(self.before, residual, self.rdt, k, branch, k, m, k, residual, None, up.had_block, up.fmt, None,
                              self.codes, self.scales, self.row_scales, st)
        Q.qvla_gemm_fp4(up, self.codes, self.scales, self.row_scales, m, self.hidden, st)
        Q.qvla_fp4_linear(down, self.hidden, m, None, self.out, self.work, self.work.numel(), st)
        Q.qvla_block_norm(self.after, residual, self.rdt, k, self.out, k, m, k, residual, self.next, st)
        return self.next[:m]
