"""One attention block of the language backbone or the action head, as it is served: the fused Q/K/V linear (W4A4), attention, the
output linear (W4A4), and a 4-bit key/value cache of its tokens.

``prefill`` takes packed prompts.  A sequence without earlier tokens attends to its fresh keys and values, which then enter the
cache; one that has tokens already attends to what the cache gives back of all its tokens, the new ones included, as it does in
``step``.  What a sequence gets does not depend on the others (but for last bits, as a call's sizes decide how it splits the
keys).  ``step`` takes the next token or tokens of every sequence: they
enter the cache and attend to it.  Every step of the computation is a libqvla call on the current stream; this file only
places buffers and pages.  Calls run one after the other, also where they are made on different streams.

Queries and keys reach attention as the linear gives them: a model with rotary positions makes the same calls itself, with its
rotation between the linear and the cache.
"""

from __future__ import annotations

import torch

from . import qvla as Q

_TORCH = {Q.F16: torch.float16, Q.BF16: torch.bfloat16}


class AttentionBlock:
    """``qkv``: a Layer with N = (heads + 2 kv_heads) head_dim, columns [Q | K | V]; ``o``: a Layer with K = heads head_dim, of
    one activation and output type.  Up to ``max_tokens`` tokens of each of ``batch`` sequences are cached."""

    def __init__(self, qkv: Q.Layer, o: Q.Layer, heads: int, kv_heads: int, head_dim: int, batch: int, max_tokens: int,
                 page_size: int = 64, rotate: bool = True, device=None):
        if qkv.N != (heads + 2 * kv_heads) * head_dim or o.K != heads * head_dim:
            raise ValueError("the layers' widths do not match the heads")
        if not qkv.xdt == qkv.ydt == o.xdt == o.ydt or qkv.ydt not in _TORCH:
            raise ValueError("the layers must share one 16-bit type")
        self.qkv, self.o, self.heads, self.kv_heads, self.dim, self.batch = qkv, o, heads, kv_heads, head_dim, batch
        self.dt, self.torch_dt = qkv.ydt, _TORCH[qkv.ydt]
        self.device = torch.device("cuda") if device is None else device
        self.scale = head_dim ** -0.5
        self.max_tokens = max_tokens
        self.width = -(-max_tokens // page_size)
        pages = batch * self.width
        self.pool = torch.zeros(Q.qvla_kv4_pool_bytes(pages, page_size, kv_heads, head_dim), dtype=torch.uint8, device=self.device)
        self.cache = Q.Kv4Cache(self.pool, pages, page_size, kv_heads, head_dim, rotate)
        self.table = torch.arange(pages, dtype=torch.int32, device=self.device).reshape(batch, self.width)
        self.lens = [0] * batch  # cached tokens, and the same on the device
        self.lens_device = torch.zeros(batch, dtype=torch.int32, device=self.device)
        self._ws = torch.empty(256, dtype=torch.uint8, device=self.device)
        self._last = torch.cuda.current_stream() if self.pool.is_cuda else None  # of the latest call

    def _stream(self) -> torch.cuda.Stream:
        """The current stream, behind the block's latest call: the cache, the lengths and the workspace serve all calls."""
        stream = torch.cuda.current_stream()
        if stream != self._last:
            stream.wait_stream(self._last)
            for t in (self.pool, self.table, self.lens_device, self._ws):
                t.record_stream(stream)
            self._last = stream
        return stream

    def _workspace(self, nbytes: int) -> torch.Tensor:
        if self._ws.numel() < nbytes:
            self._ws = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        return self._ws

    def _check(self, x, lens) -> None:
        """The library takes sizes on trust where they lie on the device: an input of other sizes would be read past its end."""
        if len(lens) != self.batch or any(n < 0 for n in lens):
            raise ValueError(f"lens must hold the tokens of {self.batch} sequences")
        if any(n + new > self.max_tokens for n, new in zip(self.lens, lens)):
            raise ValueError(f"a sequence would exceed {self.max_tokens} cached tokens")
        if tuple(x.shape) != (sum(lens), self.qkv.K) or x.dtype != self.torch_dt or not x.is_contiguous():
            raise ValueError(f"x must be contiguous {self.torch_dt} [{sum(lens)}, {self.qkv.K}]")
        if x.device.type != torch.device(self.device).type:
            raise ValueError(f"x must lie on {self.device}")

    def _linear(self, layer: Q.Layer, x, stream) -> torch.Tensor:
        m = x.shape[0]
        y = torch.empty(m, layer.N, dtype=self.torch_dt, device=self.device)
        n = Q.qvla_linear_workspace_bytes(layer, m)
        Q.qvla_w4a4_linear(layer, x, m, -1, y, self._workspace(n), n, stream)
        return y

    def _ints(self, values) -> torch.Tensor:
        return torch.tensor(values, dtype=torch.int32, device=self.device)

    def _split(self, y):
        """Queries, keys and values in the fused output, where they lie."""
        q, k = self.heads * self.dim, self.kv_heads * self.dim
        return y[:, :q], y[:, q: q + k], y[:, q + k:]

    def _store(self, y, lens, cu, stream) -> None:
        _, k, v = self._split(y)
        Q.qvla_kv4_append(self.cache, k, v, self.dt, y.stride(0), y.stride(0), self.batch, cu, y.shape[0], self.table, self.width,
                          self.lens_device, stream)
        self.lens = [n + new for n, new in zip(self.lens, lens)]
        self.lens_device = self._ints(self.lens)

    def prefill(self, x: torch.Tensor, lens, causal: bool = True) -> torch.Tensor:
        """x [sum(lens), qkv.K]: the next lens[b] tokens of every sequence (0 for none), packed.  Returns [sum(lens), o.N]."""
        self._check(x, lens)
        stream = self._stream()
        total, earlier = sum(lens), self.lens
        cu = self._ints([sum(lens[:b]) for b in range(self.batch + 1)])
        y = self._linear(self.qkv, x, stream)
        q, k, v = self._split(y)
        ks = vs = y.stride(0)
        self._store(y, lens, cu, stream)
        cu_k, total_k = cu, total
        if any(m and n for m, n in zip(earlier, lens)):
            fresh, width = (k, v), self.kv_heads * self.dim
            at = [sum(m for m, n in zip(self.lens[:b], lens) if n) for b in range(self.batch + 1)]  # keys only where there are queries
            cu_k, total_k, ks, vs = self._ints(at), at[-1], width, width
            k, v = (torch.empty(total_k, width, dtype=self.torch_dt, device=self.device) for _ in range(2))
            Q.qvla_kv4_gather(self.cache, self.batch, cu_k, total_k, self.table, self.width, None, k, v, self.dt, stream)
            for b, (m, n) in enumerate(zip(earlier, lens)):
                if n and not m:
                    new = slice(sum(lens[:b]), sum(lens[:b]) + n)
                    k[at[b]: at[b + 1]], v[at[b]: at[b + 1]] = fresh[0][new], fresh[1][new]
        a = torch.empty(total, self.heads * self.dim, dtype=self.torch_dt, device=self.device)
        Q.qvla_attention_prompt(q, k, v, self.dt, self.heads, self.kv_heads, self.dim, y.stride(0), ks, vs, self.batch, cu, total,
                                cu_k, total_k, self.scale, causal, a, stream)
        return self._linear(self.o, a, stream)

    def rewind(self, lens) -> None:
        """Back to the first lens[b] cached tokens of every sequence: those behind them are forgotten, and the next ones take their
        places.  A denoising loop goes back to its observation after each step; 0 ends a sequence."""
        if len(lens) != self.batch or any(not 0 <= n <= m for n, m in zip(lens, self.lens)):
            raise ValueError(f"lens must hold, of {self.batch} sequences, at most the cached tokens {self.lens}")
        self._stream()
        self.lens = list(lens)
        self.lens_device = self._ints(self.lens)

    def step(self, x: torch.Tensor, causal: bool = True) -> torch.Tensor:
        """x [batch * n, qkv.K]: the next n tokens of every sequence.  Returns [batch * n, o.N]."""
        total = x.shape[0]
        n = total // self.batch
        if n * self.batch != total:
            raise ValueError("x holds the same number of tokens of every sequence")
        self._check(x, [n] * self.batch)
        stream = self._stream()
        cu = self._ints([b * n for b in range(self.batch + 1)])
        y = self._linear(self.qkv, x, stream)
        self._store(y, [n] * self.batch, cu, stream)
        longest = max(self.lens)
        a = torch.empty(total, self.heads * self.dim, dtype=self.torch_dt, device=self.device)
        need = Q.qvla_attention_kv4_workspace_bytes(self.heads, self.kv_heads, self.dim, self.batch, max(total, 1), max(n, 1),
                                                    max(longest, 1))
        Q.qvla_attention_kv4(self.cache, self._split(y)[0], self.dt, self.heads, y.stride(0), self.batch, cu, total, n, self.table,
                             self.width, self.lens_device, longest, self.scale, causal, a, self._workspace(need) if need else None,
                             need, stream)
        return self._linear(self.o, a, stream)
