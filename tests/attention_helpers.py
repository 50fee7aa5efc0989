"""Shared pieces of the attention tests: packed inputs, paged pools, calls through the binding, and the elementwise bound
that a result has to keep against the float64 statement."""

import numpy as np
import torch

from oracle import attention_oracle as A
from paper_2605_28803_gb300 import qvla as Q

DEV = "cuda"
TORCH = {"f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}  # half an ulp, relative


def stream():
    return torch.cuda.current_stream()


def ints(values):
    return torch.tensor(list(values), dtype=torch.int32, device=DEV)


def offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


def draw_heads(rng, n, heads, dim, dtype, outliers=False):
    x = rng.standard_normal((n, heads, dim), dtype=np.float32)
    if outliers and n:
        x[:, :, rng.integers(0, dim, 3)] *= 5.0
    return torch.from_numpy(x).to(TORCH[dtype])


def f64(t):
    return t.double().cpu().numpy()


def prompt(q, k, v, lens_q, lens_k, causal, scale=None, cu_q=None, cu_k=None):
    """qvla_attention_prompt on device copies of q [n, heads, dim], k, v [m, kv, dim] (any token strides)."""
    heads, dim = q.shape[1:]
    scale = dim ** -0.5 if scale is None else scale
    o = torch.full((q.shape[0], heads, dim), float("nan"), dtype=q.dtype, device=DEV)
    dt = Q.F16 if q.dtype == torch.float16 else Q.BF16
    Q.qvla_attention_prompt(q, k, v, dt, heads, k.shape[1], dim, q.stride(0), k.stride(0), v.stride(0), len(lens_q),
                            ints(offsets(lens_q)) if cu_q is None else cu_q, q.shape[0],
                            ints(offsets(lens_k)) if cu_k is None else cu_k, k.shape[0], scale, causal, o, stream())
    return o


def bound(ref, mag, top, terms, dim, out, p_unit, q_unit, v_sum):
    """What the roundings may add up to, elementwise.
    - the output's rounding: UNIT |o|, and half the smallest f16 subnormal;
    - a probability: p_unit relative (rounded to 16 bits for the product with the values; its f16 form has an
      absolute floor of 2^-25, with values that sum to v_sum);
    - a score: its float32 sum of dim terms (at most (dim + 4) 2^-24 of the sum of magnitudes; products and partial sums
      on the tensor cores may be truncated instead of rounded, twice that), the query's own rounding q_unit, the
      product with scale and log2 e and the exponential (2^-22 relative and 4 ulp of the largest |score|).  An error d in
      a score is at most 2 d (1 + d) in a normalised probability, numerator and denominator both;
    - float32 sums over the keys: 2^-20."""
    d = (2 * (dim + 4) * 2.0 ** -24 + q_unit) * terms + 8 * 2.0 ** -24 * (top + 1) + 2.0 ** -21
    rel = p_unit + 2 * d * (1 + d) + 2.0 ** -20
    return UNIT[out] * np.abs(ref) * 1.01 + rel[..., None] * 1.05 * mag + 2.0 ** -25 * (1 + v_sum)


def reference(q, k, v, lens_q, lens_k, causal, scale=None):
    """float64 attention over packed sequences; (o, mag, top, terms) of all rows."""
    dim = q.shape[-1]
    scale = dim ** -0.5 if scale is None else scale
    oq, ok = offsets(lens_q), offsets(lens_k)
    parts = [A.attention(q[oq[b]: oq[b + 1]], k[ok[b]: ok[b + 1]], v[ok[b]: ok[b + 1]], scale, causal)
             for b in range(len(lens_q))]
    return [np.concatenate([p[i] for p in parts]) for i in range(4)]


class Paged:
    """A pool of random contents (also where no token lies) and a table of pages for sequences of `lens` tokens, in random
    order; entries that no token needs are -1."""

    def __init__(self, rng, lens, kv_heads, dim, page, rotate, spare=2, extra_columns=1):
        need = [-(-n // page) for n in lens]
        self.pages, self.page, self.kv, self.dim, self.rotate = sum(need) + spare, page, kv_heads, dim, rotate
        self.width = max(need + [0]) + extra_columns
        order = rng.permutation(self.pages)
        self.table = np.full((len(lens), self.width), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at: at + n]
            at += n
        self.pool = rng.integers(0, 256, (self.pages, kv_heads, page * (dim + 8)), dtype=np.uint8)
        self.device = torch.from_numpy(self.pool).to(DEV)
        self.table_device = torch.from_numpy(self.table).to(DEV)
        self.cache = Q.Kv4Cache(self.device, self.pages, page, kv_heads, dim, rotate)

    def fill(self, rng, lens, k_scale=0.3, v_scale=0.3):
        """Codes in [-7, 7] and ordinary scales at every token's place; NaN scales and any codes elsewhere."""
        kc, vc, ks, vs = A.pool_parts(self.pool, self.page, self.dim)
        ks[...] = np.nan
        vs[...] = np.nan
        for b, n in enumerate(lens):
            pos = np.arange(n)
            at, slot = self.table[b, pos // self.page], pos % self.page
            for codes, scales, s in ((kc, ks, k_scale), (vc, vs, v_scale)):
                codes[at, :, slot] = A.pack_nibbles(rng.integers(-7, 8, (n, self.kv, self.dim)))
                scales[at, :, slot] = rng.uniform(0.3, 1.0, (n, self.kv)).astype(np.float32) * s
        self.device.copy_(torch.from_numpy(self.pool))

    def heads(self, lens, first=None):
        """Cached keys and values of all sequences, packed, float32 in the cache's basis."""
        parts = [A.cached_heads(self.pool, self.page, self.dim, self.table[b], n, 0 if first is None else first[b])
                 for b, n in enumerate(lens)]
        return tuple(np.concatenate([p[i] for p in parts]) for i in range(2))

    def read_back(self, lens, first):
        """What the cache gives back, packed, float32 in the model's basis."""
        parts = [A.cached_read_back(self.pool, self.page, self.dim, self.table[b], n, first[b], self.rotate)
                 for b, n in enumerate(lens)]
        return tuple(np.concatenate([p[i] for p in parts]) for i in range(2))


def kv4(p, q, lens_q, lens_k, causal, scale=None, ws_bytes=None, max_q=None, max_len=None, cu_q=None, kv_len=None):
    """qvla_attention_kv4; ws_bytes None: the library's own size."""
    heads, dim = q.shape[1:]
    scale = dim ** -0.5 if scale is None else scale
    max_q = max(lens_q) if max_q is None else max_q
    max_len = max(lens_k) if max_len is None else max_len
    if ws_bytes is None:
        ws_bytes = Q.qvla_attention_kv4_workspace_bytes(heads, p.kv, dim, len(lens_q), max(1, q.shape[0]), max(1, max_q),
                                                        max(1, max_len))
    ws = torch.full((max(ws_bytes, 1),), 255, dtype=torch.uint8, device=DEV)
    o = torch.full((q.shape[0], heads, dim), float("nan"), dtype=q.dtype, device=DEV)
    dt = Q.F16 if q.dtype == torch.float16 else Q.BF16
    Q.qvla_attention_kv4(p.cache, q, dt, heads, q.stride(0), len(lens_q), ints(offsets(lens_q)) if cu_q is None else cu_q,
                         q.shape[0], max_q, p.table_device, p.width, ints(lens_k) if kv_len is None else kv_len, max_len,
                         scale, causal, o, ws if ws_bytes else None, ws_bytes, stream())
    return o


def kv4_reference(p, q, lens_q, lens_k, causal, scale=None):
    """float64 attention over the cache's values; (o, mag, top, terms) in the model's basis.  `mag` of a rotated cache is the
    bound of a rotated row: sum_c |H_cd| mag_c."""
    k, v = p.heads(lens_k)
    qd = f64(q)
    h = A.hadamard(p.dim)
    o, mag, top, terms = reference(qd @ h if p.rotate else qd, k, v, lens_q, lens_k, causal, scale)
    if p.rotate:
        o, mag = o @ h, mag @ np.abs(h)
    return o, mag, top, terms
