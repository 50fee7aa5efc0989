"""A row-wise bound for attention over the 4-bit cache, tight enough that a missing chunk or a rounding to too few bits shows.

The error of a row (one head of one query) is taken in the 2-norm, which a rotation of the outputs keeps.  With p_j the
probabilities and v_j the cached values of the row's key/value head, every rounding acts on single tokens, so where roundings are
independent their errors add up as sqrt(sum_j p_j^2 |v_j|^2); four times that is taken.  The terms:
- weights p_j Dv_j: rounded to float16, 2^-11 of each; those of like weights may all go the same way, which is 2^-11 |o|;
  and `floor` of the largest weight's power of two, absolutely (float16's subnormals);
- scores: an error d_j moves the row by sum_j p_j d_j (v_j - o).  The queries' rounding e_c = q_unit q_c gives scale sqrt(sum_c (e_c
  k_jc)^2).  The matrix instructions' float32 sums take D / 16 steps, each truncated (2^-23 of the partial sum, once, as these are
  worst cases): of the queries with codes offset to 1 to 15, partial sums stay below (8 4 + 7 4) |q| Dk_j.  2^-21 of the largest
  |score| stands for the product with scale and log2 e, the difference from the reference and the exponential;
- the float32 sums over the tokens: 2^-23 for each step of a warp; the rotations: 2^-19;
- the output's type: half an ulp of each channel, and half its smallest subnormal."""

import numpy as np
import torch

from oracle import attention_oracle as A
from tests import attention_helpers as H


def rows_of(p, q, lens_q, lens_k, causal, scale=None, leave=None):
    """Per sequence, head and query: row, head, the query, and the keys and values that it sees, float64 in the cache's basis, and the
    scale; `leave`: tokens (first, end) that are left out, as if a chunk of them had been lost."""
    k, v = p.heads(lens_k)
    k, v, qd = k.astype(np.float64), v.astype(np.float64), H.f64(q)
    qd = qd @ A.hadamard(p.dim) if p.rotate else qd
    scale = p.dim ** -0.5 if scale is None else scale
    at_q, at_k = H.offsets(lens_q), H.offsets(lens_k)
    group = q.shape[1] // p.kv
    for b, (n, m) in enumerate(zip(lens_q, lens_k)):
        see = np.arange(m)[None] <= (m - n + np.arange(n))[:, None] if causal else np.ones((n, m), bool)
        if leave is not None:
            see = see & ~((np.arange(m) >= leave[0]) & (np.arange(m) < leave[1]))[None]
        for h in range(q.shape[1]):
            kb, vb = k[at_k[b]: at_k[b + 1], h // group], v[at_k[b]: at_k[b + 1], h // group]
            for i in range(n):
                js = np.nonzero(see[i])[0]
                yield at_q[b] + i, h, qd[at_q[b] + i, h], kb[js], vb[js], scale


def statement(p, q, lens_q, lens_k, causal, scale=None, q_unit=0.0, warps=4, floor=2.0 ** -32, leave=None):
    """(o, bound): o [queries, heads, dim] float64 in the model's basis, and the bound of a row's 2-norm [queries, heads]."""
    o, tol = np.zeros(q.shape), np.zeros(q.shape[:2])
    out = "f16" if q.dtype == torch.float16 else "bf16"
    for i, h, qi, k, v, scale_ in rows_of(p, q, lens_q, lens_k, causal, scale, leave):
        if len(k) == 0:
            continue
        s = scale_ * (k @ qi)
        w = np.exp(s - s.max())
        pr = w / w.sum()
        o[i, h] = pr @ v
        size = np.linalg.norm(v, axis=1)
        scales = np.abs(v).max(1)  # of a token's values, up to 7 Dv
        of_queries = scale_ * q_unit * np.sqrt((k * k) @ (qi * qi))
        of_sums = scale_ * (p.dim / 16 + 4) * 2.0 ** -23 * 60 / 7 * np.linalg.norm(qi) * np.abs(k).max(1)
        d = 4 * of_queries + of_sums + 2.0 ** -21 * (np.abs(s).max() + 1)
        norm = np.linalg.norm(o[i, h])
        spread = np.sqrt(np.sum((pr * size) ** 2))
        steps = len(k) / (16 * warps) + 8
        tol[i, h] = (2.0 ** -11 * (norm + 4 * spread) + floor * (w * scales).max() * np.sqrt(p.dim) * len(k) / w.sum()
                     + np.sqrt(np.sum((pr * d * np.linalg.norm(v - o[i, h], axis=1)) ** 2))
                     + steps * 2.0 ** -23 * (norm + 4 * spread) + 2.0 ** -19 * norm
                     + H.UNIT[out] * norm + 2.0 ** -25 * np.sqrt(p.dim))
    return (o @ A.hadamard(p.dim) if p.rotate else o), tol


def error(got, want):
    return np.linalg.norm(np.asarray(got, np.float64) - want, axis=-1)
