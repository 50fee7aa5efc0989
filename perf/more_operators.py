"""The operators of microscaled 4-bit floating point whose speed and outputs are measured: quantising rows, the product
of two quantised matrices, and the norms on either side of a block with its gate and residual.

A case is a dict of plain values:
  kind     "quantize"  rows to codes and scales, then read back as values of the rows' type
           "linear"    rows quantised, then multiplied by a layer's quantised weights
           "product"   rows that are codes already, multiplied by a layer's weights
           "norm"      residual + gate * branch, then the next block's norm
           "junction"  the same with its output quantised, then the next block's first product
  m, k, n  rows (tokens), channels, output channels (0 where there are none; of a gated layer the hidden units)
  fmt      "mx": blocks of 32 channels with a power of two (E8M0);  "nv": blocks of 16 channels with an E4M3 scale, and a
           float32 scale a row
  had      the Hadamard block ahead of the quantiser (1: none)
  dtype    "f16" or "bf16", of rows, outputs, branch and norm parameters;  rdtype  the residual's, also "f32"
  gated, bias   of the layer
  norm     "rms" or "layer";  branch, post, cond: a branch is added; it is normalised first; gate, scale and shift are given
           for every `cond` tokens (0: none)

A 4-bit code is E2M1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives (bit 3).  Byte j of a row holds code 2j in its low nibble
and 2j + 1 in its high one.  Block scales lie in tiles of 128 rows x 4 blocks, 512 bytes each, tile (m / 128, b / 4) of a
row-major grid: the scale of row m and block b is byte (m % 32) * 16 + (m / 32 % 4) * 4 + b % 4 of its tile.

Layers are those of the repository's models: the backbone (816 prompt tokens, 2048 channels, MLP 2 x 16384, fused QKV
2560) and the action head (50 tokens, 1024 channels, MLP 4096); the odd sizes are generic.
"""

import math

import torch

own = False

DEV = "cuda"
_TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_BLOCK = {"mx": 32, "nv": 16}
_EPS = 1e-6


def _case(name, kind, m, k, n=0, fmt="nv", had=1, dtype="bf16", rdtype="bf16", gated=False, bias=False, norm="rms", branch=True,
          post=False, cond=0):
    return dict(name=name, kind=kind, m=m, k=k, n=n, fmt=fmt, had=had, dtype=dtype, rdtype=rdtype, gated=gated, bias=bias,
                norm=norm, branch=branch, post=post, cond=cond)


def listed():
    return [
        # one decoded token's hidden state ahead of the backbone's QKV
        _case("quantize_token", "quantize", 1, 2048, had=2048),
        # the MLP's hidden units of one observation, ahead of the down projection
        _case("quantize_prefix", "quantize", 816, 16384, had=2048),
        # a ragged batch of prompts, the short rotation, float16
        _case("quantize_batch", "quantize", 3211, 2432, fmt="mx", had=128, dtype="f16"),
        # the down projection of one decoded token: all of its time is the weights
        _case("linear_token", "linear", 1, 16384, 2048, had=2048),
        # the action head's up projection in one denoising step
        _case("linear_action", "linear", 50, 1024, 4096, fmt="mx", had=64, dtype="f16", bias=True),
        # the gated MLP over one observation
        _case("product_prefix", "product", 816, 2048, 16384, gated=True),
        # prompts of odd length through a layer of odd width
        _case("product_batch", "product", 1187, 4096, 2576, fmt="mx", dtype="f16", bias=True),
        # ten observations through a wide layer
        _case("product_large", "product", 8192, 2048, 16384, fmt="mx"),
        # the action head between attention and MLP: conditioned gate, scale and shift
        _case("norm_action", "norm", 50, 1024, dtype="f16", rdtype="f16", norm="layer", cond=50),
        # eight observations, norms on both sides of the block, the residual held in float32
        _case("norm_prefix", "norm", 6528, 2048, rdtype="f32", post=True),
        # the action heads of four robots, to the MLP's up projection
        _case("junction_action", "junction", 200, 1024, 4096, dtype="f16", rdtype="f16", had=1024, norm="layer", cond=50, bias=True),
        # the backbone between MLP and the next layer's fused QKV
        _case("junction_prefix", "junction", 816, 2048, 2560, had=2048),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["quantize", "linear", "product", "product", "norm", "junction"])
    m, k = _spread(rng, 1, 8192), 128 * _spread(rng, 1, 128)
    n = 16 * _spread(rng, 1, 1024) if kind in ("linear", "product", "junction") else 0
    gated = n > 0 and rng.random() < 0.25
    if gated:
        n = -(-n // 128) * 128
    while m * k > 1 << 25 or m * k * n * (2 if gated else 1) > 1 << 38:
        m = -(-m // 2)
    had = rng.choice([b for b in (1, 1, 16, 64, 128, 256, 512, 1024, 2048, 4096) if k % b == 0])
    dtype = rng.choice(["f16", "bf16"])
    norms = kind in ("norm", "junction")
    branch = not norms or rng.random() < 0.85
    c = _case("", kind, m, k, n, rng.choice(["mx", "nv"]), 1 if kind in ("product", "norm") else had, dtype,
              rng.choice([dtype, dtype, "f32"]) if norms else dtype, gated, n > 0 and rng.random() < 0.5,
              rng.choice(["rms", "layer"]), branch, branch and rng.random() < 0.4, rng.choice([0, m, -(-m // 3)]) if norms else 0)
    del c["name"]
    return c


# ---- shapes and inputs -------------------------------------------------------------------------------------------

def _scale_bytes(fmt, rows, k):
    return -(-rows // 128) * (k // _BLOCK[fmt] // 4) * 512


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _rows(g, m, k, dtype):
    """N(0, 1) rows with a few channels (the same in every row) twenty times larger, as a model's activations have."""
    x = torch.randn(m, k, generator=g, device=DEV)
    x[:, torch.randperm(k, generator=g, device=DEV)[: max(1, k // 200)]] *= 20.0
    return x.to(_TORCH[dtype])


def _codes(g, rows, k, fmt, size):
    """Codes, block scales and row scales of a matrix of `rows` rows whose entries are about `size`."""
    q = torch.randint(0, 256, (rows, k // 2), generator=g, device=DEV, dtype=torch.int32).to(torch.uint8)
    nbytes = _scale_bytes(fmt, rows, k)
    if fmt == "nv":  # E4M3 bytes of 64 to 448, as blocks have them whose largest entry is not far below the row's
        s = torch.randint(0x68, 0x7F, (nbytes,), generator=g, device=DEV, dtype=torch.int32).to(torch.uint8)
        row = (torch.rand(rows, generator=g, device=DEV) * 0.4 + 0.8) * (size / 800.0)
    else:
        e = 127 + round(math.log2(size / 3.0))
        s = torch.randint(e - 1, e + 2, (nbytes,), generator=g, device=DEV, dtype=torch.int32).to(torch.uint8)
        row = None
    return q, s, row


def _vector(g, k, dtype, mean, spread, rows=None):
    shape = (k,) if rows is None else (rows, k)
    return (torch.randn(shape, generator=g, device=DEV) * spread + mean).to(_TORCH[dtype])


def prepare(case, seed):
    s = dict(case)
    g = _gen(seed)
    m, k, n, fmt, dt = s["m"], s["k"], s["n"], s["fmt"], _TORCH[s["dtype"]]
    rows = 2 * n if s["gated"] else n
    if n:
        s["wq"], s["ws"], s["wrow"] = _codes(g, rows, k, fmt, 1.0 / math.sqrt(k))
        s["b"] = torch.randn(rows, generator=g, device=DEV) * 0.1 if s["bias"] else None
        s["out"] = torch.empty(m, n, dtype=dt, device=DEV)
    if s["kind"] == "product":
        s["xq"], s["xs"], s["xrow"] = _codes(g, m, k, fmt, 1.0)
    elif s["kind"] in ("quantize", "linear"):
        s["x"] = _rows(g, m, k, s["dtype"])
    else:
        s["r"] = _rows(g, m, k, s["rdtype"])
        s["y"] = _rows(g, m, k, s["dtype"]) if s["branch"] else None
        s["post_w"] = _vector(g, k, s["dtype"], 0.0, 0.3) if s["post"] else None  # stored less one
        s["pre_w"] = _vector(g, k, s["dtype"], 0.0, 0.3)
        s["pre_b"] = _vector(g, k, s["dtype"], 0.0, 0.2) if s["norm"] == "layer" else None
        if s["cond"]:
            c = -(-m // s["cond"])
            mod = _vector(g, 3 * k, s["dtype"], 0.0, 0.5, c)  # a conditioning layer's output: gate, scale, shift
            s["gate"], s["scale"], s["shift"] = mod[:, :k], mod[:, k: 2 * k], mod[:, 2 * k:]
        else:
            s["gate"] = s["scale"] = s["shift"] = None
        s["r_out"] = torch.empty_like(s["r"])
        s["h"] = torch.empty(m, k, dtype=dt, device=DEV)
    if s["kind"] in ("quantize", "junction"):
        s["hq"] = torch.empty(m, k // 2, dtype=torch.uint8, device=DEV)
        s["hs"] = torch.zeros(_scale_bytes(fmt, m, k), dtype=torch.uint8, device=DEV)
        s["hrow"] = torch.empty(m, device=DEV)
        s["values"] = torch.empty(m, k, dtype=dt, device=DEV)
    if own:
        _prepare_own(s, rows)
    return s


def _prepare_own(s, rows):
    from paper_2605_28803_gb300 import qvla as Q

    fmt = Q.MXFP4 if s["fmt"] == "mx" else Q.NVFP4
    s["code"], s["fmt_code"] = Q.DTYPE_CODES[s["dtype"]], fmt
    if s["n"]:
        host = [None if t is None else t.cpu().numpy() for t in (s["wq"], s["ws"], s["wrow"], s["b"])]
        create = Q.qvla_fp4_layer_create_gated if s["gated"] else Q.qvla_fp4_layer_create
        s["layer"] = create(s["n"], s["k"], s["had"], fmt, s["code"], s["code"], *host)
        s["ws_bytes"] = Q.qvla_fp4_linear_workspace_bytes(s["layer"], s["m"])
        s["work"] = torch.empty(max(s["ws_bytes"], 256), dtype=torch.uint8, device=DEV)
    if s["kind"] in ("norm", "junction"):
        s["plan"] = Q.BlockNorm(Q.NORM_RMS if s["norm"] == "rms" else Q.NORM_LAYER, s["code"], eps=_EPS, weight_offset=1.0,
                                residual_scale=1.0, post_norm=s["post"], post_weight=s["post_w"], pre_weight=s["pre_w"],
                                pre_bias=s["pre_b"], gate=s["gate"], scale=s["scale"], shift=s["shift"], mod_tokens=s["cond"])


# ---- the operators in their plain form ----------------------------------------------------------------------------

def _hadamard(x, b):
    """Blocks of b channels times the Hadamard matrix / sqrt(b), float32, butterflies of distance b/2, b/4, ..., 1."""
    shape, h = x.shape, b // 2
    while h >= 1:
        lo, hi = x.reshape(-1, 2, h).unbind(1)
        x = torch.stack((lo + hi, lo - hi), 1)
        h //= 2
    return x.reshape(shape) * torch.tensor(1.0 / math.sqrt(b), dtype=torch.float32, device=x.device)


def _e2m1():
    v = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV)
    return torch.cat((v, -v))


def _scale_place(rows, blocks):
    """Where the scales of row m and block b lie: byte offsets [rows, blocks]."""
    m, b = torch.arange(rows, device=DEV)[:, None], torch.arange(blocks, device=DEV)[None]
    return ((m // 128) * (blocks // 4) + b // 4) * 512 + (m % 32) * 16 + (m // 32 % 4) * 4 + b % 4


def _scale_values(fmt, tiles, rows, k):
    """float32 [rows, blocks]."""
    bytes_ = tiles[_scale_place(rows, k // _BLOCK[fmt])]
    if fmt == "nv":
        return bytes_.view(torch.float8_e4m3fn).float()
    return torch.exp2((bytes_.int() - 127).float())


def _values(fmt, q, tiles, k):
    """float32 [rows, k]: codes times block scales, without the rows' scales."""
    codes = torch.stack((q & 15, q >> 4), -1).flatten(1).long()
    return _e2m1()[codes] * _scale_values(fmt, tiles, q.shape[0], k).repeat_interleave(_BLOCK[fmt], 1)


def _round_float(x, bits, low, high):
    """float64 to the nearest number of 1 + bits significant bits, half to even, the smallest exponent `low`, at most `high`."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** low))) - bits)
    return (torch.round(x / step) * step).clamp(-high, high)


def _quantized(fmt, z):
    """z float32 [rows, k] to (codes * block scales float32 [rows, k], rows' scales float32 [rows, 1])."""
    zb = z.reshape(z.shape[0], -1, _BLOCK[fmt])
    top = zb.abs().amax(-1, keepdim=True)
    if fmt == "mx":
        e = (torch.floor(torch.log2(top.double().clamp(min=2.0 ** -149))) - 2).clamp(-127, 127)
        scale, row = torch.exp2(e), torch.ones(z.shape[0], 1, device=DEV)
        unit = scale
    else:
        row = torch.div(top.amax(1), torch.tensor(2688.0, device=DEV))
        # the quotients of float32 numbers are rounded from 64 bits, where their ties are true ones
        scale = _round_float(top.double() / (6.0 * row.double()[:, None]).clamp(min=1e-300), 3, -6, 448.0)
        unit = (scale.float() * row[:, None]).double()
    q = torch.where(unit > 0, zb.double() / unit.clamp(min=1e-300), 0.0)
    return (_round_float(q, 1, 0, 6.0) * scale).float().reshape(z.shape), row


def _rotated(s, x):
    return _hadamard(x.float(), s["had"]) if s["had"] > 1 else x.float()


def _gelu(x):
    return 0.5 * x * (1.0 + torch.tanh(0.7978845608028654 * (x + 0.044715 * x * x * x)))


def _multiply(s, x, row):
    """x float32 [m, k] and its rows' scales by the layer's weights."""
    y = x @ _values(s["fmt"], s["wq"], s["ws"], s["k"]).T
    if s["fmt"] == "nv":
        y *= row * s["wrow"]
    if s["b"] is not None:
        y += s["b"]
    if s["gated"]:
        y = _gelu(y[:, : s["n"]]) * y[:, s["n"]:]
    return y.to(_TORCH[s["dtype"]])


def _normed(s, x, weight, bias=None):
    if s["norm"] == "layer":
        x = x - x.mean(-1, keepdim=True)
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS) * (1.0 + weight.float())
    return x if bias is None else x + bias.float()


def _given(s, name):
    """The conditioning of every token, float32."""
    return s[name].float().repeat_interleave(s["cond"], 0)[: s["m"]]


def _block_norm(s):
    r = s["r"]
    if s["y"] is not None:
        u = s["y"].float()
        if s["post"]:
            u = _normed(s, u, s["post_w"])
        if s["cond"]:
            u = u * _given(s, "gate")
        r = (r.float() + u).to(r.dtype)
    h = _normed(s, r.float(), s["pre_w"], s["pre_b"])
    if s["cond"]:
        h = h * (1.0 + _given(s, "scale")) + _given(s, "shift")
    return r, h.to(_TORCH[s["dtype"]])


def _plain(s):
    kind = s["kind"]
    if kind == "product":
        return _multiply(s, _values(s["fmt"], s["xq"], s["xs"], s["k"]), None if s["xrow"] is None else s["xrow"][:, None])
    if kind in ("quantize", "linear"):
        v, row = _quantized(s["fmt"], _rotated(s, s["x"]))
        return (v * row).to(_TORCH[s["dtype"]]) if kind == "quantize" else _multiply(s, v, row)
    r, h = _block_norm(s)
    if kind == "norm":
        return {"residual": r, "h": h}
    return {"residual": r, "y": _multiply(s, *_quantized(s["fmt"], _rotated(s, h)))}


# ---- the same through the library's entry points --------------------------------------------------------------------

def _own(s):
    from paper_2605_28803_gb300 import qvla as Q

    st = torch.cuda.current_stream()
    kind, m, k, fmt, code = s["kind"], s["m"], s["k"], s["fmt_code"], s["code"]
    if kind == "quantize":
        Q.qvla_fp4_quantize_rows(s["x"], code, k, m, k, s["had"], fmt, None, s["hq"], s["hs"], s["hrow"], st)
        Q.qvla_fp4_dequantize_rows(s["hq"], s["hs"], s["hrow"], fmt, m, k, s["values"], code, st)
        return s["values"]
    if kind == "linear":
        Q.qvla_fp4_linear(s["layer"], s["x"], m, None, s["out"], s["work"], s["ws_bytes"], st)
        return s["out"]
    if kind == "product":
        Q.qvla_gemm_fp4(s["layer"], s["xq"], s["xs"], s["xrow"], m, s["out"], st)
        return s["out"]
    rcode = Q.DTYPE_CODES[s["rdtype"]]
    r_out, written = (s["r"], None) if s["y"] is None else (s["r_out"], s["r_out"])
    if kind == "norm":
        Q.qvla_block_norm(s["plan"], s["r"], rcode, k, s["y"], k, m, k, written, s["h"], st)
        return {"residual": r_out, "h": s["h"]}
    Q.qvla_block_norm_fp4(s["plan"], s["r"], rcode, k, s["y"], k, m, k, written, None, s["had"], fmt, None, s["hq"], s["hs"],
                          s["hrow"], st)
    Q.qvla_gemm_fp4(s["layer"], s["hq"], s["hs"], s["hrow"], m, s["out"], st)
    return {"residual": r_out, "y": s["out"]}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    m, k, n, kind = case["m"], case["k"], case["n"], case["kind"]
    rows = 2 * n if case["gated"] else n
    per_row = k // 2 + k // _BLOCK[case["fmt"]] + (4 if case["fmt"] == "nv" else 0)
    turns = k * m * int(math.log2(case["had"]))
    if kind == "quantize":  # the rows in, codes and scales out; those in again, values out
        return {"bytes": m * (2 * k + 2 * per_row + 2 * k), "flops": turns + 3 * m * k}
    product = {"bytes": rows * per_row + 2 * m * n + (4 * rows if case["bias"] else 0), "flops": 2 * m * k * rows}
    if kind == "product":
        return {"bytes": product["bytes"] + m * per_row, "flops": product["flops"]}
    if kind == "linear":
        return {"bytes": product["bytes"] + 2 * m * k, "flops": product["flops"] + turns + 3 * m * k}
    res = 4 if case["rdtype"] == "f32" else 2
    vectors = 2 * k * (1 + (1 if case["post"] else 0) + (1 if case["norm"] == "layer" else 0))
    mod = 2 * k * -(-m // case["cond"]) * (3 if case["branch"] else 2) if case["cond"] else 0
    read = m * k * (res + (2 if case["branch"] else 0)) + vectors + mod
    wrote = m * k * (res if case["branch"] else 0)
    if kind == "norm":
        return {"bytes": read + wrote + 2 * m * k, "flops": 10 * m * k}
    return {"bytes": read + wrote + product["bytes"], "flops": product["flops"] + turns + 13 * m * k}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

def _sylvester(b):
    h = torch.ones(1, 1, dtype=torch.float64, device=DEV)
    while h.shape[0] < b:
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)), 0)
    return h / math.sqrt(b)


def _matrix(fmt, q, tiles, row, k):
    """A quantised matrix's values, float64, from its bytes."""
    rows, per = q.shape[0], _BLOCK[fmt]
    grid = tiles.reshape(-(-rows // 128), k // per // 4, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, k // per)[:rows].long()
    if fmt == "mx":
        scale = torch.ldexp(torch.ones_like(grid, dtype=torch.float64), grid - 127)
    else:  # 1.mmm 2^(e - 7), or 0.mmm 2^-6
        e, f = grid // 8 % 16, (grid % 8).double() / 8
        scale = torch.where(e > 0, torch.ldexp(1 + f, e - 7), f / 64)
    out = torch.empty(rows, k, dtype=torch.float64, device=DEV)
    for half in (0, 1):
        c = q.long() % 16 if half == 0 else q.long() // 16
        e, f = c // 2 % 4, (c % 2).double() / 2
        v = torch.where(e > 0, torch.ldexp(1 + f, e - 1), f)
        out[:, half::2] = torch.where(c >= 8, -v, v)
    out = (out.reshape(rows, -1, per) * scale[..., None]).reshape(rows, k)
    return out if row is None else out * row.double()[:, None]


def _nearest(x, numbers, even):
    """Each entry of x >= 0 to the nearest of `numbers` (ascending), a tie to the one with an even code."""
    i = torch.bucketize(x, numbers).clamp(1, numbers.numel() - 1)
    lo, hi = numbers[i - 1], numbers[i]
    up = (x - lo > hi - x) | ((x - lo == hi - x) & even[i])
    return torch.where(x >= numbers[-1], numbers[-1], torch.where(up, hi, lo))


def _quantized_exact(fmt, z):
    """What the rows z (float64) stand for once quantised."""
    e2m1 = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEV)
    even8 = torch.arange(8, device=DEV) % 2 == 0
    out = torch.zeros_like(z)
    row = (z.abs().amax(1) / 2688).float().double()  # a float32 number
    if fmt == "nv":
        c = torch.arange(127, device=DEV)  # E4M3 from zero to 448
        e4m3 = torch.where(c >= 8, torch.ldexp(1 + (c % 8).double() / 8, c // 8 - 7), (c % 8).double() / 512)
    for at in range(0, z.shape[1], _BLOCK[fmt]):
        part = z[:, at: at + _BLOCK[fmt]]
        top = part.abs().amax(1)
        if fmt == "mx":
            scale = torch.ldexp(torch.ones_like(top), (torch.frexp(top).exponent - 3).clamp(-127, 127))
            unit = scale
        else:
            scale = _nearest(torch.nan_to_num(top / (6 * row)), e4m3, c % 2 == 0) * row
            unit = scale.float().double()  # codes are rounded against a float32 number
        q = torch.where(unit[:, None] > 0, part.abs() / unit[:, None], 0.0)
        out[:, at: at + _BLOCK[fmt]] = torch.sign(part) * _nearest(q, e2m1, even8) * scale[:, None]
    return out


def _product_exact(s, x):
    y = x @ _matrix(s["fmt"], s["wq"], s["ws"], s["wrow"], s["k"]).T
    if s["b"] is not None:
        y += s["b"].double()
    if s["gated"]:
        gate, up = y.split(s["n"], 1)
        y = gate / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (gate + 0.044715 * gate ** 3))) * up
    return y


def _norm_exact(s):
    def norm(x, w):
        d = x if s["norm"] == "rms" else x - x.sum(1, keepdim=True) / s["k"]
        return d / torch.sqrt((d ** 2).sum(1, keepdim=True) / s["k"] + _EPS) * (w.double() + 1)

    token = torch.arange(s["m"], device=DEV) // max(1, s["cond"])
    r = s["r"].double()
    if s["branch"]:
        u = norm(s["y"].double(), s["post_w"]) if s["post"] else s["y"].double()
        r = r + (u * s["gate"].double()[token] if s["cond"] else u)
        exact_r = r
        r = r.to(s["r"].dtype).double()  # the norm reads the residual as it is stored
    else:
        exact_r = r
    h = norm(r, s["pre_w"])
    if s["norm"] == "layer":
        h = h + s["pre_b"].double()
    if s["cond"]:
        h = h * (1 + s["scale"].double()[token]) + s["shift"].double()[token]
    return exact_r, h


def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]
    if kind == "product":
        return _product_exact(s, _matrix(s["fmt"], s["xq"], s["xs"], s["xrow"], s["k"]))
    if kind == "norm":
        r, h = _norm_exact(s)
        return {"residual": r, "h": h}
    r, x = None, None
    if kind == "junction":
        r, h = _norm_exact(s)
        x = h.to(_TORCH[s["dtype"]]).double()  # the quantiser reads the norm's output rounded to its type
    else:
        x = s["x"].double()
    if s["had"] > 1:
        x = (x.reshape(-1, s["had"]) @ _sylvester(s["had"])).reshape(x.shape)
    v = _quantized_exact(s["fmt"], x)
    if kind == "quantize":
        return v
    y = _product_exact(s, v)
    return {"residual": r, "y": y} if kind == "junction" else y
