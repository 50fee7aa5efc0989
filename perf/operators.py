"""The attention operators whose speed and outputs are measured: attention over packed prompts, and a paged
key/value cache of 4-bit codes -- storing tokens, reading them back, and attention over it for a few query tokens.

A case is a dict of plain values:
  kind     "prompt"  softmax attention over packed sequences: grouped heads, causal or full
           "append"  new tokens' keys and values stored in the cache, then read back as values
           "gather"  cached tokens read back as values
           "decode"  attention of the last tokens of every sequence over its part of the cache
  heads, kv_heads, dim   query heads, key/value heads, channels a head
  dtype    "f16" or "bf16", of queries, keys, values and outputs
  causal   each query sees the keys up to its own position; the last query stands at the last key
  q_lens   tokens of each sequence (text, comma separated): queries, or new tokens
  k_lens   keys of each sequence: for "append" the tokens cached before, for "gather" the tokens read
  page     tokens a cache page holds;  rotate  whether heads are Hadamard-rotated ahead of the quantiser

The cache's pool is uint8 [pages][kv_heads][page * (dim + 8)]: the keys' codes [page][dim / 2], the values' codes, the
keys' scales float32 [page], the values' scales.  A byte holds two channels, the even one in its low nibble, as
two's-complement codes in [-7, 7]; a channel stands for code * scale, scale = max |y| / 7 of the token's head, codes
rounded half to even on the exact quotient.  With `rotate`, y is the head times the Hadamard matrix / sqrt(dim).
Positions follow a table of pages for each sequence, in no order.

Heads are those of the repository's models: 8 heads of 256 channels over one key/value head (the backbone, 816
prompt tokens) and 8 of 128 (the action head, 50 tokens); the other head counts, 64 channels and the longer contexts
are generic.
"""

import math

import torch

own = False

DEV = "cuda"
_TORCH = {"f16": torch.float16, "bf16": torch.bfloat16}


def _case(name, kind, heads, kv_heads, dim, dtype, q_lens, k_lens, causal=True, page=64, rotate=True):
    return dict(name=name, kind=kind, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, causal=causal,
                q_lens=",".join(map(str, q_lens)), k_lens=",".join(map(str, k_lens)), page=page, rotate=rotate)


def listed():
    packed, over = [1, 37, 816, 129, 1500, 64, 333], [1, 37, 816, 2000, 1500, 900, 333]
    ragged = [1, 4093, 17, 816, 2500, 63, 64, 65, 1290, 6001, 128, 3, 777, 2048, 5, 950, 333, 1500, 31, 407, 2222, 90, 612]
    return [
        # the action head's self-attention of one denoising step: 50 action tokens, every head its own keys
        _case("prompt_action_50", "prompt", 8, 8, 128, "f16", [50], [50], causal=False),
        # the backbone over one observation: 816 image and text tokens that see one another
        _case("prompt_prefix_816", "prompt", 8, 1, 256, "bf16", [816], [816], causal=False),
        # prompts of seven users packed into one batch, one of a single token, two with a part that was read back from
        # the cache ahead of their own tokens
        _case("prompt_packed", "prompt", 14, 2, 64, "bf16", packed, over),
        # one long document
        _case("prompt_long", "prompt", 16, 4, 128, "bf16", [8192], [8192]),
        # one decoded token of each of sixteen sequences enters the cache
        _case("append_tokens", "append", 8, 1, 256, "bf16", [1] * 16, [50 * i + 7 for i in range(16)]),
        # eight prompts enter the cache
        _case("append_prompts", "append", 32, 8, 128, "f16", [1000, 816, 1201, 50, 333, 2048, 129, 1617],
              [0, 50, 0, 816, 0, 0, 77, 0]),
        # a cached observation is read back for the next chunk of its prompt
        _case("gather_816", "gather", 8, 1, 256, "bf16", [816], [816]),
        # a batch of long contexts is read back
        _case("gather_long", "gather", 32, 8, 128, "f16", [1] * 6, [8000, 16384, 129, 4097, 12001, 9000], page=128),
        # one token of one robot's plan over its cached observation
        _case("decode_816", "decode", 8, 1, 256, "bf16", [1], [817]),
        # 50 action tokens of four robots over their cached observations, all of which they see
        _case("decode_chunk", "decode", 8, 1, 256, "bf16", [50] * 4, [866, 866, 700, 866], causal=False),
        # single tokens of many users, contexts of one token to thousands
        _case("decode_ragged", "decode", 32, 8, 128, "f16", [1] * len(ragged), ragged, page=16, rotate=False),
        # eight long contexts
        _case("decode_long", "decode", 32, 8, 128, "bf16", [1] * 8, [65536, 65000, 40000, 65536, 60001, 65536, 32768, 65535]),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _split(rng, total, parts):
    """`total` tokens in `parts` sequences of very different lengths, each one token at least."""
    w = [rng.random() ** 2 + 0.01 for _ in range(parts)]
    return [max(1, int(total * x / sum(w))) for x in w]


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "append", "gather", "decode", "decode"])
    heads, kv_heads = rng.choice([(8, 1), (8, 2), (8, 8), (16, 4), (32, 8), (14, 2), (12, 4), (5, 5)])
    dim = rng.choice([64, 128, 256])
    dtype = rng.choice(["f16", "bf16"])
    rotate = rng.random() < 0.7
    page = rng.choice([16, 32, 64, 128])
    if kind == "prompt":
        batch = _spread(rng, 1, 12)
        q = _split(rng, _spread(rng, 16, 6000), batch)
        k = [n + (_spread(rng, 1, 2000) if rng.random() < 0.3 else 0) for n in q]
        causal = rng.random() < 0.75
        while 4 * dim * heads * _pairs(q, k, causal) > 2.5e11:
            q, k = [-(-n // 2) for n in q], [-(-n // 2) for n in k]
    elif kind == "decode":
        batch = _spread(rng, 1, 40)
        # long caches for single tokens; a chunk of up to 64 tokens over shorter ones
        n = 1 if rng.random() < 0.6 else _spread(rng, 2, 64)
        most = 300_000 // kv_heads if n == 1 else 20_000
        k = [x + n for x in _split(rng, _spread(rng, 16, most), batch)]
        q = [n] * batch
        causal = rng.random() < 0.8
    else:
        batch = _spread(rng, 1, 24)
        n = _split(rng, _spread(rng, batch, (100_000 if kind == "append" else 200_000) // kv_heads), batch)
        before = [_spread(rng, 1, 1000) - 1 for _ in n]
        q, k = (n, before) if kind == "append" else ([1] * batch, n)
        causal = True
    c = _case("", kind, heads, kv_heads, dim, dtype, q, k, causal, page, rotate)
    del c["name"]
    return c


# ---- shapes and inputs -------------------------------------------------------------------------------------------

def _lens(text):
    return [int(x) for x in text.split(",")]


def _offsets(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _tokens(g, n, heads, dim, dtype, outliers=False):
    """[n, heads, dim] N(0, 1); keys have a few channels that are several times larger, as a model's do."""
    x = torch.randn(n, heads, dim, generator=g, device=DEV)
    if outliers:
        x[:, :, :: max(1, dim // 4)] *= 4.0
    return x.to(_TORCH[dtype])


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEV).manual_seed(seed)
    H, KV, D, dt = c["heads"], c["kv_heads"], c["dim"], c["dtype"]
    q_lens, k_lens = _lens(c["q_lens"]), _lens(c["k_lens"])
    s = dict(c, q_lens=q_lens, k_lens=k_lens, scale=1.0 / math.sqrt(D), dt=_TORCH[dt])
    nq, nk = sum(q_lens), sum(k_lens)
    s["total_q"], s["total_k"], s["batch"] = nq, nk, len(q_lens)
    if c["kind"] == "prompt":
        if q_lens == k_lens:  # the fused projection's output: each token's query heads, key heads, value heads
            x = torch.cat([_tokens(g, nq, H, D, dt), _tokens(g, nq, KV, D, dt, True), _tokens(g, nq, KV, D, dt)], 1)
            s["q"], s["k"], s["v"] = x[:, :H], x[:, H: H + KV], x[:, H + KV:]
        else:
            s["q"], s["k"], s["v"] = _tokens(g, nq, H, D, dt), _tokens(g, nk, KV, D, dt, True), _tokens(g, nk, KV, D, dt)
        s["cu_q"], s["cu_k"] = _ints(_offsets(q_lens)), _ints(_offsets(k_lens))
        s["o"] = torch.empty(nq, H, D, dtype=s["dt"], device=DEV)
        return s
    # the cache: every sequence's pages, in no order, and a few pages of nobody
    page = c["page"]
    new = q_lens if c["kind"] == "append" else [0] * len(q_lens)
    need = [-(-(k + n) // page) for k, n in zip(k_lens, new)]
    pages = sum(need) + 3
    table = torch.zeros(len(need), max(need), dtype=torch.int32, device=DEV)
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at: at + n]
        at += n
    s["table"], s["pages"] = table, pages
    block = page * D // 2
    pool = torch.empty(pages, KV, page * (D + 8), dtype=torch.uint8, device=DEV)
    for i in range(2):  # codes of rotated or plain heads: near a Gaussian's, the largest channel at 7
        n = torch.randint(0, 1 << 16, (pages, KV, block), generator=g, device=DEV, dtype=torch.int32)
        lo, hi = (n & 255) % 15 - 7, (n >> 8) % 15 - 7
        pool[:, :, i * block: (i + 1) * block] = ((lo & 15) | ((hi & 15) << 4)).to(torch.uint8)
    scales = torch.rand(pages, KV, 2 * page, generator=g, device=DEV) * 0.2 + 0.1
    pool[:, :, 2 * block:] = scales.view(torch.uint8)
    s["pool"] = pool
    s["len"] = _ints(k_lens)
    if c["kind"] == "append":
        x = torch.cat([_tokens(g, nq, H, D, dt), _tokens(g, nq, KV, D, dt, True), _tokens(g, nq, KV, D, dt)], 1)
        s["k"], s["v"] = x[:, H: H + KV], x[:, H + KV:]
        s["cu_q"] = _ints(_offsets(q_lens))
        s["ko"], s["vo"] = (torch.empty(nq, KV, D, dtype=s["dt"], device=DEV) for _ in range(2))
    elif c["kind"] == "gather":
        s["cu_k"] = _ints(_offsets(k_lens))
        s["ko"], s["vo"] = (torch.empty(nk, KV, D, dtype=s["dt"], device=DEV) for _ in range(2))
    else:
        s["q"] = _tokens(g, nq, H, D, dt)
        s["cu_q"] = _ints(_offsets(q_lens))
        s["o"] = torch.empty(nq, H, D, dtype=s["dt"], device=DEV)
        # room for the partial results of a split over the keys: at most 32 MiB and 16 results of every query row
        s["ws"] = torch.empty((32 << 20) + 16 * nq * H * (D + 2) * 4, dtype=torch.uint8, device=DEV)
    return s


# ---- the operators in their plain form ----------------------------------------------------------------------------

def _hadamard(x):
    """x times the Hadamard matrix / sqrt(dim) over the last axis, float32, butterflies of distance 1, 2, 4, ..."""
    shape, dim, h = x.shape, x.shape[-1], 1
    x = x.reshape(-1, dim)
    while h < dim:
        a, b = x.reshape(-1, dim // (2 * h), 2, h).unbind(2)
        x = torch.stack((a + b, a - b), 2).reshape(-1, dim)
        h *= 2
    return (x * torch.tensor(1.0 / math.sqrt(dim), dtype=torch.float32, device=x.device)).reshape(shape)


def _places(s, lens, starts):
    """Page and slot of every token: sequence b's tokens starts[b] .. starts[b] + lens[b]."""
    lens, starts = torch.tensor(lens, device=DEV), torch.tensor(starts, device=DEV)
    seq = torch.repeat_interleave(torch.arange(len(lens), device=DEV), lens)
    pos = torch.arange(seq.numel(), device=DEV) - (torch.cumsum(lens, 0) - lens)[seq] + starts[seq]
    return s["table"][seq, pos // s["page"]].long(), pos % s["page"]


def _planes(s):
    """The pool as keys' codes, values' codes [pages, kv_heads, page, dim / 2] and their scales [pages, kv_heads, page]."""
    pool, page, D = s["pool"], s["page"], s["dim"]
    n = page * D // 2
    codes = pool[:, :, : 2 * n].unflatten(2, (2, page, D // 2))
    scales = pool.view(torch.float32)[:, :, 2 * n // 4:].unflatten(2, (2, page))
    return codes[:, :, 0], codes[:, :, 1], scales[:, :, 0], scales[:, :, 1]


def _store(s, codes, scales, where, x):
    y = x.float()
    y = _hadamard(y) if s["rotate"] else y
    d = y.abs().amax(-1) / 7.0
    # the quotient of two float32 numbers is taken in 64 bits, so that its ties are true ones
    q = torch.where(d[..., None] > 0, (y.double() / d[..., None].double()).round(), 0.0).clamp(-7, 7).to(torch.int32)
    codes[where[0], :, where[1]] = ((q[..., 0::2] & 15) | ((q[..., 1::2] & 15) << 4)).to(torch.uint8)
    scales[where[0], :, where[1]] = d


def _values(codes, scales, where):
    """float32 [tokens, kv_heads, dim] of the places, in the cache's basis."""
    b = codes[where[0], :, where[1]].to(torch.int32)
    q = torch.stack(((b & 15 ^ 8) - 8, (b >> 4 ^ 8) - 8), -1).flatten(-2)
    return q.float() * scales[where[0], :, where[1]][..., None]


def _softmax_attention(q, k, v, see, scale):
    """q [b, h, n, d], k and v [b, kv, m, d], see [b, n, m]; float32.  A row that sees nothing is zero."""
    group = q.shape[1] // k.shape[1]
    w = q.unflatten(1, (k.shape[1], group)) @ k.unsqueeze(2).transpose(-1, -2)
    w.mul_(scale).masked_fill_(~see[:, None, None], -math.inf)
    top = w.amax(-1, keepdim=True)
    top.masked_fill_(top == -math.inf, 0.0)
    w.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    return ((w @ v.unsqueeze(2)) / total.masked_fill_(total == 0, 1.0)).flatten(1, 2)


def _padded(x, lens):
    """[tokens, heads, d] of packed sequences -> [b, heads, longest, d], zeros behind each sequence."""
    at = torch.tensor(lens, device=DEV)
    i = torch.arange(max(lens), device=DEV)
    inside = i < at[:, None]
    rows = torch.where(inside, (torch.cumsum(at, 0) - at)[:, None] + i, 0)
    return torch.where(inside[..., None, None], x[rows].float(), 0.0).transpose(1, 2), inside


def _seen(s, inside_k):
    n, m = max(s["q_lens"]), inside_k.shape[1]
    see = inside_k[:, None].expand(-1, n, -1)
    if s["causal"]:
        last = torch.tensor(s["k_lens"], device=DEV) - torch.tensor(s["q_lens"], device=DEV)
        see = see & (torch.arange(m, device=DEV) <= torch.arange(n, device=DEV)[:, None] + last[:, None, None])
    return see


def _plain_attention(s, q, k, v):
    qp, inside_q = _padded(q, s["q_lens"])
    kp, inside_k = _padded(k, s["k_lens"])
    vp, _ = _padded(v, s["k_lens"])
    o = _softmax_attention(qp, kp, vp, _seen(s, inside_k), s["scale"])
    return o.transpose(1, 2)[inside_q]


def _plain(s):
    kind, dt = s["kind"], s["dt"]
    if kind == "prompt":
        return _plain_attention(s, s["q"], s["k"], s["v"]).to(dt)
    kc, vc, ks, vs = _planes(s)
    if kind == "append":
        where = _places(s, s["q_lens"], s["k_lens"])
        _store(s, kc, ks, where, s["k"])
        _store(s, vc, vs, where, s["v"])
    else:
        where = _places(s, s["k_lens"], [0] * s["batch"])
    k, v = _values(kc, ks, where), _values(vc, vs, where)
    if kind == "decode":
        q = s["q"].float()
        o = _plain_attention(s, _hadamard(q) if s["rotate"] else q, k, v)
        return (_hadamard(o) if s["rotate"] else o).to(dt)
    return {"k": (_hadamard(k) if s["rotate"] else k).to(dt), "v": (_hadamard(v) if s["rotate"] else v).to(dt)}


# ---- the same through the library's entry points --------------------------------------------------------------------

def _own(s):
    from paper_2605_28803_gb300 import qvla as Q

    st = torch.cuda.current_stream()
    code = Q.DTYPE_CODES[s["dtype"]]
    H, KV, D = s["heads"], s["kv_heads"], s["dim"]
    if s["kind"] == "prompt":
        Q.qvla_attention_prompt(s["q"], s["k"], s["v"], code, H, KV, D, s["q"].stride(0), s["k"].stride(0), s["v"].stride(0),
                                s["batch"], s["cu_q"], s["total_q"], s["cu_k"], s["total_k"], s["scale"], s["causal"], s["o"], st)
        return s["o"]
    cache = Q.Kv4Cache(s["pool"], s["pages"], s["page"], KV, D, s["rotate"])
    table, width = s["table"], s["table"].shape[1]
    if s["kind"] == "decode":
        Q.qvla_attention_kv4(cache, s["q"], code, H, s["q"].stride(0), s["batch"], s["cu_q"], s["total_q"], max(s["q_lens"]),
                             table, width, s["len"], max(s["k_lens"]), s["scale"], s["causal"], s["o"], s["ws"],
                             s["ws"].numel(), st)
        return s["o"]
    if s["kind"] == "append":
        Q.qvla_kv4_append(cache, s["k"], s["v"], code, s["k"].stride(0), s["v"].stride(0), s["batch"], s["cu_q"],
                          s["total_q"], table, width, s["len"], st)
        Q.qvla_kv4_gather(cache, s["batch"], s["cu_q"], s["total_q"], table, width, s["len"], s["ko"], s["vo"], code, st)
    else:
        Q.qvla_kv4_gather(cache, s["batch"], s["cu_k"], s["total_k"], table, width, None, s["ko"], s["vo"], code, st)
    return {"k": s["ko"], "v": s["vo"]}


def run(state):
    return _own(state) if own else _plain(state)


def _pairs(q_lens, k_lens, causal):
    """Query/key pairs that attention has to form."""
    n = 0
    for q, k in zip(q_lens, k_lens):
        first = k - q + 1  # keys that the first query sees
        n += sum(max(0, min(k, first + i)) for i in range(q)) if causal else q * k
    return n


def work(case):
    q_lens, k_lens = _lens(case["q_lens"]), _lens(case["k_lens"])
    H, KV, D = case["heads"], case["kv_heads"], case["dim"]
    nq, nk = sum(q_lens), sum(k_lens)
    if case["kind"] == "prompt":
        return {"bytes": 2 * D * (2 * nq * H + 2 * nk * KV), "flops": 4 * D * H * _pairs(q_lens, k_lens, case["causal"])}
    if case["kind"] == "decode":
        return {"bytes": nk * KV * (D + 8) + 2 * 2 * nq * H * D, "flops": 4 * D * H * _pairs(q_lens, k_lens, case["causal"])}
    n = nq if case["kind"] == "append" else nk
    turns = 2 * math.log2(D) * D * n * KV if case["rotate"] else 0
    cached, values = n * KV * (D + 8), 2 * 2 * n * KV * D
    if case["kind"] == "append":  # read the tokens, write the cache; read it back, write the values
        return {"bytes": 2 * (cached + values), "flops": int(2 * turns + 8 * D * n * KV)}
    return {"bytes": cached + values, "flops": int(turns + 2 * D * n * KV)}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

def _sylvester(dim):
    m = torch.ones(1, 1, dtype=torch.float64, device=DEV)
    while m.shape[0] < dim:
        m = torch.cat((torch.cat((m, m), 1), torch.cat((m, -m), 1)), 0)
    return m / math.sqrt(dim)


def exact(case, seed):
    s = prepare(case, seed)
    H, KV, D, page = s["heads"], s["kv_heads"], s["dim"], s["page"]
    turn = _sylvester(D) if s["rotate"] else None
    if s["kind"] == "append":
        out = {}
        for name in ("k", "v"):
            y = s[name].double()
            y = y @ turn if s["rotate"] else y
            d = (y.abs().max(-1, keepdim=True).values / 7).float().double()  # a scale is a float32 number
            y = torch.round(y / d).clamp(-7, 7) * d
            out[name] = y @ turn if s["rotate"] else y
        return out

    def cached(b, n, head):
        """Keys and values of a sequence's first n tokens for one head, float64, in the cache's basis."""
        rows = s["pool"][s["table"][b, : -(-n // page)].long(), head]
        found = []
        for i in range(2):
            b4 = rows[:, i * page * D // 2: (i + 1) * page * D // 2].reshape(-1, D // 2)
            lo, hi = (b4 % 16).double(), torch.div(b4, 16, rounding_mode="floor").double()
            c = torch.stack((lo - 16 * (lo > 7), hi - 16 * (hi > 7)), 2).reshape(-1, D)
            d = rows[:, page * D + 4 * page * i: page * D + 4 * page * (i + 1)].contiguous().view(torch.float32).double()
            found.append((c * d.reshape(-1, 1))[:n])
        return found

    if s["kind"] == "gather":
        out = {"k": [], "v": []}
        for b, n in enumerate(s["k_lens"]):
            both = [torch.stack(x, 1) for x in zip(*(cached(b, n, h) for h in range(KV)))]
            for name, x in zip(("k", "v"), both):
                out[name].append(x @ turn if s["rotate"] else x)
        return {name: torch.cat(x) for name, x in out.items()}
    o = torch.zeros(s["total_q"], H, D, dtype=torch.float64, device=DEV)
    q0, k0 = 0, 0
    for b, (n, m) in enumerate(zip(s["q_lens"], s["k_lens"])):
        q = s["q"][q0: q0 + n].double()
        for h in range(KV):
            if s["kind"] == "prompt":
                k, v = (s[x][k0: k0 + m, h].double() for x in ("k", "v"))
            else:
                k, v = cached(b, m, h)
            for j in range(h * (H // KV), (h + 1) * (H // KV)):
                qj = q[:, j] @ turn if s["kind"] == "decode" and s["rotate"] else q[:, j]
                w = qj @ k.T / math.sqrt(D)
                if s["causal"]:
                    w = w + torch.full_like(w, -math.inf).triu(m - n + 1)
                w = torch.nan_to_num(torch.softmax(w, -1)) @ v
                o[q0: q0 + n, j] = w @ turn if s["kind"] == "decode" and s["rotate"] else w
        q0, k0 = q0 + n, k0 + m
    return o
