"""Performance cases of the 8-bit KV cache and of the step that feeds a cache.

Each case is one pass of a program that serves a model with a full KV cache
beside (or before) the compressed one:

  norm    the query and key heads of new tokens normalised and rotated
          (`qk_norm_rope`), taken out of the rows of a fused projection
  cache   new rows written into the 8-bit cache (`kv8_write`) and the blocks
          that hold them read back (`kv8_read`)
  attn    attention of the newest query tokens over the 8-bit cache
          (`kv8_decode`)

listed() names the cases, draw() gives more of the same ranges, prepare()
makes what such a program holds on the GPU, run() is the pass (plain torch, or
with `own` the library's calls), work() what it cannot do without, exact() the
same results in 64 bits.

The cache: blocks of 64 tokens per sequence and KV head with one fp32 scale per
block and side.  A block's codes are 64 * head_dim contiguous bytes, keys in the
order (t / 16, d / 64, (d % 64) / 16, t % 16, d % 16), values in the order
(d / 16, (t % 16) / 4, d % 16, t % 4, t / 16).  int8: scale = amax / 127;
e4m3: the smallest power of two with amax <= 448 * scale; codes are the nearest,
ties to even, of x / scale.  Rows written into a block that holds earlier rows
raise its scale where they need it, and the earlier rows are rewritten from the
values they stood for.
"""

import math

import torch

own = False

# name: query heads, KV heads, head dim, RoPE base
SHAPES = {
    "llama8b": (32, 8, 128, 5e5),     # Llama-3.1-8B layer
    "qwen3_4b": (32, 8, 128, 1e6),    # Qwen3-4B layer, whose heads are normalised
    "qwen7b": (28, 4, 128, 1e6),      # Qwen2.5-7B layer, seven query heads per KV head
    "small": (8, 2, 64, 1e4),         # a small layer with 64-wide heads
    "wide64": (16, 4, 64, 1e4),       # 64-wide heads, four per KV head
    "mha4": (4, 4, 128, 1e4),         # no grouping
    "gqa2": (16, 8, 128, 1e6),        # two query heads per KV head
    "gqa8": (32, 4, 128, 1e6),        # eight query heads per KV head
    "mqa16": (16, 1, 128, 1e4),       # one KV head
}
EPS = 1e-6
BLOCK = 64


def _norm(shape, tokens, position, dtype="bf16", weights=True, rotate=True):
    return {"kind": "norm", "shape": shape, "tokens": tokens, "position": position, "dtype": dtype,
            "weights": weights, "rotate": rotate}


def _cache(shape, batch, rows, start, spread, format, dtype="bf16"):
    # sequence b is written from row start + b * spread on, with rows - (b * spread) % rows rows
    return {"kind": "cache", "shape": shape, "batch": batch, "rows": rows, "start": start, "spread": spread,
            "format": format, "dtype": dtype}


def _attn(shape, batch, length, format, queries=1, shortest=None, dtype="bf16"):
    # lengths fall evenly from `length` to `shortest` over the batch
    return {"kind": "attn", "shape": shape, "batch": batch, "length": length, "format": format, "queries": queries,
            "shortest": length if shortest is None else shortest, "dtype": dtype}


def listed():
    cases = [
        # one chat's new token, late in a 120k context: latency
        ("norm_one_token", _norm("qwen3_4b", 1, 120003)),
        # a 32k prompt
        ("norm_prompt_32k", _norm("qwen3_4b", 32764, 0)),
        # an odd chunk of a small fp32 model
        ("norm_fp32_4k", _norm("small", 4097, 1011, dtype="fp32")),
        # a serving batch's new tokens into blocks filled to different heights
        ("cache_append_b32", _cache("llama8b", 32, 1, 9001, 37, "int8")),
        # four long prompts
        ("cache_prompt_4x128k", _cache("llama8b", 4, 131068, 0, 0, "int8")),
        # the next chunk of three prompts of different lengths, fp32 rows
        ("cache_chunk_fp32", _cache("wide64", 3, 2051, 1003, 333, "e4m3", dtype="fp32")),
        # the shortest: a small fp32 model's chat
        ("attn_small_fp32_1k", _attn("small", 1, 1021, "int8", dtype="fp32")),
        # one chat at 32k
        ("attn_llama8b_32k", _attn("llama8b", 1, 32764, "int8")),
        # four sequences at 128k
        ("attn_llama8b_4x128k", _attn("llama8b", 4, 131068, "int8")),
        # eight at 128k, seven query heads per KV head
        ("attn_qwen7b_8x128k", _attn("qwen7b", 8, 131068, "e4m3")),
        # a serving batch of unequal conversations, one of them not begun
        ("attn_ragged_b32", _attn("llama8b", 32, 32765, "e4m3", shortest=0)),
        # four drafted tokens checked against a 120k context
        ("attn_draft4_120k", _attn("qwen3_4b", 1, 120001, "int8", queries=4)),
    ]
    return [dict(c, name=name) for name, c in cases]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "cache", "attn", "attn"])
    shape = rng.choice(["llama8b", "qwen3_4b", "qwen7b", "small", "wide64", "mha4", "gqa2", "gqa8", "mqa16"])
    format = rng.choice(["int8", "e4m3"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    hq, hkv, _, _ = SHAPES[shape]
    if kind == "norm":
        return _norm(shape, _log(rng, 1, 32764), _log(rng, 1, 131072), dtype, rng.random() < 0.8, rng.random() < 0.8)
    if kind == "cache":
        batch = rng.choice([1, 2, 3, 5, 8, 16, 32])
        rows = 1 if rng.random() < 0.3 else _log(rng, 2, 262144 // batch)
        return _cache(shape, batch, rows, rng.choice([0, _log(rng, 1, 20000)]), rng.randrange(0, 200), format, dtype)
    batch = rng.choice([1, 1, 2, 3, 4, 7, 8, 16, 32])
    length = _log(rng, 64, min(131068, 524288 // batch))
    shortest = rng.choice([length, length, rng.randrange(0, length + 1)])
    queries = rng.choice([1, 1, 1, rng.randrange(2, 9)])
    return _attn(shape, batch, length, format, min(queries, 128 * hkv // hq), shortest, dtype)


# ---------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------

def _es(case):
    return 2 if case["dtype"] == "bf16" else 4


def _capacity(rows):
    return max(BLOCK, (rows + BLOCK - 1) // BLOCK * BLOCK)


def _starts(case):
    return [case["start"] + b * case["spread"] for b in range(case["batch"])]


def _counts(case):
    return [case["rows"] - (b * case["spread"]) % case["rows"] for b in range(case["batch"])]


def _first_row(start):
    return start // BLOCK * BLOCK


def _lengths(case):
    n = case["batch"]
    return [case["length"] - (case["length"] - case["shortest"]) * b // max(1, n - 1) for b in range(n)]


def work(case):
    hq, hkv, dh, _ = SHAPES[case["shape"]]
    es, dp = _es(case), hkv * dh
    if case["kind"] == "norm":
        n = case["tokens"] * (hq + hkv) * dh
        return {"bytes": 2 * n * es + case["tokens"] * 4 + 2 * dh * es, "flops": 10 * n}
    if case["kind"] == "cache":
        new = sum(_counts(case))
        held = sum(s + c - _first_row(s) for s, c in zip(_starts(case), _counts(case)))
        blocks = sum((s + c + BLOCK - 1) // BLOCK - s // BLOCK for s, c in zip(_starts(case), _counts(case)))
        # rows in, codes out; codes in, rows out; the scales both times
        return {"bytes": 2 * (new * dp * (es + 1) + held * dp * (es + 1) + 2 * blocks * hkv * 4),
                "flops": 8 * (new + held) * dp}
    tokens = sum(_lengths(case))
    blocks = sum((n + BLOCK - 1) // BLOCK for n in _lengths(case))
    rows = case["batch"] * case["queries"] * hq * dh
    return {"bytes": 2 * tokens * dp + 2 * blocks * hkv * 4 + rows * (es + 4),
            "flops": 4 * tokens * case["queries"] * hq * dh}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _rows(gen, batch, rows, width, dh):
    """Keys or values as a layer makes them: unit noise, four channels of every head eight times larger, token sizes
    that vary by a factor of two."""
    x = torch.randn(batch, rows, width, generator=gen, device="cuda")
    big = torch.ones(dh, device="cuda")
    big[torch.randperm(dh, generator=gen, device="cuda")[:4]] = 8.0
    x = x.view(batch, rows, -1, dh).mul_(big)
    return x.mul_(torch.rand(batch, rows, 1, 1, generator=gen, device="cuda") + 0.5).view(batch, rows, width)


def _config(case):
    """The library's configuration of the case's layer, as a program keeps it."""
    if not own:
        return None
    import paper_2608_00528_amd as s4r
    hq, hkv, dh, theta = SHAPES[case["shape"]]
    kind = case["kind"]
    capacity = BLOCK if kind == "norm" else _cache_capacity(case)
    return s4r.make_config(batch=case.get("batch", 1), n_q_heads=hq, n_kv_heads=hkv, head_dim=dh, rank=32,
                           capacity=capacity, rope_theta=theta if case.get("rotate", True) else 0.0,
                           dtype=case["dtype"])


def _cache_capacity(case):
    if case["kind"] == "cache":
        return _capacity(max(s + case["rows"] for s in _starts(case)))
    return _capacity(case["length"])


def _empty_cache(case):
    _, hkv, dh, _ = SHAPES[case["shape"]]
    tiles = _cache_capacity(case) // BLOCK
    shape = (case["batch"], hkv, tiles)
    return {"k_codes": torch.zeros(*shape, BLOCK * dh, dtype=torch.uint8, device="cuda"),
            "k_scales": torch.zeros(shape, device="cuda"),
            "v_codes": torch.zeros(*shape, BLOCK * dh, dtype=torch.uint8, device="cuda"),
            "v_scales": torch.zeros(shape, device="cuda")}


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    hq, hkv, dh, theta = SHAPES[case["shape"]]
    dt, dp = _dt(case), hkv * dh
    s = {"case": dict(case), "cfg": _config(case)}
    if case["kind"] == "norm":
        n = case["tokens"]
        qkv = torch.randn(n, (hq + 2 * hkv) * dh, generator=gen, device="cuda")
        qkv.mul_(torch.rand(n, 1, generator=gen, device="cuda") * 4 + 0.25)
        s["qkv"] = qkv.to(dt)
        s["q_weight"] = s["k_weight"] = None
        if case["weights"]:
            s["q_weight"], s["k_weight"] = [(1 + 0.2 * torch.randn(dh, generator=gen, device="cuda")).to(dt)
                                            for _ in range(2)]
        s["positions"] = torch.arange(n, dtype=torch.int32, device="cuda") + case["position"]
        return s
    cache = s["cache"] = _empty_cache(case)
    if case["kind"] == "cache":
        s["k"], s["v"] = [_rows(gen, case["batch"], case["rows"], dp, dh).to(dt) for _ in range(2)]
        s["starts"] = torch.tensor(_starts(case), dtype=torch.int32, device="cuda")
        s["counts"] = torch.tensor(_counts(case), dtype=torch.int32, device="cuda")
        # the rows that the first blocks hold already, half as large as the new ones
        first = [_first_row(x) for x in _starts(case)]
        s["read_from"] = torch.tensor(first, dtype=torch.int32, device="cuda")
        s["read_rows"] = s["starts"] - s["read_from"] + s["counts"]
        s["read_most"] = max(a + c - f for a, c, f in zip(_starts(case), _counts(case), first))
        if any(x % BLOCK for x in _starts(case)):
            for side in ("k", "v"):
                old = 0.5 * _rows(gen, case["batch"], BLOCK, dp, dh)
                _plain_write(cache, side, old, s["read_from"], s["starts"] - s["read_from"], case["format"], dh)
        return s
    for side in ("k", "v"):
        x = _rows(gen, case["batch"], _cache_capacity(case), dp, dh)
        zero = torch.zeros(case["batch"], dtype=torch.int32, device="cuda")
        _plain_write(cache, side, x, zero, zero + x.shape[1], case["format"], dh)
        del x
    s["q"] = (1.2 * torch.randn(case["batch"], case["queries"], hq, dh, generator=gen, device="cuda")).to(dt)
    s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
    if own:
        import paper_2608_00528_amd as s4r
        s["ws"] = s4r.alloc_kv8_workspace(s["cfg"], case["queries"])
    return s


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------

def _keys_laid_out(x):
    """[B, H, T, 64, d] -> [B, H, T, 64 d] in the order of a block of keys."""
    b, h, t, n, d = x.shape
    return x.view(b, h, t, 4, 16, d // 64, 4, 16).permute(0, 1, 2, 3, 5, 6, 4, 7).reshape(b, h, t, n * d)


def _values_laid_out(x):
    b, h, t, n, d = x.shape
    return x.view(b, h, t, 4, 4, 4, d // 16, 16).permute(0, 1, 2, 6, 4, 7, 5, 3).reshape(b, h, t, n * d)


def _keys_in_rows(x, d):
    b, h, t, _ = x.shape
    return x.view(b, h, t, 4, d // 64, 4, 16, 16).permute(0, 1, 2, 3, 6, 4, 5, 7).reshape(b, h, t, BLOCK, d)


def _values_in_rows(x, d):
    b, h, t, _ = x.shape
    return x.view(b, h, t, d // 16, 4, 16, 4, 4).permute(0, 1, 2, 7, 4, 6, 3, 5).reshape(b, h, t, BLOCK, d)


def _held(codes, scales, side, format, d):
    """The values of blocks of codes, [B, H, T, 64, d] in fp32."""
    codes = (_keys_in_rows if side == "k" else _values_in_rows)(codes, d)
    codes = codes.view(torch.int8) if format == "int8" else codes.view(torch.float8_e4m3fn)
    return codes.float() * scales[..., None, None]


def _scale_for(amax, format):
    # a quotient of tensors: torch divides by a plain number through its rounded reciprocal
    most = torch.full_like(amax, 127.0 if format == "int8" else 448.0)
    if format == "int8":
        s = amax / most
    else:
        m, e = torch.frexp(amax.double() / most.double())
        s = torch.ldexp(torch.ones_like(m), e - (m == 0.5).to(e.dtype)).float()
    return torch.where(amax < 2.0 ** -90, torch.zeros_like(s), s)


def _plain_write(cache, side, rows, starts, counts, format, d):
    """Rows [B, n, H d] of each sequence into the cache from row starts[b] on, counts[b] of them."""
    codes, scales = cache[side + "_codes"], cache[side + "_scales"]
    b, h, tiles, _ = codes.shape
    n = rows.shape[1]
    blocks = min(tiles, (n + 2 * BLOCK - 2) // BLOCK)
    seq = torch.arange(b, device=rows.device)[:, None]
    tile = torch.div(starts, BLOCK, rounding_mode="floor")[:, None].long() + torch.arange(blocks, device=rows.device)
    inside = (tile < tiles) & (tile * BLOCK < (starts + counts)[:, None])
    tile = tile.clamp(max=tiles - 1)
    held = _held(codes[seq, :, tile].transpose(1, 2), scales[seq, :, tile].transpose(1, 2), side, format, d)
    row = (tile[:, :, None] * BLOCK + torch.arange(BLOCK, device=rows.device)).view(b, -1)
    row = torch.where(inside.repeat_interleave(BLOCK, 1), row, torch.full_like(row, -1)) - starts[:, None]
    new = (row >= 0) & (row < counts[:, None])
    older = (row < 0) & (row >= -(starts % BLOCK)[:, None])
    x = rows.float()[seq, row.clamp(0, n - 1)].view(b, blocks, BLOCK, h, d).permute(0, 3, 1, 2, 4)
    new, older = [m.view(b, 1, blocks, BLOCK, 1) for m in (new, older)]
    amax = torch.where(new, x.abs(), torch.zeros_like(x)).amax((3, 4))
    scale = _scale_for(amax, format)
    partly = older.any(3)[..., 0]
    scale = torch.where(partly, torch.maximum(scale, scales[seq, :, tile].transpose(1, 2)), scale)
    x = torch.where(new, x, held)
    s = scale[..., None, None]
    y = torch.where(s > 0, x.double() / s.double(), torch.zeros((), dtype=torch.float64, device=x.device))
    if format == "int8":
        y = y.round().clamp_(-127, 127).to(torch.int8).view(torch.uint8)
    else:
        y = y.float().clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    old = (_keys_in_rows if side == "k" else _values_in_rows)(codes[seq, :, tile].transpose(1, 2), d)
    y = torch.where(new | older, y, old)
    y = (_keys_laid_out if side == "k" else _values_laid_out)(y.contiguous())
    at, which = torch.nonzero(inside, as_tuple=True)
    codes[at, :, tile[at, which]] = y.transpose(1, 2)[at, which]
    scales[at, :, tile[at, which]] = scale.transpose(1, 2)[at, which]


def _plain_read(cache, side, starts, counts, most, format, d, dtype):
    """Rows [B, most, H d]: counts[b] of them from row starts[b] on, then zeros."""
    codes, scales = cache[side + "_codes"], cache[side + "_scales"]
    b, h, tiles, _ = codes.shape
    i = torch.arange(most, device=codes.device)
    row = (starts[:, None] + i).clamp(max=tiles * BLOCK - 1).long()
    blocks = min(tiles, (most + 2 * BLOCK - 2) // BLOCK)
    first = torch.div(starts, BLOCK, rounding_mode="floor")[:, None].long()
    tile = (first + torch.arange(blocks, device=codes.device)).clamp(max=tiles - 1)
    seq = torch.arange(b, device=codes.device)[:, None]
    x = _held(codes[seq, :, tile].transpose(1, 2), scales[seq, :, tile].transpose(1, 2), side, format, d)
    x = x.reshape(b, h, blocks * BLOCK, d).transpose(1, 2)[seq, row - first * BLOCK]
    x = torch.where((i < counts[:, None])[:, :, None, None], x, torch.zeros((), device=x.device))
    return x.reshape(b, most, h * d).to(dtype)


def _plain_norm(x, weight, positions, theta):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
    if theta == 0.0:
        return x
    half = x.shape[-1] // 2
    f = theta ** (-torch.arange(half, dtype=torch.float64, device=x.device) / half)
    angle = positions.double()[:, None, None] * f
    c, s = angle.cos().float(), angle.sin().float()
    lo, hi = x[..., :half], x[..., half:]
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)


def _plain_attn(q, k, v, lengths):
    """q [B, n, hq, d], k and v [B, H, N, d]; query i of n sees lengths - (n - 1 - i) tokens."""
    b, n, hq, d = q.shape
    h = k.shape[1]
    q = q.view(b, n, h, hq // h, d).permute(0, 2, 4, 1, 3).reshape(b, h, d, -1).contiguous()
    s = (torch.matmul(k, q) / math.sqrt(d)).transpose(2, 3).contiguous()
    limit = lengths[:, None] - torch.arange(n - 1, -1, -1, device=q.device)
    limit = limit.repeat_interleave(hq // h, 1)[:, None, :, None]
    seen = torch.arange(k.shape[2], device=q.device) < limit
    s = torch.where(seen, s, torch.full((), -math.inf, dtype=s.dtype, device=s.device))
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.double().sum(-1, keepdim=True).to(s.dtype)
    o = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    return o.view(b, h, n, hq // h, d).transpose(1, 2).reshape(b, n, hq, d)


# ---------------------------------------------------------------------------
# the pass
# ---------------------------------------------------------------------------

def _heads(s):
    """The query and key heads in the rows of the fused projection."""
    hq, hkv, dh, _ = SHAPES[s["case"]["shape"]]
    x = s["qkv"].view(-1, hq + 2 * hkv, dh)
    return x[:, :hq], x[:, hq:hq + hkv]


def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    _, hkv, dh, theta = SHAPES[case["shape"]]
    if case["kind"] == "norm":
        q, k = _heads(s)
        theta = theta if case["rotate"] else 0.0
        return {"q": _plain_norm(q, s["q_weight"], s["positions"], theta).to(q.dtype),
                "k": _plain_norm(k, s["k_weight"], s["positions"], theta).to(k.dtype)}
    cache, format = s["cache"], case["format"]
    if case["kind"] == "cache":
        _plain_write(cache, "k", s["k"], s["starts"], s["counts"], format, dh)
        _plain_write(cache, "v", s["v"], s["starts"], s["counts"], format, dh)
        back = (s["read_from"], s["read_rows"], s["read_most"], format, dh, _dt(case))
        return {"k": _plain_read(cache, "k", *back), "v": _plain_read(cache, "v", *back),
                "k_scales": cache["k_scales"], "v_scales": cache["v_scales"]}
    k = _held(cache["k_codes"], cache["k_scales"], "k", format, dh).flatten(2, 3)
    v = _held(cache["v_codes"], cache["v_scales"], "v", format, dh).flatten(2, 3)
    return _plain_attn(s["q"].float(), k, v, s["lengths"])


def _run_own(s, case):
    import paper_2608_00528_amd as s4r
    cfg = s["cfg"]
    if case["kind"] == "norm":
        q, k = _heads(s)
        q, k = s4r.qk_norm_rope(cfg, q, k, s["positions"], s["q_weight"], s["k_weight"], eps=EPS)
        return {"q": q, "k": k}
    cache = s4r.KV8Cache(case["format"], **s["cache"])
    if case["kind"] == "cache":
        s4r.kv8_write(cfg, cache, s["k"], s["v"], starts=s["starts"], counts=s["counts"])
        k, v = s4r.kv8_read(cfg, cache, s["read_most"], starts=s["read_from"], counts=s["read_rows"])
        return {"k": k, "v": v, "k_scales": cache.k_scales, "v_scales": cache.v_scales}
    return s4r.kv8_decode(cfg, cache, case["length"], s["q"], s["ws"], lengths=s["lengths"])


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------

def _exact_norm(case, s):
    hq, hkv, dh, theta = SHAPES[case["shape"]]
    x = s["qkv"].double().view(-1, hq + 2 * hkv, dh)
    pos = s["positions"].double()

    def one(y, w):
        if w is not None:
            y = y / ((y * y).sum(-1, keepdim=True) / dh + EPS).sqrt() * w.double()
        if not case["rotate"]:
            return y
        pair = torch.complex(y[..., :dh // 2], y[..., dh // 2:])
        speed = torch.exp(torch.arange(dh // 2, device=y.device).double() * (-2.0 * math.log(theta) / dh))
        turn = pos[:, None] * speed
        pair = pair * torch.complex(turn.cos(), turn.sin())[:, None]
        return torch.cat([pair.real, pair.imag], -1)

    return {"q": one(x[:, :hq], s["q_weight"]), "k": one(x[:, hq:hq + hkv], s["k_weight"])}


def _exact_scale(amax, format):
    """The block's scale as it is stored."""
    if amax < 2.0 ** -90:
        return 0.0
    if format == "int8":
        return float(torch.tensor(amax / 127.0, dtype=torch.float64).float())
    e = math.floor(math.log2(amax / 448.0)) - 1
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def _exact_nearest(y, format):
    if format == "int8":
        return y.round()
    e = torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -30))).clamp_min(-6.0)
    e = torch.where(torch.exp2(e) > y.abs(), e - 1, e).clamp_min(-6.0)
    step = torch.exp2(e - 3.0)
    return (y / step).round() * step


def _exact_blocks(x, format, least=None):
    """x [..., 64, d] (rows that a block does not take are zeros): the values that the block's codes stand for."""
    amax = x.abs().amax((-1, -2))
    flat = [_exact_scale(a, format) for a in amax.flatten().tolist()] if least is not None else None
    if flat is not None:
        scale = torch.maximum(torch.tensor(flat, dtype=torch.float64, device=x.device).view(amax.shape), least)
    elif format == "int8":
        scale = (amax / torch.full_like(amax, 127.0)).float().double()
    else:
        scale = torch.exp2(torch.ceil(torch.log2(amax / torch.full_like(amax, 448.0))))
    s = scale[..., None, None]
    return _exact_nearest(x / torch.where(s > 0, s, torch.ones_like(s)), format) * s, scale


def _exact_cache(case, s):
    _, h, d, _ = SHAPES[case["shape"]]
    out = {}
    for side in ("k", "v"):
        codes, scales = s["cache"][side + "_codes"], s["cache"][side + "_scales"].double().clone()
        back = torch.zeros(case["batch"], s["read_most"], h * d, dtype=torch.float64, device="cuda")
        for b, (start, count) in enumerate(zip(_starts(case), _counts(case))):
            first, high = _first_row(start), start - _first_row(start)
            t0, n = first // BLOCK, (high + count + BLOCK - 1) // BLOCK
            x = torch.zeros(n * BLOCK, h, d, dtype=torch.float64, device="cuda")
            x[high:high + count] = s[side][b, :count].double().view(count, h, d)
            x = x.view(n, BLOCK, h, d).transpose(1, 2)
            got, scale = _exact_blocks(x, case["format"])
            if high:
                # the block that holds older rows: their values, found byte by byte
                least = scales[b, :, t0]
                t, c = torch.meshgrid(torch.arange(high, device="cuda"), torch.arange(d, device="cuda"), indexing="ij")
                if side == "k":
                    at = ((((t // 16) * (d // 64) + c // 64) * 4 + c % 64 // 16) * 16 + t % 16) * 16 + c % 16
                else:
                    at = ((((c // 16) * 4 + t % 16 // 4) * 16 + c % 16) * 4 + t % 4) * 4 + t // 16
                raw = codes[b, :, t0][:, at]
                raw = raw.view(torch.int8 if case["format"] == "int8" else torch.float8_e4m3fn).double()
                block = x[0].clone()
                new, scale[0] = _exact_blocks(block, case["format"], least)
                older = (raw * least[:, None, None]).float().double()
                sc = torch.where(scale[0] > 0, scale[0], torch.ones_like(scale[0]))[:, None, None]
                new[:, :high] = _exact_nearest(older / sc, case["format"]) * scale[0][:, None, None]
                got[0] = new
            scales[b, :, t0:t0 + n] = scale.transpose(0, 1)
            back[b, :high + count] = got.transpose(1, 2).reshape(n * BLOCK, h * d)[:high + count]
        out[side], out[side + "_scales"] = back, scales
    return out


def _exact_attn(case, s):
    hq, h, d, _ = SHAPES[case["shape"]]
    g, nq = hq // h, case["queries"]
    t = torch.arange(BLOCK, device="cuda")[:, None]
    c = torch.arange(d, device="cuda")[None, :]
    at_k = ((((t // 16) * (d // 64) + c // 64) * 4 + c % 64 // 16) * 16 + t % 16) * 16 + c % 16
    at_v = ((((c // 16) * 4 + t % 16 // 4) * 16 + c % 16) * 4 + t % 4) * 4 + t // 16
    kind = torch.int8 if case["format"] == "int8" else torch.float8_e4m3fn
    out = torch.zeros(case["batch"], nq, hq, d, dtype=torch.float64, device="cuda")
    for b, length in enumerate(_lengths(case)):
        for j in range(h):
            k, v = [(s["cache"][n + "_codes"][b, j][:, at.flatten()].view(kind).double()
                     * s["cache"][n + "_scales"][b, j].double()[:, None]).view(-1, d)[:length]
                    for n, at in (("k", at_k), ("v", at_v))]
            for i in range(nq):
                n = length - (nq - 1 - i)
                if n <= 0:
                    continue
                q = s["q"][b, i, j * g:(j + 1) * g].double()
                out[b, i, j * g:(j + 1) * g] = torch.softmax(torch.mm(q, k[:n].t().contiguous()) * d ** -0.5, -1) @ v[:n]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "cache": _exact_cache, "attn": _exact_attn}[case["kind"]](case, s)
