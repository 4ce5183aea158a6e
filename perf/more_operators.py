"""Cases for measuring prompt attention over contiguous slabs and the parking of slabs in fewer bits.

Three operators, each in a plain form (elementary torch operations in 32 bits, rounded once at the
end) and through the library:

  prefill  causal attention of a step's new tokens, any number per request, over the requests' slabs
           (Pool.prefill_attention)
  pack     rows of slabs, all layers, to a dense store: 8-bit floats, 8-bit or 4-bit integers with a
           scale per group of elements                                    (Pool.pack_kv)
  unpack   the same rows back into slabs, of the same or of another pool   (Pool.unpack_kv)

`own` chooses: False runs the plain forms, True makes the calls that a user of the library makes.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.bfloat16}
KV_SCALES = (0.0140625, 0.015625)      # what a code of 1 stands for in an 8-bit pool: keys, values
TOP = {"e4m3": 448.0, "int8": 127.0, "int4": 7.0}
TINY_GROUP = 2.0 ** -100               # a group whose largest element is below this counts as zeros


# ---- cases -------------------------------------------------------------------------------------

def _prefill(name, batch, tokens, context, heads, dtype, salt=1):
    q, kv, d = heads
    return {"name": name, "op": "prefill", "batch": batch, "tokens": tokens, "context": context, "q_heads": q,
            "kv_heads": kv, "head_dim": d, "dtype": dtype, "salt": salt}


def _store(op, name, batch, tokens, layers, heads, dtype, fmt, group, salt=1):
    return {"name": name, "op": op, "batch": batch, "tokens": tokens, "layers": layers, "kv_heads": heads[1],
            "head_dim": heads[2], "dtype": dtype, "format": fmt, "group": group, "salt": salt}


QWEN = (28, 4, 128)     # the repository's Qwen-7B-shaped layer
TINY = (2, 1, 64)       # its fp32 reference layer


def listed():
    return [
        # a request's single new token through the prompt path: the smallest call, latency only
        _prefill("prefill, one token behind 900", 1, 1, 900, QWEN, "bf16"),
        # the repository's chunked prefill: eight requests, chunks of 128 behind about 1,920 tokens
        _prefill("prefill, chunks of 128 behind 1920", 8, 1024, 1920, QWEN, "bf16"),
        # a batch of whole prompts of different lengths, nothing in the cache yet
        _prefill("prefill, 24 ragged prompts", 24, 12001, 0, QWEN, "bf16"),
        # one long prompt: the largest
        _prefill("prefill, one prompt of 16384", 1, 16384, 0, QWEN, "bf16"),
        # a chunk far into a long document, 8-bit pool: few rows, many keys
        _prefill("prefill, 509 behind 30001, 8-bit", 1, 509, 30001, QWEN, "e4m3"),
        # the fp32 reference layer, odd sizes
        _prefill("prefill, fp32, 5 requests", 5, 613, 77, TINY, "f32"),
        # a request of a few tokens is parked from one layer: the smallest call
        _store("pack", "pack, 17 tokens of one layer, int8", 1, 17, 1, QWEN, "bf16", "int8", 128),
        # twelve preempted requests leave the pool, all layers
        _store("pack", "pack, 12 requests, 28 layers, e4m3", 12, 8191, 28, QWEN, "bf16", "e4m3", 128),
        # a long one is parked in 4 bits, scales for every 32 elements, and comes back into another slab
        _store("park", "park and return, 5001 tokens, int4", 1, 5001, 28, QWEN, "bf16", "int4", 32),
        # a few tokens come back into an 8-bit pool
        _store("unpack", "unpack, 90 tokens of two layers, int8, 8-bit pool", 3, 90, 2, QWEN, "e4m3", "int8", 64),
        # the twelve come back
        _store("unpack", "unpack, 12 requests, 28 layers, e4m3", 12, 8191, 28, QWEN, "bf16", "e4m3", 128),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["prefill", "prefill", "prefill", "pack", "unpack", "park"])
    salt = rng.randrange(1, 1 << 20)
    if op == "prefill":
        dtype = rng.choice(["bf16", "bf16", "bf16", "e4m3", "f32"])
        heads = rng.choice([QWEN, (16, 8, 128), (8, 2, 128)])
        if dtype == "bf16":
            heads = rng.choice([QWEN, (16, 8, 128), (32, 2, 128), (16, 4, 64), (10, 2, 64), (8, 8, 64)])
        if dtype == "f32":
            heads = rng.choice([TINY, (4, 2, 128), (8, 2, 32)])
        tokens = _log(rng, 1, 8192 if dtype != "f32" else 1024)
        batch = min(tokens, _log(rng, 1, 64))
        # new tokens times keys, and tokens in the cache, bounded
        most = min(30000, 60_000_000 // tokens, 200_000 // batch) if dtype != "f32" else 2000
        context = 0 if rng.random() < 0.25 else _log(rng, 1, max(2, most))
        c = _prefill("", batch, tokens, context, heads, dtype, salt)
    else:
        dtype = rng.choice(["bf16", "bf16", "e4m3", "f32"])
        heads = rng.choice([QWEN, (16, 8, 128), (5, 1, 128)])
        if dtype != "e4m3":
            heads = rng.choice([QWEN, TINY, (16, 8, 128), (10, 2, 64), (6, 2, 32)])
        fmt = "int4" if op == "park" else rng.choice(["e4m3", "int8"])
        group = rng.choice([g for g in (16, 32, 64, 128) if g <= heads[2]])
        layers = _log(rng, 1, 28)
        tokens = _log(rng, 1, 200_000_000 // (layers * 2 * heads[1] * heads[2] * 4))
        tokens = min(tokens, 16384)
        c = _store(op, "", min(tokens, _log(rng, 1, 64)), tokens, layers, heads, dtype, fmt, group, salt)
    del c["name"]
    return c


# ---- shapes: the same for every seed -------------------------------------------------------------

def _up16(x):
    return (x + 15) // 16 * 16


def _shares(n, tokens, salt, spread=1.0):
    """`tokens` dealt to n requests, at least one each, ragged."""
    r = random.Random(tokens * 4099 + n * 31 + salt)
    weight = [math.exp(r.gauss(0.0, 0.8 * spread)) for _ in range(n)]
    out = [1 + int((tokens - n) * w / sum(weight)) for w in weight]
    out[n // 2] += tokens - sum(out)
    return out


def _shape(case):
    """New tokens and context of every request."""
    n, salt = case["batch"], case["salt"]
    r = random.Random(salt * 1000003 + n)
    new = _shares(n, case["tokens"], salt, 0.1 if case["context"] > 1000 else 1.0)
    if case["context"] == 0:
        return new, [0] * n
    return new, [max(0, int(case["context"] * r.uniform(0.8, 1.2))) if n > 1 else case["context"] for _ in range(n)]


def _esize(case):
    return {"bf16": 2, "f32": 4, "e4m3": 1}[case["dtype"]]


# ---- inputs ------------------------------------------------------------------------------------

def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _handle(case, memory, layers, tokens, boundaries, max_batch, max_group):
    """The library's pool over `memory`, no Large Bucket."""
    from paper_2512_09427_b200 import odma
    cfg = odma.config_default()
    cfg.safety_pct, cfg.max_len, cfg.window = 0, boundaries[-1], 16
    cfg.max_batch, cfg.max_group = max_batch, max_group
    kind = {"bf16": odma.DTYPE_BF16, "f32": odma.DTYPE_F32, "e4m3": odma.DTYPE_FP8_E4M3}[case["dtype"]]
    pool = odma.Pool(memory.data_ptr(), memory.numel() * memory.element_size(), layers, case["kv_heads"], case["head_dim"],
                     kind, cfg)
    if pool.set_buckets(boundaries) != odma.OK or pool.get_stats()["total_tokens"] != tokens:
        raise RuntimeError("the pool has another size")
    if case["dtype"] == "e4m3":
        pool.set_kv_scales([KV_SCALES[0]] * layers, [KV_SCALES[1]] * layers)
    return pool


def _slabs(lengths):
    """Two slab sizes, one for the shorter half of the requests: (capacities, bases, boundaries)."""
    small, large = _up16(sorted(lengths)[len(lengths) // 2]), _up16(max(lengths))
    cap = [small if x <= small else large for x in lengths]
    base = [sum(cap[:i]) for i in range(len(cap))]
    return cap, base, sorted({small, large})


def _admit(pool, req, cap, length, base):
    rc, slab = pool.alloc(req, cap)
    if rc or slab[:2] != (base, cap) or (length and pool.commit_step([req], [length])):
        raise RuntimeError("the slab is not where it was expected")


def _fill(case, gen, arrays, rows):
    """Keys and values with a few strong channels, as the pool holds them."""
    d = case["head_dim"]
    store = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.uint8}[case["dtype"]]
    mem = torch.empty(arrays, rows, d, dtype=store, device="cuda")
    for a in range(arrays):
        x = _normal(gen, rows, d)
        if case["op"] != "prefill":
            x.mul_(torch.exp(0.5 * _normal(gen, d)))
        if case["dtype"] == "e4m3":
            mem[a] = (x / KV_SCALES[a & 1]).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        else:
            mem[a] = x.to(store)
    return mem


def prepare(case, seed):
    return _prepare_prefill(case, seed) if case["op"] == "prefill" else _prepare_store(case, seed)


def _prepare_prefill(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    hq, hkv, d, dt = case["q_heads"], case["kv_heads"], case["head_dim"], DTYPES[case["dtype"]]
    new, ctx = _shape(case)
    n, tokens = case["batch"], case["tokens"]
    length = [a + b for a, b in zip(new, ctx)]
    cap, base, bounds = _slabs(length)
    total = sum(cap)
    mem = _fill(case, gen, 2, total * hkv)
    state = {"case": case, "mem": mem, "q": _normal(gen, tokens, hq, d).mul_(1.5).to(dt), "new": new, "len": length,
             "cap": cap, "base": base}
    if own:
        pool = _handle(case, mem, 1, total, bounds, n, hq // hkv)
        for i in range(n):
            _admit(pool, i, cap[i], ctx[i], base[i])
        stream = torch.cuda.current_stream().cuda_stream
        state["table"] = torch.empty(pool.tables_bytes(n), dtype=torch.uint8, device="cuda")
        state["tables"] = pool.build_tables(list(range(n)), state["table"].data_ptr(), state["table"].numel(), stream, new)
        state["workspace"] = torch.empty(pool.prefill_workspace_bytes(hq, state["tables"]), dtype=torch.uint8, device="cuda")
        state["out"] = torch.empty_like(state["q"])
        state["lse"] = torch.empty(tokens, hq, dtype=torch.float32, device="cuda")
        state["pool"] = pool
    return state


def _prepare_store(case, seed):
    """Source slabs filled (pack, park) or zero (unpack: they are the destination); park's destination lies behind them."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n, hkv, d, layers = case["batch"], case["kv_heads"], case["head_dim"], case["layers"]
    length = _shares(n, case["tokens"], case["salt"])
    cap, base, bounds = _slabs(length)
    copies = 2 if case["op"] == "park" else 1
    half = sum(cap)
    total, tokens, arrays = copies * half, case["tokens"], 2 * layers
    if case["op"] == "unpack":
        store = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.uint8}[case["dtype"]]
        mem = torch.zeros(arrays, total * hkv, d, dtype=store, device="cuda")
    else:
        mem = _fill(case, gen, arrays, total * hkv)
        if copies == 2:
            mem[:, half * hkv:] = 0
    # the row of every (token, head), tokens in request order
    rows = []
    for i in range(n):
        t = torch.arange(length[i], dtype=torch.int64)
        rows.append(base[i] * hkv + torch.arange(hkv)[None] * cap[i] + t[:, None])
    rows = torch.cat(rows).to("cuda")
    wide = {"int4": d // 2}.get(case["format"], d)
    shape_c, shape_s = (arrays, tokens, hkv, wide), (arrays, tokens, hkv, d // case["group"])
    kind = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8, "int4": torch.uint8}[case["format"]]
    if case["op"] == "unpack":
        x = _normal(gen, arrays, tokens, hkv, d).view(*shape_s, case["group"])
        top = x.abs().amax(-1, keepdim=True)
        codes = x / top * TOP[case["format"]]
        codes = (codes.round() if case["format"] == "int8" else codes).to(kind).view(shape_c)
        scales = (top[..., 0] * (1.5 / TOP[case["format"]])).contiguous()
    else:
        codes = torch.empty(shape_c, dtype=torch.uint8, device="cuda").view(kind)
        scales = torch.empty(shape_s, dtype=torch.float32, device="cuda")
    state = {"case": case, "mem": mem, "rows": rows, "half": half * hkv, "codes": codes, "scales": scales}
    if own:
        from paper_2512_09427_b200 import odma
        pool = _handle(case, mem, layers, total, bounds, n, 1)
        for k in range(copies):
            for i in range(n):
                _admit(pool, k * n + i, cap[i], length[i] if k == 0 and case["op"] != "unpack" else 0, k * half + base[i])
        fmt = {"e4m3": odma.STORE_E4M3, "int8": odma.STORE_INT8, "int4": odma.STORE_INT4}[case["format"]]
        state["store"] = odma.KvStore(fmt, case["group"], 0, layers, codes.data_ptr(), codes.numel(), scales.data_ptr(),
                                      scales.numel() * 4)
        state["length"], state["pool"] = length, pool
    return state


# ---- one pass ----------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return _own_prefill(state) if op == "prefill" else _own_store(state)
    return _plain_prefill(state) if op == "prefill" else _plain_store(state)


def _own_prefill(s):
    s["pool"].prefill_attention(0, s["q"].data_ptr(), s["case"]["q_heads"], s["tables"], s["workspace"].data_ptr(),
                                s["workspace"].numel(), s["out"].data_ptr(), s["lse"].data_ptr(),
                                torch.cuda.current_stream().cuda_stream)
    return s["out"], s["lse"]


def _own_store(s):
    c, pool = s["case"], s["pool"]
    n, stream = c["batch"], torch.cuda.current_stream().cuda_stream
    if c["op"] != "unpack":
        pool.pack_kv(range(n), s["store"], stream=stream)
    if c["op"] != "pack":
        first = n if c["op"] == "park" else 0
        pool.unpack_kv(range(first, first + n), s["store"], count=s["length"], stream=stream)
    return _store_outputs(s)


def _store_outputs(s):
    """What the pass has written: codes as the values they stand for in units of their scales, or the slabs' rows."""
    c = s["case"]
    if c["op"] == "pack":
        return s["codes"], s["scales"]
    mem = s["mem"].view(torch.float8_e4m3fn) if c["dtype"] == "e4m3" else s["mem"]
    return (mem, s["scales"]) if c["op"] == "park" else mem


def _dequantised(x, case, a):
    return x.view(torch.float8_e4m3fn).float() * KV_SCALES[a] if case["dtype"] == "e4m3" else x.float()


def _plain_prefill(s):
    c, mem = s["case"], s["mem"]
    hq, hkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    g = hq // hkv
    out = torch.empty_like(s["q"])
    lse = torch.empty(s["q"].shape[0], hq, dtype=torch.float32, device="cuda")
    at = 0
    for new, length, cap, base in zip(s["new"], s["len"], s["cap"], s["base"]):
        slab = slice(base * hkv, (base + cap) * hkv)
        keys = _dequantised(mem[0][slab], c, 0).view(hkv, cap, d)
        vals = _dequantised(mem[1][slab], c, 1).view(hkv, cap, d)
        block = max(1, min(new, (1 << 27) // (hq * length)))            # new tokens at a time
        for t0 in range(0, new, block):
            t1 = min(new, t0 + block)
            end = length - new + t1                                     # keys that the last of them sees
            q = s["q"][at + t0:at + t1].float().view(t1 - t0, hkv, g, d).permute(1, 2, 0, 3) * (1.0 / math.sqrt(d))
            score = q.reshape(hkv, g * (t1 - t0), d) @ keys[:, :end].transpose(1, 2)
            score = score.view(hkv, g, t1 - t0, end)
            behind = torch.arange(end, device="cuda")[None] > torch.arange(end - (t1 - t0), end, device="cuda")[:, None]
            score = score.masked_fill_(behind, -math.inf)
            top = score.amax(-1, keepdim=True)
            score = score.sub_(top).exp_()
            den = score.sum(-1, keepdim=True)
            o = (score.view(hkv, -1, end) @ vals[:, :end]).view(hkv, g, t1 - t0, d) / den
            out[at + t0:at + t1] = o.permute(2, 0, 1, 3).reshape(t1 - t0, hq, d).to(out.dtype)
            lse[at + t0:at + t1] = (top + den.log())[..., 0].permute(2, 0, 1).reshape(t1 - t0, hq)
        at += new
    return out, lse


def _plain_store(s):
    c, mem, rows = s["case"], s["mem"], s["rows"]
    fmt, group, op = c["format"], c["group"], c["op"]
    one = torch.ones((), dtype=torch.float32, device="cuda")
    for a in range(2 * c["layers"]):
        if op != "unpack":
            x = _dequantised(mem[a][rows], c, a & 1)
            x = x.view(*x.shape[:-1], -1, group)                        # [tokens, heads, groups, group]
            top = x.abs().amax(-1)
            zero = top < TINY_GROUP
            scale = top / (one * TOP[fmt])                              # a true division, not a product with 1 / TOP
            inv = torch.where(zero, 0.0, one / scale)[..., None]
            s["scales"][a] = torch.where(zero, 0.0, scale)
            y = (x * inv).flatten(-2).clamp_(-TOP[fmt], TOP[fmt])
            if fmt == "int4":
                n = y.round().to(torch.int32) & 15
                y = n[..., 0::2] | (n[..., 1::2] << 4)
            elif fmt == "int8":
                y = y.round()
            s["codes"][a] = y.to(s["codes"].dtype)
        if op != "pack":
            code = s["codes"][a]
            if fmt == "int4":
                n = code.to(torch.int32)
                code = torch.stack((n & 15, n >> 4), -1).flatten(-2)
                code = torch.where(code > 7, code - 16, code)
            x = code.float()
            x = (x.view(*x.shape[:-1], -1, group) * s["scales"][a][..., None]).flatten(-2)
            if c["dtype"] == "e4m3":
                x = (x * (one / KV_SCALES[a & 1])).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            mem[a][rows + (s["half"] if op == "park" else 0)] = x.to(mem.dtype)
    return _store_outputs(s)


# ---- what a pass cannot do without, and the results in 64 bits -----------------------------------

def work(case):
    if case["op"] == "prefill":
        new, ctx = _shape(case)
        hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
        io = 4 if case["dtype"] == "f32" else 2
        seen = sum(a * c + a * (a + 1) // 2 for a, c in zip(new, ctx))
        return {"bytes": sum(new + ctx) * 2 * hkv * d * _esize(case) + case["tokens"] * hq * (2 * d * io + 4),
                "flops": 4 * d * hq * seen}
    rows = 2 * case["layers"] * case["tokens"] * case["kv_heads"]
    row, wide = case["head_dim"] * _esize(case), case["head_dim"] // (2 if case["format"] == "int4" else 1)
    kept = wide + 4 * case["head_dim"] // case["group"]
    trips = 2 if case["op"] == "park" else 1
    return {"bytes": trips * rows * (row + kept), "flops": trips * rows * case["head_dim"] * 2}


def exact(case, seed):
    return _exact_prefill(case, seed) if case["op"] == "prefill" else _exact_store(case, seed)


def _exact_prefill(case, seed):
    s = _prepare_prefill(case, seed)
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    g = hq // hkv
    out = torch.empty(case["tokens"], hq, d, dtype=torch.float64, device="cuda")
    lse = torch.empty(case["tokens"], hq, dtype=torch.float64, device="cuda")
    first = 0
    for i in range(case["batch"]):
        new, length = s["new"][i], s["len"][i]
        for h in range(hkv):
            at = s["base"][i] * hkv + h * s["cap"][i]
            kv = []
            for a in range(2):
                x = s["mem"][a][at:at + length]
                kv.append(x.view(torch.float8_e4m3fn).to(torch.float64) * KV_SCALES[a] if case["dtype"] == "e4m3" else x.to(torch.float64))
            step = max(1, (1 << 26) // (g * length))
            for t in range(0, new, step):
                e = min(new, t + step)
                rows = s["q"][first + t:first + e, h * g:(h + 1) * g].to(torch.float64)
                score = torch.einsum("tgd,kd->tgk", rows, kv[0]) / math.sqrt(d)
                position = torch.arange(length - new + t, length - new + e, device="cuda")
                score = torch.where(torch.arange(length, device="cuda")[None, None] <= position[:, None, None], score, -math.inf)
                lse[first + t:first + e, h * g:(h + 1) * g] = torch.logsumexp(score, -1)
                out[first + t:first + e, h * g:(h + 1) * g] = torch.einsum("tgk,kd->tgd", torch.softmax(score, -1), kv[1])
        first += new
    return out, lse


def _exact_store(case, seed):
    s = _prepare_store(case, seed)
    fmt, group, d = case["format"], case["group"], case["head_dim"]
    if case["op"] == "unpack":
        out = torch.zeros(s["mem"].shape, dtype=torch.float64, device="cuda")
        for a in range(out.shape[0]):
            x = s["codes"][a].to(torch.float64) * s["scales"][a].to(torch.float64).repeat_interleave(group, -1)
            if case["dtype"] == "e4m3":
                x = (x / KV_SCALES[a & 1]).clamp(-448, 448)
            out[a].index_copy_(0, s["rows"].flatten(), x.reshape(-1, d))
        return out
    scales = torch.empty(s["scales"].shape, dtype=torch.float64, device="cuda")
    codes = torch.empty(s["codes"].shape, dtype=torch.float64, device="cuda") if case["op"] == "pack" and fmt == "e4m3" else None
    for a in range(scales.shape[0]):
        x = s["mem"][a][s["rows"].flatten()]
        x = x.view(torch.float8_e4m3fn).to(torch.float64) * KV_SCALES[a & 1] if case["dtype"] == "e4m3" else x.to(torch.float64)
        x = x.view(*scales.shape[1:], group)
        scales[a] = x.abs().amax(-1) / TOP[fmt]
        if codes is not None:
            codes[a] = (x / scales[a][..., None].clamp(min=1e-300)).reshape(codes.shape[1:])
    # integers are decided in 32 bits by definition: no value between them to compare with
    return (codes, scales) if case["op"] == "pack" else (None, scales)
