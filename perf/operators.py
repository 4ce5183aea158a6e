"""Cases for measuring the operators that surround decode attention over contiguous slabs.

Three operators, each in a plain form (elementary torch operations in 32 bits, rounded once at the
end) and through the library:

  append   norm of every query and key head, rotation by position (one axis or several) and the
           append of the new rows into the slabs, in one pass          (Pool.append_qkv)
  prefix   decode attention of a batch whose requests share a long prefix: softmax over the
           prefix's keys and then the request's own                    (Pool.decode_attention_prefix)
  tables   per-step tables, slot map and positions from lengths that live in device memory
                                                                       (Pool.build_tables_device)

`own` chooses: False runs the plain forms, True makes the calls that a user of the library makes.
"""
import math
import random

import numpy as np
import torch

own = False

TILE = 64           # tokens per tile of the split plan
CTAS = 148          # shares the split plan deals the batch into
EPS = 1e-6
THETA = 1e6
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.bfloat16}
KV_SCALES = (0.0140625, 0.015625)      # what a code of 1 stands for in an 8-bit pool: keys, values


# ---- cases -------------------------------------------------------------------------------------

def _append(name, batch, tokens, context, heads, dtype, rot, axes=1, interleaved=False, norm=True):
    q, kv, d = heads
    return {"name": name, "op": "append", "batch": batch, "tokens": tokens, "context": context, "q_heads": q,
            "kv_heads": kv, "head_dim": d, "dtype": dtype, "rot": rot, "axes": axes, "interleaved": interleaved,
            "norm": norm}


def _prefix(name, batch, prefix, suffix, heads, dtype, salt=1):
    q, kv, d = heads
    return {"name": name, "op": "prefix", "batch": batch, "prefix": prefix, "suffix": suffix, "q_heads": q,
            "kv_heads": kv, "head_dim": d, "dtype": dtype, "salt": salt}


def _tables(name, batch, mean, kv_heads, new):
    return {"name": name, "op": "tables", "batch": batch, "mean": mean, "kv_heads": kv_heads, "new": new}


QWEN = (28, 4, 128)     # the repository's Qwen-7B-shaped layer
TINY = (2, 1, 64)       # its fp32 reference layer


def listed():
    return [
        # a single stream decoding: one token, latency only
        _append("append, one token", 1, 1, 900, QWEN, "bf16", 128),
        # the decode step of the 256-request batch on an 8-bit pool
        _append("append, decode of 256, 8-bit", 256, 256, 700, QWEN, "e4m3", 128),
        # a ragged prefill chunk with image positions (time, height, width), q/k/v cut out of one projection
        _append("append, chunk of 8192, 3 axes", 9, 8192, 500, QWEN, "bf16", 128, axes=3),
        # the fp32 reference layer, half of each head rotated, adjacent pairs, no norm
        _append("append, fp32, part rotated", 4, 431, 250, TINY, "f32", 32, interleaved=True, norm=False),
        # a few requests behind a short system prompt: the smallest calls
        _prefix("prefix 777, batch 3", 3, 777, 20, QWEN, "bf16"),
        # the 64-request batch behind a system prompt, own parts as long as in that workload
        _prefix("prefix 2048, batch 64", 64, 2048, 512, QWEN, "bf16"),
        # many requests behind one long document, short own parts: the largest
        _prefix("prefix 32768, batch 256", 256, 32768, 96, QWEN, "bf16"),
        # an 8-bit pool, odd sizes
        _prefix("prefix 5001, batch 47, 8-bit", 47, 5001, 301, QWEN, "e4m3"),
        # the fp32 reference layer
        _prefix("prefix 1000, fp32", 4, 1000, 100, TINY, "f32"),
        # one long stream, cut over all shares
        _tables("tables, one request", 1, 16384, 4, "one"),
        # the 256-request decode batch with heavy-tailed lengths
        _tables("tables, batch of 256", 256, 96, 4, "one"),
        # the largest batch, a ragged number of new tokens each, some none
        _tables("tables, batch of 1024, ragged", 1024, 500, 4, "ragged"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "prefix", "prefix", "tables"])
    if op == "append":
        dtype = rng.choice(["bf16", "bf16", "bf16", "e4m3", "f32"])
        heads = rng.choice([QWEN, (16, 8, 128), (5, 1, 128)])
        if dtype != "e4m3":
            heads = rng.choice([QWEN, TINY, (16, 8, 128), (10, 2, 64), (24, 24, 64), (6, 2, 32)])
        tokens = _log(rng, 1, 8192 if dtype != "f32" else 2048)
        batch = min(tokens, _log(rng, 1, 256))
        d = heads[2]
        axes = rng.choice([1, 1, 2, 3])
        rot = rng.choice([d, d, d // 2, 16])
        c = _append("", batch, tokens, _log(rng, 1, 800), heads, dtype, rot, axes, rng.random() < 0.4, rng.random() < 0.8)
    elif op == "prefix":
        dtype = rng.choice(["bf16", "bf16", "bf16", "e4m3", "f32"])
        heads = rng.choice([QWEN, (16, 8, 128), (8, 2, 128)])
        if dtype == "bf16":
            heads = rng.choice([QWEN, (16, 8, 128), (32, 2, 128), (16, 4, 64), (8, 8, 64)])
        if dtype == "f32":
            heads = rng.choice([TINY, (4, 2, 128), (8, 2, 32)])
            batch, prefix, suffix = _log(rng, 1, 16), _log(rng, 1, 2000), _log(rng, 1, 300)
        else:
            batch = _log(rng, 1, 256)
            prefix = _log(rng, 1, 32768)
            suffix = _log(rng, 1, max(2, min(2000, 60000 // batch)))
        c = _prefix("", batch, prefix, suffix, heads, dtype, rng.randrange(1, 1 << 20))
    else:
        c = _tables("", _log(rng, 1, 1024), _log(rng, 1, 600), rng.choice([1, 2, 4, 8]), rng.choice(["one", "ragged"]))
    del c["name"]
    return c


# ---- inputs ------------------------------------------------------------------------------------

def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _up16(x):
    return (x + 15) // 16 * 16


def _esize(case):
    return {"bf16": 2, "f32": 4, "e4m3": 1}[case["dtype"]]


def _lengths(case):
    """Ragged lengths of the requests' own parts, the same for every seed."""
    r = random.Random(case["salt"] * 1000003 + case["batch"])
    m = case["suffix"]
    return [max(1, min(8 * m, int(m * math.exp(r.gauss(0.0, 0.7) - 0.245)))) for _ in range(case["batch"])]


def _shares(n, tokens):
    """New tokens of the requests, one each at least, ragged, the same for every seed."""
    r = random.Random(tokens * 4099 + n)
    weight = [r.random() + 0.05 for _ in range(n)]
    new = [1 + int((tokens - n) * w / sum(weight)) for w in weight]
    new[n // 2] += tokens - sum(new)
    return new


def _handle(case, memory, tokens, boundaries, max_batch, max_group):
    """The library's pool over `memory`: one layer, no Large Bucket."""
    from paper_2512_09427_b200 import odma
    cfg = odma.config_default()
    cfg.safety_pct, cfg.max_len, cfg.window = 0, boundaries[-1], 16
    cfg.max_batch, cfg.max_group, cfg.plan_ctas = max_batch, max_group, CTAS
    kind = {"bf16": odma.DTYPE_BF16, "f32": odma.DTYPE_F32, "e4m3": odma.DTYPE_FP8_E4M3}[case["dtype"]]
    pool = odma.Pool(memory.data_ptr(), memory.numel() * memory.element_size(), 1, case["kv_heads"], case["head_dim"],
                     kind, cfg)
    if pool.set_buckets(boundaries) != odma.OK or pool.get_stats()["total_tokens"] != tokens:
        raise RuntimeError("the pool has another size")
    if case["dtype"] == "e4m3":
        pool.set_kv_scales([KV_SCALES[0]], [KV_SCALES[1]])
    return pool


def _admit(pool, req, cap, length, base):
    rc, slab = pool.alloc(req, cap)
    if rc or slab[:2] != (base, cap) or pool.commit_step([req], [length]):
        raise RuntimeError("the slab is not where it was expected")


def prepare(case, seed):
    return {"append": _prepare_append, "prefix": _prepare_prefix, "tables": _prepare_tables}[case["op"]](case, seed)


def _prepare_append(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = random.Random(seed)
    n, tokens, dt = case["batch"], case["tokens"], DTYPES[case["dtype"]]
    hq, hkv, d, rot, axes = case["q_heads"], case["kv_heads"], case["head_dim"], case["rot"], case["axes"]
    new = _shares(n, tokens)
    length = [r.randint(0, case["context"]) for _ in range(n)]
    cap = _up16(case["context"] + max(new))
    total = n * cap
    # one projection's output, cut into queries, keys and values
    qkv = _normal(gen, tokens, hq + 2 * hkv, d).mul_(2.0).to(dt)
    store = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.uint8}[case["dtype"]]
    mem = torch.zeros(2, total * hkv, d, dtype=store, device="cuda")
    pos1 = np.concatenate([np.arange(a, a + b) for a, b in zip(length, new)])
    owner = np.repeat(np.arange(n), new)
    if axes == 1:
        far = r.randrange(1 << 17)
        pos = pos1[None] + far
    else:                               # rows of a picture: time stands still, height and width walk
        pos = np.stack([pos1 // 256 + 1000 * owner, pos1 // 16 % 16, pos1 % 16][:axes]) + r.randrange(1 << 15)
    pairs = rot // 2
    section = [pairs] if axes == 1 else [pairs // axes + (1 if a < pairs % axes else 0) for a in range(axes)]
    slot = (owner * cap * hkv + pos1)[:, None] + np.arange(hkv)[None] * cap
    state = {
        "case": case, "q": qkv[:, :hq], "k": qkv[:, hq:hq + hkv], "v": qkv[:, hq + hkv:], "mem": mem,
        "q_norm": (1.0 + 0.2 * _normal(gen, d)).to(dt) if case["norm"] else None,
        "k_norm": (1.0 + 0.2 * _normal(gen, d)).to(dt) if case["norm"] else None,
        "inv_freq": torch.tensor([THETA ** (-2.0 * i / rot) for i in range(pairs)], dtype=torch.float32, device="cuda"),
        "pos": torch.tensor(pos, dtype=torch.int32, device="cuda"),
        "axis": torch.tensor(np.repeat(np.arange(axes), section), dtype=torch.int64, device="cuda"),
        "section": section,
        "slot": torch.tensor(slot, dtype=torch.int64, device="cuda"),
    }
    if own:
        from paper_2512_09427_b200 import odma
        pool = _handle(case, mem, total, [cap], n, hq // hkv)
        for i in range(n):
            _admit(pool, i, cap, length[i], i * cap)
        stream = torch.cuda.current_stream().cuda_stream
        state["table"] = torch.empty(pool.tables_bytes(n), dtype=torch.uint8, device="cuda")
        state["tables"] = pool.build_tables(list(range(n)), state["table"].data_ptr(), state["table"].numel(), stream, new)
        state["q_out"] = torch.empty(tokens, hq, d, dtype=dt, device="cuda")
        row = (hq + 2 * hkv) * d
        state["prep"] = odma.QkvPrep(
            rot_dim=rot, interleaved=case["interleaved"], section=section, inv_freq=state["inv_freq"].data_ptr(),
            positions=state["pos"].data_ptr(), q_norm=state["q_norm"].data_ptr() if case["norm"] else 0,
            k_norm=state["k_norm"].data_ptr() if case["norm"] else 0, eps=EPS, q_stride=row, k_stride=row, v_stride=row)
        state["pool"] = pool
    return state


def _prepare_prefix(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n, p, dt = case["batch"], case["prefix"], DTYPES[case["dtype"]]
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    lens = _lengths(case)
    cap_p, cap_s = _up16(p), _up16(max(lens))
    total = cap_p + n * cap_s
    kv = _normal(gen, 2, total * hkv, d)
    if case["dtype"] == "e4m3":
        for a in range(2):
            kv[a].mul_(1.0 / KV_SCALES[a])
        mem = kv.clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        mem = kv.to(dt)
    del kv
    state = {
        "case": case, "mem": mem, "q": _normal(gen, n, hq, d).to(dt), "cap_p": cap_p, "cap_s": cap_s,
        "len": torch.tensor(lens, dtype=torch.int64, device="cuda"), "longest": max(lens),
    }
    if own:
        pool = _handle(case, mem, total, sorted({cap_p, cap_s}), n, hq // hkv)
        _admit(pool, n, cap_p, p, 0)
        for i in range(n):
            _admit(pool, i, cap_s, lens[i], cap_p + i * cap_s)
        stream = torch.cuda.current_stream().cuda_stream
        state["table"] = torch.empty(pool.tables_bytes(n), dtype=torch.uint8, device="cuda")
        state["tables"] = pool.build_tables(list(range(n)), state["table"].data_ptr(), state["table"].numel(), stream, [0] * n)
        state["workspace"] = torch.empty(pool.prefix_workspace_bytes(hq, n, p), dtype=torch.uint8, device="cuda")
        state["out"] = torch.empty_like(state["q"])
        state["lse"] = torch.empty(n, hq, dtype=torch.float32, device="cuda")
        state["pool"] = pool
    return state


def _prepare_tables(case, seed):
    r = random.Random(seed)
    n, hkv = case["batch"], case["kv_heads"]
    # heavy-tailed lengths, some requests still empty; now and then one whose slab is full
    length = [0 if r.random() < 0.03 else int(case["mean"] * min(64.0, r.paretovariate(1.5)) / 3.0) for _ in range(n)]
    if case["new"] == "one":
        new = [1] * n
    else:
        new = [0 if r.random() < 0.2 else r.randint(1, 17) for _ in range(n)]
    cap = [_up16(a + b + r.randint(0, 40)) for a, b in zip(length, new)]
    cap = [max(16, c - 16 * (-(-(c - a - b + 1) // 16))) if r.random() < 0.01 else c for a, b, c in zip(length, new, cap)]
    order = list(range(n))
    r.shuffle(order)
    base, at = [0] * n, 0
    for i in order:
        base[i], at = at, at + cap[i]
    dev = {"dtype": torch.int32, "device": "cuda"}
    state = {
        # a program that captured the step has rows for this many new tokens, used or not
        "case": case, "total": at, "n_new": n if case["new"] == "one" else 8 * n + 16,
        "slabs": torch.tensor([[a, b] for a, b in zip(base, cap)], **dev),
        "len": torch.tensor(length, **dev), "new": torch.tensor(new, **dev) if case["new"] != "one" else None,
    }
    if own:
        geometry = {"kv_heads": hkv, "head_dim": 64, "dtype": "bf16"}
        room = max(at, 16)                # slabs may all be empty; a pool has room for some tokens
        state["mem"] = torch.empty(room * hkv * 2 * 64, dtype=torch.bfloat16, device="cuda")
        pool = _handle(geometry, state["mem"], room, [max(16, _up16(max(cap)))], n, 8)
        state["table"] = torch.empty(pool.tables_bytes(n), dtype=torch.uint8, device="cuda")
        state["next"] = torch.empty(n, **dev)
        state["slots"] = torch.empty(state["n_new"], **dev)
        state["positions"] = torch.empty(state["n_new"], **dev)
        state["pool"] = pool
    return state


# ---- one pass ----------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return {"append": _own_append, "prefix": _own_prefix, "tables": _own_tables}[op](state)
    return {"append": _plain_append, "prefix": _plain_prefix, "tables": _plain_tables}[op](state)


def _own_append(s):
    s["pool"].append_qkv(0, s["tables"], s["q"].data_ptr(), s["k"].data_ptr(), s["v"].data_ptr(), s["q_out"].data_ptr(),
                         s["case"]["q_heads"], s["prep"], torch.cuda.current_stream().cuda_stream)
    return _append_outputs(s["q_out"], s["mem"], s["case"])


def _own_prefix(s):
    c = s["case"]
    s["pool"].decode_attention_prefix(0, s["q"].data_ptr(), c["q_heads"], c["batch"], c["prefix"], s["tables"],
                                      s["workspace"].data_ptr(), s["workspace"].numel(), s["out"].data_ptr(),
                                      s["lse"].data_ptr(), torch.cuda.current_stream().cuda_stream)
    return s["out"], s["lse"]


def _own_tables(s):
    n = s["case"]["batch"]
    t = s["pool"].build_tables_device(
        s["slabs"].data_ptr(), s["len"].data_ptr(), n, s["n_new"], s["table"].data_ptr(), s["table"].numel(),
        d_n_new=s["new"].data_ptr() if s["new"] is not None else 0, d_len_next=s["next"].data_ptr(),
        d_slots=s["slots"].data_ptr(), d_positions=s["positions"].data_ptr(),
        stream=torch.cuda.current_stream().cuda_stream)
    return s["table"].view(torch.int32)[:t.words], s["next"], s["slots"], s["positions"]


def _append_outputs(q_out, mem, case):
    mem = mem.view(torch.float8_e4m3fn) if case["dtype"] == "e4m3" else mem
    return q_out, mem[0], mem[1]


def _rotated(x, weight, angle, case):
    """Norm over the head, then the rotation; x [tokens, heads, d] in 32 bits, angle [tokens, pairs] in 64."""
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
    rot = case["rot"]
    if case["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    ra, rb = a * cos - b * sin, a * sin + b * cos
    r = torch.stack((ra, rb), -1).flatten(-2) if case["interleaved"] else torch.cat((ra, rb), -1)
    return torch.cat((r, x[..., rot:]), -1)


def _plain_append(s):
    c, mem = s["case"], s["mem"]
    angle = s["pos"].double()[s["axis"]].t() * s["inv_freq"].double()[None]
    q = _rotated(s["q"].float(), s["q_norm"], angle, c).to(s["q"].dtype)
    k, v, slot = _rotated(s["k"].float(), s["k_norm"], angle, c), s["v"].float(), s["slot"]
    if c["dtype"] == "e4m3":
        one = torch.ones((), dtype=torch.float32, device="cuda")
        k = (k * (one / KV_SCALES[0])).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        v = (v * (one / KV_SCALES[1])).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    mem[0][slot] = k.to(mem.dtype)
    mem[1][slot] = v.to(mem.dtype)
    return _append_outputs(q, mem, c)


def _dequantised(x, case, a):
    return x.view(torch.float8_e4m3fn).float() * KV_SCALES[a] if case["dtype"] == "e4m3" else x.float()


def _plain_prefix(s):
    c, mem = s["case"], s["mem"]
    n, p, hq, hkv, d = c["batch"], c["prefix"], c["q_heads"], c["kv_heads"], c["head_dim"]
    head = torch.arange(hkv, device="cuda")
    rows = head[:, None] * s["cap_p"] + torch.arange(p, device="cuda")[None]                     # [hkv, p]
    t = torch.arange(s["longest"], device="cuda")
    base = s["cap_p"] + torch.arange(n, device="cuda") * s["cap_s"]
    own_rows = base[:, None, None] * hkv + head[None, :, None] * s["cap_s"] + t[None, None]      # [n, hkv, longest]
    q = s["q"].float().view(n, hkv, hq // hkv, d) * (1.0 / math.sqrt(d))
    kp, vp = _dequantised(mem[0][rows], c, 0), _dequantised(mem[1][rows], c, 1)
    ks, vs = _dequantised(mem[0][own_rows], c, 0), _dequantised(mem[1][own_rows], c, 1)
    sp = q.transpose(0, 1).reshape(hkv, -1, d) @ kp.transpose(1, 2)                               # [hkv, n*g, p]
    ss = q @ ks.transpose(2, 3)                                                                   # [n, hkv, g, longest]
    ss = ss.masked_fill(t[None, None, None] >= s["len"][:, None, None, None], -math.inf)
    mp = sp.amax(-1).view(hkv, n, -1).transpose(0, 1)                                             # [n, hkv, g]
    m = torch.maximum(mp, ss.amax(-1))
    sp = (sp - m.transpose(0, 1).reshape(hkv, -1)[..., None]).exp_()
    ss = (ss - m[..., None]).exp_()
    den = sp.sum(-1).view(hkv, n, -1).transpose(0, 1) + ss.sum(-1)
    out = (sp @ vp).view(hkv, n, -1, d).transpose(0, 1) + ss @ vs
    out = (out / den[..., None]).reshape(n, hq, d).to(s["q"].dtype)
    return out, (m + den.log()).reshape(n, hq)


MIN_PIECE, MIN_SHARE = 3, 4      # tiles: shortest piece of a cut stream, least cost of a share


def _plain_tables(s):
    """The table that include/odma.h describes at odma_build_tables_device, by sums, searches and scatters."""
    c = s["case"]
    n, hkv, total, n_new = c["batch"], c["kv_heads"], s["total"], s["n_new"]
    bound, n_comb = n * hkv + CTAS, min(n * hkv, CTAS)
    where = {"dtype": torch.long, "device": s["len"].device}
    base, cap = s["slabs"].long().unbind(1)
    length = s["len"].long()
    new = s["new"].long() if s["new"] is not None else torch.ones_like(length)
    zero, nought = torch.zeros_like(length), torch.zeros(1, **where)
    ok = (base >= 0) & (base % 16 == 0) & (cap >= 0) & (base + cap <= total) & (length >= 0) & (new >= 0) & (new <= n_new)
    counted = torch.where((new >= 0) & (new <= n_new), new, zero)
    cu = torch.cat((nought, counted.cumsum(0)))
    ok &= (length + new <= cap) & (cu[:-1] + new <= n_new)
    cu = cu.clamp(max=n_new)
    base, cap, after = torch.where(ok, base, zero), torch.where(ok, cap, zero), torch.where(ok, length + new, zero)

    # streams, numbered over the requests that hold a token: tiles, and cost with one for the start
    held = torch.nonzero_static(after > 0, size=n, fill_value=0)[:, 0]
    streams = (after > 0).sum() * hkv
    q_all = torch.arange(n * hkv + 1, **where)
    req_of = held[(q_all // hkv).clamp(max=n - 1)]
    tiles = torch.where(q_all < streams, (after[req_of] + TILE - 1) // TILE, 0)
    cost = torch.where(q_all < streams, tiles + 1, 0)
    ends = cost.cumsum(0)
    # where the shares begin: stream q, tile t; a cut close to a stream's end moves to that end
    share = ((ends[-1] + CTAS - 1) // CTAS).clamp(min=MIN_SHARE)
    x = (torch.arange(CTAS + 1, **where) * share).clamp(max=ends[-1])
    q = torch.searchsorted(ends, x, right=True).clamp(max=n * hkv)
    u, of = x - (ends - cost)[q], tiles[q]
    low = torch.where(of < 2 * MIN_PIECE, 2 * u <= of, u <= MIN_PIECE)
    high = ~low & ((of < 2 * MIN_PIECE) | (u > of - MIN_PIECE + 1))
    t = torch.where(low | high, 0, u - 1)
    q = torch.where(x >= ends[-1], streams, q + high.long())
    t = torch.where(x >= ends[-1], 0, t)
    q[CTAS], t[CTAS] = streams, 0
    # pieces in stream order: one per stream and one per cut inside a stream
    begin = q + (t > 0).long().cumsum(0)
    cut_q = torch.where(t > 0, q, n * hkv + 1).sort().values
    first = q_all + torch.searchsorted(cut_q, q_all)
    piece_q = torch.full((bound + 2,), -1, **where)
    piece_t = torch.zeros(bound + 2, **where)
    piece_q[torch.where(q_all < streams, first, bound + 1)] = q_all
    at = torch.where(t > 0, begin, bound + 1)
    piece_q[at], piece_t[at] = q, t
    pi = torch.arange(bound, **where)
    live, pq, pt = pi < begin[CTAS], piece_q[:bound].clamp(min=0), piece_t[:bound]
    last = (pi + 1 >= begin[CTAS]) | (piece_q[1:bound + 1] != pq)
    stop = torch.where(last, tiles[pq], piece_t[1:bound + 1])
    cuts = first[1:] - first[:-1] - 1
    cut = torch.where(q_all[:-1] < streams, cuts, 0) > 0
    split = cut[pq.clamp(max=n * hkv - 1)]
    comb_of = cut.long().cumsum(0) - 1
    req, head = req_of[pq], pq % hkv
    tok0 = pt * TILE
    row0 = base[req] * hkv + head * cap[req] + tok0
    flags = (~split).long() + 2 * last.long()
    comb = torch.where(split, comb_of[pq.clamp(max=n * hkv - 1)], -1)
    item = torch.stack((req, head, tok0, torch.minimum(stop * TILE, after[req]) - tok0, flags, pi, row0, comb), 1)
    item = torch.where(live[:, None], item, torch.tensor([-1, 0, 0, 0, 0, 0, 0, -1], **where))
    # inside a share, the pieces of cut streams (its first and its last at most) come first
    owner = torch.searchsorted(begin, pi, right=True).clamp(max=CTAS) - 1
    b0, m = begin[owner], begin[owner + 1] - begin[owner]
    lead = split[b0.clamp(max=bound - 1)]
    tail = split[(b0 + m - 1).clamp(min=0, max=bound - 1)] & (m > 1)
    j = pi - b0
    place = torch.where((j == 0) & lead, 0, torch.where((j == m - 1) & tail, lead.long(), j + tail.long()))
    items = torch.empty_like(item)
    items[torch.where(live, b0 + place, pi)] = item
    rec = torch.zeros(CTAS, 12, **where)
    rec[:, 0], rec[:, 1] = begin[:-1], begin[1:]
    rec[:, 4:] = torch.where((begin[1:] > begin[:-1])[:, None], items[begin[:-1].clamp(max=bound - 1)], 0)
    cs = torch.nonzero_static(cut, size=n_comb, fill_value=0)[:, 0]
    combine = torch.stack((req_of[cs], cs % hkv, first[cs], cuts[cs] + 1), 1)
    combine = torch.where((torch.arange(n_comb, **where) < cut.sum())[:, None], combine, 0)

    def padded(v):
        return torch.cat((v, torch.zeros(-len(v) % 4, **where)))

    words = torch.cat((padded(base), padded(cap), padded(after), padded(cu), rec.flatten(), items.flatten(),
                       combine.flatten()))
    # slot map and positions of the new tokens
    tok = torch.arange(n_new, **where)
    r = (torch.searchsorted(cu, tok, right=True) - 1).clamp(max=n - 1)
    there = (tok < cu[-1]) & ok[r]
    pos = length[r] + tok - cu[r]
    slots, pos = torch.where(there, base[r] * hkv + pos, -1), torch.where(there, pos, -1)
    return words.int(), torch.where(ok, length + new, length).int(), slots.int(), pos.int()


# ---- what a pass cannot do without, and the results in 64 bits -----------------------------------

def work(case):
    if case["op"] == "append":
        io = 4 if case["dtype"] == "f32" else 2
        row, hq, hkv = case["head_dim"] * case["tokens"], case["q_heads"], case["kv_heads"]
        return {"bytes": row * (2 * hq * io + 2 * hkv * (io + _esize(case))), "flops": row * (hq + hkv) * 6}
    if case["op"] == "prefix":
        n, hq, hkv, d = case["batch"], case["q_heads"], case["kv_heads"], case["head_dim"]
        own_tokens = sum(_lengths(case))
        io = 4 if case["dtype"] == "f32" else 2
        return {"bytes": (case["prefix"] + own_tokens) * 2 * hkv * d * _esize(case) + n * hq * (2 * d * io + 4),
                "flops": 4 * d * hq * (n * case["prefix"] + own_tokens)}
    n, hkv = case["batch"], case["kv_heads"]
    return {"bytes": 4 * (9 * n + 12 * CTAS + 8 * (n * hkv + CTAS) + 4 * min(n * hkv, CTAS)), "flops": 16 * (n * hkv + CTAS)}


def exact(case, seed):
    if case["op"] == "append":
        return _exact_append(case, seed)
    if case["op"] == "prefix":
        return _exact_prefix(case, seed)
    return None


def _exact_append(case, seed):
    s = _prepare_append(case, seed)
    rot, d = case["rot"], case["head_dim"]
    pairs = rot // 2
    lo = torch.arange(pairs, device="cuda") * (2 if case["interleaved"] else 1)
    hi = lo + (1 if case["interleaved"] else pairs)
    pos = s["pos"].to(torch.float64)
    theta = torch.stack([pos[a] for a in s["axis"].tolist()], 1) * s["inv_freq"].to(torch.float64)

    def head(x, w):
        y = x.to(torch.float64)
        if w is not None:
            y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / d + EPS) * w.to(torch.float64)
        z = y.clone()
        z[..., lo] = y[..., lo] * torch.cos(theta)[:, None] - y[..., hi] * torch.sin(theta)[:, None]
        z[..., hi] = y[..., hi] * torch.cos(theta)[:, None] + y[..., lo] * torch.sin(theta)[:, None]
        return z

    k, v = head(s["k"], s["k_norm"]), s["v"].to(torch.float64)
    if case["dtype"] == "e4m3":
        k, v = (k / KV_SCALES[0]).clamp(-448, 448), (v / KV_SCALES[1]).clamp(-448, 448)
    both = torch.zeros(s["mem"].shape, dtype=torch.float64, device="cuda")
    both[0].index_copy_(0, s["slot"].flatten(), k.reshape(-1, d))
    both[1].index_copy_(0, s["slot"].flatten(), v.reshape(-1, d))
    return head(s["q"], s["q_norm"]), both[0], both[1]


def _exact_prefix(case, seed):
    s = _prepare_prefix(case, seed)
    n, p, hq, hkv, d = case["batch"], case["prefix"], case["q_heads"], case["kv_heads"], case["head_dim"]
    g = hq // hkv

    def wide(rows, a):
        x = rows.view(torch.float8_e4m3fn).to(torch.float64) * KV_SCALES[a] if case["dtype"] == "e4m3" else rows.to(torch.float64)
        return x

    out = torch.empty(n, hq, d, dtype=torch.float64, device="cuda")
    lse = torch.empty(n, hq, dtype=torch.float64, device="cuda")
    lens = s["len"].tolist()
    for h in range(hkv):
        keys = wide(s["mem"][0][h * s["cap_p"]:h * s["cap_p"] + p], 0)
        vals = wide(s["mem"][1][h * s["cap_p"]:h * s["cap_p"] + p], 1)
        for i in range(n):
            at = (s["cap_p"] + i * s["cap_s"]) * hkv + h * s["cap_s"]
            k = torch.cat((keys, wide(s["mem"][0][at:at + lens[i]], 0)))
            v = torch.cat((vals, wide(s["mem"][1][at:at + lens[i]], 1)))
            score = s["q"][i, h * g:(h + 1) * g].to(torch.float64) @ k.T / math.sqrt(d)
            lse[i, h * g:(h + 1) * g] = torch.logsumexp(score, -1)
            out[i, h * g:(h + 1) * g] = torch.softmax(score, -1) @ v
    return out, lse
