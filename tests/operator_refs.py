"""Plain references of the operators around slab attention (fp64 and integers), and a small pool to run them on."""
import math

import torch

TILE, MIN_PIECE, MIN_SHARE = 64, 3, 4


def lib():
    from paper_2512_09427_b200 import odma
    return odma


# ---- tables ------------------------------------------------------------------------------------

def up4(v):
    return (v + 3) // 4 * 4


def share_starts(lengths, kv_heads, ctas):
    """(streams, cuts): streams [(request, head, tiles)] that hold a token, and where each share begins (stream, tile)."""
    streams = [(i, h, (a + TILE - 1) // TILE) for i, a in enumerate(lengths) if a > 0 for h in range(kv_heads)]
    start = [0]
    for _, _, t in streams:
        start.append(start[-1] + t + 1)
    share = max(-(-start[-1] // ctas), MIN_SHARE)
    cuts, s = [], 0
    for c in range(ctas + 1):
        x = c * share
        if c == ctas or x >= start[-1]:
            cuts.append((len(streams), 0))
            continue
        while start[s + 1] <= x:
            s += 1
        u, t = x - start[s], streams[s][2]
        if t < 2 * MIN_PIECE:
            cuts.append((s, 0) if 2 * u <= t else (s + 1, 0))
        elif u - 1 < MIN_PIECE:
            cuts.append((s, 0))
        elif u - 1 > t - MIN_PIECE:
            cuts.append((s + 1, 0))
        else:
            cuts.append((s, u - 1))
    return streams, cuts


def device_tables(base, cap, length, new, n_new_total, tokens, kv_heads, ctas):
    """(words, lengths after, slot map, positions) of odma_build_tables_device, request by request, piece by piece."""
    n = len(base)
    cu, ok = [0], []
    for i in range(n):
        counted = 0 <= new[i] <= n_new_total
        ok.append(counted and base[i] >= 0 and base[i] % 16 == 0 and cap[i] >= 0 and base[i] + cap[i] <= tokens and
                  length[i] >= 0 and length[i] + new[i] <= cap[i] and cu[-1] + new[i] <= n_new_total)
        cu.append(cu[-1] + (new[i] if counted else 0))
    b = [x if o else 0 for x, o in zip(base, ok)]
    k = [x if o else 0 for x, o in zip(cap, ok)]
    after = [x + y if o else 0 for x, y, o in zip(length, new, ok)]
    streams, cuts = share_starts(after, kv_heads, ctas)
    pieces = []                                     # (stream, first tile, end tile, share)
    for c in range(ctas):
        s, t = cuts[c]
        while (s, t) < cuts[c + 1]:
            e = cuts[c + 1][1] if s == cuts[c + 1][0] else streams[s][2]
            pieces.append((s, t, e, c))
            s, t = s + 1, 0
    count, record, combine, items = {}, {}, [], []
    for p in pieces:
        count[p[0]] = count.get(p[0], 0) + 1
    for slot, (s, t, e, c) in enumerate(pieces):
        i, h, of = streams[s]
        if count[s] > 1 and s not in record:
            record[s] = len(combine)
            combine.append([i, h, slot, count[s]])
        item = [i, h, TILE * t, min(TILE * e, after[i]) - TILE * t, (1 if count[s] == 1 else 0) | (2 if e == of else 0), slot,
                b[i] * kv_heads + h * k[i] + TILE * t, record.get(s, -1)]
        items.append((c, count[s] > 1, item))
    out, rec = [], []
    for c in range(ctas):
        first = len(out)
        out += [it for cc, sp, it in items if cc == c and sp] + [it for cc, sp, it in items if cc == c and not sp]
        rec += [first, len(out), 0, 0] + (out[first] if len(out) > first else [0] * 8)
    out += [[-1, 0, 0, 0, 0, 0, 0, -1]] * (n * kv_heads + ctas - len(out))
    combine += [[0] * 4] * (min(n * kv_heads, ctas) - len(combine))

    def pad(v):
        return v + [0] * (up4(len(v)) - len(v))

    words = pad(b) + pad(k) + pad(after) + pad([min(x, n_new_total) for x in cu]) + rec + sum(out, []) + sum(combine, [])
    slots, pos = [-1] * n_new_total, [-1] * n_new_total
    for i in range(n):
        for j in range(new[i] if ok[i] else 0):
            slots[cu[i] + j], pos[cu[i] + j] = b[i] * kv_heads + length[i] + j, length[i] + j
    return words, [x + y if o else x for x, y, o in zip(length, new, ok)], slots, pos


# ---- norm, rotation -----------------------------------------------------------------------------

def prepared(x, weight, eps, inv_freq, positions, axis, rot_dim, interleaved):
    """x [tokens, heads, D] -> (z, slack): fp64 result of norm and rotation, and a bound on what fp32 arithmetic may
    differ from it by.  positions [axes, tokens], axis [pairs].

    fp32: the sum of D squares is off by (D + 2) 2^-24 relative at most, half of that after the root; the root, two
    products and the product with the turn add at most 8 roundings or units of 2^-23; the angle, reduced to
    [-pi, pi] and rounded to fp32, is off by 2^-24 pi < 2e-7, its sine and cosine by two units (2.4e-7) more."""
    d = x.shape[-1]
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps) * weight.double()
    pairs = rot_dim // 2
    a = torch.arange(pairs) * (2 if interleaved else 1)
    b = a + (1 if interleaved else pairs)
    z, size = y.clone(), y.abs()
    if pairs:
        t = (positions.double()[axis].t() * inv_freq.double()[None])[:, None]
        z[..., a] = y[..., a] * t.cos() - y[..., b] * t.sin()
        z[..., b] = y[..., b] * t.cos() + y[..., a] * t.sin()
        both = y[..., a].abs() + y[..., b].abs()
        size[..., a] = both
        size[..., b] = both
    return z, size * ((d / 2 + 16) * 2.0 ** -24 + 5e-7)


def rounding(z, dtype):
    """Half a step of `dtype` at z: eps/2 relative, and half the smallest subnormal."""
    fi = torch.finfo(dtype)
    return z.abs() * (fi.eps / 2) + fi.smallest_normal * fi.eps / 2


# ---- attention ------------------------------------------------------------------------------------

def attention(q, keys, values, dtype):
    """One request: q [g, D], keys and values [N, D] -> (out, lse, out bound, lse bound), all fp64.

    A score is a sum of D fp32 products: off by (D + 4) 2^-24 times the sum of their sizes (scale and the log2
    factor included in the 4).  Weights: twice that relative (numerator and denominator), 2^-21 for 2^x, and a half
    step of bf16 (2^-8) where the weights go through 16-bit (or split 8-bit) tensor-core operands.  Sums over N keys and the
    merges: (N + 64) 2^-24.  The result: one rounding to `dtype`."""
    d, n = q.shape[-1], keys.shape[0]
    if n == 0:
        z = torch.zeros_like(q, dtype=torch.float64)
        return z, torch.full((q.shape[0],), -math.inf, dtype=torch.float64), z, torch.zeros(q.shape[0], dtype=torch.float64)
    qd, k, v = q.double(), keys.double(), values.double()
    s = qd @ k.t() / math.sqrt(d)
    slip = ((d + 4) * 2.0 ** -24 * (qd.abs() @ k.abs().t()) / math.sqrt(d)).amax(-1)
    w = torch.softmax(s, -1)
    out, size = w @ v, w @ v.abs()
    sums = (n + 64) * 2.0 ** -24
    rel = 2 * slip + 2.0 ** -21 + sums + (2.0 ** -8 if dtype != torch.float32 else 0.0)
    lse = torch.logsumexp(s, -1)
    # the denominator may be summed over rounded weights or unrounded ones: 2^-8 once more where they are rounded
    bound = size * rel[:, None] + rounding(out, dtype)
    lse_bound = slip + 2.0 ** -21 + sums + lse.abs() * 2.0 ** -22 + (s.abs().amax(-1) * 2.0 ** -22)
    return out, lse, bound, lse_bound


# ---- a pool ---------------------------------------------------------------------------------------

class SlabPool:
    """A device pool with every row NaN but those of live tokens, and its contents on the host."""

    def __init__(self, caps, lens, layers=1, kv_heads=4, head_dim=128, kind="bf16", ctas=0, max_batch=None, max_group=16,
                 seed=1, scale=1.0, **cfg_over):
        odma = lib()
        self.odma, self.kind, self.layers, self.kv_heads, self.head_dim = odma, kind, layers, kv_heads, head_dim
        self.caps, self.lens = list(caps), list(lens)
        n = len(caps)
        cfg = odma.config_default()
        cfg.safety_pct, cfg.window = 0, 16
        cfg.max_len = max(caps)
        cfg.max_batch = max_batch or n
        cfg.max_group = min(8, max_group) if kind == "e4m3" else max_group
        cfg.plan_ctas = ctas
        for k, v in cfg_over.items():
            setattr(cfg, k, v)
        dt = {"bf16": (odma.DTYPE_BF16, torch.bfloat16), "f32": (odma.DTYPE_F32, torch.float32),
              "e4m3": (odma.DTYPE_FP8_E4M3, torch.uint8)}[kind]
        self.io = torch.float32 if kind == "f32" else torch.bfloat16
        self.T = sum(caps)
        shape = (layers * 2, self.T * kv_heads, head_dim)
        if kind == "e4m3":
            self.mem = torch.full(shape, 0x7F, dtype=torch.uint8, device="cuda")        # the code of NaN
        else:
            self.mem = torch.full(shape, float("nan"), dtype=dt[1], device="cuda")
        self.pool = odma.Pool(self.mem.data_ptr(), self.mem.numel() * self.mem.element_size(), layers, kv_heads, head_dim, dt[0], cfg)
        self.ctas = cfg.plan_ctas or torch.cuda.get_device_properties(0).multi_processor_count
        self.k_scale = [0.014 + 0.001 * i for i in range(layers)] if kind == "e4m3" else [1.0] * layers
        self.v_scale = [0.016 - 0.001 * i for i in range(layers)] if kind == "e4m3" else [1.0] * layers
        if kind == "e4m3":
            self.pool.set_kv_scales(self.k_scale, self.v_scale)
        gen = torch.Generator().manual_seed(seed)
        self.base = []
        for r, (c, ln) in enumerate(zip(caps, lens)):
            assert self.pool.set_buckets([c]) == 0
            rc, slab = self.pool.alloc(r, c)
            assert rc == 0 and slab[1] == c
            self.base.append(slab[0])
            if ln:
                assert self.pool.commit_step([r], [ln]) == 0
                for a in range(layers * 2):
                    x = torch.randn(ln, kv_heads, head_dim, generator=gen) * (scale if a % 2 == 0 else 1.0)
                    rows = self.stored(x, a)
                    for h in range(kv_heads):
                        at = slab[0] * kv_heads + h * c
                        self.mem[a, at:at + ln] = rows[:, h].cuda()
        self.gen = gen
        self.stream = torch.cuda.current_stream().cuda_stream
        self.table = torch.empty(self.pool.tables_bytes(cfg.max_batch), dtype=torch.uint8, device="cuda")

    def stored(self, x, array):
        if self.kind != "e4m3":
            return x.to(self.io)
        inv = torch.ones(()) / torch.tensor((self.v_scale if array % 2 else self.k_scale)[array // 2], dtype=torch.float32)
        return (x.to(self.io).float() * inv).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)

    def values(self, array, req, head, n):
        """The first n rows of one stream as fp64."""
        at = self.base[req] * self.kv_heads + head * self.caps[req]
        x = self.mem[array, at:at + n].cpu()
        if self.kind != "e4m3":
            return x.double()
        scale = torch.tensor((self.v_scale if array % 2 else self.k_scale)[array // 2], dtype=torch.float32)
        return x.view(torch.float8_e4m3fn).double() * scale.double()

    def randn(self, *shape, scale=1.0):
        return (torch.randn(*shape, generator=self.gen) * scale).to(self.io).cuda()

    def tables(self, reqs, n_new=None):
        return self.pool.build_tables(reqs, self.table.data_ptr(), self.table.numel(), self.stream, n_new)

    def sync(self):
        torch.cuda.synchronize()
        return self.pool.check_status(self.stream)

    def reference(self, layer, q, reqs, lens, prefix=None, prefix_len=0):
        """fp64 attention of q [n, q_heads, D] (host) over the slabs: stacked (out, lse, bounds)."""
        g = q.shape[1] // self.kv_heads
        rows = []
        for i, r in enumerate(reqs):
            per_head = []
            for h in range(self.kv_heads):
                k, v = self.values(2 * layer, r, h, lens[i]), self.values(2 * layer + 1, r, h, lens[i])
                if prefix_len:
                    k = torch.cat((self.values(2 * layer, prefix, h, prefix_len), k))
                    v = torch.cat((self.values(2 * layer + 1, prefix, h, prefix_len), v))
                per_head.append(attention(q[i, h * g:(h + 1) * g].cpu(), k, v, self.io))
            rows.append([torch.cat([p[j] for p in per_head]) for j in range(4)])
        return [torch.stack([r[j] for r in rows]) for j in range(4)]


def within(got, want, bound, what=""):
    got = got.detach().cpu().double()
    far = (got - want).abs() - bound
    same = (got == want) | ((got - want).abs() <= bound)
    assert bool(same.all()), f"{what}: {int((~same).sum())} of {same.numel()} values out of bounds, worst excess {far[~same].max().item()}"
