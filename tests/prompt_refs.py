"""Plain references (fp64 and integers) of prompt attention over slabs and of the store of parked rows, and how the calls are
made on an operator_refs.SlabPool."""
import math

import torch

from operator_refs import SlabPool, lib, rounding, within

# ---- prompt attention ---------------------------------------------------------------------------


def causal(q, keys, values, dtype, seen, twice=False):
    """One KV head of one request: q [a, g, D], keys and values [N, D]; token j sees the first N - a + 1 + j keys.
    -> (out, lse, out bound, lse bound), fp64.

    The bounds are those of operator_refs.attention (scores (D + 4) 2^-24, weights 2^-21 for 2^x, sums
    (N + 64) 2^-24, a half step of bf16 where weights go through 16-bit operands, one rounding at the end), with 2^-18 for 2^x
    where weights go to the tensor cores (a polynomial good to 2.6e-6, and the argument's rounding); `twice`: weights that
    may be rounded again when a reference has risen within a step."""
    a, g, d = q.shape
    n = keys.shape[0]
    qd, k, v = q.double(), keys.double(), values.double()
    # rows that a token does not see may be anything
    k = torch.where(seen[:, None], k, torch.zeros_like(k))
    v = torch.where(seen[:, None], v, torch.zeros_like(v))
    s = torch.einsum("tgd,kd->tgk", qd, k) / math.sqrt(d)
    hidden = torch.arange(n)[None, None] > torch.arange(n - a, n)[:, None, None]
    s = s.masked_fill(hidden, -math.inf)
    slip = ((d + 4) * 2.0 ** -24 * torch.einsum("tgd,kd->tgk", qd.abs(), k.abs()) / math.sqrt(d)).masked_fill(hidden, 0.0).amax(-1)
    w = torch.softmax(s, -1)
    out, size = torch.einsum("tgk,kd->tgd", w, v), torch.einsum("tgk,kd->tgd", w, v.abs())
    sums = (n + 64) * 2.0 ** -24
    wide = dtype == torch.float32
    power = 2.0 ** -21 if wide else 2.0 ** -18
    rel = 2 * slip + power + sums + (0.0 if wide else 2.0 ** (-7 if twice else -8))
    lse = torch.logsumexp(s, -1)
    top = s.masked_fill(hidden, 0.0).abs().amax(-1)
    return out, lse, size * rel[..., None] + rounding(out, dtype), slip + power + sums + lse.abs() * 2.0 ** -22 + top * 2.0 ** -22


def append_new(s, tables, layer, new, scale=1.0):
    """Random rows for the step's tokens, through odma_append_kv."""
    total = sum(new)
    k, v = s.randn(max(1, total), s.kv_heads, s.head_dim, scale=scale), s.randn(max(1, total), s.kv_heads, s.head_dim)
    s.pool.append_kv(layer, tables, k.data_ptr(), v.data_ptr(), s.stream)
    return k, v


def prefill_reference(s, layer, q, reqs, ctx, new, twice=False):
    """fp64 results of q [tokens, q_heads, D] over the slabs: (out, lse, bounds)."""
    g = q.shape[1] // s.kv_heads
    q, rows, at = q.cpu(), [], 0
    for r, c, a in zip(reqs, ctx, new):
        if a == 0:
            continue
        heads = []
        for h in range(s.kv_heads):
            k, v = s.values(2 * layer, r, h, c + a), s.values(2 * layer + 1, r, h, c + a)
            heads.append(causal(q[at:at + a, h * g:(h + 1) * g], k, v, s.io, torch.ones(c + a, dtype=torch.bool), twice))
        rows.append([torch.cat([x[j] for x in heads], 1) for j in range(4)])
        at += a
    return [torch.cat([x[j] for x in rows]) for j in range(4)]


def call_prefill(s, layer, q, tables, spare=0, want_lse=True, workspace=None):
    """The call, with a workspace of NaN, canaries behind it and behind the results."""
    tokens, q_heads, d = q.shape
    nbytes = s.pool.prefill_workspace_bytes(q_heads, tables)
    assert nbytes > 0
    ws = workspace if workspace is not None else torch.full((nbytes + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.full((tokens + 1, q_heads, d), -77.0, dtype=s.io, device="cuda")
    lse = torch.full((tokens + 1, q_heads), -77.0, device="cuda")
    s.pool.prefill_attention(layer, q.data_ptr(), q_heads, tables, ws.data_ptr(), nbytes, out.data_ptr(), lse.data_ptr() if want_lse else 0,
                             s.stream)
    assert s.sync() == 0
    if workspace is None:
        assert (ws[nbytes:] == 0xFF).all()
    assert (out[tokens - spare:] == -77).all() and (lse[tokens - spare:] == -77).all()
    if not want_lse:
        assert (lse == -77).all()
    return out[:tokens - spare], lse[:tokens - spare]


def run_prefill(s, reqs, ctx, new, q_heads, layer=0, qscale=1.0, kscale=1.0, tables=None, repeat=1, want_lse=True, twice=False):
    t = tables or s.tables(reqs, new)
    append_new(s, t, layer, new, kscale)
    q = s.randn(sum(new), q_heads, s.head_dim, scale=qscale)
    got = [call_prefill(s, layer, q, t, want_lse=want_lse) for _ in range(repeat)]
    for o, l in got[1:]:
        assert torch.equal(o, got[0][0]) and torch.equal(l, got[0][1])
    out, lse, bound, lse_bound = prefill_reference(s, layer, q, reqs, ctx, new, twice)
    within(got[0][0], out, bound, "out")
    if want_lse:
        within(got[0][1], lse, lse_bound, "lse")
    return q, got[0]


def up16(x):
    return (x + 15) // 16 * 16


# ---- the store ------------------------------------------------------------------------------------

TOP = {"e4m3": 448.0, "int8": 127.0, "int4": 7.0}


def formats():
    odma = lib()
    return {"raw": odma.STORE_RAW, "e4m3": odma.STORE_E4M3, "int8": odma.STORE_INT8, "int4": odma.STORE_INT4}


def quantised(x, fmt, group):
    """x [..., D] fp32 -> (codes as the store holds them, uint8; scales fp32): the header's arithmetic, step by step in fp32."""
    y = x.float().unflatten(-1, (-1, group))
    top = y.abs().amax(-1)
    bad = ~torch.isfinite(y).all(-1)
    small = (top < 2.0 ** -100) & ~bad
    one = torch.ones((), dtype=torch.float32)
    scale = torch.where(small, torch.zeros(()), top / torch.full((), TOP[fmt]))
    inv = torch.where(small | bad, torch.zeros(()), one / scale)
    z = torch.where(bad[..., None], torch.zeros(()), y) * inv[..., None]
    scale = torch.where(bad, torch.full((), math.nan), scale)
    z = z.clamp(-TOP[fmt], TOP[fmt]).flatten(-2)
    if fmt == "e4m3":
        codes = z.to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        n = z.round().to(torch.int32)
        codes = (n & 255).to(torch.uint8) if fmt == "int8" else ((n[..., 0::2] & 15) | (n[..., 1::2] & 15) << 4).to(torch.uint8)
    return codes, scale


def restored(codes, scale, fmt, group):
    """Codes and scales -> fp32 values."""
    if fmt == "e4m3":
        x = codes.view(torch.float8_e4m3fn).float()
    elif fmt == "int8":
        x = codes.view(torch.int8).float()
    else:
        n = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).to(torch.int32)
        x = torch.where(n > 7, n - 16, n).float()
    return (x.unflatten(-1, (-1, group)) * scale[..., None]).flatten(-2)


def slab_rows(s, array, req, first, count):
    """The stored rows of a run of tokens: [count, kv_heads, D], on the host."""
    out = []
    for h in range(s.kv_heads):
        at = s.base[req] * s.kv_heads + h * s.caps[req] + first
        out.append(s.mem[array, at:at + count].cpu())
    return torch.stack(out, 1)


def row_values(s, rows, array):
    """Stored rows as the fp32 numbers they stand for."""
    if s.kind != "e4m3":
        return rows.float()
    return rows.view(torch.float8_e4m3fn).float() * torch.tensor((s.v_scale if array % 2 else s.k_scale)[array // 2], dtype=torch.float32)


class Store:
    """A store of NaN and canaries for `tokens` tokens of layers [layer, layer + n_layers)."""

    def __init__(self, s, fmt, group, layer, n_layers, tokens):
        self.fmt, self.group, self.arrays, self.tokens = fmt, group, range(2 * layer, 2 * (layer + n_layers)), tokens
        cb, sb = s.pool.kv_store_bytes(formats()[fmt], group, n_layers, tokens)
        self.codes = torch.full((cb + 32,), 0x7F, dtype=torch.uint8, device="cuda")
        self.scales = torch.full((sb // 4 + 8,), math.nan, device="cuda")
        self.cb, self.sb = cb, sb
        self.c = lib().KvStore(formats()[fmt], group, layer, n_layers, self.codes.data_ptr(), cb, self.scales.data_ptr() if sb else 0, sb)

    def parts(self, kv_heads):
        shape = (len(self.arrays), self.tokens, kv_heads)
        codes = self.codes[:self.cb].cpu().view(*shape, -1)
        scales = self.scales[:self.sb // 4].cpu().view(*shape, -1) if self.sb else None
        assert (self.codes[self.cb:] == 0x7F).all() and torch.isnan(self.scales[self.sb // 4:]).all()
        return codes, scales


def same_bits(a, b):
    """Equal, NaN equal to NaN."""
    if a.dtype.is_floating_point:
        return bool((((a == b) | (torch.isnan(a) & torch.isnan(b)))).all())
    return torch.equal(a, b)
