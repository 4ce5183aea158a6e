// The split of a step's causal attention over the blocks of one launch, worked out by every block for
// itself from the lengths in the step's table.  Included by .cu files only.
//
// Work is a list of tiles: request by request, KV head by KV head, `tile_tokens` new tokens at a time.
// Tile j of a request with c tokens before the step sees the keys up to its last token, in steps of
// STEP keys.  In units of 1 / STEP of a step it is charged c + tile_tokens * (j + 1) + start, so that
// the tiles before the j-th cost
//     F(j) = j (c + start) + tile_tokens j (j + 1) / 2
// and share s of S, which begins at cost s * ceil(total / S), is found by three searches in closed form.  A
// share that begins inside a tile cuts it: the pieces leave partial results and a second kernel merges them.
// A cut costs some steps too (its rows are written in 32 bits and read again), so when there are no more tiles than shares
// and the longest tile ends before an equal share and a cut would, every share takes a tile; and a cut closer than
// `min_piece` steps to an end of its tile moves to that end.
//
// Equal charges are not equal times: the SMs of one launch differ by a tenth (one prompt of 16,384 tokens: 2.22 M cycles on
// average, 2.47 M on the slowest), and a cut costs time on both its sides.  So, with up to 32 requests, blocks take whole tiles
// one by one from a common counter, requests with the longest slabs and their last tiles first, unless the tiles are so few
// and long that the last ones would end a tenth and a cut later than equal shares.  (In a row, prompts of
// 1,500 tokens: 36 us, by equal shares 41; of 16,384: 1,647 and 1,769; 4,096 tokens behind 16,000, three tiles a block and 12 left
// over: 1,003 and 919; 1,400 behind 30,000: 773 and 547.)  More requests keep equal shares: taking them 32 at a time made ragged
// batches faster (64 of them 93 -> 85 us), but single tokens slower (512 of them 106 -> 121, one 14.3 -> 15.4).
#pragma once

#include "device_utils.cuh"

namespace odma {
namespace dev {

struct alignas(16) PlanScratch {                // shared memory of one block
    int64_t sums[3][32];
    int64_t total_cost, total_tiles;
    int4 cut[2];                    // where its share begins and ends: {request, KV head, tile, step}; n: behind everything
    int32_t longest, wide_at;       // wide_at: see PrefillItem, of the first
    int32_t queued;                 // tiles are taken from the common counter (`cut` is behind everything)
};

__device__ __forceinline__ int prefill_tiles(int new_tokens, int tile_tokens) { return (new_tokens + tile_tokens - 1) / tile_tokens; }

// New tokens of request i, 0 where its words do not fit together (a refused request has length 0).
__device__ __forceinline__ int prefill_new(const PrefillParams& p, int i, int len) {
    const int add = __ldg(p.cu_new + i + 1) - __ldg(p.cu_new + i);
    return add > 0 && add <= len ? add : 0;
}

// The place of cost `x` inside one request: KV head, tile, step.  `whole`: tiles count, and not what they cost.  Called by a
// whole warp; returns false where the cut moves behind the request.
template <int STEP>
__device__ __forceinline__ bool prefill_place(const PrefillParams& p, bool whole, int64_t x, int len, int add, int4& c) {
    const int64_t OV = STEP / 8 * p.plan_start;
    const int lane = threadIdx.x & 31;
    const int ctx = len - add, nt = prefill_tiles(add, p.tile_tokens);
    auto tile_sum = [&](int64_t j) { return j * (ctx + OV) + static_cast<int64_t>(p.tile_tokens) * (j * (j + 1) / 2); };
    const int64_t head_cost = whole ? nt : tile_sum(nt);
    c.y = static_cast<int>(x / head_cost);
    const int64_t y = x - c.y * head_cost;
    c.w = 0;
    if (whole) {
        c.z = static_cast<int>(y);
        return true;
    }
    int a = 0, n = nt;                                   // the last tile in [a, a + n) with F(tile) <= y, 32 of them at a time
    while (n > 1) {
        const int by = (n + 31) / 32, j = a + lane * by;
        const int hit = __popc(__ballot_sync(0xFFFFFFFFu, lane * by < n && tile_sum(j) <= y)) - 1;
        n = min(by, n - hit * by);
        a += hit * by;
    }
    c.z = a;
    const int64_t before = tile_sum(a), tile_cost = tile_sum(a + 1) - before;
    const int steps = (ctx + min((a + 1) * p.tile_tokens, add) + STEP - 1) / STEP;
    int t = static_cast<int>((y - before) * steps / tile_cost);
    bool next = false;
    if (steps < 2 * p.min_piece) {
        next = 2 * t >= steps;
        t = 0;
    } else if (t < p.min_piece) {
        t = 0;
    } else if (t > steps - p.min_piece) {
        next = true;
    }
    c.w = next ? 0 : t;
    if (next && ++c.z == nt) {
        c.z = 0;
        if (++c.y == p.kv_heads) {
            c.y = 0;
            return false;
        }
    }
    return true;
}

// Finds where this block's share begins and ends.  `cum` and `lens` [n] and, for an 8-bit pool, `wide_of` [n] are scratch.
// Every thread of the block calls; a barrier is behind the last access.  Up to 32 requests the first two warps find a cut
// each by themselves, with nothing but shuffles (one request: 2,100 cycles instead of 3,900); more go through the scratch.
template <int STEP, int THREADS, bool QUEUE>
__device__ void prefill_plan(const PrefillParams& p, PlanScratch* s, int64_t* cum, int32_t* lens, int32_t* wide_of) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t OV = STEP / 8 * p.plan_start, CUT = STEP / 8 * p.plan_cut;
    const int64_t S = p.shares;
    auto tile_sum = [&](int64_t ctx, int64_t j) { return j * (ctx + OV) + static_cast<int64_t>(p.tile_tokens) * (j * (j + 1) / 2); };
    auto warp_scan = [&](int64_t v) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t x = __shfl_up_sync(0xFFFFFFFFu, v, o);
            if (lane >= o) v += x;
        }
        return v;
    };
    // a tile each, or shares of equal cost
    auto is_whole = [&](int64_t tiles, int64_t cost, int longest) {
        return tiles <= S && (static_cast<int64_t>(longest) * STEP + OV) * S <= cost + CUT * S;
    };
    auto share_cost = [&](bool whole, int64_t total) {
        if (whole) return int64_t(1);
        const int64_t share = (total + S - 1) / S, least = static_cast<int64_t>(p.min_piece) * STEP + OV;
        return share < least ? least : share;
    };
    const int mine = static_cast<int>(blockIdx.x) + warp;        // the cut that warps 0 and 1 look for
    auto set_cut = [&](const int4& c, int wide_at) {
        if (lane != 0) return;
        s->cut[warp] = c;
        if (warp == 0) s->wide_at = wide_at;
        if (warp == 0 || mine == p.shares) p.starts[mine] = c;
    };
    if (p.n <= 32) {
        if (warp < 2) {
            int len = 0, add = 0;
            if (lane < p.n) {
                len = __ldg(p.len + lane);
                add = prefill_new(p, lane, len);
            }
            const int nt = prefill_tiles(add, p.tile_tokens);
            const int64_t cost = tile_sum(len - add, nt) * p.kv_heads, tiles = static_cast<int64_t>(nt) * p.kv_heads;
            const int64_t cost_to = warp_scan(cost), tiles_to = warp_scan(tiles);
            const int longest = __reduce_max_sync(0xFFFFFFFFu, add > 0 ? (len + STEP - 1) / STEP : 0);
            const int64_t total_cost = __shfl_sync(0xFFFFFFFFu, cost_to, 31), total_tiles = __shfl_sync(0xFFFFFFFFu, tiles_to, 31);
            const bool whole = is_whole(total_tiles, total_cost, longest);
            const int64_t at = whole ? tiles_to - tiles : cost_to - cost, total = whole ? total_tiles : total_cost;
            const int64_t x = mine * share_cost(whole, total);
            int4 c = make_int4(p.n, 0, 0, 0);
            bool queued = false;
            if (QUEUE && p.queue && total_tiles > S) {
                // Tiles one by one: with more than k S of them above a (k + 1)-th of a time, some block takes k + 1 and longer than that.
                const float time = (1.1f * static_cast<float>(total_cost)) / static_cast<float>(S) + static_cast<float>(CUT);
                const float first = static_cast<float>(len - add + OV), per_tile = 1.f / static_cast<float>(p.tile_tokens);
                queued = true;
#pragma unroll 1
                for (int k = 0; k < 10; ++k) {
                    const float below = fminf(fmaxf((time / (k + 1) - first) * per_tile, 0.f), static_cast<float>(nt));
                    queued &= __reduce_add_sync(0xFFFFFFFFu, (nt - static_cast<int>(below)) * p.kv_heads) <= k * S;
                }
            }
            if (warp == 0 && lane == 0) s->queued = queued;
            if (!queued && x < total && mine != p.shares) {
                const uint32_t some = __ballot_sync(0xFFFFFFFFu, add > 0);
                // the last request with something to do whose cost before it is at most x
                const int r = 31 - __clz(__ballot_sync(0xFFFFFFFFu, at <= x) & some);
                c.x = r;
                if (!prefill_place<STEP>(p, whole, x - __shfl_sync(0xFFFFFFFFu, at, r), __shfl_sync(0xFFFFFFFFu, len, r), __shfl_sync(0xFFFFFFFFu, add, r), c)) {
                    const uint32_t behind = r == 31 ? 0u : some >> (r + 1);
                    c.x = behind ? r + __ffs(behind) : p.n;
                }
            }
            int wide_at = 0;
            if (p.wide) {
                const int64_t wide = add > 0 ? (len + 15) & ~15 : 0, wide_to = warp_scan(wide) - wide;
                wide_at = static_cast<int>(min(__shfl_sync(0xFFFFFFFFu, wide_to, min(c.x, 31)), p.wide_tokens));
            }
            set_cut(c, wide_at);
        }
        __syncthreads();
        return;
    }
    if (tid == 0) s->queued = 0;
    // a thread takes `per` requests in a row
    const int per = (p.n + THREADS - 1) / THREADS;
    int64_t cost = 0, tiles = 0, wide = 0;
    int longest = 0;
    for (int k = 0; k < per; ++k) {
        const int i = tid * per + k;
        if (i >= p.n) break;
        const int len = __ldg(p.len + i), add = prefill_new(p, i, len), nt = prefill_tiles(add, p.tile_tokens);
        cost += tile_sum(len - add, nt) * p.kv_heads;
        tiles += static_cast<int64_t>(nt) * p.kv_heads;
        if (add > 0) {
            wide += (len + 15) & ~15;
            longest = max(longest, (len + STEP - 1) / STEP);
        }
    }
    int64_t cost_to = warp_scan(cost), tiles_to = warp_scan(tiles), wide_to = warp_scan(wide);
    longest = __reduce_max_sync(0xFFFFFFFFu, longest);
    if (tid == 0) s->longest = 0;
    if (lane == 31) {
        s->sums[0][warp] = cost_to;
        s->sums[1][warp] = tiles_to;
        s->sums[2][warp] = wide_to;
    }
    __syncthreads();
    if (lane == 0) atomicMax(&s->longest, longest);
    if (warp == 0) {
        const bool in = lane < THREADS / 32;
        const int64_t a = warp_scan(in ? s->sums[0][lane] : 0), b = warp_scan(in ? s->sums[1][lane] : 0),
                      c = warp_scan(in ? s->sums[2][lane] : 0);
        if (in) {
            s->sums[0][lane] = a;
            s->sums[1][lane] = b;
            s->sums[2][lane] = c;
        }
        if (lane == 31) {
            s->total_cost = a;
            s->total_tiles = b;
        }
    }
    __syncthreads();
    if (warp > 0) {
        cost_to += s->sums[0][warp - 1];
        tiles_to += s->sums[1][warp - 1];
        wide_to += s->sums[2][warp - 1];
    }
    const int64_t total_cost = s->total_cost, total_tiles = s->total_tiles;
    const bool whole = is_whole(total_tiles, total_cost, s->longest);
    int64_t at = (whole ? tiles_to - tiles : cost_to - cost), wide_at = wide_to - wide;
    for (int k = 0; k < per; ++k) {
        const int i = tid * per + k;
        if (i >= p.n) break;
        const int len = __ldg(p.len + i), add = prefill_new(p, i, len), nt = prefill_tiles(add, p.tile_tokens);
        cum[i] = at;
        lens[i] = len;
        if (p.wide) {
            wide_of[i] = static_cast<int32_t>(min(wide_at, p.wide_tokens));
            if (add > 0) wide_at += (len + 15) & ~15;
        }
        at += whole ? static_cast<int64_t>(nt) * p.kv_heads : tile_sum(len - add, nt) * p.kv_heads;
    }
    __syncthreads();
    if (warp < 2) {
        const int64_t total = whole ? total_tiles : total_cost, x = mine * share_cost(whole, total);
        int4 c = make_int4(p.n, 0, 0, 0);
        if (x < total && mine != p.shares) {
            int lo = 0, hi = p.n;                       // the last request whose cost before it is at most x
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (cum[mid] <= x) lo = mid; else hi = mid;
            }
            c.x = lo;
            const int len = lens[lo];
            if (!prefill_place<STEP>(p, whole, x - cum[lo], len, prefill_new(p, lo, len), c))
                for (++c.x; c.x < p.n && prefill_new(p, c.x, lens[c.x]) == 0;) ++c.x;
        }
        set_cut(c, p.wide && c.x < p.n ? wide_of[c.x] : 0);
    }
    __syncthreads();
}

// One piece of work: steps [t0, t1) of a tile.
struct PrefillItem {
    int head;
    int tok0;               // first token of the tile among the request's new ones
    int add, ctx;           // new tokens and tokens before them
    int cu;                 // the request's first row of q
    int t0, t1;             // t1 = 0: no more items
    int slot;               // partial result, -1: the tile is whole
    int base, cap;
    int wide_at;            // 8-bit pools: the request's first token in the widened rows
};

// Walks the items of a share, or (QUEUE, and the plan says so) takes tiles from the common counter.  Called by one whole warp
// (or by every thread, which then reads the same words).
template <int STEP, bool QUEUE>
struct PrefillWalk {
    const PrefillParams& p;
    int4 at, end;
    int len, add, ctx, cu, base, cap, wide_at;
    // the counter's: lane r keeps the request with the r-th longest slab, and the tiles of all heads up to and with it
    bool queued;
    int request = 0, first_wide = 0, tiles_to = 0, taken = static_cast<int>(blockIdx.x);

    __device__ __forceinline__ PrefillWalk(const PrefillParams& params, const PlanScratch& s)
        : p(params), at(s.cut[0]), end(s.cut[1]), wide_at(s.wide_at), queued(QUEUE && s.queued) {
        if (at.x < p.n) fetch();
    }
    // One warp, before the first item, where `queued` is set.
    __device__ __forceinline__ void sort() {
        const int lane = threadIdx.x & 31;
        const int mine = lane < p.n ? __ldg(p.len + lane) : 0, fresh = lane < p.n ? prefill_new(p, lane, mine) : 0;
        auto sum_to = [&](auto v) {
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const auto x = __shfl_up_sync(0xFFFFFFFFu, v, o);
                if (lane >= o) v += x;
            }
            return v;
        };
        const int64_t wide = fresh > 0 ? (mine + 15) & ~15 : 0, before = sum_to(wide) - wide;
        first_wide = static_cast<int>(min(before, p.wide_tokens));
        const int key = fresh > 0 ? mine : -1;
        int rank = 0;
#pragma unroll 1
        for (int k = 0; k < 32; ++k) {
            const int other = __shfl_sync(0xFFFFFFFFu, key, k);
            rank += other > key || (other == key && k < lane);
        }
#pragma unroll 1
        for (int k = 0; k < 32; ++k)
            if (__shfl_sync(0xFFFFFFFFu, rank, k) == lane) request = k;
        first_wide = __shfl_sync(0xFFFFFFFFu, first_wide, request);
        tiles_to = sum_to(prefill_tiles(__shfl_sync(0xFFFFFFFFu, fresh, request), p.tile_tokens) * p.kv_heads);
    }
    // The next tile of the counter's: the first is the block's own number.
    __device__ __forceinline__ bool take() {
        if (taken < 0) {
            if ((threadIdx.x & 31) == 0) taken = p.shares + static_cast<int>(atomicAdd(p.queue, 1u));
            taken = __shfl_sync(0xFFFFFFFFu, taken, 0);
        }
        const uint32_t behind = __ballot_sync(0xFFFFFFFFu, tiles_to > taken);          // the first of these holds it
        if (behind == 0) return false;
        const int r = __ffs(behind) - 1, from = __shfl_sync(0xFFFFFFFFu, tiles_to, max(r - 1, 0));
        at.x = __shfl_sync(0xFFFFFFFFu, request, r);
        wide_at = __shfl_sync(0xFFFFFFFFu, first_wide, r);
        fetch();
        const int y = taken - (r > 0 ? from : 0), tile = y / p.kv_heads;
        at.y = y - tile * p.kv_heads;
        at.z = prefill_tiles(add, p.tile_tokens) - 1 - tile;
        at.w = 0;
        return true;
    }
    __device__ __forceinline__ void fetch() {
        len = __ldg(p.len + at.x);
        add = prefill_new(p, at.x, len);
        ctx = len - add;
        cu = __ldg(p.cu_new + at.x);
        base = __ldg(p.base + at.x);
        cap = __ldg(p.cap + at.x);
    }
    __device__ __forceinline__ bool next(PrefillItem& it) {
        if (QUEUE && queued && !take()) return false;
        if (at.x >= p.n || (at.x == end.x && at.y == end.y && at.z == end.z && at.w == end.w)) return false;
        const bool last = at.x == end.x && at.y == end.y && at.z == end.z;      // the share ends inside this tile
        const int tok0 = at.z * p.tile_tokens;
        const int steps = (ctx + min(tok0 + p.tile_tokens, add) + STEP - 1) / STEP;
        it.head = at.y;
        it.tok0 = tok0;
        it.add = add;
        it.ctx = ctx;
        it.cu = cu;
        it.t0 = at.w;
        it.t1 = last ? end.w : steps;
        it.slot = at.w > 0 ? 2 * static_cast<int>(blockIdx.x) : last ? 2 * static_cast<int>(blockIdx.x) + 1 : -1;
        it.base = base;
        it.cap = cap;
        it.wide_at = wide_at;
        if (QUEUE && queued) {
            taken = -1;
        } else if (last) {
            at = end;
        } else {
            at.w = 0;
            if ((at.z + 1) * p.tile_tokens < add) {
                ++at.z;
            } else {
                at.z = 0;
                if (++at.y == p.kv_heads) {
                    at.y = 0;
                    wide_at += (len + 15) & ~15;
                    for (++at.x; at.x < p.n; ++at.x) {
                        fetch();
                        if (add > 0) break;
                    }
                }
            }
        }
        return true;
    }
};

}  // namespace dev
}  // namespace odma
