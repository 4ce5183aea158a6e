// The per-step table of a batch, its slot map and its positions, built on the GPU from lengths that
// live there (odma_build_tables_device).
//
// The batch's streams (request, KV head) that hold a token are lined up in order; a stream of t
// tiles of 64 tokens costs t + 1.  Share c of `ctas` begins at cost x_c = c * C, with C the average
// cost rounded up.  A cut that falls within kMinPieceTiles tiles of an end of its stream moves to
// that end.  Everything then follows in closed form: with (q_c, t_c) the stream and tile where share
// c begins,
//     item_begin(c) = q_c + #{c' <= c : t_c' > 0}                (one piece per stream start or inner cut)
//     combine record of the stream that cut c splits = #{first inner cuts of a stream up to c} - 1
// and share c's pieces are streams q_c .. q_{c+1}, whole but for its first and last.
//
// What bounds it is latency (a batch of 1,024 requests writes 190 KB): one launch of a cluster of
// eight CTAs, each of which redoes the two block-wide sums over the requests (a few KB from L2) and
// the binary searches of the cuts (shared memory) and then writes its part of the table, a thread per
// item, so nothing is exchanged between CTAs (one CTA for all: 11.6 us for one request, 26 us for 1,024;
// eight: 7.1 and 9.9).  The cluster barrier orders the last read of the lengths before their
// update, which may be in place.
#include "device_utils.cuh"
#include "planner.hpp"

namespace odma {
namespace {

constexpr int kThreads = 512;
constexpr int kCluster = 8;
constexpr int kPerThread = kMaxDeviceBatch / kThreads;

// Inclusive sum over the block of one 64-bit value per thread; `total` to every thread.
__device__ __forceinline__ int64_t block_sum(int64_t v, int64_t* warp_sums, int64_t& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t x = __shfl_up_sync(0xFFFFFFFFu, v, o);
        if (lane >= o) v += x;
    }
    __syncthreads();                                   // the previous call's readers are done
    if (lane == 31) warp_sums[warp] = v;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        const int64_t x = warp_sums[w];
        if (w < warp) before += x;
        total += x;
    }
    return before + v;
}

// Index of the first element of the ascending a[0, n) that is greater than x.
template <typename A, typename X>
__device__ __forceinline__ int upper_bound(const A* a, int n, X x) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (static_cast<X>(a[mid]) > x) hi = mid; else lo = mid + 1;
    }
    return lo;
}

__global__ void __launch_bounds__(kThreads) __cluster_dims__(kCluster, 1, 1) build_tables_kernel(const DeviceTablesParams p) {
    extern __shared__ int64_t smem[];
    __shared__ int64_t warp_sums[kThreads / 32];
    const int n = p.n, hkv = p.kv_heads, ctas = p.n_ctas;
    // over the requests that hold a token ("held", in order): cost of all heads before each, request, length
    int64_t* cost_before = smem;                                        // [n]
    int32_t* held_req = reinterpret_cast<int32_t*>(cost_before + n);    // [n]
    int32_t* held_len = held_req + n;                                   // [n]
    int32_t* held_base = held_len + n;                                  // [n]
    int32_t* held_cap = held_base + n;                                  // [n]
    // over all requests: first new token, committed length (-1: refused)
    int32_t* cu = held_cap + n;                                         // [n + 1]
    int32_t* len0 = cu + n + 1;                                         // [n]
    // over the shares' starts
    int32_t* cut_q = len0 + n;                                          // [ctas + 1] stream
    int32_t* cut_t = cut_q + ctas + 1;                                  // [ctas + 1] tile
    int32_t* begin = cut_t + ctas + 1;                                  // [ctas + 1] first item
    int32_t* firsts = begin + ctas + 1;                                 // [ctas + 1] streams cut so far
    const int tid = threadIdx.x;
    const int rank = blockIdx.x % kCluster;
    const int all = kCluster * kThreads, me = rank * kThreads + tid;    // thread of the cluster

    // ---- the requests: thread t of the block takes requests t*per .. t*per + per - 1
    const int per = (n + kThreads - 1) / kThreads;
    int base[kPerThread], cap[kPerThread], len[kPerThread], add[kPerThread];
    int64_t mine = 0;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
        const int i = tid * per + k;
        base[k] = cap[k] = len[k] = add[k] = 0;
        if (k < per && i < n) {
            const int2 s = __ldg(reinterpret_cast<const int2*>(p.slabs) + i);
            base[k] = s.x;
            cap[k] = s.y;
            len[k] = p.len[i];
            add[k] = p.n_new ? p.n_new[i] : 1;
            if (add[k] >= 0 && add[k] <= p.n_new_total) mine += add[k];
        }
    }
    int64_t total;
    int64_t at = block_sum(mine, warp_sums, total) - mine;
    int64_t cost = 0, held = 0;
    bool bad = false;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
        const int i = tid * per + k;
        if (k >= per || i >= n) continue;
        const bool counted = add[k] >= 0 && add[k] <= p.n_new_total;
        const bool ok = counted && base[k] >= 0 && (base[k] & 15) == 0 && cap[k] >= 0 &&
                        static_cast<int64_t>(base[k]) + cap[k] <= p.tokens && len[k] >= 0 &&
                        static_cast<int64_t>(len[k]) + add[k] <= cap[k] && at + add[k] <= p.n_new_total;
        cu[i] = static_cast<int32_t>(min(at, static_cast<int64_t>(p.n_new_total)));
        if (counted) at += add[k];
        if (i == n - 1) cu[n] = static_cast<int32_t>(min(at, static_cast<int64_t>(p.n_new_total)));
        len0[i] = ok ? len[k] : -1;
        const int after = ok ? len[k] + add[k] : 0;
        bad = bad || !ok;
        if (after > 0) {
            cost += (after + kTileTokens - 1) / kTileTokens + 1;
            held += 1;
        }
        if ((i & (kCluster - 1)) == rank) {
            p.table[p.off_base + i] = ok ? base[k] : 0;
            p.table[p.off_cap + i] = ok ? cap[k] : 0;
            p.table[p.off_len + i] = after;
        }
        add[k] = after;                                // from here on: the length after the step
    }
    // one sum for both counts: held requests above bit 48 (n <= 4096), cost below (< 2^40)
    int64_t both;
    int64_t pre = block_sum((held << 48) | cost, warp_sums, both) - ((held << 48) | cost);
    const int n_held = static_cast<int>(both >> 48);
    const int64_t req_cost = both & ((int64_t(1) << 48) - 1);
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
        if (k >= per || tid * per + k >= n || add[k] <= 0) continue;
        const int r = static_cast<int>(pre >> 48);
        held_req[r] = tid * per + k;
        held_len[r] = add[k];
        held_base[r] = base[k];
        held_cap[r] = cap[k];
        cost_before[r] = (pre & ((int64_t(1) << 48) - 1)) * hkv;
        pre += (int64_t(1) << 48) + (add[k] + kTileTokens - 1) / kTileTokens + 1;
    }
    if (rank == 0 && bad) atomicOr(p.status, kStatusOverflow);
    __syncthreads();

    // ---- the shares' starts
    const int streams = n_held * hkv;
    const int64_t work = req_cost * hkv;
    // (both below 2^41, so the rounded quotient's floor is the quotient's)
    const int64_t share = max(static_cast<int64_t>(static_cast<double>(work + ctas - 1) / ctas), static_cast<int64_t>(kMinShareTiles));
    int64_t sums = 0;                                  // of this thread's starts: inner cuts (low), first ones (high)
    const int cper = (ctas + 1 + kThreads - 1) / kThreads;
    for (int c = tid * cper; c < min((tid + 1) * cper, ctas + 1); ++c) {
        const int64_t x = c * share;
        int q = streams, t = 0;
        if (x < work && c < ctas) {
            const int r = upper_bound(cost_before, n_held, x) - 1;
            const int of = (held_len[r] + kTileTokens - 1) / kTileTokens;
            const int64_t in = x - cost_before[r];     // < kv_heads * (of + 1)
            const int h = in < (int64_t(1) << 32) ? static_cast<int>(static_cast<uint32_t>(in) / static_cast<uint32_t>(of + 1))
                                                  : static_cast<int>(in / (of + 1));
            const int u = static_cast<int>(in - static_cast<int64_t>(h) * (of + 1));
            q = r * hkv + h;
            t = u - 1;
            if (of < 2 * kMinPieceTiles) {             // never cut: to the nearer end
                q += 2 * u <= of ? 0 : 1;
                t = 0;
            } else if (t < kMinPieceTiles) {
                t = 0;
            } else if (t > of - kMinPieceTiles) {
                q += 1;
                t = 0;
            }
        }
        cut_q[c] = q;
        cut_t[c] = t;
    }
    __syncthreads();
    for (int c = tid * cper; c < min((tid + 1) * cper, ctas + 1); ++c)
        if (cut_t[c] > 0) sums += 1 + ((c == 0 || cut_t[c - 1] == 0 || cut_q[c - 1] != cut_q[c]) ? int64_t(1) << 32 : 0);
    int64_t cuts;
    int64_t run = block_sum(sums, warp_sums, cuts) - sums;
    for (int c = tid * cper; c < min((tid + 1) * cper, ctas + 1); ++c) {
        if (cut_t[c] > 0) run += 1 + ((c == 0 || cut_t[c - 1] == 0 || cut_q[c - 1] != cut_q[c]) ? int64_t(1) << 32 : 0);
        begin[c] = cut_q[c] + static_cast<int32_t>(run & 0xFFFFFFFF);
        firsts[c] = static_cast<int32_t>(run >> 32);
    }
    __syncthreads();

    // ---- items, a thread each
    const int n_items = begin[ctas], n_comb = firsts[ctas];
    int4* items = reinterpret_cast<int4*>(p.table + p.off_items);
    int4* recs = reinterpret_cast<int4*>(p.table + p.off_cta);
    for (int i = me; i < p.n_items; i += all) {
        if (i >= n_items) {                            // what no piece fills
            items[2 * i] = make_int4(-1, 0, 0, 0);
            items[2 * i + 1] = make_int4(0, 0, 0, -1);
            continue;
        }
        const int c = upper_bound(begin, ctas + 1, i) - 1;          // the share that begins with this piece or before it
        const int q0 = cut_q[c], t0 = cut_t[c], q1 = cut_q[c + 1], t1 = cut_t[c + 1];
        const int b = begin[c], m = q1 - q0 + (t1 > 0 ? 1 : 0), j = i - b;
        const bool lead = t0 > 0 || (q0 == q1 && t1 > 0), tail = m > 1 && t1 > 0;
        const int q = q0 + j, r = q / hkv, h = q - r * hkv;
        const int L = held_len[r], of = (L + kTileTokens - 1) / kTileTokens;
        const int start = j == 0 ? t0 : 0, stop = j == m - 1 && t1 > 0 ? t1 : of;
        const bool split = start > 0 || stop < of;
        const int tok0 = start * kTileTokens;
        const int comb = !split ? -1 : (start > 0 ? firsts[c] : firsts[c + 1]) - 1;
        const int4 lo = make_int4(held_req[r], h, tok0, min(stop * kTileTokens, L) - tok0);
        const int4 hi = make_int4((split ? 0 : 1) | (stop == of ? 2 : 0), i, held_base[r] * hkv + h * held_cap[r] + tok0, comb);
        // the share's pieces of split streams come first
        const int place = j == 0 && lead ? 0 : (j == m - 1 && tail ? (lead ? 1 : 0) : j + (tail ? 1 : 0));
        items[2 * (b + place)] = lo;
        items[2 * (b + place) + 1] = hi;
        if (place == 0) {
            recs[3 * c + 1] = lo;
            recs[3 * c + 2] = hi;
        }
    }
    // ---- CTA records and combine records, a thread per share
    for (int c = me; c < ctas; c += all) {
        recs[3 * c] = make_int4(begin[c], begin[c + 1], 0, 0);
        if (begin[c] == begin[c + 1]) recs[3 * c + 1] = recs[3 * c + 2] = make_int4(0, 0, 0, 0);
        const int q = cut_q[c];
        if (cut_t[c] > 0 && (cut_t[c - 1] == 0 || cut_q[c - 1] != q)) {      // the first cut of stream q
            const int last = upper_bound(cut_q, ctas + 1, q);               // cuts c .. last - 1 lie inside it
            const int r = q / hkv;
            reinterpret_cast<int4*>(p.table + p.off_combine)[firsts[c] - 1] = make_int4(held_req[r], q - r * hkv, begin[c] - 1, 1 + last - c);
        }
    }
    for (int i = n_comb + me; i < p.n_combine; i += all)
        reinterpret_cast<int4*>(p.table + p.off_combine)[i] = make_int4(0, 0, 0, 0);
    for (int i = me; i <= n; i += all) p.table[p.off_cu_new + i] = cu[i];
    for (int i = n + me; i < p.off_cap - p.off_base; i += all)
        p.table[p.off_base + i] = p.table[p.off_cap + i] = p.table[p.off_len + i] = 0;
    for (int i = n + 1 + me; i < p.off_cta - p.off_cu_new; i += all) p.table[p.off_cu_new + i] = 0;
    // ---- the new tokens
    if (p.slots || p.positions)
        for (int tok = me; tok < p.n_new_total; tok += all) {
            int slot = -1, pos = -1;
            if (tok < cu[n]) {
                const int r = upper_bound(cu, n + 1, tok) - 1;
                if (len0[r] >= 0) {
                    pos = len0[r] + tok - cu[r];
                    slot = __ldg(p.slabs + 2 * r) * hkv + pos;
                }
            }
            if (p.slots) p.slots[tok] = slot;
            if (p.positions) p.positions[tok] = pos;
        }
    // ---- the lengths after the step: every CTA of the cluster has read the old ones by now
    if (p.len_next) {
        __syncwarp();
        asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) {
            const int i = tid * per + k;
            if (k < per && i < n && (i & (kCluster - 1)) == rank) p.len_next[i] = len0[i] >= 0 ? add[k] : len[k];
        }
    }
}

int smem_bytes(int n, int ctas) { return 8 * n + 4 * (6 * n + 1) + 4 * 4 * (ctas + 1); }

}  // namespace

cudaError_t launch_build_tables(const DeviceTablesParams& p, cudaStream_t stream) {
    static bool configured[64] = {false};              // the opt-in to large shared memory is per device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!configured[dev]) {
        e = cudaFuncSetAttribute(build_tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 smem_bytes(kMaxDeviceBatch, kMaxDeviceCtas));
        if (e != cudaSuccess) return e;
        configured[dev] = true;
    }
    build_tables_kernel<<<kCluster, kThreads, smem_bytes(p.n, p.n_ctas), stream>>>(p);
    return cudaGetLastError();
}

}  // namespace odma
