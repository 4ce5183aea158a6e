// The prefix part of attention behind a shared prefix on the fifth-generation tensor cores (bf16 rows,
// head_dim 64 or 128; 8-bit prefixes come here as bf16).  See prefix.cu for the operator.
//
// A block takes one KV head, one split of the prefix's keys and up to 256 query rows (row = request,
// query head of the group).  With rows on the M side and 128 keys per tile
//     S[128 x 128] = Q[128 x D] . K[128 x D]^T        Q, K from shared memory, K-major
//     O[128 x D]  += P[128 x 128] . V[128 x D]        P from tensor memory, V MN-major
// with S, P and O in tensor memory: S takes 128 columns, P (bf16) overwrites its first 64 once S has
// been read, O takes D more.  Two such sets ("lanes") share the SM's tensor pipe: while one lane's
// softmax runs, the other's products do.  More than 128 rows: the lanes hold two row tiles and use
// every K and V tile twice; otherwise both hold the same rows and take the tiles in turn, each with
// a partial result of its own.
//
// Warps 0-7 and 8-15: softmax of lane 0 and 1, two threads per row, 64 keys each (no shuffles; with one
// thread per row a scheduler has one warp of the lane and waits out every instruction's latency:
// 4,200 cycles per pair of tiles against PAIR_CYCLES); warp 16: TMA producer; warp 17: issues all products, in the
// order PV0(j) QK0(j+1) PV1(j) QK1(j+1), so S of a lane is only overwritten by a product issued after the
// one that reads its P, and a full S tells that the lane's O is complete up to the tile before.
//
// The softmax keeps a reference m per row, raised only when a tile's maximum passes it by 2^8: P stays
// below 256, which bf16 relative to the fp32 accumulator does not mind, and O is rescaled in tensor
// memory only then.  P is rounded to bf16 for the product (half a step: 2^-9 to 2^-8 of a weight, random
// in sign over the keys); sums, maxima and O are fp32.
#include "odma.h"
#include "tcgen05.cuh"

namespace odma {
namespace {

using namespace dev;

constexpr int kTile = kPrefixTile;                  // keys per tile
constexpr int kM = 128;                             // rows per lane
constexpr int kSoftmaxWarps = 16;                   // four warpgroups: lane 0 and 1, left and right 64 keys
constexpr int kThreads = (kSoftmaxWarps + 2) * 32;
constexpr int kProducerWarp = kSoftmaxWarps, kMmaWarp = kSoftmaxWarps + 1;
constexpr int kLaneThreads = kSoftmaxWarps * 16;    // softmax threads of a lane
constexpr int kMaxStages = 8;
constexpr float kRescaleAbove = 8.f;
constexpr int kHalfBytes = kTile * 128;             // 64 elements of 128 rows
// barriers
constexpr int kBarFull = 0, kBarEmpty = kMaxStages, kBarQ = 2 * kMaxStages, kBarS = kBarQ + 2, kBarP = kBarS + 2,
              kBarO = kBarP + 2, kBarDrain = kBarO + 2, kNumBars = kBarDrain + 1;

template <int D>
struct Config {
    static constexpr int kHalves = D / 64;
    static constexpr int kTileBytes = kHalves * kHalfBytes;      // of K, of V, and of a lane's Q
    static constexpr int kStages = D == 128 ? 5 : 8;
    static constexpr int kSmem = (2 + kStages) * kTileBytes + 2 * kM * 4 + kNumBars * 8 + 64 + 1024;
};

// D[tmem] (+)= A[tmem] . B[smem]
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%5, %5, %5, %5}, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b), "r"(idesc), "r"(accumulate), "r"(0u)
        : "memory");
}

// 16 columns of the thread's own row (tensor-memory lane = 32 * (warp mod 4) + lane); stores of 16 and of 8.
__device__ __forceinline__ void tmem_ld_row16(uint32_t addr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_st_row16(uint32_t addr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}

__device__ __forceinline__ void tmem_st_row8(uint32_t addr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(addr), "r"(r[0]), "r"(r[1]),
                 "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 fma2(const float2& a, const float2& b, const float2& c) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, z, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
        "fma.rn.f32x2 w, x, y, z;\n\tmov.b64 {%0, %1}, w;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(const float2& a, const float2& b) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
        "add.rn.f32x2 w, x, y;\n\tmov.b64 {%0, %1}, w;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}

constexpr int kCols = kTile / 2;                    // scores per softmax thread

__device__ __forceinline__ float row_max(const uint32_t (&s)[kCols]) {
    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int i = 0; i < kCols; i += 8)
#pragma unroll
        for (int k = 0; k < 4; ++k) mx[k] = fmaxf(fmaxf(mx[k], __uint_as_float(s[i + 2 * k])), __uint_as_float(s[i + 2 * k + 1]));
    return fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
}

// The thread's weights 2^(s * scale - m), rounded to bf16, to tensor memory; their sum (unrounded).
__device__ __forceinline__ float row_weights(const uint32_t (&s)[kCols], float scale, float m, uint32_t t_p) {
    const float ref = m == -INFINITY ? 0.f : m;     // every score so far is -inf: weights 0, not NaN
    const float2 sc = make_float2(scale, scale), neg = make_float2(-ref, -ref);
    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
    for (int c = 0; c < kCols / 16; ++c) {
        uint32_t pk[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float2 x = fma2(make_float2(__uint_as_float(s[16 * c + 2 * i]), __uint_as_float(s[16 * c + 2 * i + 1])), sc, neg);
            x = make_float2(fast_exp2(x.x), fast_exp2(x.y));
            sum[i & 1] = add2(sum[i & 1], x);
            pk[i] = pack_bf16(x.x, x.y);
        }
        tmem_st_row8(t_p + 8u * c, pk);
    }
    return (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
}

// Barrier over `threads` threads; the second form tells whether any of them says yes.  Every thread of a lane
// comes to every one of its barriers, also after a wait has given up.
__device__ __forceinline__ void lane_sync(int id, int threads) {
    asm volatile("barrier.cta.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
__device__ __forceinline__ bool lane_any(int id, int threads, bool yes) {
    uint32_t any;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, %3, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
        : "=r"(any)
        : "r"(static_cast<uint32_t>(yes)), "r"(id), "r"(threads)
        : "memory");
    return any != 0;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
prefix_umma_kernel(const __grid_constant__ CUtensorMap map, const PrefixParams p) {
    using Cfg = Config<D>;
    constexpr int STAGES = Cfg::kStages;
    constexpr uint32_t IDESC_QK = umma_idesc(kM, kTile, false), IDESC_PV = umma_idesc(kM, D, true);
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    uint8_t* qbuf = smem;
    uint8_t* kv = qbuf + 2 * Cfg::kTileBytes;
    float* xch = reinterpret_cast<float*>(kv + STAGES * Cfg::kTileBytes);    // [lane][row], between a row's two threads
    uint64_t* bars = reinterpret_cast<uint64_t*>(xch + 2 * kM);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + kNumBars);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(const_cast<int*>(abort_flag) + 1);
    const uint32_t bar0 = smem_u32(bars);
    auto bar = [&](int i) { return bar0 + 8u * static_cast<uint32_t>(i); };
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int64_t limit = p.wait_limit_ns;

    // the block's work
    const int head = blockIdx.y;
    const int rows = p.n * p.group, r0 = blockIdx.x * 2 * kM;
    const bool in_turn = p.in_turn != 0;             // both lanes on the same rows, tiles in turn
    const bool lane1 = in_turn || r0 + kM < rows;    // is there a second lane?
    const int blocks = in_turn ? p.splits >> 1 : p.splits;      // splits of the keys over the blocks
    const int all_tiles = (p.len + kTile - 1) / kTile;
    const int t0 = static_cast<int>(static_cast<int64_t>(all_tiles) * blockIdx.z / blocks);
    const int t1 = static_cast<int>(static_cast<int64_t>(all_tiles) * (blockIdx.z + 1) / blocks);
    const int tiles = t1 - t0;
    const int ahead = in_turn ? 2 : 1;               // K tiles requested before the first V tile

    if (tid < kNumBars) {
        const bool many = (tid >= kBarQ && tid < kBarS) || (tid >= kBarP && tid < kBarO);   // a lane's threads
        mbar_init(bar(tid), many ? static_cast<uint32_t>(kLaneThreads) : 1u);
    }
    if (tid == 0) {
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const uint32_t kv_u32 = smem_u32(kv), q_u32 = smem_u32(qbuf);
    bool ok = true;
    if (warp == kProducerWarp) {
        // ------------------------------------------------------------------ producer
        // Ring order: the first `ahead` K tiles, then V(j), K(j + ahead) for each j.
        if (lane == 0) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map)) : "memory");
        uint32_t issued = 0;
        auto load = [&](bool is_v, int t) {
            const uint32_t stage = issued % STAGES, use = issued / STAGES;
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarEmpty + stage), (use & 1u) ^ 1u, abort_flag, p.status, limit));
            if (!ok) return;
            // a tile is two boxes of 64 rows per 128-byte column block; the prefix's last tile may need one only
            const int boxes = p.len - (t0 + t) * kTile > 64 ? 2 : 1;
            if (lane == 0) mbar_expect_tx(bar(kBarFull + stage), static_cast<uint32_t>(boxes * Cfg::kHalves) * 8192u);
            __syncwarp();
            const int h = lane >> 1, b = lane & 1;
            if (h < Cfg::kHalves && b < boxes)
                tma_load_2d(kv_u32 + stage * Cfg::kTileBytes + h * kHalfBytes + b * 8192, &map, h * 64,
                            static_cast<int32_t>((is_v ? p.v_row0 : p.k_row0) + head * p.head_rows + (t0 + t) * kTile + b * 64),
                            bar(kBarFull + stage));
            ++issued;
        };
        for (int t = 0; t < min(ahead, tiles) && ok; ++t) load(false, t);
        for (int t = 0; t < tiles && ok; ++t) {
            load(true, t);
            if (ok && t + ahead < tiles) load(false, t + ahead);
        }
        if (lane == 0 && (!ok || *abort_flag)) {
            // something timed out: wait (bounded) for the loads in flight before shared memory is given up
            for (uint32_t i = issued > STAGES ? issued - STAGES : 0; i < issued; ++i)
                mbar_wait_slow(bar(kBarFull + i % STAGES), (i / STAGES) & 1u, nullptr, p.status, limit / 4 + 1);
        }
    } else if (warp == kMmaWarp) {
        // ------------------------------------------------------------------ products
        uint32_t elected;
        asm volatile("{\n\t.reg .pred P;\n\telect.sync _|P, 0xFFFFFFFF;\n\tselp.b32 %0, 1, 0, P;\n\t}" : "=r"(elected));
        uint32_t used = 0;                           // ring position
        auto wait_tile = [&]() {                     // the next tile of the ring; its stage
            const uint32_t stage = used % STAGES;
            ok = ok && __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarFull + stage), (used / STAGES) & 1u, abort_flag, p.status, limit));
            tc_fence_after();
            ++used;
            return stage;
        };
        auto wait_bar = [&](int b, uint32_t parity) {
            ok = ok && __all_sync(0xFFFFFFFFu, mbar_wait_spin(bar(b), parity, abort_flag, p.status, limit));
            tc_fence_after();
        };
        auto first = [&](int L, uint32_t stage) {    // S of lane L from the K tile in `stage`
            const uint32_t qb = q_u32 + (in_turn ? 0u : static_cast<uint32_t>(L) * Cfg::kTileBytes), kb = kv_u32 + stage * Cfg::kTileBytes;
            if (ok && elected) {
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                    umma<false>(tmem + static_cast<uint32_t>(L) * 256u, smem_desc(qb + (ks >> 2) * kHalfBytes + (ks & 3) * 32, 16, 1024),
                                smem_desc(kb + (ks >> 2) * kHalfBytes + (ks & 3) * 32, 16, 1024), IDESC_QK, ks > 0 ? 1u : 0u);
                umma_commit(bar(kBarS + L));
            }
            __syncwarp();
        };
        auto second = [&](int L, int t, uint32_t stage, bool start, bool last) {     // O of lane L += P V
            const uint32_t base = tmem + static_cast<uint32_t>(L) * 256u, vb = kv_u32 + stage * Cfg::kTileBytes;
            const int keys = min(kTile, p.len - (t0 + t) * kTile), steps = (keys + 15) >> 4;
            if (ok && elected) {
                for (int ks = 0; ks < steps; ++ks)
                    umma_ts(base + 128u, base + static_cast<uint32_t>(ks) * 8u, smem_desc(vb + ks * 2048, kHalfBytes, 1024), IDESC_PV,
                            (start && ks == 0) ? 0u : 1u);
                if (last) umma_commit(bar(kBarO + L));
            }
            __syncwarp();
        };
        auto release = [&](uint32_t stage) {
            if (ok && elected) umma_commit(bar(kBarEmpty + stage));
            __syncwarp();
        };
        // value rows between the prefix's end and the next multiple of 16: whatever the slab holds there,
        // and 0 times a NaN would not be 0
        auto clear_tail = [&](int t, uint32_t stage) {
            const int keys = min(kTile, p.len - (t0 + t) * kTile), end = (keys + 15) & ~15;
            if (keys == end || !ok) return;
            uint8_t* vb = kv + stage * Cfg::kTileBytes;
            for (int i = lane; i < (end - keys) * 8 * Cfg::kHalves; i += 32) {
                const int row = keys + i / (8 * Cfg::kHalves), c = i % (8 * Cfg::kHalves);
                *reinterpret_cast<uint4*>(vb + (c >> 3) * kHalfBytes + row * 128 + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            fence_proxy_async();
            __syncwarp();
        };
        wait_bar(kBarQ, 0);
        if (!in_turn) {
            if (lane1) wait_bar(kBarQ + 1, 0);
            uint32_t ks = wait_tile();
            first(0, ks);
            if (lane1) first(1, ks);
            release(ks);
            for (int t = 0; t < tiles && ok; ++t) {
                const bool last = t + 1 == tiles;
                const uint32_t vs = wait_tile();
                clear_tail(t, vs);
                wait_bar(kBarP, t & 1u);
                second(0, t, vs, t == 0, last);
                if (!last) {
                    ks = wait_tile();
                    first(0, ks);
                }
                if (lane1) {
                    wait_bar(kBarP + 1, t & 1u);
                    second(1, t, vs, t == 0, last);
                }
                release(vs);
                if (!last) {
                    if (lane1) first(1, ks);
                    release(ks);
                }
            }
        } else {
            for (int t = 0; t < min(2, tiles) && ok; ++t) {
                const uint32_t ks = wait_tile();
                first(t, ks);
                release(ks);
            }
            for (int t = 0; t < tiles && ok; ++t) {
                const int L = t & 1;
                const uint32_t vs = wait_tile();
                clear_tail(t, vs);
                wait_bar(kBarP + L, static_cast<uint32_t>(t >> 1) & 1u);
                second(L, t, vs, t < 2, t + 2 >= tiles);
                release(vs);
                if (t + 2 < tiles) {
                    const uint32_t ks = wait_tile();
                    first(L, ks);
                    release(ks);
                }
            }
        }
        // nothing may still be running when tensor memory is given back
        if (elected) umma_commit(bar(kBarDrain));
        __syncwarp();
        mbar_wait_slow(bar(kBarDrain), 0, nullptr, p.status, limit / 4 + 1);
    } else {
        // ------------------------------------------------------------------ softmax
        const int L = warp >> 3, side = (warp >> 2) & 1;     // lane; left or right 64 keys of a tile
        const int row = (warp & 3) * 32 + lane;      // of the lane's tile
        const int g_row = r0 + (in_turn ? 0 : L * kM) + row;
        const int sync_id = 1 + L;
        auto out_row = [&](int r) { return static_cast<int64_t>(r / p.group) * p.q_heads + head * p.group + r % p.group; };
        if (L == 0 || (lane1 && !in_turn)) {
            // queries to shared memory in the swizzled order; rows behind the last are zero
            constexpr int CH = D / 8;                // 16-byte chunks per row
            constexpr int RSTEP = kLaneThreads / CH;
            const uint4* q = static_cast<const uint4*>(p.q);
            uint8_t* dst = qbuf + L * Cfg::kTileBytes;
            uint4 v[kM / RSTEP];
            const int c = tid % CH, rr = (tid & (kLaneThreads - 1)) / CH;       // chunk, first of the thread's rows
#pragma unroll
            for (int i = 0; i < kM / RSTEP; ++i) {   // all loads before the first store
                const int g = r0 + L * kM + rr + i * RSTEP;
                v[i] = make_uint4(0u, 0u, 0u, 0u);
                if (g < rows) v[i] = __ldg(q + out_row(g) * CH + c);
            }
#pragma unroll
            for (int i = 0; i < kM / RSTEP; ++i) {
                const int r = rr + i * RSTEP;
                *reinterpret_cast<uint4*>(dst + (c >> 3) * kHalfBytes + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = v[i];
            }
            fence_proxy_async();
            mbar_arrive(bar(kBarQ + L));
        }
        const uint32_t t_s = tmem + (static_cast<uint32_t>(warp & 3) << 21) + static_cast<uint32_t>(L) * 256u, t_o = t_s + 128u;
        const float scale = p.scale_log2;
        float m = -INFINITY, l = 0.f;                // reference (log2 units, the same in a row's two threads) and sum
        const int first_t = in_turn ? L : 0, step = in_turn ? 2 : 1;
        const bool active = L == 0 || lane1;
        uint32_t done = 0;                           // tiles of this lane so far
        for (int t = first_t; t < tiles && active; t += step, ++done) {
            if (ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait_spin(bar(kBarS + L), done & 1u, abort_flag, p.status, limit));
            uint32_t s[kCols];
            float top = -INFINITY;
            if (ok) {
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < kCols / 16; ++c) tmem_ld_row16(t_s + static_cast<uint32_t>(side * kCols + 16 * c), s + 16 * c);
                tmem_wait_ld();
                const int keys = p.len - (t0 + t) * kTile - side * kCols;
                if (keys < kCols) {
#pragma unroll
                    for (int i = 0; i < kCols; ++i)
                        if (i >= keys) s[i] = 0xFF800000u;       // -inf
                }
                top = row_max(s) * scale;
            }
            // The barrier says whether some row of the lane has a maximum past its reference's limit (or no
            // reference yet), and that all of S has been read: from here P may take its place.
            if (lane_any(sync_id, kLaneThreads, done == 0 || top > m + kRescaleAbove)) {
                float* x = xch + L * kM + row;
                if (side == 0) *x = top;
                lane_sync(sync_id, kLaneThreads);
                if (side == 1) *x = top = fmaxf(*x, top);
                lane_sync(sync_id, kLaneThreads);
                if (side == 0) top = *x;
                const bool raise = done == 0 ? top > m : top > m + kRescaleAbove;
                const float before = m;
                if (raise) m = top;
                if (ok && done > 0) {                // the row's O, complete up to the tile before, to the new reference
                    const float f = raise ? fast_exp2(before - m) : 1.f;
                    l *= f;
#pragma unroll
                    for (int c = 0; c < D / 32; ++c) {
                        uint32_t o[16];
                        const uint32_t at = t_o + static_cast<uint32_t>(side * (D / 2) + 16 * c);
                        tmem_ld_row16(at, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                        tmem_st_row16(at, o);
                    }
                }
            }
            if (ok) {
                l += row_weights(s, scale, m, t_s + static_cast<uint32_t>(side * kCols / 2));
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(bar(kBarP + L));
            }
        }
        // the lane's result
        if (done > 0 && ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarO + L), 0, abort_flag, p.status, limit));
        // Products are complete in the order of their issue.  Lane 0's O is complete: so are all products
        // that read queries.  Lane 1's: so are all products of the block, unless the lanes take tiles in turn
        // and lane 0 has the last one.
        if (in_turn && L == 1 && ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarO), 0, abort_flag, p.status, limit));
        tc_fence_after();
        if (active) {
            // O by rows from tensor memory into shared memory (16-byte chunks in an order that spreads them over
            // the banks), then whole rows to global memory.  Lane 0's rows lie on the queries, lane 1's on
            // the first two stages: nothing reads them any more (see the waits above).
            constexpr int CH = D / 4;                // 16-byte chunks of a row of fp32
            static_assert(kM * D * 4 == 2 * Cfg::kTileBytes, "a lane's result takes the place of two tiles");
            uint8_t* st = smem + (L * kM + (warp & 3) * 32) * D * 4;
            if (side == 1) xch[L * kM + row] = l;
            if (ok) {
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[16];
                    if (done > 0) {
                        tmem_ld_row16(t_o + static_cast<uint32_t>(side * (D / 2) + 16 * c), o);
                        tmem_wait_ld();
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] = 0u;
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<uint4*>(st + (lane * CH + ((side * (CH / 2) + c * 4 + i) ^ (lane & 7))) * 16) =
                            make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                }
            }
            lane_sync(sync_id, kLaneThreads);
            if (ok) {
                const int part = in_turn ? 2 * blockIdx.z + L : blockIdx.z;
                const int64_t part0 = static_cast<int64_t>(part) * p.n * p.q_heads;
                const int w0 = r0 + (in_turn ? 0 : L * kM) + (warp & 3) * 32, ch = lane % CH;
                for (int r = side * 16 + lane / CH; r < side * 16 + 16 && w0 + r < rows; r += 32 / CH) {
                    const uint4 v = *reinterpret_cast<const uint4*>(st + (r * CH + (ch ^ (r & 7))) * 16);
                    reinterpret_cast<uint4*>(p.part_o)[(part0 + out_row(w0 + r)) * CH + ch] = v;
                }
                if (side == 0 && g_row < rows)
                    *reinterpret_cast<float2*>(p.part_ml + 2 * (part0 + out_row(g_row))) = make_float2(m, l + xch[L * kM + row]);
            }
        }
    }
    // ---- tear-down: every role comes here, on every path, and tensor memory is given back
    if (!ok) *abort_flag = 1;
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

template <int D>
cudaError_t launch_t(const CUtensorMap& map, const PrefixParams& p, cudaStream_t stream) {
    static bool configured[64] = {false};             // the opt-in to large shared memory is per device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!configured[dev]) {
        e = cudaFuncSetAttribute(prefix_umma_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Config<D>::kSmem);
        if (e != cudaSuccess) return e;
        configured[dev] = true;
    }
    const int rows = p.n * p.group;
    const dim3 grid(static_cast<unsigned>((rows + 2 * kM - 1) / (2 * kM)), static_cast<unsigned>(p.kv_heads),
                    static_cast<unsigned>(p.in_turn ? p.splits / 2 : p.splits));
    prefix_umma_kernel<D><<<grid, kThreads, Config<D>::kSmem, stream>>>(map, p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_prefix_umma(const CUtensorMap& map, const PrefixParams& p, cudaStream_t stream) {
    if (p.splits < 1 || p.len < 1) return cudaSuccess;
    return p.head_dim == 128 ? launch_t<128>(map, p, stream) : launch_t<64>(map, p, stream);
}

}  // namespace odma
