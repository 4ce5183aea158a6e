// The prefix part of attention behind a shared prefix on the fifth-generation tensor cores (bf16 rows,
// head_dim 64 or 128; 8-bit prefixes come here as bf16).  See prefix.cu for the operator.
//
// A block takes one KV head, one split of the prefix's keys and up to 256 query rows (row = request,
// query head of the group).  With rows on the M side and steps of 64 keys
//     S[128 x 64] = Q[128 x D] . K[64 x D]^T          Q, K from shared memory, K-major
//     O[128 x D] += P[128 x 64] . V[64 x D]           P from tensor memory, V MN-major
// with S, P and O in tensor memory.  Two such sets ("lanes") share the SM.  More than 128 rows: the lanes
// hold two row tiles and use every step's K and V twice; otherwise both hold the same rows and take the
// steps in turn, each with a partial result of its own.
//
// Tensor memory (512 columns): a lane has two S buffers of 64 columns and O (D columns).  P (bf16)
// overwrites the first half of the left and of the right 32 columns of its S once they have been read.
// Two buffers let S of the next step be there when a step's softmax begins: with one buffer of 128 keys per
// lane (all that fits) a lane's softmax and products took turns, 4,100 cycles per pair of tiles
// where the products alone take 2,100.
//
// Warps 0-7 and 8-15: softmax of lane 0 and 1, two threads per row, 32 keys each (no shuffles); warp 16: TMA
// producer; warps 17 and 18: issue of lane 0's and 1's products, QK(0) QK(1), then PV(u) QK(u + 2) for every step u, so a
// buffer is only overwritten by a product issued after the one that reads its P.
//
// The softmax keeps a reference m per row, raised only when a step's maximum passes it by 2^8: P stays
// below 256, which bf16 relative to the fp32 accumulator does not mind, and O is rescaled in tensor
// memory only then.  P is rounded to bf16 for the product (half a step: 2^-9 to 2^-8 of a weight, random
// in sign over the keys); sums, maxima and O are fp32.
//
// What bounds it: the tensor pipe.  32,768 keys and 7,168 rows (120 GFLOP): 108 us for this kernel alone, 1.1 PFLOP/s
// (0.66 of the measured burst rate), the whole call 137 us in a burst and 146 to 152 sustained (the GPU then sits at its
// power limit, 985 W); 1,570 cycles per step of 64 keys and 256 rows.  An instruction takes 64 cycles, the first
// product's, 64 keys wide, no less than one of 128 keys (2 x (8 + 4) x 64 = 1,536); with a quarter of the first
// product's instructions the call took 124 us instead of 140, of the second's 130, without the exponentials 132,
// without loads 138.  Steps of 128 keys would halve the first product's count and leave one S buffer per lane, whose
// chain of softmax and products is about as long.  A block's set-up, queries and hand-over cost 6.5 us, of which the
// 128 KB of its partial results are 2.4: that is what short prefixes pay for.
#include "odma.h"
#include "tcgen05.cuh"

namespace odma {
namespace {

using namespace dev;

constexpr int kM = 128;                             // rows per lane
constexpr int kStep = 64;                           // keys per step
constexpr int kCols = kStep / 2;                    // scores per softmax thread
constexpr int kSoftmaxWarps = 16;                   // four warpgroups: lane 0 and 1, left and right half of a step's keys
constexpr int kThreads = (kSoftmaxWarps + 3) * 32;
constexpr int kProducerWarp = kSoftmaxWarps, kMmaWarp = kSoftmaxWarps + 1;    // and kMmaWarp + 1: one per lane
constexpr int kLaneThreads = kSoftmaxWarps * 16;    // softmax threads of a lane
constexpr int kMaxStages = 16;
constexpr float kRescaleAbove = 8.f;
constexpr int kQHalfBytes = kM * 128;               // 64 elements of a lane's queries
constexpr int kHalfBytes = kStep * 128;             // 64 elements of a step's keys or values
// barriers
constexpr int kBarFull = 0, kBarEmpty = kMaxStages, kBarP = 2 * kMaxStages, kBarS = kBarP + 4,
              kBarPv = kBarS + 4, kBarO = kBarPv + 2, kBarDrain = kBarO + 2, kNumBars = kBarDrain + 2;   // S, P: [lane][buffer]

template <int D>
struct Config {
    static constexpr int kHalves = D / 64;
    static constexpr int kQBytes = kHalves * kQHalfBytes;        // a lane's queries
    static constexpr int kStageBytes = kHalves * kHalfBytes;     // a step's keys, or its values
    static constexpr int kStages = D == 128 ? 10 : 16;
    static constexpr int kSmem = 2 * kQBytes + kStages * kStageBytes + 2 * kM * 4 + kNumBars * 8 + 64 + 1024;
};

// Products and commits by the elected lane of a converged warp.  The election is a predicate of the instruction and
// not a branch around it: the code stays uniform, so descriptors and addresses stay in uniform registers, where these
// instructions want them (behind a branch every one of them is moved there for every instruction).
// D[tmem] (+)= A[smem] . B[smem]^T
__device__ __forceinline__ void umma_ss(uint32_t elected, uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(elected)
        : "memory");
}
// D[tmem] (+)= A[tmem] . B[smem]
__device__ __forceinline__ void umma_ts(uint32_t elected, uint32_t d_tmem, uint32_t a_tmem, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b), "r"(idesc), "r"(accumulate), "r"(elected)
        : "memory");
}
__device__ __forceinline__ void commit(uint32_t elected, uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(elected)
        : "memory");
}

// 16 columns of the thread's own row (tensor-memory lane = 32 * (warp mod 4) + lane).
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

__device__ __forceinline__ float row_max(const uint32_t (&s)[kCols]) {
    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int i = 0; i < kCols; i += 8)
#pragma unroll
        for (int k = 0; k < 4; ++k) mx[k] = fmaxf(fmaxf(mx[k], __uint_as_float(s[i + 2 * k])), __uint_as_float(s[i + 2 * k + 1]));
    return fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
}

// The thread's weights 2^(s * scale - ref), rounded to bf16, to tensor memory; their sum (unrounded).
__device__ __forceinline__ float row_weights(const uint32_t (&s)[kCols], float scale, float ref, uint32_t t_p) {
    const float2 sc = make_float2(scale, scale), neg = make_float2(-ref, -ref);
    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    uint32_t pk[kCols / 2];
#pragma unroll
    for (int i = 0; i < kCols / 2; ++i) {
        float2 x = fma2(make_float2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), sc, neg);
        x = make_float2(fast_exp2(x.x), fast_exp2(x.y));
        sum[i & 1] = add2(sum[i & 1], x);
        pk[i] = pack_bf16(x.x, x.y);
    }
    tmem_st_row16(t_p, pk);
    return (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
}

// Barrier over `threads` threads; the second form tells whether any of them says yes.  Every thread comes to every
// one of its barriers, also after a wait has given up.
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
    constexpr uint32_t IDESC_QK = umma_idesc(kM, kStep, false), IDESC_PV = umma_idesc(kM, D, true);
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    uint8_t* qbuf = smem;
    uint8_t* kv = qbuf + 2 * Cfg::kQBytes;
    float* xch = reinterpret_cast<float*>(kv + STAGES * Cfg::kStageBytes);    // [lane][row], between a row's two threads
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
    const bool in_turn = p.in_turn != 0;             // both lanes on the same rows, steps in turn
    const bool lane1 = in_turn || r0 + kM < rows;    // is there a second lane?
    const int blocks = in_turn ? p.splits >> 1 : p.splits;      // splits of the keys over the blocks, in tiles of 128
    const int all_tiles = (p.len + kPrefixTile - 1) / kPrefixTile;
    const int z = static_cast<int>(blockIdx.z);      // below 128, and tiles below 2^24: no product leaves 32 bits
    const int k0 = all_tiles * z / blocks * kPrefixTile, k1 = min(p.len, all_tiles * (z + 1) / blocks * kPrefixTile);
    const int steps = (k1 - k0 + kStep - 1) / kStep; // of the block; a lane takes all of them, or every second one
    const int turn = in_turn ? 2 : 1, ahead = 2 * turn;         // K of a step is asked for `ahead` steps before its V
    auto lane_steps = [&](int L) { return in_turn ? (steps - L + 1) / 2 : steps; };

    const uint32_t kv_u32 = smem_u32(kv), q_u32 = smem_u32(qbuf);
    bool ok = true;
    auto out_row = [&](int r) { return (r / p.group) * p.q_heads + head * p.group + r % p.group; };    // row of q and of a partial result

    // ---- set-up, the roles side by side: barriers and the first loads; tensor memory; the queries
    uint32_t issued = 0;
    auto load = [&](bool is_v, int u) {              // the producer's next stage
        const uint32_t stage = issued % STAGES, use = issued / STAGES;
        if (use > 0) ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarEmpty + stage), (use & 1u) ^ 1u, abort_flag, p.status, limit));
        if (!ok) return;
        if (lane == 0) mbar_expect_tx(bar(kBarFull + stage), static_cast<uint32_t>(Cfg::kStageBytes));
        __syncwarp();
        if (lane < Cfg::kHalves)                     // a box of 64 rows per 128-byte column block
            tma_load_2d(kv_u32 + stage * Cfg::kStageBytes + lane * kHalfBytes, &map, lane * 64,
                        static_cast<int32_t>((is_v ? p.v_row0 : p.k_row0) + head * p.head_rows + k0 + u * kStep), bar(kBarFull + stage));
        ++issued;
    };
    constexpr int QCH = D / 8;                       // 16-byte chunks of a query row
    constexpr int QLOADS = kM * QCH / kLaneThreads;  // per thread of a lane
    constexpr int QROWS = 32 / QCH;                  // rows per warp and load
    if (warp == kProducerWarp) {
        for (int i = lane; i < kNumBars; i += 32) {
            const bool softmax = i >= kBarP && i < kBarS;                        // arrivals of a lane's softmax warps
            const bool shared = i >= kBarEmpty && i < kBarP && lane1;            // both lanes hand every stage back
            mbar_init(bar(i), softmax ? kLaneThreads / 32u : shared ? 2u : 1u);
        }
        if (lane == 0) *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        __syncwarp();
        asm volatile("griddepcontrol.wait;" ::: "memory");                       // 8-bit pools: the kernel ahead writes these rows
        for (int u = 0; u < min(ahead, steps) && ok; ++u) load(false, u);        // (as many stages as this are free)
    } else if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        // The kernel behind this one (the requests' own parts) reads nothing that this one or the one ahead of it writes: its
        // blocks may begin on every SM that this one leaves idle or is done with.  They begin once every block of this
        // kernel has come here, and so holds its tensor memory: theirs keep their columns until this kernel has ended, and a
        // block of this one that still waited for columns on the same SM would never end.
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    } else if (warp < kSoftmaxWarps && (warp < 8 || (lane1 && !in_turn))) {
        // Queries to shared memory, in the swizzled order: a warp takes 16 of its lane's 128 rows, QROWS at a time, all
        // loads before the first store; one thread works out one row's place.
        const int w0 = (warp & 7) * (QROWS * QLOADS), g0 = r0 + (warp >> 3) * kM + w0;
        const int mine = out_row(min(g0 + (lane & (QROWS * QLOADS - 1)), rows - 1));
        uint4 qv[QLOADS];
#pragma unroll
        for (int i = 0; i < QLOADS; ++i) {
            const int r = i * QROWS + lane / QCH, at = __shfl_sync(0xFFFFFFFFu, mine, r);
            qv[i] = make_uint4(0u, 0u, 0u, 0u);      // rows behind the last are zero
            if (g0 + r < rows) qv[i] = __ldg(static_cast<const uint4*>(p.q) + static_cast<int64_t>(at) * QCH + lane % QCH);
        }
        uint8_t* dst = qbuf + (warp >> 3) * Cfg::kQBytes;
#pragma unroll
        for (int i = 0; i < QLOADS; ++i) {
            const int r = w0 + i * QROWS + lane / QCH, c = lane % QCH;
            *reinterpret_cast<uint4*>(dst + (c >> 3) * kQHalfBytes + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = qv[i];
        }
        fence_proxy_async();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp == kProducerWarp) {
        // ------------------------------------------------------------------ producer
        // Ring order: K of the first `ahead` steps, then V(u), K(u + ahead) for each step u.
        for (int u = 0; u < steps && ok; ++u) {
            load(true, u);
            if (ok && u + ahead < steps) load(false, u + ahead);
        }
        if (lane == 0 && (!ok || *abort_flag)) {
            // something timed out: wait (bounded) for the loads in flight before shared memory is given up
            for (uint32_t i = issued > STAGES ? issued - STAGES : 0; i < issued; ++i)
                mbar_wait_slow(bar(kBarFull + i % STAGES), (i / STAGES) & 1u, nullptr, p.status, limit / 4 + 1);
        }
    } else if (warp >= kMmaWarp) {
        // ------------------------------------------------------------------ products of one lane
        const int L = warp - kMmaWarp;
        uint32_t elected;
        asm volatile("{\n\t.reg .pred P;\n\telect.sync _|P, 0xFFFFFFFF;\n\tselp.b32 %0, 1, 0, P;\n\t}" : "=r"(elected));
        uint32_t stage_next = 0, phase_next = 0;     // ring position
        auto wait = [&](uint32_t b, uint32_t parity) {
            if (!__all_sync(0xFFFFFFFFu, mbar_try(b, parity)))
                ok = ok && __all_sync(0xFFFFFFFFu, mbar_wait_slow(b, parity, abort_flag, p.status, limit));
        };
        auto wait_stage = [&]() {
            const uint32_t stage = stage_next;
            wait(bar(kBarFull + stage), phase_next);
            if (++stage_next == STAGES) {
                stage_next = 0;
                phase_next ^= 1u;
            }
            return stage;
        };
        const uint64_t q_desc = smem_desc(q_u32 + (in_turn ? 0u : static_cast<uint32_t>(L) * Cfg::kQBytes), 16, 1024),
                       k_desc = smem_desc(kv_u32, 16, 1024), v_desc = smem_desc(kv_u32, kHalfBytes, 1024);
        const uint32_t base = tmem + static_cast<uint32_t>(L) * 256u;
        // S of the lane's step v; the keys' stage is handed back
        auto first = [&](int v, uint32_t stage) {
            const uint64_t kd = k_desc + stage * (Cfg::kStageBytes >> 4);
            const uint32_t t_s = base + static_cast<uint32_t>(v & 1) * kStep;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
                umma_ss(elected, t_s, q_desc + (((ks >> 2) * kQHalfBytes + (ks & 3) * 32) >> 4), kd + (((ks >> 2) * kHalfBytes + (ks & 3) * 32) >> 4),
                        IDESC_QK, ks > 0 ? 1u : 0u);
            commit(elected, bar(kBarS + 2 * L + (v & 1)));
            commit(elected, bar(kBarEmpty + stage));
        };
        // O += P V of the lane's step v; so is the values'
        auto second = [&](int v, uint32_t stage, int keys) {
            const uint64_t vd = v_desc + stage * (Cfg::kStageBytes >> 4);
            const uint32_t t_p = base + static_cast<uint32_t>(v & 1) * kStep;
            auto product = [&](int ks) {             // 16 keys; P of the step's right half begins at its column kCols
                umma_ts(elected, base + 128u, t_p + static_cast<uint32_t>((ks >> 1) * kCols + (ks & 1) * 8), vd + ((ks * 2048) >> 4), IDESC_PV,
                        (v == 0 && ks == 0) ? 0u : 1u);
            };
            if (keys >= kStep) {
                product(0);
                product(1);
                product(2);
                product(3);
            } else {
                for (int ks = 0; ks * 16 < keys; ++ks) product(ks);
            }
            commit(elected, bar(kBarPv + L));
            commit(elected, bar(kBarEmpty + stage));
        };
        // value rows between the prefix's end and the next multiple of 16: whatever the slab holds there,
        // and 0 times a NaN would not be 0 (both lanes' warps may do it: they write the same)
        auto clear_tail = [&](int keys, uint32_t stage) {
            const int end = (keys + 15) & ~15;
            uint8_t* vb = kv + stage * Cfg::kStageBytes;
            for (int i = lane; i < (end - keys) * 8 * Cfg::kHalves; i += 32) {
                const int row = keys + i / (8 * Cfg::kHalves), c = i % (8 * Cfg::kHalves);
                *reinterpret_cast<uint4*>(vb + (c >> 3) * kHalfBytes + row * 128 + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            fence_proxy_async();
            __syncwarp();
        };
        if (L == 0 || lane1) {
            const int mine = in_turn ? L : 0;
            // Every stage is waited for and handed back, used or not: a wait tells a phase from its neighbours only.
            auto pass = [&](uint32_t stage) {
                if (elected && ok) mbar_arrive(bar(kBarEmpty + stage));
                __syncwarp();
            };
            for (int u = 0; u < min(ahead, steps) && ok; ++u) {
                const uint32_t ks = wait_stage();
                if (u % turn != mine)
                    pass(ks);
                else if (ok)
                    first(u / turn, ks);
            }
            int v = 0;
            for (int u = 0; u < steps && ok; ++u) {
                const uint32_t vs = wait_stage();
                const bool more = u + ahead < steps;
                if (u % turn != mine) {
                    pass(vs);
                    if (more) pass(wait_stage());
                    continue;
                }
                const int keys = p.len - (k0 + u * kStep);
                if (keys < kStep) clear_tail(keys, vs);
                wait(bar(kBarP + 2 * L + (v & 1)), static_cast<uint32_t>(v >> 1) & 1u);
                if (!ok) break;
                tc_fence_after();
                second(v, vs, keys);
                if (more) {
                    const uint32_t ks = wait_stage();
                    if (ok) first(v + 2, ks);
                }
                ++v;
            }
            commit(elected, bar(kBarO + L));
        }
        // nothing may still be running when tensor memory is given back
        commit(elected, bar(kBarDrain + L));
        __syncwarp();
        mbar_wait_slow(bar(kBarDrain + L), 0, nullptr, p.status, limit / 4 + 1);
    } else {
        // ------------------------------------------------------------------ softmax
        const int L = warp >> 3, side = (warp >> 2) & 1;     // lane; left or right half of a step's keys
        const int row = (warp & 3) * 32 + lane;      // of the lane's tile
        const int g_row = r0 + (in_turn ? 0 : L * kM) + row;
        const int pair_id = 1 + L * 4 + (warp & 3);  // barrier of the row's two warps
        const uint32_t t_s = tmem + (static_cast<uint32_t>(warp & 3) << 21) + static_cast<uint32_t>(L) * 256u, t_o = t_s + 128u;
        const float scale = p.scale_log2;
        float m = -INFINITY, l = 0.f;                // reference (log2 units, the same in a row's two threads) and sum
        const bool active = L == 0 || lane1;
        const int own = active ? lane_steps(L) : 0;  // steps of the lane
        for (int u = 0; u < own; ++u) {
            if (ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarS + 2 * L + (u & 1)), static_cast<uint32_t>(u >> 1) & 1u, abort_flag, p.status, limit));
            const uint32_t t_u = t_s + static_cast<uint32_t>((u & 1) * kStep + side * kCols);
            uint32_t s[kCols];
            float top = -INFINITY;
            if (ok) {
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < kCols / 16; ++c) tmem_ld_row16(t_u + 16u * c, s + 16 * c);
                tmem_wait_ld();
                const int keys = p.len - (k0 + (in_turn ? 2 * u + L : u) * kStep + side * kCols);
                if (keys < kCols) {
#pragma unroll
                    for (int i = 0; i < kCols; ++i)
                        if (i >= keys) s[i] = 0xFF800000u;       // -inf
                }
                top = row_max(s) * scale;
            }
            // The two warps of these 32 rows agree whether some row's maximum has passed its reference's limit (or
            // there is no reference yet).
            if (lane_any(pair_id, 64, u == 0 || top > m + kRescaleAbove)) {
                float* x = xch + L * kM + row;
                if (side == 0) *x = top;
                lane_sync(pair_id, 64);
                if (side == 1) *x = top = fmaxf(*x, top);
                lane_sync(pair_id, 64);
                if (side == 0) top = *x;
                const bool raise = u == 0 ? top > m : top > m + kRescaleAbove;
                const float before = m;
                if (raise) m = top;
                if (u > 0) {
                    // O to the new reference, once it is complete up to the step before (S of this step says so up to
                    // the step before that one, so the barrier is at most one phase behind)
                    if (ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarPv + L), static_cast<uint32_t>(u - 1) & 1u, abort_flag, p.status, limit));
                    const float f = raise ? fast_exp2(before - m) : 1.f;
                    l *= f;
                    if (ok) {
                        tc_fence_after();
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
            }
            if (ok) {
                const float ref = m == -INFINITY ? 0.f : m;      // every score so far is -inf: weights 0, not NaN
                l += row_weights(s, scale, ref, t_u);            // P over the left half of the columns just read
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(kBarP + 2 * L + (u & 1)));
            }
        }
        // the lane's result
        // Both lanes' products are complete before either lane writes over queries and stages.
        const bool two = lane1 && (!in_turn || steps > 1);
        if (ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarO), 0, abort_flag, p.status, limit));
        if (ok && two) ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarO + 1), 0, abort_flag, p.status, limit));
        tc_fence_after();
        if (active) {
            // O by rows from tensor memory into shared memory (over queries and stages; a row's pitch is 16 bytes more than
            // its size, which spreads 16-byte chunks over the banks), then a bulk copy per row to global memory.
            constexpr uint32_t PITCH = D * 4 + 16;
            static_assert(2 * kM * PITCH <= 2 * Cfg::kQBytes + Cfg::kStages * Cfg::kStageBytes, "where the results go");
            const uint32_t st = static_cast<uint32_t>(L * kM + row) * PITCH;
            if (side == 1) xch[L * kM + row] = l;
            if (ok) {
                uint32_t o[D / 32][16];
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    if (own > 0) {
                        tmem_ld_row16(t_o + static_cast<uint32_t>(side * (D / 2) + 16 * c), o[c]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[c][i] = 0u;
                    }
                }
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < D / 32; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<uint4*>(smem + st + (side * (D / 2) + 16 * c + 4 * i) * 4) =
                            make_uint4(o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]);
            }
            fence_proxy_async();
            lane_sync(pair_id, 64);
            if (ok && side == 0 && g_row < rows) {
                const int part = in_turn ? 2 * blockIdx.z + L : blockIdx.z;
                const int64_t at = static_cast<int64_t>(part) * p.n * p.q_heads + out_row(g_row);
                asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(p.part_o + at * D), "r"(smem_u32(smem) + st), "r"(D * 4)
                             : "memory");
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                *reinterpret_cast<float2*>(p.part_ml + 2 * at) = make_float2(m, l + xch[L * kM + row]);
                asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");        // written: the block may end
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
cudaError_t launch_t(const CUtensorMap& map, const PrefixParams& p, bool behind_dequant, cudaStream_t stream) {
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
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Config<D>::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = behind_dequant ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, prefix_umma_kernel<D>, map, p);
}

}  // namespace

cudaError_t launch_prefix_umma(const CUtensorMap& map, const PrefixParams& p, bool behind_dequant, cudaStream_t stream) {
    if (p.splits < 1 || p.len < 1) return cudaSuccess;
    return p.head_dim == 128 ? launch_t<128>(map, p, behind_dequant, stream) : launch_t<64>(map, p, behind_dequant, stream);
}

}  // namespace odma
