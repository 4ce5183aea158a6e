// Causal attention of a step's new tokens over the slabs on the fifth-generation tensor cores (bf16 rows, head_dim
// 64 or 128; the rows of an 8-bit pool come here as bf16).  See prefill.cu for the operator, prefill_plan.cuh for
// the split of the work.
//
// A persistent block walks its share of tiles.  A tile is one KV head of one request and up to 256 query rows (row =
// token, query head of the group: the group's heads share every key), in two lanes of up to 128; it is taken in steps of
// 128 keys,
//     S[128 x 128] = Q[128 x D] . K[128 x D]^T        Q, K from shared memory, K-major
//     O[128 x D]  += P[128 x 128] . V[128 x D]        P from tensor memory, V MN-major
// and both lanes use every step's K and V.  The lanes are out of phase: while one's softmax runs, the tensor pipe
// has the other's products.
//
// Tensor memory (512 columns): a lane has S (128 columns) and O (D columns); P (bf16) overwrites S from the left, 16
// columns for the 32 just read.
//
// Warps 0-3 and 4-7: softmax of lane 0 and 1, a thread per row; warp 8: TMA producer; warps 9 and 10: issue of lane 0's
// and 1's products, QK(0), then PV(u) QK(u + 1) for every step u, so S is only overwritten by a product issued after the one
// that reads P from it.
//
// The softmax keeps a reference m per row, raised only when a maximum passes it by 2^8: P stays below 256, which bf16
// relative to the fp32 accumulator does not mind.  So the 32 columns of a chunk need not wait for the other 96: the weights
// are computed with the standing reference while the chunk's maximum is found, and where it turns out too low (a tile's
// first chunk, and rarely later) the chunk is done again and what is already there, sum, O, and P of the step, is scaled.
// P is rounded to bf16 for the product (half a step: at most 2^-8 of a weight, random in sign over the keys); sums,
// maxima and O are fp32.
#include "odma.h"
#include "prefill_plan.cuh"
#include "tcgen05.cuh"

namespace odma {
namespace {

using namespace dev;

constexpr int kM = kPrefillRows / 2;                // rows per lane
constexpr int kStep = kPrefillStep;
constexpr int kChunk = 32;                          // scores of a row in registers at a time
constexpr int kThreads = 384;
constexpr int kProducerWarp = 8, kMmaWarp = 9;      // and kMmaWarp + 1
constexpr int kMaxStages = 10;
constexpr int kItemSlots = 4;
constexpr float kRescaleAbove = 8.f;
constexpr int kHalfBytes = 128 * 128;               // 64 elements of 128 rows: of a lane's queries, of a step's keys or values
// barriers
constexpr int kBarFull = 0, kBarEmpty = kMaxStages, kBarItem = 2 * kMaxStages, kBarQFull = kBarItem + kItemSlots,
              kBarQFree = kBarQFull + 1, kBarS = kBarQFree + 1, kBarPa = kBarS + 2, kBarPb = kBarPa + 2, kBarHalf = kBarPb + 2,
              kBarO = kBarHalf + 2, kBarDrain = kBarO + 2, kNumBars = kBarDrain + 2;

template <int D>
struct Config {
    static constexpr int kHalves = D / 64;
    static constexpr int kQBytes = kHalves * kHalfBytes;         // a lane's queries
    static constexpr int kStageBytes = kHalves * kHalfBytes;     // a step's keys, or its values
    static constexpr int kStages = D == 128 ? 5 : 10;
    static constexpr int kRing = kStages * kStageBytes;
    static constexpr int kSmem = 2 * kQBytes + kRing + kItemSlots * static_cast<int>(sizeof(PrefillItem)) + kNumBars * 8 + 64 + 1024;
};
static_assert(Config<128>::kSmem <= 232448 && Config<64>::kSmem <= 232448, "shared memory of a block");
// the plan's scratch lies in the ring, before the first load
static_assert(sizeof(PlanScratch) + kMaxPrefillBatch * 16 + 64 <= Config<128>::kRing, "room for the plan");

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, int32_t z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}

// Maxima that a NaN goes through.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float row_max(const uint32_t (&s)[kChunk]) {
    float mx[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) mx[k] = __uint_as_float(s[k]);
#pragma unroll
    for (int i = 4; i < kChunk - 4; i += 8)
#pragma unroll
        for (int k = 0; k < 4; ++k) mx[k] = max3(mx[k], __uint_as_float(s[i + 2 * k]), __uint_as_float(s[i + 2 * k + 1]));
    const float a = max3(mx[0], __uint_as_float(s[kChunk - 4]), __uint_as_float(s[kChunk - 3])),
                b = max3(mx[1], __uint_as_float(s[kChunk - 2]), __uint_as_float(s[kChunk - 1]));
    return max3(a, b, max3(mx[2], mx[3], mx[3]));
}

// 2^x on the fused multiply-add pipe, for finite x <= 127: x = n + f with |f| <= 1/2, 2^f by the polynomial of degree 4
// with the least relative error on that interval (2.6e-6, far below the rounding of P), n added to the exponent.  Below 2^-126 the
// result is some number below 2^-125.  Two at a time.
__device__ __forceinline__ float2 poly_exp2(float2 x) {
    x.x = fmaxf(x.x, -126.f);
    x.y = fmaxf(x.y, -126.f);
    const float2 round = make_float2(12582912.f, 12582912.f), back = make_float2(-12582912.f, -12582912.f);
    const float2 t = add2(x, round), n = add2(t, back);
    const float2 f = fma2(n, make_float2(-1.f, -1.f), x);
    float2 y = fma2(f, make_float2(0.0095701f, 0.0095701f), make_float2(0.05591786f, 0.05591786f));
    y = fma2(y, f, make_float2(0.24024745f, 0.24024745f));
    y = fma2(y, f, make_float2(0.69312181f, 0.69312181f));
    y = fma2(y, f, make_float2(0.99999926f, 0.99999926f));
    return make_float2(__uint_as_float(__float_as_uint(y.x) + (__float_as_uint(t.x) << 23)),
                       __uint_as_float(__float_as_uint(y.y) + (__float_as_uint(t.y) << 23)));
}

// Weights 2^(s * scale - ref) of a chunk, rounded to bf16, and their sum (unrounded).  The first POLY of its 16 pairs
// take the fused multiply-add pipe, the others the special-function unit.
template <int POLY>
__device__ __forceinline__ float weights(const uint32_t (&s)[kChunk], float scale, float ref, uint32_t (&pk)[kChunk / 2]) {
    const float2 sc = make_float2(scale, scale), neg = make_float2(-ref, -ref);
    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
    for (int i = 0; i < kChunk / 2; ++i) {
        float2 x = fma2(make_float2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), sc, neg);
        if (i * POLY / 16 != (i + 1) * POLY / 16)
            x = poly_exp2(x);
        else
            x = make_float2(fast_exp2(x.x), fast_exp2(x.y));
        sum[i & 1] = add2(sum[i & 1], x);
        pk[i] = pack_bf16(x.x, x.y);
    }
    return (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
}
constexpr int kPolyPairs = 5;

// 32 bytes, a whole sector, in one instruction.
__device__ __forceinline__ void store8(void* p, const uint32_t* v) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
                 "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
prefill_umma_kernel(const __grid_constant__ CUtensorMap kv_map, const __grid_constant__ CUtensorMap q_map, const PrefillParams p) {
    using Cfg = Config<D>;
    constexpr int STAGES = Cfg::kStages;
    constexpr uint32_t IDESC_QK = umma_idesc(kM, kStep, false), IDESC_PV = umma_idesc(kM, D, true);
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    uint8_t* qbuf = smem;
    uint8_t* kv = qbuf + 2 * Cfg::kQBytes;
    PrefillItem* items = reinterpret_cast<PrefillItem*>(kv + Cfg::kRing);
    uint64_t* bars = reinterpret_cast<uint64_t*>(items + kItemSlots);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + kNumBars);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(const_cast<int*>(abort_flag) + 1);
    PlanScratch* plan = reinterpret_cast<PlanScratch*>(kv);
    const uint32_t bar0 = smem_u32(bars);
    auto bar = [&](int i) { return bar0 + 8u * static_cast<uint32_t>(i); };
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int64_t limit = p.wait_limit_ns;
    const int lane_tokens = p.tile_tokens >> 1, lane_rows = lane_tokens * p.group;
    const uint32_t kv_u32 = smem_u32(kv), q_u32 = smem_u32(qbuf);
    bool ok = true;

    // ---- set-up: barriers, tensor memory, query rows that no token has, the share
    if (warp == kProducerWarp) {
        for (int i = lane; i < kNumBars; i += 32) {
            const bool softmax = i >= kBarPa && i < kBarHalf;                    // a lane's four softmax warps
            const bool both = (i >= kBarEmpty && i < kBarItem) || i == kBarQFree;
            mbar_init(bar(i), softmax ? 4u : both ? 2u : 1u);
        }
        if (lane == 0) *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    } else if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else if (warp < 8) {
        const int spare = (kM - lane_rows) * 8 * Cfg::kHalves;                   // 16-byte chunks behind a lane's rows
        uint8_t* q_lane = qbuf + (warp >> 2) * Cfg::kQBytes;
        for (int i = tid & 127; i < spare; i += 128) {
            const int row = lane_rows + i / (8 * Cfg::kHalves), c = i % (8 * Cfg::kHalves);
            *reinterpret_cast<uint4*>(q_lane + (c >> 3) * kHalfBytes + row * 128 + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    int64_t* cum = reinterpret_cast<int64_t*>(kv + sizeof(PlanScratch));
    int32_t* lens = reinterpret_cast<int32_t*>(cum + p.n);
    prefill_plan<kStep, kThreads>(p, plan, cum, lens, lens + p.n);
    PrefillWalk<kStep> walk(p, *plan);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    fence_proxy_async();                             // the plan's words and the spare rows, before loads and products
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    // steps of lane L in item `it`: [it.t0, it.t0 + count)
    auto lane_end = [&](const PrefillItem& it, int L) {          // the keys that its last token sees
        const int first = it.tok0 + L * lane_tokens;
        return first < it.add ? it.ctx + min(first + lane_tokens, it.add) : 0;
    };
    auto lane_steps = [&](const PrefillItem& it, int L) {
        return max(0, min(it.t1, (lane_end(it, L) + kStep - 1) / kStep) - it.t0);
    };

    if (warp == kProducerWarp) {
        // ------------------------------------------------------------------ producer
        uint32_t stage = 0, phase = 0, filled = 0;
        int n_items = 0;
        PrefillItem it;
        int32_t k_row = 0, v_row = 0;
        auto load = [&](bool is_v, int u) {
            if (filled >= STAGES) ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarEmpty + stage), phase ^ 1u, abort_flag, p.status, limit));
            if (!ok) return;
            if (lane == 0) mbar_expect_tx(bar(kBarFull + stage), static_cast<uint32_t>(Cfg::kStageBytes));
            __syncwarp();
            if (lane < 2 * Cfg::kHalves)                 // boxes of 64 rows and 64 elements
                tma_load_2d(kv_u32 + stage * Cfg::kStageBytes + (lane >> 1) * kHalfBytes + (lane & 1) * (kHalfBytes / 2), &kv_map, (lane >> 1) * 64,
                            (is_v ? v_row : k_row) + u * kStep + (lane & 1) * 64, bar(kBarFull + stage));
            ++filled;
            if (++stage == STAGES) {
                stage = 0;
                phase ^= 1u;
            }
        };
        bool more = walk.next(it);
        while (ok) {
            // The slot's last item lies four back: its readers have all come to a later one (see the waits on kBarQFree).
            PrefillItem* to = items + (n_items & (kItemSlots - 1));
            if (!more) it.t1 = 0;
            if (lane == 0) {
                *to = it;
                mbar_arrive(bar(kBarItem + (n_items & (kItemSlots - 1))));
            }
            __syncwarp();
            if (!more) break;
            const int64_t rows = static_cast<int64_t>(p.wide ? it.wide_at : it.base) * p.kv_heads +
                                 static_cast<int64_t>(it.head) * (p.wide ? (it.ctx + it.add + 15) & ~15 : it.cap);
            k_row = static_cast<int32_t>(p.k_row0 + rows);
            v_row = static_cast<int32_t>(p.v_row0 + rows);
            load(false, it.t0);
            // the queries, once the products of the item before have read theirs
            if (ok && n_items > 0)
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarQFree), static_cast<uint32_t>(n_items - 1) & 1u, abort_flag, p.status, limit));
            if (!ok) break;
            const int lanes = it.tok0 + lane_tokens < it.add ? 2 : 1;
            if (lane == 0) mbar_expect_tx(bar(kBarQFull), static_cast<uint32_t>(lanes * Cfg::kHalves * lane_rows * 128));
            __syncwarp();
            if (lane < lanes * Cfg::kHalves) {
                const int L = lane / Cfg::kHalves, hf = lane % Cfg::kHalves;
                tma_load_3d(q_u32 + L * Cfg::kQBytes + hf * kHalfBytes, &q_map, hf * 64, it.head * p.group, it.cu + it.tok0 + L * lane_tokens,
                            bar(kBarQFull));
            }
            ++n_items;
            const int t0 = it.t0, t1 = it.t1;
            for (int u = t0; u < t1 && ok; ++u) {
                load(true, u);
                if (ok && u + 1 < t1) load(false, u + 1);
            }
            more = walk.next(it);
        }
        if (lane == 0 && (!ok || *abort_flag)) {
            // something timed out: wait (bounded) for the loads in flight before shared memory is given up
            for (uint32_t i = filled > STAGES ? filled - STAGES : 0; i < filled; ++i)
                mbar_wait_slow(bar(kBarFull + i % STAGES), (i / STAGES) & 1u, nullptr, p.status, limit / 4 + 1);
            if (n_items > 0) mbar_wait_slow(bar(kBarQFull), static_cast<uint32_t>(n_items - 1) & 1u, nullptr, p.status, limit / 4 + 1);
        }
    } else if (warp == kMmaWarp || warp == kMmaWarp + 1) {
        // ------------------------------------------------------------------ products of one lane
        const int L = warp - kMmaWarp;
        uint32_t elected;
        asm volatile("{\n\t.reg .pred P;\n\telect.sync _|P, 0xFFFFFFFF;\n\tselp.b32 %0, 1, 0, P;\n\t}" : "=r"(elected));
        uint32_t stage_next = 0, phase_next = 0, p_count = 0;
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
        const uint64_t q_desc = smem_desc(q_u32 + static_cast<uint32_t>(L) * Cfg::kQBytes, 16, 1024), k_desc = smem_desc(kv_u32, 16, 1024),
                       v_desc = smem_desc(kv_u32, kHalfBytes, 1024);
        const uint32_t t_s = tmem + static_cast<uint32_t>(L) * 256u, t_o = t_s + 128u;
        // Every stage is waited for and handed back, used or not: a wait tells a phase from its neighbours only.
        auto pass = [&](uint32_t stage) {
            if (elected && ok) mbar_arrive(bar(kBarEmpty + stage));
            __syncwarp();
        };
        // value rows between a tile's last key and the next multiple of 16: whatever the slab holds there, and 0 times
        // a NaN would not be 0 (both lanes' warps may do it: they write the same)
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
        for (int n_items = 0; ok; ++n_items) {
            const int slot = n_items & (kItemSlots - 1);
            wait(bar(kBarItem + slot), static_cast<uint32_t>(n_items / kItemSlots) & 1u);
            if (!ok) break;
            const PrefillItem it = items[slot];
            if (it.t1 == 0) break;
            const int own = lane_steps(it, L), steps = it.t1 - it.t0;
            const int lane_keys = lane_end(it, L), tile_keys = it.ctx + min(it.tok0 + 2 * lane_tokens, it.add);
            wait(bar(kBarQFull), static_cast<uint32_t>(n_items) & 1u);
            if (own == 0) {
                if (elected && ok) mbar_arrive(bar(kBarQFree));
                __syncwarp();
            }
            auto first = [&](int u) {                    // S of step u; the keys' stage is handed back, and after the last the queries
                const uint32_t stage = wait_stage();
                if (!ok) return;
                if (u >= own) {
                    pass(stage);
                    return;
                }
                const uint64_t kd = k_desc + stage * (Cfg::kStageBytes >> 4);
                tc_fence_after();
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                    umma_ss(elected, t_s, q_desc + (((ks >> 2) * kHalfBytes + (ks & 3) * 32) >> 4), kd + (((ks >> 2) * kHalfBytes + (ks & 3) * 32) >> 4),
                            IDESC_QK, ks > 0 ? 1u : 0u);
                commit(elected, bar(kBarS + L));
                commit(elected, bar(kBarEmpty + stage));
                if (u + 1 == own) commit(elected, bar(kBarQFree));
            };
            first(0);
            for (int u = 0; u < steps && ok; ++u) {
                const uint32_t vs = wait_stage();
                if (!ok) break;
                if (u < own) {
                    const int k0 = (it.t0 + u) * kStep;
                    const int slices = (min(kStep, lane_keys - k0) + 15) >> 4;           // of 16 keys
                    if (tile_keys - k0 < slices * 16) clear_tail(tile_keys - k0, vs);
                    const uint64_t vd = v_desc + vs * (Cfg::kStageBytes >> 4);
                    auto product = [&](int ks) {
                        umma_ts(elected, t_o, t_s + static_cast<uint32_t>(ks * 8), vd + ((ks * 2048) >> 4), IDESC_PV, (u == 0 && ks == 0) ? 0u : 1u);
                    };
                    wait(bar(kBarPa + L), p_count & 1u);
                    if (!ok) break;
                    tc_fence_after();
                    if (slices >= 4) {
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks) product(ks);
                    } else {
                        for (int ks = 0; ks < slices; ++ks) product(ks);
                    }
                    commit(elected, bar(kBarHalf + L));
                    wait(bar(kBarPb + L), p_count & 1u);
                    if (!ok) break;
                    tc_fence_after();
                    if (slices == 8) {
#pragma unroll
                        for (int ks = 4; ks < 8; ++ks) product(ks);
                    } else {
                        for (int ks = 4; ks < slices; ++ks) product(ks);
                    }
                    ++p_count;
                    commit(elected, bar(kBarEmpty + vs));
                    if (u + 1 == own) commit(elected, bar(kBarO + L));
                } else {
                    pass(vs);
                }
                if (u + 1 < steps) first(u + 1);
            }
        }
        // nothing may still be running when tensor memory is given back
        commit(elected, bar(kBarDrain + L));
        __syncwarp();
        mbar_wait_slow(bar(kBarDrain + L), 0, nullptr, p.status, limit / 4 + 1);
    } else if (warp < 8) {
        // ------------------------------------------------------------------ softmax
        const int L = warp >> 2;
        const int row = (warp & 3) * 32 + lane;          // of the lane's tile
        const int row_tok = min(row / p.group, lane_tokens - 1), row_head = row % p.group;
        const uint32_t t_s = tmem + (static_cast<uint32_t>(warp & 3) << 21) + static_cast<uint32_t>(L) * 256u, t_o = t_s + 128u;
        const float scale = p.scale_log2;
        uint32_t s_count = 0, o_count = 0;
        for (int n_items = 0; ok; ++n_items) {
            const int slot = n_items & (kItemSlots - 1);
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarItem + slot), static_cast<uint32_t>(n_items / kItemSlots) & 1u, abort_flag, p.status, limit));
            if (!ok) break;
            const PrefillItem it = items[slot];
            if (it.t1 == 0) break;
            const int own = lane_steps(it, L);
            const int tok = it.tok0 + L * lane_tokens + row_tok;
            const int sees = it.ctx + min(tok, it.add - 1) + 1;                  // keys of this row
            const int all_see = it.ctx + it.tok0 + L * lane_tokens + 1;          // keys of the lane's first row
            float m = -INFINITY, l = 0.f;                // reference (log2 units) and sum
            float most = NAN;                            // a maximum above it raises the reference (no reference yet: any)
            for (int u = 0; u < own && ok; ++u) {
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarS + L), s_count & 1u, abort_flag, p.status, limit));
                if (!ok) break;
                tc_fence_after();
                const int k0 = (it.t0 + u) * kStep;
                // The reference of the warp's rows goes up: what has been computed with the one before is scaled.  `c`: chunks of
                // this step already in P; `o`: O holds something.
                auto raise = [&](float top, int c, bool o) {
                    const bool up = m == -INFINITY ? top > m : top > most;
                    const float before = m;
                    if (up) {
                        m = top;
                        most = top + kRescaleAbove;
                    }
                    const float f = up ? fast_exp2(before - m) : 1.f;
                    l *= f;
                    if (c >= 2 && ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarHalf + L), s_count & 1u, abort_flag, p.status, limit));
                    if (!ok) return;
                    tc_fence_after();
                    if (o || c >= 2) {
#pragma unroll 1
                        for (int k = 0; k < D / 16; ++k) {
                            uint32_t v[16];
                            tmem_ld_row16(t_o + 16u * k, v);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
                            tmem_st_row16(t_o + 16u * k, v);
                        }
                    }
                    if (c & 1) {                         // the first chunk of this half
                        uint32_t v[16];
                        tmem_ld_row16(t_s + 16u * (c - 1), v);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            v[i] = pack_bf16(__uint_as_float(v[i] << 16) * f, __uint_as_float(v[i] & 0xFFFF0000u) * f);
                        tmem_st_row16(t_s + 16u * (c - 1), v);
                    }
                    tmem_wait_st();
                };
                auto step = [&](auto masked) {
                    constexpr bool MASK = decltype(masked)::value;
                    uint32_t s[2][kChunk];
                    tmem_ld_row32(t_s, s[0]);
#pragma unroll
                    for (int c = 0; c < kStep / kChunk; ++c) {
                        uint32_t(&x)[kChunk] = s[c & 1];
                        tmem_wait_row32(x);
                        if (c + 1 < kStep / kChunk) tmem_ld_row32(t_s + static_cast<uint32_t>((c + 1) * kChunk), s[(c + 1) & 1]);
                        if (MASK) {
                            const int keys = sees - k0 - c * kChunk;
#pragma unroll
                            for (int i = 0; i < kChunk; ++i)
                                if (i >= keys) x[i] = 0xFF800000u;       // -inf
                        }
                        uint32_t pk[kChunk / 2];
                        float sum = weights<MASK ? 0 : kPolyPairs>(x, scale, m == -INFINITY ? 0.f : m, pk);
                        const float top = row_max(x) * scale;
                        if (__any_sync(0xFFFFFFFFu, !(top <= most))) {
                            raise(top, c, u > 0);
                            sum = weights<0>(x, scale, m == -INFINITY ? 0.f : m, pk);
                        }
                        l += sum;
                        tmem_st_row16(t_s + 16u * c, pk);
                        if (c == 1 || c == 3) {
                            tmem_wait_st();
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(bar((c == 1 ? kBarPa : kBarPb) + L));
                        }
                    }
                };
                if (k0 + kStep <= all_see)
                    step(std::false_type());
                else
                    step(std::true_type());
                ++s_count;
            }
            if (!ok) break;
            // ---- the tile's result
            if (own > 0) {
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarO + L), o_count & 1u, abort_flag, p.status, limit));
                if (!ok) break;
                ++o_count;
                tc_fence_after();
            }
            const bool mine = row < lane_rows && tok < it.add;
            const float inv = it.slot >= 0 ? 1.f : p.v_scale / l;
            const int64_t out_row = static_cast<int64_t>(it.cu + tok) * p.q_heads + it.head * p.group + row_head;
            const int64_t part_row = static_cast<int64_t>(it.slot) * p.part_rows + L * lane_rows + row;
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
                uint32_t v[32];
                if (own > 0) {
                    tmem_ld_row32(t_o + 32u * c, v);
                    tmem_wait_row32(v);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = 0u;
                }
                if (mine && it.slot >= 0) {
                    float* to = p.part_o + part_row * D + 32 * c;
#pragma unroll
                    for (int i = 0; i < 32; i += 8) store8(static_cast<void*>(to + i), v + i);
                } else if (mine) {
                    uint32_t w[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) w[i] = pack_bf16(__uint_as_float(v[2 * i]) * inv, __uint_as_float(v[2 * i + 1]) * inv);
                    uint8_t* to = static_cast<uint8_t*>(p.out) + (out_row * D + 32 * c) * 2;
                    store8(to, w);
                    store8(to + 32, w + 8);
                }
                __syncwarp();
            }
            if (mine) {
                if (it.slot >= 0)
                    *reinterpret_cast<float2*>(p.part_ml + 2 * part_row) = make_float2(m, l);
                else if (p.lse)
                    p.lse[out_row] = (m + log2f(l)) * 0.6931471805599453f;
            }
            tc_fence_before();                           // O has been read: the next item's products may write it
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
cudaError_t launch_t(const CUtensorMap& kv, const CUtensorMap& q, const PrefillParams& p, cudaStream_t stream) {
    static bool configured[64] = {false};             // the opt-in to large shared memory is per device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!configured[dev]) {
        e = cudaFuncSetAttribute(prefill_umma_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Config<D>::kSmem);
        if (e != cudaSuccess) return e;
        configured[dev] = true;
    }
    prefill_umma_kernel<D><<<static_cast<unsigned>(p.shares), kThreads, Config<D>::kSmem, stream>>>(kv, q, p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_prefill_umma(const CUtensorMap& kv, const CUtensorMap& q, const PrefillParams& p, cudaStream_t stream) {
    return p.head_dim == 128 ? launch_t<128>(kv, q, p, stream) : launch_t<64>(kv, q, p, stream);
}

}  // namespace odma
