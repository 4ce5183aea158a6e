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
// Tensor memory (512 columns): a lane has S (128 columns) and O (D columns); P (bf16) overwrites S from the left, 32
// columns for the 64 just read.
//
// Warps 0-3 and 4-7: softmax of lane 0 and 1, a thread per row; warp 8: TMA producer; warp 9: issue of the products, QK(0) of
// both lanes, then PV(u) QK(u + 1) of one and of the other for every step u, so S is only overwritten by a product issued
// after the one that reads P from it.
//
// The softmax keeps a reference m per row, and no maximum is looked for while it stands: a half step's weights are taken
// against it, and their sum, which is needed anyway, tells when it is too low (above 2^16; a NaN too).  Then the half is done
// again with a new reference, and sum and O are scaled.  A tile's first step and the steps that a mask cuts look for their
// maximum first.  bf16 and the fp32 sums have the range for weights above 1.  P is rounded to bf16 for the product (half a
// step: at most 2^-8 of a weight, random in sign over the keys); sums, references and O are fp32.
//
// What bounds it: the tensor pipe, shared memory and the exponentials in turn.  A step's products want 2,048 cycles of the pipe
// (256 x 128 x D twice), and the first product's operands as many of shared memory's; a lane's own chain, scores to weights to
// products, is about 2,700, of which the other lane's covers what the pipe can take: 2,900 to 3,240 per step.  One prompt of
// 16,384 tokens, 28 + 4 heads of 128: 1,400 to 1,480 us (1.35 PFLOP/s, tensor pipe 70 % busy), 1,605 to 1,650
// back to back, at the card's power limit (1.2).  8 chunks of 128 tokens behind 1,920: 43.0 us (703 TFLOP/s).  With heads
// of 64 the products want half as much and the lane's own chain is as long: a step still takes 3,000 cycles (4,096 tokens, 16 + 4
// heads: 61 to 65 us, 530 to 560 TFLOP/s, tensor pipe 27 % busy, special-function unit 45 %).
// A tile costs 4,000 cycles beside its steps (results 2,300: tensor memory to registers to rows; first loads and scores), the
// launch about 7 us: set-up, plan, first loads, and the merge behind it.
#include "odma.h"
#include "prefill_plan.cuh"
#include "tcgen05.cuh"

namespace odma {
namespace {

using namespace dev;

constexpr int kM = kPrefillRows / 2;                // rows per lane
constexpr int kStep = kPrefillStep;
constexpr int kChunk = 32;                          // scores of a row in registers at a time
constexpr int kSoftmaxWarps = 8;                    // lane 0 and 1, four times 32 rows
constexpr int kProducerWarp = kSoftmaxWarps, kMmaWarp = kSoftmaxWarps + 1;
constexpr int kThreads = (kSoftmaxWarps + 2) * 32;
constexpr int kMaxStages = 10;
constexpr int kItemSlots = 4;
constexpr int kPolyPairs = 3;
constexpr float kRaiseAbove = 16.f, kTooLarge = 65536.f;         // how far a maximum, in log2, or a half step's sum of weights may pass the reference
constexpr int kHalfBytes = 128 * 128;               // 64 elements of 128 rows: of a lane's queries, of a step's keys or values
// barriers
constexpr int kBarFull = 0, kBarEmpty = kMaxStages, kBarItem = 2 * kMaxStages, kBarRead = kBarItem + kItemSlots, kBarQFull = kBarRead + kItemSlots,
              kBarQFree = kBarQFull + 2, kBarS = kBarQFree + 2, kBarPa = kBarS + 2, kBarPb = kBarPa + 2, kBarHalf = kBarPb + 2,
              kBarO = kBarHalf + 2, kBarDrain = kBarO + 2, kNumBars = kBarDrain + 1;

template <int D>
struct Config {
    static constexpr int kHalves = D / 64;
    static constexpr int kQBytes = kHalves * kHalfBytes;         // a lane's queries
    static constexpr int kStageBytes = kHalves * kHalfBytes;     // a step's keys, or its values
    static constexpr int kStages = D == 128 ? 5 : 10;
    static constexpr int kRing = kStages * kStageBytes;
    static constexpr int kSmem = 2 * kQBytes + kRing + kItemSlots * static_cast<int>(sizeof(PrefillItem)) + kNumBars * 8 + 64 + 1024;
};
static_assert(kItemSlots * sizeof(PrefillItem) % 8 == 0, "barriers lie behind the items");
static_assert(Config<128>::kSmem <= 232448 && Config<64>::kSmem <= 232448, "shared memory of a block");
// the plan's scratch lies in the ring, before the first load
static_assert(sizeof(PlanScratch) + kMaxPrefillBatch * 16 + 64 <= Config<128>::kRing, "room for the plan");

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, int32_t z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}

__device__ __forceinline__ float row_max(const uint32_t (&s)[kChunk]) {
    float mx[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) mx[k] = __uint_as_float(s[k]);
#pragma unroll
    for (int i = 4; i < kChunk; i += 4)
#pragma unroll
        for (int k = 0; k < 4; ++k) mx[k] = fmaxf(mx[k], __uint_as_float(s[i + k]));
    return fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
}

// 2^x on the fused multiply-add pipe: x = n + f with |f| <= 1/2, 2^f by the polynomial of degree 4 with the least relative
// error on that interval (2.6e-6, by Remez exchange), times 2^n, whose exponent n + 127 is held to [0, 254] by one
// instruction.  So below 2^-126 the result is 0, and above 2^127 it is one of that size and not what an exponent that has run into
// the sign makes of it: the sum of weights is too large then and the caller takes the special-function unit instead, as it does
// for infinities and NaN, which end as NaN, and for x below -2^23, where n's bits no longer mean n.  Two at a time.
__device__ __forceinline__ float2 poly_exp2(float2 x) {
    constexpr float kRound = 12582912.f;             // 1.5 * 2^23: the sum's low bits are n (and 127 with it)
    const float2 t = add2(x, make_float2(kRound + 127.f, kRound + 127.f)), n = add2(t, make_float2(-kRound - 127.f, -kRound - 127.f));
    const float2 f = fma2(n, make_float2(-1.f, -1.f), x);
    float2 y = fma2(f, make_float2(0.0095701f, 0.0095701f), make_float2(0.05591786f, 0.05591786f));
    y = fma2(y, f, make_float2(0.24024745f, 0.24024745f));
    y = fma2(y, f, make_float2(0.69312181f, 0.69312181f));
    y = fma2(y, f, make_float2(0.99999926f, 0.99999926f));
    auto power = [](float v) { return __int_as_float(__viaddmin_s32_relu(__float_as_int(v), -0x4B400000, 254) << 23); };
    return mul2(y, make_float2(power(t.x), power(t.y)));
}

// Weights 2^(s * scale - ref) of a chunk, rounded to bf16, and their sum (unrounded).  POLY of its 16 pairs take the fused
// multiply-add pipe, the others the special-function unit, which is the busier of the two: both lanes' weights alone keep
// it for 2,048 of a step's cycles (8 requests, chunks of 128 behind 1,920, head_dim 128: 45.1 us with 0 pairs, 43.1 with 2, 43.0 with 3,
// 43.0 with 4; 16 + 4 heads of 64: 46.8, 45.0, 43.3, 44.4; one prompt of 16,384 in a row, where the card's power limit decides: 1,717, 1,632,
// 1,616, 1,604).
template <int POLY = 0>
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
        if (lane < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(lane == 0 ? &kv_map : &q_map) : "memory");
        for (int i = lane; i < kNumBars; i += 32) {
            const bool read = i >= kBarRead && i < kBarQFull;        // all softmax warps; a lane's
            mbar_init(bar(i), read ? kSoftmaxWarps : i >= kBarPa && i < kBarHalf ? 4u : 1u);
        }
        if (lane == 0) *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    } else if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else if (warp < kSoftmaxWarps) {
        const int spare = (kM - lane_rows) * 8 * Cfg::kHalves;                   // 16-byte chunks behind a lane's rows
        uint8_t* q_lane = qbuf + (warp >> 2) * Cfg::kQBytes;
        for (int i = tid & 127; i < spare; i += 128) {
            const int row = lane_rows + i / (8 * Cfg::kHalves), c = i % (8 * Cfg::kHalves);
            *reinterpret_cast<uint4*>(q_lane + (c >> 3) * kHalfBytes + row * 128 + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
    }
    int64_t* cum = reinterpret_cast<int64_t*>(kv + sizeof(PlanScratch));
    int32_t* lens = reinterpret_cast<int32_t*>(cum + p.n);
    prefill_plan<kStep, kThreads, true>(p, plan, cum, lens, lens + p.n);
    PrefillWalk<kStep, true> walk(p, *plan);
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
        if (walk.queued) walk.sort();
        bool more = walk.next(it);
        asm volatile("griddepcontrol.wait;" ::: "memory");               // the kernel ahead writes the counter and the rows of 8-bit pools
        while (ok) {
            // The slot's last item lies four back.  The softmax warps say when they have read it; the issuing warp has come to the
            // one two back at least (kBarQFree).
            const int slot = n_items & (kItemSlots - 1);
            if (n_items >= kItemSlots)
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarRead + slot), static_cast<uint32_t>(n_items / kItemSlots - 1) & 1u, abort_flag, p.status, limit));
            if (!ok) break;
            PrefillItem* to = items + slot;
            if (!more) it.t1 = 0;
            if (lane == 0) {
                *to = it;
                mbar_arrive(bar(kBarItem + slot));
            }
            __syncwarp();
            if (!more) break;
            const int64_t rows = static_cast<int64_t>(p.wide ? it.wide_at : it.base) * p.kv_heads +
                                 static_cast<int64_t>(it.head) * (p.wide ? (it.ctx + it.add + 15) & ~15 : it.cap);
            k_row = static_cast<int32_t>(p.k_row0 + rows);
            v_row = static_cast<int32_t>(p.v_row0 + rows);
            // a lane's queries, once its products of the item before have read theirs
            auto queries = [&](int L) {
                if (ok && n_items > 0)
                    ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarQFree + L), static_cast<uint32_t>(n_items - 1) & 1u, abort_flag, p.status, limit));
                if (!ok) return;
                const bool some = it.tok0 + L * lane_tokens < it.add;
                if (lane == 0) mbar_expect_tx(bar(kBarQFull + L), some ? static_cast<uint32_t>(Cfg::kHalves * lane_rows * 128) : 0u);
                __syncwarp();
                if (some && lane < Cfg::kHalves)
                    tma_load_3d(q_u32 + L * Cfg::kQBytes + lane * kHalfBytes, &q_map, lane * 64, it.head * p.group, it.cu + it.tok0 + L * lane_tokens,
                                bar(kBarQFull + L));
            };
            const int t0 = it.t0, t1 = it.t1;
            load(false, t0);
            queries(0);
            if (ok) load(true, t0);
            queries(1);
            ++n_items;
            for (int u = t0 + 1; u < t1 && ok; ++u) {
                load(false, u);
                if (ok) load(true, u);
            }
            more = walk.next(it);
        }
        if (lane == 0 && (!ok || *abort_flag)) {
            // something timed out: wait (bounded) for the loads in flight before shared memory is given up
            for (uint32_t i = filled > STAGES ? filled - STAGES : 0; i < filled; ++i)
                mbar_wait_slow(bar(kBarFull + i % STAGES), (i / STAGES) & 1u, nullptr, p.status, limit / 4 + 1);
            for (int L = 0; L < 2 && n_items > 0; ++L)
                mbar_wait_slow(bar(kBarQFull + L), static_cast<uint32_t>(n_items - 1) & 1u, nullptr, p.status, limit / 4 + 1);
        }
    } else if (warp == kMmaWarp) {
        // ------------------------------------------------------------------ products of both lanes
        // One warp issues them all, lane 0's PV(u) QK(u + 1) and then lane 1's: the tensor pipe takes them in this order, which
        // keeps the lanes half a step apart.  It takes few instructions ahead, so whatever this warp does between them is
        // time in which the pipe stands still.
        uint32_t elected;
        asm volatile("{\n\t.reg .pred P;\n\telect.sync _|P, 0xFFFFFFFF;\n\tselp.b32 %0, 1, 0, P;\n\t}" : "=r"(elected));
        uint32_t stage = 0, phase = 0, p_count[2] = {0, 0};
        auto wait = [&](uint32_t b, uint32_t parity) {
            if (!__all_sync(0xFFFFFFFFu, mbar_try(b, parity)))
                ok = ok && __all_sync(0xFFFFFFFFu, mbar_wait_slow(b, parity, abort_flag, p.status, limit));
        };
        auto wait_stage = [&]() {
            const uint32_t now = stage;
            wait(bar(kBarFull + stage), phase);
            if (++stage == STAGES) {
                stage = 0;
                phase ^= 1u;
            }
            return now;
        };
        const uint64_t q_desc = smem_desc(q_u32, 16, 1024), k_desc = smem_desc(kv_u32, 16, 1024), v_desc = smem_desc(kv_u32, kHalfBytes, 1024);
        // value rows between a tile's last key and the next multiple of 16: whatever the slab holds there, and 0 times
        // a NaN would not be 0
        auto clear_tail = [&](int keys, uint32_t at) {
            const int end = (keys + 15) & ~15;
            uint8_t* vb = kv + at * Cfg::kStageBytes;
            for (int i = lane; i < (end - keys) * 8 * Cfg::kHalves; i += 32) {
                const int row = keys + i / (8 * Cfg::kHalves), c = i % (8 * Cfg::kHalves);
                *reinterpret_cast<uint4*>(vb + (c >> 3) * kHalfBytes + row * 128 + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            fence_proxy_async();
            __syncwarp();
        };
        // What the products need to know of an item.
        struct Work {
            int steps, k0, tile_keys;                    // steps, the first one's first key, keys that the tile's last token sees
            int own[2], keys[2];                         // of each lane
        };
        int n_items = 0;
        auto next_item = [&](Work& w) {                  // steps = 0: there is none
            const int slot = n_items & (kItemSlots - 1);
            wait(bar(kBarItem + slot), static_cast<uint32_t>(n_items / kItemSlots) & 1u);
            ++n_items;
            w.steps = 0;
            if (!ok) return;
            const PrefillItem& it = items[slot];
            w.steps = it.t1 == 0 ? 0 : it.t1 - it.t0;
            w.k0 = it.t0 * kStep;
#pragma unroll
            for (int L = 0; L < 2; ++L) {
                w.own[L] = lane_steps(it, L);
                w.keys[L] = lane_end(it, L);
            }
            w.tile_keys = max(w.keys[0], w.keys[1]);
        };
        // S of lane L
        auto scores = [&](int L, uint32_t at) {
            const uint64_t qd = q_desc + static_cast<uint32_t>(L) * (Cfg::kQBytes >> 4), kd = k_desc + at * (Cfg::kStageBytes >> 4);
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
                umma_ss(elected, tmem + static_cast<uint32_t>(L) * 256u, qd + (((k >> 2) * kHalfBytes + (k & 3) * 32) >> 4),
                        kd + (((k >> 2) * kHalfBytes + (k & 3) * 32) >> 4), IDESC_QK, k > 0 ? 1u : 0u);
            commit(elected, bar(kBarS + L));
        };
        // The same for step u of an item; after its last the queries are handed back
        auto first = [&](int L, const Work& w, int u, uint32_t at) {
            if (u == 0) {
                wait(bar(kBarQFull + L), static_cast<uint32_t>(n_items - 1) & 1u);
                if (!ok) return;
                tc_fence_after();
            }
            if (u < w.own[L]) scores(L, at);
            if (u == max(w.own[L] - 1, 0)) commit(elected, bar(kBarQFree + L));
        };
        // O of lane L += P V of step u.  INNER: not the lane's last step, nor the tile's first.
        auto second = [&](auto inner, int L, const Work& w, int u, uint32_t at) {
            constexpr bool INNER = decltype(inner)::value;
            const uint32_t t_s = tmem + static_cast<uint32_t>(L) * 256u, t_o = t_s + 128u;
            const uint64_t vd = v_desc + at * (Cfg::kStageBytes >> 4);
            auto product = [&](int k) {                  // 16 keys
                umma_ts(elected, t_o, t_s + static_cast<uint32_t>(k * 8), vd + ((k * 2048) >> 4), IDESC_PV, (!INNER && u == 0 && k == 0) ? 0u : 1u);
            };
            const bool full = INNER || u + 1 < w.own[L];
            int slices = 8;
            wait(bar(kBarPa + L), p_count[L] & 1u);
            if (!ok) return;
            tc_fence_after();
            if (!full) {                                 // the lane's last step: as many keys as there are
                const int k0 = w.k0 + u * kStep;
                slices = (min(kStep, w.keys[L] - k0) + 15) >> 4;
                if (w.tile_keys - k0 < kStep) clear_tail(w.tile_keys - k0, at);
            }
            auto products = [&](int from) {
                if (slices >= from + 4) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) product(from + k);
                } else {
                    for (int k = from; k < slices; ++k) product(k);
                }
            };
            products(0);
            commit(elected, bar(kBarHalf + L));
            wait(bar(kBarPb + L), p_count[L] & 1u);
            if (!ok) return;
            tc_fence_after();
            products(4);
            ++p_count[L];
            if (!full) commit(elected, bar(kBarO + L));
        };
        // The steps of all items in one sequence, a lane's PV of one and QK of the next at a time: the end of a tile for
        // one lane is under way beside the other's.  Both stages are waited for ahead of the weights: between a lane's two
        // products the tensor pipe would idle.
        Work now, next;
        next_item(now);
        if (ok && now.steps > 0) {
            const uint32_t ks = wait_stage();
            if (ok) first(0, now, 0, ks);
            if (ok) first(1, now, 0, ks);
            commit(elected, bar(kBarEmpty + ks));
        }
        for (int u = 0; ok && now.steps > 0;) {
            const int inner = min(now.own[0], now.own[1]) - 2;       // both lanes have this step, the next, and one more
            while (u > 0 && u < inner) {
                const uint32_t vs = wait_stage(), ks = wait_stage();
                if (!ok) break;
                second(std::true_type(), 0, now, u, vs);
                if (!ok) break;
                scores(0, ks);
                second(std::true_type(), 1, now, u, vs);
                if (!ok) break;
                commit(elected, bar(kBarEmpty + vs));
                scores(1, ks);
                commit(elected, bar(kBarEmpty + ks));
                ++u;
            }
            if (!ok) break;
            const bool last = u + 1 == now.steps;
            next = now;
            if (last) next_item(next);
            const int v = last ? 0 : u + 1;              // the next step
            const uint32_t vs = wait_stage();
            uint32_t ks = 0;
            if (next.steps > 0) ks = wait_stage();
            if (!ok) break;
            if (u < now.own[0]) second(std::false_type(), 0, now, u, vs);
            if (ok && next.steps > 0) first(0, next, v, ks);
            if (ok && u < now.own[1]) second(std::false_type(), 1, now, u, vs);
            if (!ok) break;
            commit(elected, bar(kBarEmpty + vs));
            if (next.steps > 0) {
                first(1, next, v, ks);
                commit(elected, bar(kBarEmpty + ks));
            }
            now = next;
            u = v;
        }
        // nothing may still be running when tensor memory is given back
        commit(elected, bar(kBarDrain));
        __syncwarp();
        mbar_wait_slow(bar(kBarDrain), 0, nullptr, p.status, limit / 4 + 1);
    } else if (warp < kSoftmaxWarps) {
        // ------------------------------------------------------------------ softmax
        const int L = warp >> 2;
        const int row = (warp & 3) * 32 + lane;          // of the lane's tile
        const int row_tok = min(row / p.group, lane_tokens - 1), row_head = row % p.group;
        const uint32_t t_s = tmem + (static_cast<uint32_t>(warp & 3) << 21) + static_cast<uint32_t>(L) * 256u, t_o = t_s + 128u;
        const float scale = p.scale_log2;
        const bool out_sectors = (reinterpret_cast<uintptr_t>(p.out) & 31u) == 0;        // (16 bytes are promised)
        uint32_t s_count = 0, o_count = 0;
        for (int n_items = 0; ok; ++n_items) {
            const int slot = n_items & (kItemSlots - 1);
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarItem + slot), static_cast<uint32_t>(n_items / kItemSlots) & 1u, abort_flag, p.status, limit));
            if (!ok) break;
            const PrefillItem it = items[slot];
            if (it.t1 == 0) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kBarRead + slot));
            __syncwarp();
            const int own = lane_steps(it, L);
            const int tok = it.tok0 + L * lane_tokens + row_tok;
            const int sees = it.ctx + min(tok, it.add - 1) + 1;                  // keys of this row
            const int all_see = it.ctx + it.tok0 + L * lane_tokens + 1;          // keys of the lane's first row
            const int2 warp_sees = make_int2(__shfl_sync(0xFFFFFFFFu, sees, 0), __shfl_sync(0xFFFFFFFFu, sees, 31));     // of the warp's first and last
            float m = -INFINITY, l = 0.f;                // reference (log2 units) and sum
            for (int u = 0; u < own && ok; ++u) {
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarS + L), s_count & 1u, abort_flag, p.status, limit));
                if (!ok) break;
                tc_fence_after();
                const int k0 = (it.t0 + u) * kStep;
                const bool masked = k0 + kStep > all_see;            // some row of the lane does not see all of the step
                // The reference of the warp's rows goes up to `top` where that is higher: O and the sum, computed with the one
                // before, are scaled.  `half`: of this step, whose first product may be under way when the second raises it.
                auto raise = [&](float top, int half) {
                    const float before = m;
                    if (top > m) m = top;
                    const float f = top > before ? fast_exp2(before - m) : 1.f;
                    l *= f;
                    if (half == 0 && u == 0) return;     // nothing in O yet
                    if (half == 1) ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(kBarHalf + L), s_count & 1u, abort_flag, p.status, limit));
                    if (!ok) return;
                    tc_fence_after();
#pragma unroll 1
                    for (int k = 0; k < D / 16; ++k) {
                        uint32_t v[16];
                        tmem_ld_row16(t_o + 16u * k, v);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
                        tmem_st_row16(t_o + 16u * k, v);
                    }
                    tmem_wait_st();
                };
                auto chunk = [&](uint32_t(&x)[kChunk], int c) {      // 32 scores, those of keys that the row does not see -inf
                    tmem_ld_row32(t_s + static_cast<uint32_t>(c * kChunk), x);
                    tmem_wait_row32(x);
                    if (k0 + (c + 1) * kChunk > warp_sees.x) {
                        const int keys = sees - k0 - c * kChunk;
                        const uint32_t in = keys >= kChunk ? 0xFFFFFFFFu : keys <= 0 ? 0u : (1u << keys) - 1u;
#pragma unroll
                        for (int i = 0; i < kChunk; ++i)
                            if (!(in >> i & 1u)) x[i] = 0xFF800000u;
                    }
                };
                auto hand_over = [&](int half) {
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar((half == 0 ? kBarPa : kBarPb) + L));
                    __syncwarp();                        // the loads and stores of tensor memory want the whole warp
                };
                if (u == 0 || masked) {                  // the maximum first: there may be no reference yet
                    float top = -INFINITY;
#pragma unroll 1
                    for (int c = 0; c < kStep / kChunk; ++c) {
                        if (k0 + c * kChunk >= warp_sees.y) break;
                        uint32_t x[kChunk];
                        chunk(x, c);
                        top = fmaxf(top, row_max(x));
                    }
                    top *= scale;
                    if (__any_sync(0xFFFFFFFFu, top > m + kRaiseAbove || (m == -INFINITY && top > m))) raise(top, 0);
                    if (!ok) break;
                }
                if (masked) {
#pragma unroll 1
                    for (int c = 0; c < kStep / kChunk; ++c) {
                        uint32_t pk[kChunk / 2];
                        if (k0 + c * kChunk < warp_sees.y) {
                            uint32_t x[kChunk];
                            chunk(x, c);
                            l += weights(x, scale, m == -INFINITY ? 0.f : m, pk);
                        } else {                         // nobody sees any of it
#pragma unroll
                            for (int i = 0; i < kChunk / 2; ++i) pk[i] = 0u;
                        }
                        tmem_st_row16(t_s + 16u * c, pk);
                        if (c & 1) hand_over(c >> 1);
                    }
                } else {
                    uint32_t s[2][kChunk];
                    tmem_ld_row32(t_s, s[0]);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        uint32_t pk[2][kChunk / 2];
                        float sum = 0.f;
                        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const int c = 2 * half + k;
                            tmem_wait_row32(s[k]);
                            if (c < 3) tmem_ld_row32(t_s + static_cast<uint32_t>((c + 1) * kChunk), s[k ^ 1]);
                            sum += weights<kPolyPairs>(s[k], scale, ref, pk[k]);
                        }
                        // no reference yet, or one that is too low (or a NaN, which stays)
                        if (__any_sync(0xFFFFFFFFu, m == -INFINITY || !(sum <= kTooLarge))) {
                            float top = -INFINITY;
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                uint32_t x[kChunk];      // again from tensor memory, where P has not come yet
                                chunk(x, 2 * half + k);
                                top = fmaxf(top, row_max(x));
                            }
                            raise(top * scale, half);
                            const float up = m == -INFINITY ? 0.f : m;
                            sum = 0.f;
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                uint32_t x[kChunk];
                                chunk(x, 2 * half + k);
                                sum += weights(x, scale, up, pk[k]);
                            }
                        }
                        l += sum;
                        tmem_st_row16(t_s + 32u * half, pk[0]);
                        tmem_st_row16(t_s + 32u * half + 16u, pk[1]);
                        hand_over(half);
                    }
                }
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
            const float inv = p.v_scale / l;
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
                    if (out_sectors) {
                        store8(to, w);
                        store8(to + 32, w + 8);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            reinterpret_cast<uint4*>(to)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
                    }
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
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(p.shares));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Config<D>::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.wide || p.queue ? 1 : 0;         // behind prefill_widen_kernel or prefill_begin_kernel: set up beside it
    return cudaLaunchKernelEx(&cfg, prefill_umma_kernel<D>, kv, q, p);
}

}  // namespace

cudaError_t launch_prefill_umma(const CUtensorMap& kv, const CUtensorMap& q, const PrefillParams& p, cudaStream_t stream) {
    return p.head_dim == 128 ? launch_t<128>(kv, q, p, stream) : launch_t<64>(kv, q, p, stream);
}

}  // namespace odma
