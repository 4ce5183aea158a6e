// Causal attention of a step's new tokens over the slabs (odma_prefill_attention).
//
// Request i has c tokens in its slab before the step and a new ones behind them (already appended).  For its new
// token t and query head of KV head h, with the slab's keys and values K, V
//     out = softmax_{k <= c + t}(q . K[k] / sqrt(D)) V[k]
// The query rows of a tile (tokens x heads of the group) share every key, so K and V are read once per tile, and the
// softmax is taken in one pass: per row a reference m (log2 units), the sum l of 2^(x - m) and the unnormalised O.
//
//  prefill_umma_kernel     tcgen05 tensor cores (prefill_umma.cu): 16- and 8-bit slabs, head_dim 64 and 128
//  prefill_plain_kernel    plain ALUs, fp32 arithmetic: fp32 slabs, head_dim 32.  64 query rows and 64 keys in
//                          shared memory, 4 x 4 scores and 4 rows of O per thread in registers.  Bound by shared memory's
//                          reads beside the multiply-adds (8 vectors for 64 of them; larger tiles per thread would read less), and
//                          nothing runs beside a step's loads: 30 TFLOP/s (1,024 tokens behind 2,000, fp32, 4 + 2 heads of 128: 168 to 173 us;
//                          shared memory 65 % busy, the multiply-add pipe 50 %; heads of 64: 94 us, 68 and 50 %)
//  prefill_widen_kernel    8-bit slabs: the codes of the requests with new tokens as bf16 (exact: a code has 4 significant
//                          bits); the scales stay outside, in the score factor and in the result.  Bound by memory: 1 byte
//                          in and 2 out per element, 31 MB of 30,510 tokens of 4 heads of 128 to 62 MB: 15.3 us cold (6.1 TB/s)
//  prefill_merge_kernel    tiles that were cut between blocks: their pieces to out and lse, with the log-sum-exp rule.  4 us
//                          where nothing was cut, 12.6 for 509 tokens' 15 x 4 tiles in 148 pieces (cold)
//  prefill_begin_kernel    zeroes the counter that tiles are taken from, where there may be one
#include <algorithm>

#include "odma.h"
#include "prefill_plan.cuh"

namespace odma {
namespace {

using namespace dev;

// ---- plain ALUs

constexpr int kRows = kPrefillPlainRows, kKeys = kPrefillPlainStep;
constexpr int kPlainThreads = 256;                  // 16 x 16: four rows (ty + 16 i) by four keys (tx + 16 j) each

__device__ __forceinline__ float4 load4(const float* p) { return __ldg(reinterpret_cast<const float4*>(p)); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
    const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
    return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16),
                       __uint_as_float(v.y & 0xFFFF0000u));
}

template <int D>
struct PlainShared {
    PlanScratch plan;
    float q[kRows][D + 4];          // rows 16 bytes apart modulo 128: sixteen of them are read without conflicts
    float k[kKeys][D + 4];
    float v[kKeys][D];
    float p[kRows][kKeys + 4];
};
// the plan's words lie over the rows
template <int D>
constexpr int plain_smem() {
    constexpr int rows = static_cast<int>(sizeof(PlainShared<D>)), plan = static_cast<int>(sizeof(PlanScratch)) + kMaxPrefillBatch * 12;
    return rows > plan ? rows : plan;
}
static_assert(sizeof(PlanScratch) % 16 == 0, "rows of vectors lie behind it");
// Blocks that an SM holds: two, where its 228 KB of shared memory have room for them and for the 1 KB that each takes beside its own (not at
// head_dim 128, where a share per block more would be a second wave: 178 us instead of 168 for 1,024 tokens behind 2,000, 4 + 2 heads).
template <int D>
constexpr int plain_blocks() {
    return 2 * (plain_smem<D>() + 1024) <= 228 * 1024 ? 2 : 1;
}

template <typename T, int D>
__global__ void __launch_bounds__(kPlainThreads, plain_blocks<D>()) prefill_plain_kernel(const PrefillParams p) {
    extern __shared__ __align__(16) uint8_t smem_raw[];
    PlainShared<D>& sm = *reinterpret_cast<PlainShared<D>*>(smem_raw);
    constexpr int OC = D / 16;                      // O columns of a thread: tx * CW + 16 * CW * c + e
    constexpr int CW = OC < 4 ? OC : 4;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    int64_t* cum = reinterpret_cast<int64_t*>(smem_raw + sizeof(PlanScratch));
    prefill_plan<kKeys, kPlainThreads, false>(p, &sm.plan, cum, reinterpret_cast<int32_t*>(cum + p.n), nullptr);
    PrefillWalk<kKeys, false> walk(p, sm.plan);
    const T* pool = static_cast<const T*>(p.pool);
    const T* Q = static_cast<const T*>(p.q);
    PrefillItem it;
    while (walk.next(it)) {
        const T* K = pool + (p.k_row0 + static_cast<int64_t>(it.base) * p.kv_heads + static_cast<int64_t>(it.head) * it.cap) * D;
        const T* V = K + static_cast<int64_t>(p.v_row0 - p.k_row0) * D;
        const int tokens = min(p.tile_tokens, it.add - it.tok0), rows = tokens * p.group;
        const int last = it.ctx + it.tok0 + tokens;  // keys that the tile's last token sees
        auto row_at = [&](int r) { return static_cast<int64_t>(it.cu + it.tok0 + r / p.group) * p.q_heads + it.head * p.group + r % p.group; };
        __syncthreads();                             // the plan's words, the item before
        for (int i = tid; i < kRows * (D / 4); i += kPlainThreads) {
            const int r = i / (D / 4), c = i % (D / 4);
            const float4 x = r < rows ? load4(Q + row_at(r) * D + 4 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
            *reinterpret_cast<float4*>(&sm.q[r][4 * c]) = x;
        }
        float m[4], l[4], o[4][OC];
        int sees[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m[i] = -INFINITY;
            l[i] = 0.f;
            sees[i] = it.ctx + it.tok0 + min(ty + 16 * i, rows - 1) / p.group + 1;
#pragma unroll
            for (int c = 0; c < OC; ++c) o[i][c] = 0.f;
        }
        for (int u = it.t0; u < it.t1; ++u) {
            const int k0 = u * kKeys, count = min(kKeys, last - k0);
            __syncthreads();                         // the step before has been read
            for (int i = tid; i < kKeys * (D / 4); i += kPlainThreads) {
                const int r = i / (D / 4), c = i % (D / 4);
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;       // rows behind the last key: zero
                if (r < count) {
                    x = load4(K + static_cast<int64_t>(k0 + r) * D + 4 * c);
                    y = load4(V + static_cast<int64_t>(k0 + r) * D + 4 * c);
                }
                *reinterpret_cast<float4*>(&sm.k[r][4 * c]) = x;
                *reinterpret_cast<float4*>(&sm.v[r][4 * c]) = y;
            }
            __syncthreads();
            float s[4][4] = {};
#pragma unroll 4
            for (int d = 0; d < D; d += 4) {
                float4 a[4], b[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4*>(&sm.q[ty + 16 * i][d]);
#pragma unroll
                for (int j = 0; j < 4; ++j) b[j] = *reinterpret_cast<const float4*>(&sm.k[tx + 16 * j][d]);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        s[i][j] = fmaf(a[i].x, b[j].x, s[i][j]);
                        s[i][j] = fmaf(a[i].y, b[j].y, s[i][j]);
                        s[i][j] = fmaf(a[i].z, b[j].z, s[i][j]);
                        s[i][j] = fmaf(a[i].w, b[j].w, s[i][j]);
                    }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float top = -INFINITY;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s[i][j] = k0 + tx + 16 * j < sees[i] ? s[i][j] * p.scale_log2 : -INFINITY;
                    top = fmaxf(top, s[i][j]);
                }
#pragma unroll
                for (int off = 8; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, off));
                const float m_new = fmaxf(m[i], top);
                // a maximum of -inf (every key so far is hidden) contributes nothing and must not make NaN of it
                const float ref = m_new == -INFINITY ? 0.f : m_new;
                const float corr = exp2f(m[i] - ref);
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float w = exp2f(s[i][j] - ref);
                    sum += w;
                    sm.p[ty + 16 * i][tx + 16 * j] = w;
                }
#pragma unroll
                for (int off = 8; off > 0; off >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off);
                l[i] = fmaf(l[i], corr, sum);
                m[i] = m_new;
#pragma unroll
                for (int c = 0; c < OC; ++c) o[i][c] *= corr;
            }
            __syncwarp();                            // a row's weights come from its own half warp
#pragma unroll 2
            for (int k = 0; k < kKeys; k += 4) {
                float4 w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const float4*>(&sm.p[ty + 16 * i][k]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float v[OC];
#pragma unroll
                    for (int c = 0; c < OC; ++c) v[c] = sm.v[k + e][(c / CW) * 16 * CW + tx * CW + c % CW];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float x = e == 0 ? w[i].x : e == 1 ? w[i].y : e == 2 ? w[i].z : w[i].w;
#pragma unroll
                        for (int c = 0; c < OC; ++c) o[i][c] = fmaf(x, v[c], o[i][c]);
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = ty + 16 * i;
            if (r >= rows) continue;
            if (it.slot >= 0) {
                const int64_t at = static_cast<int64_t>(it.slot) * p.part_rows + r;
#pragma unroll
                for (int c = 0; c < OC; ++c) p.part_o[at * D + (c / CW) * 16 * CW + tx * CW + c % CW] = o[i][c];
                if (tx == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * at) = make_float2(m[i], l[i]);
            } else {
                const int64_t at = row_at(r);
                const float inv = 1.f / l[i];
#pragma unroll
                for (int c = 0; c < OC; ++c)
                    static_cast<T*>(p.out)[at * D + (c / CW) * 16 * CW + tx * CW + c % CW] = static_cast<T>(o[i][c] * inv);
                if (tx == 0 && p.lse) p.lse[at] = (m[i] + log2f(l[i])) * 0.6931471805599453f;
            }
        }
    }
}

template <typename T, int D>
cudaError_t launch_plain_t(const PrefillParams& p, cudaStream_t stream) {
    static bool configured[64] = {false};             // the opt-in to large shared memory is per device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!configured[dev]) {
        e = cudaFuncSetAttribute(prefill_plain_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, plain_smem<D>());
        if (e != cudaSuccess) return e;
        configured[dev] = true;
    }
    prefill_plain_kernel<T, D><<<static_cast<unsigned>(p.shares), kPlainThreads, plain_smem<D>(), stream>>>(p);
    return cudaGetLastError();
}

// ---- 8-bit pools

// The counter that blocks take tiles from, for the kernel behind it, which is set up meanwhile.
__global__ void prefill_begin_kernel(uint32_t* queue) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    *queue = 0u;
}

// Rows [0, len) of every head, K and V, of the requests with new tokens to the place that the plan gives them: blockIdx.y the
// request, blockIdx.z the array and head; a thread takes kWiden vectors of 16 codes, all loads before the first
// store, each to 32 bytes in one instruction (in two, half sectors at a time: 24.5 us instead of 15.3).
constexpr int kWiden = 4;
__global__ void __launch_bounds__(256) prefill_widen_kernel(const PrefillParams p) {
    __shared__ int64_t sums[8];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (p.queue && blockIdx.x + blockIdx.y + blockIdx.z + threadIdx.x == 0) *p.queue = 0u;
    const int i = blockIdx.y, len = __ldg(p.len + i), D = p.head_dim;
    if (prefill_new(p, i, len) == 0) return;
    int64_t before = 0;                              // tokens of the requests ahead
    for (int k = threadIdx.x; k < i; k += 256) {
        const int n = __ldg(p.len + k);
        if (prefill_new(p, k, n) > 0) before += (n + 15) & ~15;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) before += __shfl_xor_sync(0xFFFFFFFFu, before, o);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = before;
    __syncthreads();
    before = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) before += sums[w];
    const int pad = (len + 15) & ~15;
    if (before + pad > p.wide_tokens) {              // slabs that overlap: not all of them fit
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(p.status, kStatusOverflow);
        return;
    }
    const int h = blockIdx.z >> 1, is_v = blockIdx.z & 1;
    const int64_t vecs = static_cast<int64_t>(len) * D / 16, step = static_cast<int64_t>(gridDim.x) * 256;
    const int64_t slab = static_cast<int64_t>(__ldg(p.base + i)) * p.kv_heads, cap = __ldg(p.cap + i);
    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(p.pool) + ((is_v ? p.v_row0 : p.k_row0) + slab + h * cap) * D);
    uint4* dst = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.wide) +
                                          ((is_v * p.wide_tokens + before) * p.kv_heads + static_cast<int64_t>(h) * pad) * D);
    for (int64_t v = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; v < vecs; v += kWiden * step) {
        uint4 c[kWiden];
#pragma unroll
        for (int u = 0; u < kWiden; ++u)
            if (v + u * step < vecs) c[u] = __ldg(src + v + u * step);
#pragma unroll
        for (int u = 0; u < kWiden; ++u) {
            if (v + u * step >= vecs) break;
            const uint32_t w[4] = {c[u].x, c[u].y, c[u].z, c[u].w};
            uint32_t o[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 lo = unpack_e4m3(w[j]), hi = unpack_e4m3(w[j] >> 16);
                o[2 * j] = pack_bf16(lo.x, lo.y);
                o[2 * j + 1] = pack_bf16(hi.x, hi.y);
            }
            store8(dst + 2 * (v + u * step), o);
        }
    }
}

// ---- tiles cut between blocks

constexpr int kMergeWarps = 8;

__device__ __forceinline__ bool same_tile(const int4& a, const int4& b) { return a.x == b.x && a.y == b.y && a.z == b.z; }

template <int V>
struct RowPart {
    float2 ml;
    float x[V];
    __device__ __forceinline__ void load(const PrefillParams& p, int64_t at, int lane) {
        ml = __ldcg(reinterpret_cast<const float2*>(p.part_ml + 2 * at));
        const float* from = p.part_o + (at * 32 + lane) * V;
        if constexpr (V == 4) {
            const float4 v = ldcg4(from);
            x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
        } else if constexpr (V == 2) {
            const float2 v = __ldcg(reinterpret_cast<const float2*>(from));
            x[0] = v.x, x[1] = v.y;
        } else {
            x[0] = __ldcg(from);
        }
    }
};

// The rows of all cut tiles, dealt to the warps of the grid; a warp takes a row, kUnder pieces under way at a time.  If share s
// begins inside a tile and is the first to do so, the tile's pieces are those of share s - 1 (its last), s, s + 1, ... up to
// the one that ends the tile.  Launched programmatically: a block is there when the kernel ahead ends.
template <typename T, int V>        // head_dim = 32 * V
__global__ void __launch_bounds__(kMergeWarps * 32) prefill_merge_kernel(const PrefillParams p) {
    constexpr int kUnder = 4;
    extern __shared__ int4 start[];                  // [shares + 1]
    int32_t* tile = reinterpret_cast<int32_t*>(start + p.shares + 1);        // shares that are the first to cut their tile
    __shared__ int tiles;
    const int tid = threadIdx.x, lane = tid & 31;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int i = tid; i <= p.shares; i += kMergeWarps * 32) start[i] = __ldcg(p.starts + i);
    __syncthreads();
    if (tid < 32) {
        int n = 0;
        for (int s0 = 1; s0 < p.shares; s0 += 32) {
            const int s = s0 + lane;
            bool cut = s < p.shares && start[s].w > 0 && start[s].x < p.n;
            cut = cut && !(start[s - 1].w > 0 && same_tile(start[s - 1], start[s]));
            const uint32_t all = __ballot_sync(0xFFFFFFFFu, cut);
            if (cut) tile[n + __popc(all & ((1u << lane) - 1u))] = s;
            n += __popc(all);
        }
        if (lane == 0) tiles = n;
    }
    __syncthreads();
    const int work = tiles * p.part_rows;
    for (int i = static_cast<int>(blockIdx.x) * kMergeWarps + (tid >> 5); i < work; i += static_cast<int>(gridDim.x) * kMergeWarps) {
        const int s = tile[i / p.part_rows], r = i % p.part_rows;
        const int4 c = start[s];
        const int add = prefill_new(p, c.x, __ldg(p.len + c.x)), tok0 = c.z * p.tile_tokens, cu = __ldg(p.cu_new + c.x);
        if (r >= min(p.tile_tokens, add - tok0) * p.group) continue;
        float M = -INFINITY, L = 0.f, acc[V];
#pragma unroll
        for (int k = 0; k < V; ++k) acc[k] = 0.f;
        bool more = true;
        for (int k0 = 0; more; k0 += 32) {           // piece 0: of share s - 1
            const int k = s + k0 + lane;             // the share behind the piece's
            // (an empty share, between two equal cuts, has none)
            const bool in = k <= p.shares && (k == s || (k - 1 < p.shares && start[k - 1].w > 0 && same_tile(start[k - 1], c)));
            const bool none = in && k > s && same_tile(start[k - 1], start[k]) && start[k - 1].w == start[k].w;
            const int slot = !in || none ? -1 : k == s ? 2 * s - 1 : 2 * (k - 1);
            const uint32_t all = __ballot_sync(0xFFFFFFFFu, in);
            more = all == 0xFFFFFFFFu;
            const int count = more ? 32 : __ffs(~all) - 1;
            for (int j0 = 0; j0 < count; j0 += kUnder) {
                RowPart<V> part[kUnder];
                int from[kUnder];
#pragma unroll
                for (int j = 0; j < kUnder; ++j) {
                    from[j] = __shfl_sync(0xFFFFFFFFu, slot, (j0 + j) & 31);
                    if (j0 + j >= count) from[j] = -1;
                    if (from[j] >= 0) part[j].load(p, static_cast<int64_t>(from[j]) * p.part_rows + r, lane);
                }
#pragma unroll
                for (int j = 0; j < kUnder; ++j) {
                    if (from[j] < 0 || part[j].ml.y == 0.f) continue;    // (a piece whose keys the row does not see has no sum)
                    const float top = fmaxf(M, part[j].ml.x);
                    const float a = M == -INFINITY ? 0.f : fast_exp2(M - top), b = part[j].ml.x == -INFINITY ? 1.f : fast_exp2(part[j].ml.x - top);
                    L = fmaf(L, a, part[j].ml.y * b);
                    M = top;
#pragma unroll
                    for (int e = 0; e < V; ++e) acc[e] = fmaf(acc[e], a, part[j].x[e] * b);
                }
            }
        }
        const float inv = p.v_scale / L;
        const int64_t row = static_cast<int64_t>(cu + tok0 + r / p.group) * p.q_heads + c.y * p.group + r % p.group;
        T* to = static_cast<T*>(p.out) + (row * 32 + lane) * V;
#pragma unroll
        for (int k = 0; k < V; ++k) acc[k] *= inv;
        if constexpr (V == 4)
            store4(to, acc[0], acc[1], acc[2], acc[3]);
        else
#pragma unroll
            for (int k = 0; k < V; ++k) to[k] = static_cast<T>(acc[k]);
        if (lane == 0 && p.lse) p.lse[row] = (M + log2f(L)) * 0.6931471805599453f;
    }
}

template <typename T, int V>
cudaError_t launch_merge_t(const PrefillParams& p, cudaStream_t stream) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(std::min(4 * p.shares, (p.shares * p.part_rows + kMergeWarps - 1) / kMergeWarps)));
    cfg.blockDim = dim3(kMergeWarps * 32);
    cfg.dynamicSmemBytes = static_cast<size_t>(p.shares + 1) * 20;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, prefill_merge_kernel<T, V>, p);
}

}  // namespace

int32_t prefill_plain_blocks(int32_t head_dim) { return head_dim == 32 ? plain_blocks<32>() : head_dim == 64 ? plain_blocks<64>() : plain_blocks<128>(); }

cudaError_t launch_prefill_plain(const PrefillParams& p, bool fp32, cudaStream_t stream) {
    if (p.head_dim == 32) return fp32 ? launch_plain_t<float, 32>(p, stream) : launch_plain_t<__nv_bfloat16, 32>(p, stream);
    if (!fp32) return cudaErrorInvalidValue;         // wider 16-bit rows: prefill_umma_kernel
    return p.head_dim == 64 ? launch_plain_t<float, 64>(p, stream) : p.head_dim == 128 ? launch_plain_t<float, 128>(p, stream) : cudaErrorInvalidValue;
}

cudaError_t launch_prefill_begin(const PrefillParams& p, cudaStream_t stream) {
    prefill_begin_kernel<<<1, 1, 0, stream>>>(p.queue);
    return cudaGetLastError();
}

cudaError_t launch_prefill_widen(const PrefillParams& p, cudaStream_t stream) {
    // some blocks per SM in all, whatever the number of requests (their lengths are the device's)
    const int columns = p.n * 2 * p.kv_heads;
    const dim3 grid(static_cast<unsigned>(std::max(1, std::min(256, 1184 / columns))), static_cast<unsigned>(p.n), static_cast<unsigned>(2 * p.kv_heads));
    prefill_widen_kernel<<<grid, 256, 0, stream>>>(p);
    return cudaGetLastError();
}

cudaError_t launch_prefill_merge(const PrefillParams& p, bool fp32, cudaStream_t stream) {
    switch (p.head_dim) {
        case 32: return fp32 ? launch_merge_t<float, 1>(p, stream) : launch_merge_t<__nv_bfloat16, 1>(p, stream);
        case 64: return fp32 ? launch_merge_t<float, 2>(p, stream) : launch_merge_t<__nv_bfloat16, 2>(p, stream);
        case 128: return fp32 ? launch_merge_t<float, 4>(p, stream) : launch_merge_t<__nv_bfloat16, 4>(p, stream);
    }
    return cudaErrorInvalidValue;
}

}  // namespace odma
