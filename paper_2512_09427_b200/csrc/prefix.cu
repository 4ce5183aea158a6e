// Decode attention of a batch whose requests share a prefix (odma_decode_attention_prefix).
//
// For query row r = (request, query head) of KV head h, prefix keys K_P (one slab, shared) and the
// request's own keys K_i:
//     out_r = softmax([q_r . K_P^T, q_r . K_i^T] / sqrt(D)) [V_P; V_i]
// The prefix part is computed for all n * g rows of a KV head at once, so the prefix is read once (per
// tile of rows) and not once per request: per split s of its keys a row leaves (m, l, o) = (running
// maximum in log2 units, sum of 2^(x - m), unnormalised output) in the caller's workspace.  The
// requests' own parts come from the decode kernels, every piece left as a partial result.
// merge_prefix_kernel folds both with the log-sum-exp rule and rounds once.
//
//  prefix_umma_kernel      tcgen05 tensor cores (prefix_umma.cu): 16- and 8-bit slabs, head_dim 64 and 128
//  prefix_generic_kernel   plain ALUs, fp32 arithmetic: fp32 slabs, head_dim 32.  Eight rows per block share every
//                          key; small calls are a chain of latencies (4 requests, 1,000 keys, head_dim 64: the whole
//                          call 16.6 us, this kernel alone and cold 10.6)
//  dequant_prefix_kernel   8-bit slabs: the prefix's codes as bf16 (exact: a code has 4 significant
//                          bits); the scales stay outside, in the score factor and in the merge
//  merge_prefix_kernel     own pieces and prefix splits to out and lse
#include <algorithm>

#include "device_utils.cuh"
#include "odma.h"

namespace odma {
namespace {

using namespace dev;

constexpr int kRows = 8;            // query rows a block of the generic kernel carries
constexpr int kWarps = 4;
constexpr int kMergeWarps = 8;
constexpr int kBatch = 8;            // parts of a row that are under way at a time in the merge

__device__ __forceinline__ void unpack16(const uint4& v, float (&x)[4], float) {
    x[0] = __uint_as_float(v.x);
    x[1] = __uint_as_float(v.y);
    x[2] = __uint_as_float(v.z);
    x[3] = __uint_as_float(v.w);
}
__device__ __forceinline__ void unpack16(const uint4& v, float (&x)[8], __nv_bfloat16) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }

__device__ __forceinline__ void load_row(const float* p, float (&x)[1]) { x[0] = __ldcg(p); }
__device__ __forceinline__ void load_row(const float* p, float (&x)[2]) {
    const float2 v = __ldcg(reinterpret_cast<const float2*>(p));
    x[0] = v.x;
    x[1] = v.y;
}
__device__ __forceinline__ void load_row(const float* p, float (&x)[4]) {
    const float4 v = ldcg4(p);
    x[0] = v.x;
    x[1] = v.y;
    x[2] = v.z;
    x[3] = v.w;
}
__device__ __forceinline__ void store_row(float* p, const float (&x)[1]) { *p = x[0]; }
__device__ __forceinline__ void store_row(float* p, const float (&x)[2]) { *reinterpret_cast<float2*>(p) = make_float2(x[0], x[1]); }
__device__ __forceinline__ void store_row(float* p, const float (&x)[4]) { store4(p, x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void store_row(__nv_bfloat16* p, const float (&x)[1]) { *p = __float2bfloat16_rn(x[0]); }
__device__ __forceinline__ void store_row(__nv_bfloat16* p, const float (&x)[2]) { *reinterpret_cast<uint32_t*>(p) = pack_bf16(x[0], x[1]); }
__device__ __forceinline__ void store_row(__nv_bfloat16* p, const float (&x)[4]) { store4(p, x[0], x[1], x[2], x[3]); }

// Keys [first, last) of split s: the prefix's tiles of 128 keys dealt evenly.
__device__ __forceinline__ void split_range(const PrefixParams& p, int s, int& first, int& last) {
    const int tiles = (p.len + kPrefixTile - 1) / kPrefixTile;
    first = static_cast<int>(static_cast<int64_t>(tiles) * s / p.splits) * kPrefixTile;
    last = min(p.len, static_cast<int>(static_cast<int64_t>(tiles) * (s + 1) / p.splits) * kPrefixTile);
}

template <typename T, int DPL>      // head_dim = 32 * DPL
__global__ void __launch_bounds__(kWarps * 32) prefix_generic_kernel(const PrefixParams p) {
    constexpr int D = 32 * DPL;
    constexpr int VE = 16 / sizeof(T);
    __shared__ float q_s[kRows][D];
    __shared__ float p_s[kWarps][kRows][32];
    __shared__ float mrg_o[kWarps][kRows][D];
    __shared__ float mrg_ml[kWarps][kRows][2];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");      // the requests' own parts run beside this
    const int head = blockIdx.y, rows = p.n * p.group, r0 = blockIdx.x * kRows;
    int first, last;
    split_range(p, blockIdx.z, first, last);
    const T* K = static_cast<const T*>(p.k) + static_cast<int64_t>(head) * p.head_rows * D;
    const T* V = static_cast<const T*>(p.v) + static_cast<int64_t>(head) * p.head_rows * D;
    auto out_row = [&](int r) { return static_cast<int64_t>(r / p.group) * p.q_heads + head * p.group + r % p.group; };
    for (int i = tid; i < kRows * D; i += kWarps * 32) {
        const int r = r0 + i / D;
        q_s[i / D][i % D] = r < rows ? as_float(static_cast<const T*>(p.q)[out_row(r) * D + i % D]) : 0.f;
    }
    __syncthreads();
    float m[kRows], l[kRows], o[kRows][DPL];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        m[r] = -INFINITY;
        l[r] = 0.f;
#pragma unroll
        for (int c = 0; c < DPL; ++c) o[r][c] = 0.f;
    }
    for (int j0 = first + warp * 32; j0 < last; j0 += kWarps * 32) {
        const bool valid = j0 + lane < last;
        // the first value rows are asked for before the scores need their keys
        const int cnt = min(32, last - j0);
        constexpr int VB = DPL > 2 ? 8 : 16;         // value rows under way at a time
        float v[VB][DPL];
        auto values = [&](int b0) {
#pragma unroll
            for (int u = 0; u < VB; ++u)
                if (b0 + u < cnt)
#pragma unroll
                    for (int c = 0; c < DPL; ++c) v[u][c] = as_float(V[static_cast<int64_t>(j0 + b0 + u) * D + lane + 32 * c]);
        };
        values(0);
        float s[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) s[r] = 0.f;
        if (valid) {
            const uint4* kp = reinterpret_cast<const uint4*>(K + static_cast<int64_t>(j0 + lane) * D);
            constexpr int KB = D / VE < 16 ? D / VE : 16;    // vectors of the row under way at a time
            for (int v0 = 0; v0 < D / VE; v0 += KB) {
                uint4 kv[KB];
#pragma unroll
                for (int v = 0; v < KB; ++v) kv[v] = __ldg(kp + v0 + v);
#pragma unroll
                for (int v = 0; v < KB; ++v) {
                    float x[VE];
                    unpack16(kv[v], x, T());
#pragma unroll
                    for (int e = 0; e < VE; ++e)
#pragma unroll
                        for (int r = 0; r < kRows; ++r) s[r] = fmaf(q_s[r][(v0 + v) * VE + e], x[e], s[r]);
                }
            }
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const float x = valid ? s[r] * p.scale_log2 : -INFINITY;
            float mx = x;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, off));
            const float m_new = fmaxf(m[r], mx);
            // a maximum of -inf (every score so far is) contributes nothing and must not make NaN of it
            const float pr = m_new == -INFINITY ? 0.f : exp2f(x - m_new);
            const float corr = m_new == -INFINITY ? 1.f : exp2f(m[r] - m_new);
            float ps = pr;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) ps += __shfl_xor_sync(0xFFFFFFFFu, ps, off);
            l[r] = fmaf(l[r], corr, ps);
            m[r] = m_new;
#pragma unroll
            for (int c = 0; c < DPL; ++c) o[r][c] *= corr;
            p_s[warp][r][lane] = pr;
        }
        __syncwarp();
        for (int b0 = 0; b0 < cnt; b0 += VB) {
#pragma unroll
            for (int u = 0; u < VB; ++u) {
                if (b0 + u >= cnt) break;
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    const float pr = p_s[warp][r][b0 + u];
#pragma unroll
                    for (int c = 0; c < DPL; ++c) o[r][c] = fmaf(pr, v[u][c], o[r][c]);
                }
            }
            values(b0 + VB);
        }
        __syncwarp();
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
#pragma unroll
        for (int c = 0; c < DPL; ++c) mrg_o[warp][r][lane + 32 * c] = o[r][c];
        if (lane == 0) {
            mrg_ml[warp][r][0] = m[r];
            mrg_ml[warp][r][1] = l[r];
        }
    }
    __syncthreads();
    for (int i = tid; i < kRows * D; i += kWarps * 32) {
        const int r = i / D, d = i % D;
        if (r0 + r >= rows) break;
        float M = -INFINITY, L = 0.f, O = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) M = fmaxf(M, mrg_ml[w][r][0]);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float e = mrg_ml[w][r][0] == -INFINITY ? 0.f : exp2f(mrg_ml[w][r][0] - M);
            L = fmaf(mrg_ml[w][r][1], e, L);
            O = fmaf(mrg_o[w][r][d], e, O);
        }
        const int64_t at = static_cast<int64_t>(blockIdx.z) * p.n * p.q_heads + out_row(r0 + r);
        p.part_o[at * D + d] = O;
        if (d == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * at) = make_float2(M, L);
    }
}

// Codes [kv_heads][len][D] of K and V (rows of a head head_rows apart) to bf16 [2][kv_heads][pad][D].  A thread takes
// kDequant vectors of 16 codes, all loads before the first store, and the prefix's kernel sets itself up beside this
// one, which its set-up needs nothing of (47 requests, 5,001 keys, the whole call: 30.4 us with one vector and the
// kernels in a row, 29.1 to 30.5 so; 64 requests, 32,768 keys: 75.5 and 73.6).
constexpr int kDequant = 4;
__global__ void __launch_bounds__(256) dequant_prefix_kernel(const uint8_t* k, const uint8_t* v, int64_t head_rows, int len,
                                                             int pad, int kv_heads, int D, __nv_bfloat16* out) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int head = blockIdx.y % kv_heads;
    const uint8_t* src = (blockIdx.y < kv_heads ? k : v) + head * head_rows * D;
    __nv_bfloat16* dst = out + static_cast<int64_t>(blockIdx.y) * pad * D;
    const int64_t vecs = static_cast<int64_t>(len) * D / 16, step = static_cast<int64_t>(gridDim.x) * blockDim.x;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < vecs; i += kDequant * step) {
        uint4 c[kDequant];
#pragma unroll
        for (int u = 0; u < kDequant; ++u)
            if (i + u * step < vecs) c[u] = __ldg(reinterpret_cast<const uint4*>(src) + i + u * step);
#pragma unroll
        for (int u = 0; u < kDequant; ++u) {
            if (i + u * step >= vecs) break;
            const uint32_t w[4] = {c[u].x, c[u].y, c[u].z, c[u].w};
            uint32_t o[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 lo = unpack_e4m3(w[j]), hi = unpack_e4m3(w[j] >> 16);
                o[2 * j] = pack_bf16(lo.x, lo.y);
                o[2 * j + 1] = pack_bf16(hi.x, hi.y);
            }
            uint4* to = reinterpret_cast<uint4*>(dst) + 2 * (i + u * step);
            to[0] = make_uint4(o[0], o[1], o[2], o[3]);
            to[1] = make_uint4(o[4], o[5], o[6], o[7]);
        }
    }
}

// Blocks [0, n_items): the stream that begins with this item, a warp per query head.  Blocks behind
// them: the requests, for those without a token of their own.  A row's parts are the prefix's splits and
// then its own pieces, in that order, up to 32 at a time: a lane fetches one part's (m, l), the warp finds
// the maximum and every part's factor 2^(m - M), and the rows are added up, kBatch loads under way at a time
// (folded one after the other, a chain of L2 round trips, 15 parts took 13 us).
//
// Launched programmatically: a block begins once every block of the kernel ahead (the requests' own parts)
// has begun and knows the prefix's kernel complete.  So the plan and the prefix's parts, most of the
// work, are read before the wait for that kernel's end, and only the own pieces after it.
template <int V>
struct MergeRow {
    float M = -INFINITY, L = 0.f, acc[V];

    // `count` parts: rows of D floats `o_stride` apart from `o` (the lane's own elements), (m, l) pairs
    // `ml_stride` apart from `ml`; every row times `scale`.
    __device__ __forceinline__ void add(const float* o, int64_t o_stride, const float* ml, int64_t ml_stride, int parts, float scale) {
        const int lane = threadIdx.x & 31;
        for (int s0 = 0; s0 < parts; s0 += 32) {
            const int count = min(32, parts - s0);
            float2 v = make_float2(-INFINITY, 0.f);
            if (lane < count) v = __ldcg(reinterpret_cast<const float2*>(ml + (s0 + lane) * ml_stride));
            float x[kBatch][V];
#pragma unroll
            for (int k = 0; k < kBatch; ++k)
                if (k < count) load_row(o + (s0 + k) * o_stride, x[k]);
            float top = fmaxf(M, v.x);
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
            const float e = v.x == -INFINITY ? 0.f : fast_exp2(v.x - top), old = M == -INFINITY ? 0.f : fast_exp2(M - top);
            float sum = v.y * e;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
            L = fmaf(L, old, sum);
            M = top;
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] *= old;
            const float f = e * scale;
            for (int k0 = 0; k0 < count; k0 += kBatch) {
#pragma unroll
                for (int k = 0; k < kBatch; ++k) {
                    const float w = __shfl_sync(0xFFFFFFFFu, f, (k0 + k) & 31);
                    if (k0 + k < count)
#pragma unroll
                        for (int i = 0; i < V; ++i) acc[i] = fmaf(x[k][i], w, acc[i]);
                }
#pragma unroll
                for (int k = 0; k < kBatch; ++k)
                    if (k0 + kBatch + k < count) load_row(o + (s0 + k0 + kBatch + k) * o_stride, x[k]);
            }
        }
    }
};

template <typename T, int V>        // head_dim = 32 * V
__global__ void __launch_bounds__(kMergeWarps * 32) merge_prefix_kernel(const MergePrefixParams p) {
    constexpr int D = 32 * V;
    int req, head, heads = 1, slot0 = 0, pieces = 0;
    if (static_cast<int>(blockIdx.x) < p.n_items) {
        const int4 a = __ldg(p.items + 2 * blockIdx.x), b = __ldg(p.items + 2 * blockIdx.x + 1);
        if (a.x < 0 || a.z != 0) return;               // unused, or not a stream's first piece
        req = a.x;
        head = a.y;
        slot0 = b.y;
        pieces = b.w < 0 ? 1 : __ldg(p.combine + b.w).w;
    } else {
        req = static_cast<int>(blockIdx.x) - p.n_items;
        if (__ldg(p.len + req) > 0) return;
        head = 0;
        heads = p.kv_heads;
    }
    const int lane = threadIdx.x & 31;
    const int64_t split_rows = static_cast<int64_t>(p.n) * p.q_heads;
    for (int g = threadIdx.x >> 5; g < heads * p.group; g += kMergeWarps) {
        const int64_t row = static_cast<int64_t>(req) * p.q_heads + head * p.group + g;
        const int64_t own_row = static_cast<int64_t>(slot0) * p.group + g;
        MergeRow<V> r;
#pragma unroll
        for (int i = 0; i < V; ++i) r.acc[i] = 0.f;
        r.add(p.part_o + row * D + lane * V, split_rows * D, p.part_ml + 2 * row, 2 * split_rows, p.splits, p.v_scale);
        asm volatile("griddepcontrol.wait;" ::: "memory");
        r.add(p.own_o + own_row * D + lane * V, static_cast<int64_t>(p.group) * D, p.own_ml + 2 * own_row, 2ll * p.group, pieces, 1.f);
        const float inv = r.L > 0.f ? 1.f / r.L : (r.L == 0.f ? 0.f : r.L);      // no key at all: zeros
#pragma unroll
        for (int i = 0; i < V; ++i) r.acc[i] *= inv;
        store_row(static_cast<T*>(p.out) + row * D + lane * V, r.acc);
        if (lane == 0 && p.lse) p.lse[row] = r.L == 0.f ? -INFINITY : (r.M + log2f(r.L)) * 0.6931471805599453f;
    }
}

template <typename T>
cudaError_t launch_generic_t(const PrefixParams& p, cudaStream_t s) {
    const dim3 grid(static_cast<unsigned>((p.n * p.group + kRows - 1) / kRows), static_cast<unsigned>(p.kv_heads),
                    static_cast<unsigned>(p.splits));
    if (p.head_dim == 32) {
        prefix_generic_kernel<T, 1><<<grid, kWarps * 32, 0, s>>>(p);
    } else if constexpr (sizeof(T) == 4) {            // wider 16-bit rows: prefix_umma_kernel
        if (p.head_dim == 64)
            prefix_generic_kernel<T, 2><<<grid, kWarps * 32, 0, s>>>(p);
        else if (p.head_dim == 128)
            prefix_generic_kernel<T, 4><<<grid, kWarps * 32, 0, s>>>(p);
        else
            return cudaErrorInvalidValue;
    } else {
        return cudaErrorInvalidValue;
    }
    return cudaGetLastError();
}

}  // namespace

// Blocks along the prefix's keys: the number that minimises (waves of blocks) x (a block's time) + (what the
// partial results cost), by measured figures in ns.  Tensor cores (one block per SM): 6,500 for a block's set-up,
// queries and hand-over, and per step of 64 keys 1,100 with two row tiles, 900 with one; when one row tile's steps
// go to the two lanes in turn, 7,500 and 750 (it pays from four tiles of 128 keys per block on: 3 requests, 777
// keys, 2 blocks: 14.1 us against 14.4; 7 blocks: 12.4 against 11.0).  Plain ALUs (8 rows, blocks_per_sm of them on an
// SM): 3,000 and 5,000 per tile of 128 keys.  A row's partial result costs its write and its read in the merge, 0.2.
PrefixSplit prefix_split(int32_t rows, int32_t q_rows, int32_t kv_heads, int32_t len, int32_t sms, int32_t blocks_per_sm, bool tensor) {
    const int64_t tiles = (len + kPrefixTile - 1) / kPrefixTile;
    const int64_t blocks = kv_heads * static_cast<int64_t>(tensor ? (rows + 255) / 256 : (rows + kRows - 1) / kRows);
    const int64_t room = static_cast<int64_t>(blocks_per_sm) * sms;
    PrefixSplit best{1, 0};
    int64_t least = INT64_MAX;
    for (int32_t s = 1; s <= std::min<int64_t>(tiles, kMaxPrefixSplits); ++s) {
        const int64_t waves = (blocks * s + room - 1) / room, each = (tiles + s - 1) / s;
        for (int32_t turn = 0; turn <= (tensor && rows <= 128 ? 1 : 0); ++turn) {
            const int64_t block = !tensor ? 3000 + 5000 * each
                                  : turn    ? 7500 + 2 * each * 750
                                            : 6500 + 2 * each * (rows <= 128 ? 900 : 1100);
            const int64_t parts = turn ? 2 * s : s, cost = waves * block + parts * q_rows / 5;
            if (cost < least) {
                least = cost;
                best = PrefixSplit{static_cast<int32_t>(parts), turn};
            }
        }
    }
    return best;
}

// Blocks of prefix_generic_kernel that an SM holds: the runtime's answer, or what it is on sm_100a where there is no device
// to ask (122 to 126 registers at head_dim 32, 150 and 156 at 64 and 128).
int32_t prefix_generic_blocks(bool fp32, int32_t head_dim, bool ask) {
    int blocks = 0;
    cudaError_t e = cudaErrorNotSupported;
    if (ask) {
        const void* kernel = !fp32            ? reinterpret_cast<const void*>(&prefix_generic_kernel<__nv_bfloat16, 1>)
                             : head_dim == 32 ? reinterpret_cast<const void*>(&prefix_generic_kernel<float, 1>)
                             : head_dim == 64 ? reinterpret_cast<const void*>(&prefix_generic_kernel<float, 2>)
                                              : reinterpret_cast<const void*>(&prefix_generic_kernel<float, 4>);
        e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&blocks, kernel, kWarps * 32, 0);
        if (e != cudaSuccess) cudaGetLastError();      // not the next launch's
    }
    return e == cudaSuccess && blocks > 0 ? blocks : head_dim == 32 ? 4 : 3;
}

cudaError_t launch_prefix(const PrefixParams& p, bool fp32, cudaStream_t stream) {
    if (p.splits < 1 || p.len < 1) return cudaSuccess;
    return fp32 ? launch_generic_t<float>(p, stream) : launch_generic_t<__nv_bfloat16>(p, stream);
}

cudaError_t launch_dequant_prefix(const void* k, const void* v, int64_t head_rows, int32_t len, int32_t pad,
                                  int32_t kv_heads, int32_t head_dim, void* out, cudaStream_t stream) {
    const int64_t blocks = (static_cast<int64_t>(len) * head_dim / 16 + 256 * kDequant - 1) / (256 * kDequant);
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(blocks, 256)), static_cast<unsigned>(2 * kv_heads));
    dequant_prefix_kernel<<<grid, 256, 0, stream>>>(static_cast<const uint8_t*>(k), static_cast<const uint8_t*>(v), head_rows, len,
                                                    pad, kv_heads, head_dim, static_cast<__nv_bfloat16*>(out));
    return cudaGetLastError();
}

namespace {
// Launched with programmatic stream serialization: the blocks are there when the kernel ahead ends.
template <typename T, int V>
cudaError_t launch_merge_t(const MergePrefixParams& p, cudaStream_t stream) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(p.n_items + p.n));
    cfg.blockDim = dim3(kMergeWarps * 32);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, merge_prefix_kernel<T, V>, p);
}
}  // namespace

cudaError_t launch_merge_prefix(const MergePrefixParams& p, bool fp32, cudaStream_t stream) {
    switch (p.head_dim) {
        case 32: return fp32 ? launch_merge_t<float, 1>(p, stream) : launch_merge_t<__nv_bfloat16, 1>(p, stream);
        case 64: return fp32 ? launch_merge_t<float, 2>(p, stream) : launch_merge_t<__nv_bfloat16, 2>(p, stream);
        case 128: return fp32 ? launch_merge_t<float, 4>(p, stream) : launch_merge_t<__nv_bfloat16, 4>(p, stream);
    }
    return cudaErrorInvalidValue;
}

}  // namespace odma
