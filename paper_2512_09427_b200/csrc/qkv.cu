// What lies between the projections of a layer and its attention, in one pass (odma_append_qkv): the
// norm of every query and key head, the rotation by position, and the append of the new keys and
// values to the slabs.
//
// For a head x of D elements with weight w, position(s) of its token and pair frequencies f:
//     y = x / sqrt(mean(x^2) + eps) * w                                  (when a weight is given)
//     (z_a, z_b) = (y_a cos t - y_b sin t, y_b cos t + y_a sin t),  t = position[axis(i)] * f_i
// for the i-th pair (a, b) of the first rot_dim elements; the rest passes through.  Everything is
// fp32 and rounded once, to the io type (queries, 16- and 32-bit slabs) or to the E4M3 code of z * (1 /
// scale).  The angle is taken in fp64 and reduced by whole turns before its sine and cosine are taken
// in fp32: a position of 10^6 times an fp32 frequency keeps no digits of the turn in 32 bits.
//
// Each input element is read once and each output element written once: a chunk of 8,192 tokens of the
// 28 + 4 + 4-head layer moves 151 MB, 23.4 us at the measured copy rate; the kernel takes 35.8 us (4.2 TB/s).
// Neither the memory nor instruction issue (59 % of the slots) is full: a block's way to its first store
// (owner, length, angle, barrier) is the rest.  A row of 128 elements over 16 lanes of eight took 245
// instructions per warp and 43 us, over 8 lanes of sixteen, with a token's addresses, turns and weights in
// registers and packed arithmetic, 35.8.  Into an 8-bit pool (143 MB, 22.1 us) it takes 34.3.  One token, or 256: 3.0
// and 3.8 us, a chain of latencies (owner, position, angle, row).  A token's rot_dim / 2 sines and cosines are
// computed once, into shared memory, under the latency of the first row loads, and serve all its heads.
// A row is held by D / 16 (D / 8) lanes, laid out so that both elements of a pair sit in the same lane
// (pairs (i, i + rot_dim / 2): a run of eight (four) of each half; adjacent pairs: a run of twice that);
// the norm's sum is a shuffle tree over those lanes.
#include "device_utils.cuh"

namespace odma {
namespace {

using namespace dev;

constexpr int kMaxThreads = 384;
// Tokens per block: one while that fills the GPU (a token's way through a block, some 3 us, is all a small step costs),
// several for more, whose rows then stream behind one another (chunk of 8,192: 50 us with one per block, 43 with four).
constexpr int kTokens = 4, kManyTokens = 1024, kManyThreads = 128, kManyBlocks = 5;

// N consecutive elements of a row, in pairs of two.
template <typename T, int N>
struct Run;
template <>
struct Run<float, 4> {
    typedef float4 Raw;
    __device__ static void unpack(const Raw& r, float2 (&x)[2]) {
        x[0] = make_float2(r.x, r.y);
        x[1] = make_float2(r.z, r.w);
    }
    __device__ static Raw pack(const float2 (&x)[2]) { return make_float4(x[0].x, x[0].y, x[1].x, x[1].y); }
};
__device__ __forceinline__ float2 bf16_pair(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
template <>
struct Run<__nv_bfloat16, 4> {
    typedef uint2 Raw;
    __device__ static void unpack(const Raw& r, float2 (&x)[2]) {
        x[0] = bf16_pair(r.x);
        x[1] = bf16_pair(r.y);
    }
    __device__ static Raw pack(const float2 (&x)[2]) { return make_uint2(pack_bf16(x[0].x, x[0].y), pack_bf16(x[1].x, x[1].y)); }
};
template <>
struct Run<__nv_bfloat16, 8> {
    typedef uint4 Raw;
    __device__ static void unpack(const Raw& r, float2 (&x)[4]) {
        x[0] = bf16_pair(r.x);
        x[1] = bf16_pair(r.y);
        x[2] = bf16_pair(r.z);
        x[3] = bf16_pair(r.w);
    }
    __device__ static Raw pack(const float2 (&x)[4]) {
        return make_uint4(pack_bf16(x[0].x, x[0].y), pack_bf16(x[1].x, x[1].y), pack_bf16(x[2].x, x[2].y), pack_bf16(x[3].x, x[3].y));
    }
};
// The elements times `inv` in fp32, as E4M3 codes
template <int H>
__device__ __forceinline__ void store_codes(uint8_t* dst, const float2 (&z)[H], float inv) {
    uint32_t c[H / 2];
#pragma unroll
    for (int i = 0; i < H / 2; ++i)
        c[i] = pack_e4m3(__fmul_rn(z[2 * i].x, inv), __fmul_rn(z[2 * i].y, inv)) |
               (pack_e4m3(__fmul_rn(z[2 * i + 1].x, inv), __fmul_rn(z[2 * i + 1].y, inv)) << 16);
    if constexpr (H == 4)
        *reinterpret_cast<uint2*>(dst) = make_uint2(c[0], c[1]);
    else
        *reinterpret_cast<uint32_t*>(dst) = c[0];
}

// Last request r with cu[r] <= tok, by a whole warp: 32 probes a round.
__device__ __forceinline__ int owner_of(const int32_t* cu, int n, int tok) {
    const int lane = threadIdx.x & 31;
    int lo = 0, len = n;                            // the answer lies in [lo, lo + len)
    while (len > 1) {
        const int step = (len + 31) >> 5;
        const int i = lo + lane * step;
        const bool le = lane * step < len && __ldg(cu + i) <= tok;
        const int k = 31 - __clz(__ballot_sync(0xFFFFFFFFu, le) | 1u);
        lo += k * step;
        len = min(step, len - k * step);
    }
    return lo;
}

template <typename T, int N, bool QUANT, int G, int TOK>     // 2 N elements per lane, G lanes per row, TOK tokens per block
__global__ void __launch_bounds__(TOK > 1 ? kManyThreads : kMaxThreads, TOK > 1 ? kManyBlocks : 1) append_qkv_kernel(const QkvParams p) {
    typedef Run<T, N> R;
    typedef typename R::Raw Raw;
    __shared__ float2 turn[TOK][kMaxRotPairs];      // (cos, sin) of the tokens' angles
    __shared__ int owner[TOK], place[TOK];          // request; position in the slab, -1: nowhere
    const int tok0 = blockIdx.x * TOK, toks = min(TOK, p.n_new_total - tok0);
    const int tid = threadIdx.x, lane = tid & (G - 1);
    const int D = p.head_dim, pairs = p.rot_pairs;
    const int k_row = p.q_heads, v_row = k_row + p.kv_heads, rows = v_row + p.kv_heads;
    const bool in_row = lane * 2 * N < D;

    // element offsets of the lane's two runs in a row
    const bool rotated = lane * N < pairs;
    const bool halves = rotated && !p.interleaved;
    const int off_a = in_row ? (halves ? lane * N : lane * 2 * N) : 0, off_b = in_row ? (halves ? pairs + lane * N : lane * 2 * N + N) : 0;

    // A lane group works on one token; it takes every `step`-th of its rows (queries, then keys, then values), two
    // of them loaded ahead.
    const int step = blockDim.x / G / TOK;
    const int t = TOK == 1 ? 0 : (tid / G) / step;
    const int64_t tok = tok0 + min(t, toks - 1);
    const T* q_src = static_cast<const T*>(p.q) + tok * p.q_stride + off_a;
    const T* k_src = static_cast<const T*>(p.k_new) + tok * p.k_stride - k_row * D + off_a;
    const T* v_src = static_cast<const T*>(p.v_new) + tok * p.v_stride - v_row * D + off_a;
    const int gap = off_b - off_a;
    int r = TOK == 1 ? tid / G : (tid / G) % step;
    auto load = [&](int row, Raw& a, Raw& b) {
        if (row >= rows) return;
        const T* src = (row < k_row ? q_src : row < v_row ? k_src : v_src) + row * D;
        a = *reinterpret_cast<const Raw*>(src);
        b = *reinterpret_cast<const Raw*>(src + gap);
    };
    Raw a0{}, b0{}, a1{}, b1{};                     // in flight while the angles are computed
    load(r, a0, b0);
    load(r + step, a1, b1);

    for (int i = tid >> 5; i < toks; i += blockDim.x >> 5) {         // a warp per token
        int req = tok0 + i;
        if (!p.one_new_each) req = owner_of(p.cu_new, p.n, tok0 + i);
        const int first = __ldg(p.cu_new + req), end = __ldg(p.cu_new + req + 1);
        if ((tid & 31) == 0) {
            owner[i] = req;
            place[i] = tok0 + i < end ? __ldg(p.len + req) - (end - first) + (tok0 + i - first) : -1;
        }
    }
    if (p.positions == nullptr) __syncthreads();    // the token's place in its slab is its position
    for (int i = tid; i < toks * pairs; i += blockDim.x) {
        const int j = TOK == 1 ? 0 : i / pairs, k = i - j * pairs;
        int axis = 0;
        while (axis + 1 < p.n_axes && k >= p.section_end[axis]) ++axis;
        const int pos = p.positions ? __ldg(p.positions + axis * p.pos_stride + tok0 + j) : place[j];
        const double angle = static_cast<double>(pos) * static_cast<double>(__ldg(p.inv_freq + k));
        // In half turns, whole turns off: 1 / (2 pi) = hi + lo, hi the nearest double, and the product with hi is
        // taken exactly (fma), so the fraction keeps its digits however many turns there are.
        constexpr double HI = 0.15915494309189535, LO = -9.839338337591243e-18;
        const double turns = rint(angle * HI);
        const double part = fma(angle, LO, fma(angle, HI, -turns));
        float sn, cs;
        sincospif(static_cast<float>(2.0 * part), &sn, &cs);
        turn[j][k] = make_float2(cs, sn);
    }
    __syncthreads();
    const int pos = place[t < toks ? t : 0];
    if (t >= toks || pos < 0) return;               // no request has this token, or its request was refused

    // where the rows go: queries D apart, keys and values a slab's capacity of rows apart
    const int req = owner[t];
    const int64_t head_step = static_cast<int64_t>(__ldg(p.cap + req)) * D;
    const int64_t slab = (static_cast<int64_t>(p.layer) * 2 * p.rows_per_array + static_cast<int64_t>(__ldg(p.base + req)) * p.kv_heads + pos) * D + off_a;
    const int64_t k_dst = slab - k_row * head_step, v_dst = slab + p.rows_per_array * D - v_row * head_step;
    T* q_dst = static_cast<T*>(p.q_out) + tok * k_row * D + off_a;
    // the lane's turns, and the norm's weights of its elements (the queries', then the keys')
    constexpr int H = N / 2;
    float2 cs[H], sn[H], wa[H], wb[H];
#pragma unroll
    for (int k = 0; k < H; ++k) {
        const float2 lo = rotated && in_row ? turn[t][lane * N + 2 * k] : make_float2(1.f, 0.f);
        const float2 hi = rotated && in_row ? turn[t][lane * N + 2 * k + 1] : make_float2(1.f, 0.f);
        cs[k] = make_float2(lo.x, hi.x);
        sn[k] = make_float2(lo.y, hi.y);
    }
    auto weights = [&](const void* w) {
        if (!w) return;
        R::unpack(__ldg(reinterpret_cast<const Raw*>(static_cast<const T*>(w) + off_a)), wa);
        R::unpack(__ldg(reinterpret_cast<const Raw*>(static_cast<const T*>(w) + off_b)), wb);
    };
    const float per = 1.f / static_cast<float>(D);
    const unsigned group = G == 32 ? 0xFFFFFFFFu : ((1u << G) - 1u) << ((tid & 31) & ~(G - 1));
    const bool norm_q = p.q_norm != nullptr, norm_k = p.k_norm != nullptr;
    bool keys = false;                              // are these the keys' weights?
    weights(p.q_norm);
    for (; r < rows; r += step) {
        float2 xa[H], xb[H];
        R::unpack(a0, xa);
        R::unpack(b0, xb);
        a0 = a1;
        b0 = b1;
        load(r + 2 * step, a1, b1);
        const bool is_q = r < k_row, is_v = r >= v_row;
        if (!is_v) {
            if (!is_q && !keys) {
                keys = true;
                weights(p.k_norm);
            }
            if (is_q ? norm_q : norm_k) {           // the same for the G lanes of a row
                float2 sq = make_float2(0.f, 0.f);
                if (in_row)
#pragma unroll
                    for (int k = 0; k < H; ++k) sq = fma2(xa[k], xa[k], fma2(xb[k], xb[k], sq));
                float ss = sq.x + sq.y;
#pragma unroll
                for (int o = G / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(group, ss, o);
                const float inv = rsqrtf(fmaf(ss, per, p.eps));
                const float2 inv2 = make_float2(inv, inv);
#pragma unroll
                for (int k = 0; k < H; ++k) {
                    xa[k] = mul2(xa[k], mul2(inv2, wa[k]));
                    xb[k] = mul2(xb[k], mul2(inv2, wb[k]));
                }
            }
            if (halves) {
#pragma unroll
                for (int k = 0; k < H; ++k) {
                    const float2 u = xa[k], v = xb[k];
                    xa[k] = fma2(u, cs[k], mul2(v, make_float2(-sn[k].x, -sn[k].y)));
                    xb[k] = fma2(v, cs[k], mul2(u, sn[k]));
                }
            } else if (rotated) {                    // pair k of the lane: its elements 2k and 2k + 1 of both runs
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    float2& z = k < H ? xa[k] : xb[k - H];
                    const float c = k & 1 ? cs[k / 2].y : cs[k / 2].x, s = k & 1 ? sn[k / 2].y : sn[k / 2].x;
                    z = make_float2(z.x * c - z.y * s, z.y * c + z.x * s);
                }
            }
        }
        if (!in_row) continue;
        if (is_q) {
            T* dst = q_dst + r * D;
            *reinterpret_cast<Raw*>(dst) = R::pack(xa);
            *reinterpret_cast<Raw*>(dst + gap) = R::pack(xb);
            continue;
        }
        const int64_t at = (is_v ? v_dst : k_dst) + r * head_step;
        if (QUANT) {
            const float inv = is_v ? p.v_inv : p.k_inv;
            uint8_t* dst = static_cast<uint8_t*>(p.pool) + at;
            store_codes(dst, xa, inv);
            store_codes(dst + gap, xb, inv);
        } else {
            T* dst = static_cast<T*>(p.pool) + at;
            *reinterpret_cast<Raw*>(dst) = R::pack(xa);
            *reinterpret_cast<Raw*>(dst + gap) = R::pack(xb);
        }
    }
}

template <typename T, int N, bool QUANT, int G>
void launch_tok(const QkvParams& p, cudaStream_t stream) {
    if (p.n_new_total >= kManyTokens) {
        append_qkv_kernel<T, N, QUANT, G, kTokens><<<(p.n_new_total + kTokens - 1) / kTokens, kManyThreads, 0, stream>>>(p);
        return;
    }
    // as few passes over a token's rows as the block's limit allows, evenly filled
    const int rows = p.q_heads + 2 * p.kv_heads, passes = (rows * G + kMaxThreads - 1) / kMaxThreads;
    const int threads = ((rows + passes - 1) / passes * G + 31) / 32 * 32;
    append_qkv_kernel<T, N, QUANT, G, 1><<<p.n_new_total, threads, 0, stream>>>(p);
}

template <typename T, int N, bool QUANT>
cudaError_t launch_t(const QkvParams& p, cudaStream_t stream) {
    const int lanes = (p.head_dim + 2 * N - 1) / (2 * N);
    if (lanes <= 4)
        launch_tok<T, N, QUANT, 4>(p, stream);
    else if (lanes <= 8)
        launch_tok<T, N, QUANT, 8>(p, stream);
    else if (lanes <= 16)
        launch_tok<T, N, QUANT, 16>(p, stream);
    else if constexpr (N == 4)                      // heads of more than 128 elements, eight to a lane
        launch_tok<T, N, QUANT, 32>(p, stream);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_append_qkv(const QkvParams& p, bool fp32, cudaStream_t stream) {
    if (p.n_new_total <= 0) return cudaSuccess;
    if (fp32) return launch_t<float, 4, false>(p, stream);
    // Many tokens: sixteen elements per lane, in 16-byte loads, where head and rotated part divide into such runs; what a
    // row costs beside its elements is shared by more of them (chunk of 8,192: 43 -> 36 us).  Few: eight, a shorter way
    // through the block (256 tokens of an 8-bit pool: 4.0 us against 6.1).
    if (p.n_new_total >= kManyTokens && p.head_dim % 16 == 0 && p.rot_pairs % 8 == 0)
        return p.quantize ? launch_t<__nv_bfloat16, 8, true>(p, stream) : launch_t<__nv_bfloat16, 8, false>(p, stream);
    return p.quantize ? launch_t<__nv_bfloat16, 4, true>(p, stream) : launch_t<__nv_bfloat16, 4, false>(p, stream);
}

}  // namespace odma
