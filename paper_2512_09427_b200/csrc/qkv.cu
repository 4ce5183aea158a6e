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
// 28 + 4 + 4-head layer moves 151 MB.  A token's rot_dim / 2 sines and cosines are computed
// once, into shared memory, under the latency of the first row loads, and serve all its heads.  A
// row is held by D / 8 lanes of a warp, eight elements each, laid out so that both elements of a pair
// sit in the same lane (pairs (i, i + rot_dim / 2): four elements of each half; adjacent pairs: eight
// in a row); the norm's sum is a shuffle tree over those lanes.
#include "device_utils.cuh"

namespace odma {
namespace {

using namespace dev;

constexpr int kMaxThreads = 384;
// Tokens per block: one while that fills the GPU (a token's way through a block, some 3 us, is all a small step costs),
// several for more, whose rows then stream behind one another while the next tokens' angles are there already.
constexpr int kTokens = 4, kManyTokens = 1024;

template <typename T>
struct Quad;                                       // four elements of a row
template <>
struct Quad<float> {
    typedef float4 Raw;
    __device__ static void unpack(const Raw& r, float (&x)[4]) {
        x[0] = r.x;
        x[1] = r.y;
        x[2] = r.z;
        x[3] = r.w;
    }
    __device__ static Raw pack(const float (&x)[4]) { return make_float4(x[0], x[1], x[2], x[3]); }
};
template <>
struct Quad<__nv_bfloat16> {
    typedef uint2 Raw;
    __device__ static void unpack(const Raw& r, float (&x)[4]) {
        x[0] = __uint_as_float(r.x << 16);
        x[1] = __uint_as_float(r.x & 0xFFFF0000u);
        x[2] = __uint_as_float(r.y << 16);
        x[3] = __uint_as_float(r.y & 0xFFFF0000u);
    }
    __device__ static Raw pack(const float (&x)[4]) { return make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])); }
};

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

template <typename T, bool QUANT, int G, int TOK>   // G lanes per row, TOK tokens per block
__global__ void __launch_bounds__(kMaxThreads) append_qkv_kernel(const QkvParams p) {
    typedef typename Quad<T>::Raw Raw;
    __shared__ float2 turn[TOK][kMaxRotPairs];      // (cos, sin) of the tokens' angles
    __shared__ int owner[TOK], place[TOK];          // request; position in the slab, -1: nowhere
    const int tok0 = blockIdx.x * TOK, toks = min(TOK, p.n_new_total - tok0);
    const int tid = threadIdx.x, lane = tid & (G - 1);
    const int D = p.head_dim, pairs = p.rot_pairs;
    const int rows = p.q_heads + 2 * p.kv_heads, per_pass = blockDim.x / G;
    const bool in_row = lane * 8 < D;

    // element offsets of the lane's two quads in a query or key row
    const bool rotated = lane * 4 < pairs;
    const bool halves = rotated && !p.interleaved;
    const int off_a = halves ? lane * 4 : lane * 8, off_b = halves ? pairs + lane * 4 : lane * 8 + 4;

    // The rows of the block's tokens go to the lane groups in turn; two of a group's rows are loaded ahead.
    struct Row {
        int t, r;                                   // token of the block, row of the token (queries, keys, values)
        Raw a, b;
    };
    const int step_t = per_pass / rows, step_r = per_pass % rows;
    int next_t = (tid / G) / rows, next_r = (tid / G) % rows;
    auto fetch = [&](Row& x) {                      // the group's next row
        x.t = next_t;
        x.r = next_r;
        if (x.t >= toks) return;
        next_t += step_t;
        next_r += step_r;
        if (next_r >= rows) {
            next_r -= rows;
            ++next_t;
        }
        if (!in_row) return;
        const int64_t tok = tok0 + x.t;
        const T* src;
        int oa = off_a, ob = off_b;
        if (x.r < p.q_heads) {
            src = static_cast<const T*>(p.q) + tok * p.q_stride + x.r * D;
        } else if (x.r < p.q_heads + p.kv_heads) {
            src = static_cast<const T*>(p.k_new) + tok * p.k_stride + (x.r - p.q_heads) * D;
        } else {
            src = static_cast<const T*>(p.v_new) + tok * p.v_stride + (x.r - p.q_heads - p.kv_heads) * D;
            oa = lane * 8;
            ob = oa + 4;
        }
        x.a = *reinterpret_cast<const Raw*>(src + oa);
        x.b = *reinterpret_cast<const Raw*>(src + ob);
    };
    Row x0, x1;                                     // in flight while the angles are computed
    fetch(x0);
    fetch(x1);

    for (int t = tid >> 5; t < toks; t += blockDim.x >> 5) {         // a warp per token
        const int tok = tok0 + t;
        int req = tok;
        if (!p.one_new_each) req = owner_of(p.cu_new, p.n, tok);
        const int first = __ldg(p.cu_new + req), end = __ldg(p.cu_new + req + 1);
        if ((tid & 31) == 0) {
            owner[t] = req;
            place[t] = tok < end ? __ldg(p.len + req) - (end - first) + (tok - first) : -1;
        }
    }
    if (p.positions == nullptr) __syncthreads();    // the token's place in its slab is its position
    for (int i = tid; i < toks * pairs; i += blockDim.x) {
        const int t = i / pairs, k = i - t * pairs;
        int axis = 0;
        while (axis + 1 < p.n_axes && k >= p.section_end[axis]) ++axis;
        const int pos = p.positions ? __ldg(p.positions + axis * p.pos_stride + tok0 + t) : place[t];
        const double angle = static_cast<double>(pos) * static_cast<double>(__ldg(p.inv_freq + k));
        // whole turns off, in two steps: 2 pi = hi + lo, hi the nearest double
        const double turns = rint(angle * 0.15915494309189535);
        const double r = fma(-turns, 2.4492935982947064e-16, fma(-turns, 6.283185307179586, angle));
        float sn, cs;
        sincosf(static_cast<float>(r), &sn, &cs);
        turn[t][k] = make_float2(cs, sn);
    }
    __syncthreads();

    auto finish = [&](const Row& x) {
        const int pos = place[x.t];
        if (pos < 0) return;                        // no request has this token, or its request was refused
        const bool is_q = x.r < p.q_heads, is_v = x.r >= p.q_heads + p.kv_heads;
        float xa[4], xb[4];
        Quad<T>::unpack(x.a, xa);
        Quad<T>::unpack(x.b, xb);
        const void* w = is_v ? nullptr : (is_q ? p.q_norm : p.k_norm);
        if (w) {                                    // the same for the G lanes of a row
            float ss = 0.f;
            if (in_row)
#pragma unroll
                for (int k = 0; k < 4; ++k) ss = fmaf(xa[k], xa[k], fmaf(xb[k], xb[k], ss));
            const unsigned group = G == 32 ? 0xFFFFFFFFu : ((1u << G) - 1u) << ((tid & 31) & ~(G - 1));
#pragma unroll
            for (int o = G / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(group, ss, o);
            const float inv = rsqrtf(ss / static_cast<float>(D) + p.eps);
            if (in_row) {
                float wa[4], wb[4];
                Quad<T>::unpack(__ldg(reinterpret_cast<const Raw*>(static_cast<const T*>(w) + off_a)), wa);
                Quad<T>::unpack(__ldg(reinterpret_cast<const Raw*>(static_cast<const T*>(w) + off_b)), wb);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    xa[k] = xa[k] * inv * wa[k];
                    xb[k] = xb[k] * inv * wb[k];
                }
            }
        }
        if (!in_row) return;
        if (!is_v && rotated) {
            const float2* t4 = turn[x.t] + lane * 4;
            if (halves) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float2 t = t4[k];
                    const float u = xa[k], v = xb[k];
                    xa[k] = u * t.x - v * t.y;
                    xb[k] = v * t.x + u * t.y;
                }
            } else {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float2 t = t4[k], s = t4[2 + k];
                    const float u = xa[2 * k], v = xa[2 * k + 1], y = xb[2 * k], z = xb[2 * k + 1];
                    xa[2 * k] = u * t.x - v * t.y;
                    xa[2 * k + 1] = v * t.x + u * t.y;
                    xb[2 * k] = y * s.x - z * s.y;
                    xb[2 * k + 1] = z * s.x + y * s.y;
                }
            }
        }
        const int oa = is_v ? lane * 8 : off_a, ob = is_v ? lane * 8 + 4 : off_b;
        if (is_q) {
            T* dst = static_cast<T*>(p.q_out) + (static_cast<int64_t>(tok0 + x.t) * p.q_heads + x.r) * D;
            *reinterpret_cast<Raw*>(dst + oa) = Quad<T>::pack(xa);
            *reinterpret_cast<Raw*>(dst + ob) = Quad<T>::pack(xb);
            return;
        }
        const int req = owner[x.t], head = x.r - p.q_heads - (is_v ? p.kv_heads : 0);
        const int64_t row = (static_cast<int64_t>(p.layer) * 2 + (is_v ? 1 : 0)) * p.rows_per_array +
                            static_cast<int64_t>(__ldg(p.base + req)) * p.kv_heads + static_cast<int64_t>(head) * __ldg(p.cap + req) + pos;
        if (QUANT) {
            const float inv = is_v ? p.v_inv : p.k_inv;
            uint8_t* dst = static_cast<uint8_t*>(p.pool) + row * D;
            auto codes = [&](const float (&z)[4]) {
                return pack_e4m3(__fmul_rn(z[0], inv), __fmul_rn(z[1], inv)) |
                       (pack_e4m3(__fmul_rn(z[2], inv), __fmul_rn(z[3], inv)) << 16);
            };
            *reinterpret_cast<uint32_t*>(dst + oa) = codes(xa);
            *reinterpret_cast<uint32_t*>(dst + ob) = codes(xb);
        } else {
            T* dst = static_cast<T*>(p.pool) + row * D;
            *reinterpret_cast<Raw*>(dst + oa) = Quad<T>::pack(xa);
            *reinterpret_cast<Raw*>(dst + ob) = Quad<T>::pack(xb);
        }
    };
    while (x0.t < toks) {
        Row x = x0;
        x0 = x1;
        fetch(x1);
        finish(x);
    }
}

template <typename T, bool QUANT, int TOK>
void launch_g(const QkvParams& p, int G, int threads, cudaStream_t stream) {
    const int grid = (p.n_new_total + TOK - 1) / TOK;
    switch (G) {
        case 4: append_qkv_kernel<T, QUANT, 4, TOK><<<grid, threads, 0, stream>>>(p); break;
        case 8: append_qkv_kernel<T, QUANT, 8, TOK><<<grid, threads, 0, stream>>>(p); break;
        case 16: append_qkv_kernel<T, QUANT, 16, TOK><<<grid, threads, 0, stream>>>(p); break;
        default: append_qkv_kernel<T, QUANT, 32, TOK><<<grid, threads, 0, stream>>>(p); break;
    }
}

template <typename T, bool QUANT>
cudaError_t launch_t(const QkvParams& p, cudaStream_t stream) {
    const int G = p.head_dim <= 32 ? 4 : p.head_dim <= 64 ? 8 : p.head_dim <= 128 ? 16 : 32;
    const int rows = p.q_heads + 2 * p.kv_heads;
    // as few passes over a token's rows as the block's limit allows, evenly filled
    const int passes = (rows * G + kMaxThreads - 1) / kMaxThreads;
    const int threads = ((rows + passes - 1) / passes * G + 31) / 32 * 32;
    if (p.n_new_total >= kManyTokens)
        launch_g<T, QUANT, kTokens>(p, G, threads, stream);
    else
        launch_g<T, QUANT, 1>(p, G, threads, stream);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_append_qkv(const QkvParams& p, bool fp32, cudaStream_t stream) {
    if (p.n_new_total <= 0) return cudaSuccess;
    if (fp32) return launch_t<float, false>(p, stream);
    return p.quantize ? launch_t<__nv_bfloat16, true>(p, stream) : launch_t<__nv_bfloat16, false>(p, stream);
}

}  // namespace odma
