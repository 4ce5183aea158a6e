// Rows of slabs to a dense store in fewer bits, and back (odma_pack_kv, odma_unpack_kv).
//
// A row is one token's key or value of one KV head.  For every group of G elements of a row
//     scale = max |x| / top (top = 448, 127, 7),   code = the nearest number of the format to x * (1 / scale)
// in fp32, and back x = code * scale, rounded once to the pool's type (an 8-bit pool: times its own 1 / scale, nearest
// code).  The largest magnitude is found on the bits: without the sign, the order of a floating-point format is that of
// its bits as an integer, and infinities and NaN lie above all finite numbers.
//
// What bounds it: memory.  A thread takes 16 elements, 32 bytes of a bf16 row in one load and 16 or 8 bytes of codes in one
// store, kUnits of them with all loads before the first store; the threads of a warp follow the store, where rows of a
// token lie side by side, and meet whole rows of a slab.  A group's maximum goes through log2(G / 16) shuffles.
#include "device_utils.cuh"
#include "odma.h"

namespace odma {
namespace {

using namespace dev;

constexpr int kThreads = 256;
constexpr int kUnits = 4;                            // units of 16 elements per thread

// Division by a number that all threads share: x / d = (x * m) >> (31 + s) for x below 2^31, with 2^s the first power of two that
// reaches d and m = 2^(31 + s) / d rounded up: m d exceeds 2^(31 + s) by less than d, so the quotient is off by less than
// x / 2^(31 + s) <= 2^-s, too little to reach the next whole number (Granlund and Montgomery 1994).
struct Divider {
    uint32_t m, s, d;
};
__host__ __device__ inline Divider divider(uint32_t d) {
    uint32_t s = 0;
    while ((1u << s) < d) ++s;
    const uint64_t m = ((uint64_t(1) << (31 + s)) + d - 1) / d;
    return Divider{static_cast<uint32_t>(m), s, d};
}
__device__ __forceinline__ uint32_t quotient(uint32_t x, const Divider& v) {
    return static_cast<uint32_t>((static_cast<uint64_t>(x) * v.m) >> 31 >> v.s);
}

template <int BYTES>
struct Words {
    uint32_t w[BYTES / 4];
};
__device__ __forceinline__ void load(const void* p, Words<16>& x) {
    const uint4 v = __ldcs(static_cast<const uint4*>(p));
    x.w[0] = v.x, x.w[1] = v.y, x.w[2] = v.z, x.w[3] = v.w;
}
__device__ __forceinline__ void load(const void* p, Words<8>& x) {
    const uint2 v = __ldcs(static_cast<const uint2*>(p));
    x.w[0] = v.x, x.w[1] = v.y;
}
__device__ __forceinline__ void load(const void* p, Words<32>& x) {
    const uint4 a = __ldcs(static_cast<const uint4*>(p)), b = __ldcs(static_cast<const uint4*>(p) + 1);
    x.w[0] = a.x, x.w[1] = a.y, x.w[2] = a.z, x.w[3] = a.w;
    x.w[4] = b.x, x.w[5] = b.y, x.w[6] = b.z, x.w[7] = b.w;
}
__device__ __forceinline__ void load(const void* p, Words<64>& x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint4 v = __ldcs(static_cast<const uint4*>(p) + i);
        x.w[4 * i] = v.x, x.w[4 * i + 1] = v.y, x.w[4 * i + 2] = v.z, x.w[4 * i + 3] = v.w;
    }
}
template <int BYTES>
__device__ __forceinline__ void store(void* p, const Words<BYTES>& x) {
    if constexpr (BYTES == 8) {
        __stcs(static_cast<uint2*>(p), make_uint2(x.w[0], x.w[1]));
    } else {
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i)
            __stcs(static_cast<uint4*>(p) + i, make_uint4(x.w[4 * i], x.w[4 * i + 1], x.w[4 * i + 2], x.w[4 * i + 3]));
    }
}

// ---- the pool's element types: 16 elements as floats, the bits of their largest magnitude

template <int DTYPE>
struct Elem;
template <>
struct Elem<ODMA_DTYPE_F32> {
    static constexpr int kBytes = 64;
    static constexpr uint32_t kInf = 0x7F800000u;    // bits from here on are not finite
    __device__ static uint32_t top(const Words<64>& x) {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) t = max(t, x.w[i] & 0x7FFFFFFFu);
        return t;
    }
    __device__ static float value(uint32_t bits, float) { return __uint_as_float(bits); }
    __device__ static void floats(const Words<64>& x, float, float (&f)[16]) {
#pragma unroll
        for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(x.w[i]);
    }
    __device__ static void pack(const float (&f)[16], float, Words<64>& x) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x.w[i] = __float_as_uint(f[i]);
    }
};
template <>
struct Elem<ODMA_DTYPE_BF16> {
    static constexpr int kBytes = 32;
    static constexpr uint32_t kInf = 0x7F80u;
    __device__ static uint32_t top(const Words<32>& x) {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) t = __vmaxu2(t, x.w[i] & 0x7FFF7FFFu);
        return max(t & 0xFFFFu, t >> 16);
    }
    __device__ static float value(uint32_t bits, float) { return __uint_as_float(bits << 16); }
    __device__ static void floats(const Words<32>& x, float, float (&f)[16]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            f[2 * i] = __uint_as_float(x.w[i] << 16);
            f[2 * i + 1] = __uint_as_float(x.w[i] & 0xFFFF0000u);
        }
    }
    __device__ static void pack(const float (&f)[16], float, Words<32>& x) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x.w[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
    }
};
template <>
struct Elem<ODMA_DTYPE_FP8_E4M3> {
    static constexpr int kBytes = 16;
    static constexpr uint32_t kInf = 0x7Fu;          // a NaN; the format has no infinities
    __device__ static uint32_t top(const Words<16>& x) {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) t = __vmaxu4(t, x.w[i] & 0x7F7F7F7Fu);
        return max(max(t & 0xFFu, t >> 8 & 0xFFu), max(t >> 16 & 0xFFu, t >> 24));
    }
    __device__ static float value(uint32_t bits, float scale) { return __fmul_rn(unpack_e4m3(bits).x, scale); }
    __device__ static void floats(const Words<16>& x, float scale, float (&f)[16]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 v = unpack_e4m3(x.w[i >> 1] >> (16 * (i & 1)));
            f[2 * i] = __fmul_rn(v.x, scale);
            f[2 * i + 1] = __fmul_rn(v.y, scale);
        }
    }
    __device__ static void pack(const float (&f)[16], float inv, Words<16>& x) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x.w[i] = pack_e4m3(__fmul_rn(f[4 * i], inv), __fmul_rn(f[4 * i + 1], inv)) |
                     pack_e4m3(__fmul_rn(f[4 * i + 2], inv), __fmul_rn(f[4 * i + 3], inv)) << 16;
    }
};

// ---- the store's formats

constexpr float kMagic = 12582912.f;                 // 1.5 * 2^23: adding it rounds to the nearest whole number, ties to even,
                                                     // which then stands in the low bits
template <int FORMAT>
struct Format;
template <>
struct Format<ODMA_STORE_E4M3> {
    static constexpr int kBytes = 16;
    static constexpr float kTop = 448.f;
    __device__ static void pack(const float (&f)[16], float inv, Words<16>& c) { Elem<ODMA_DTYPE_FP8_E4M3>::pack(f, inv, c); }
    __device__ static void floats(const Words<16>& c, float scale, float (&f)[16]) { Elem<ODMA_DTYPE_FP8_E4M3>::floats(c, scale, f); }
};
template <>
struct Format<ODMA_STORE_INT8> {
    static constexpr int kBytes = 16;
    static constexpr float kTop = 127.f;
    // |x * inv| is at most 127 and three roundings, which the sum rounds to 127
    __device__ static void pack(const float (&f)[16], float inv, Words<16>& c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t b[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) b[k] = __float_as_uint(__fadd_rn(__fmul_rn(f[4 * i + k], inv), kMagic));
            c.w[i] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
        }
    }
    __device__ static void floats(const Words<16>& c, float scale, float (&f)[16]) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            // 2^23 + 128 + code, exactly
            const uint32_t b = __byte_perm(c.w[i >> 2] ^ 0x80808080u, 0x4B000000u, 0x7440 | (i & 3));
            f[i] = __fmul_rn(__uint_as_float(b) - 8388736.f, scale);
        }
    }
};
template <>
struct Format<ODMA_STORE_INT4> {
    static constexpr int kBytes = 8;
    static constexpr float kTop = 7.f;
    __device__ static void pack(const float (&f)[16], float inv, Words<8>& c) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t w = 0;
#pragma unroll
            for (int k = 7; k >= 0; --k) w = w << 4 | (__float_as_uint(__fadd_rn(__fmul_rn(f[8 * i + k], inv), kMagic)) & 15u);
            c.w[i] = w;
        }
    }
    __device__ static void floats(const Words<8>& c, float scale, float (&f)[16]) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t b = ((c.w[i >> 3] ^ 0x88888888u) >> (4 * (i & 7)) & 15u) | 0x4B000000u;
            f[i] = __fmul_rn(__uint_as_float(b) - 8388616.f, scale);
        }
    }
};

// Place of unit `u` of an array of the launch: unit of the store's array, offset in elements inside the pool's array.
// `i` is the request of an earlier unit.
struct Place {
    int64_t store, slab;
};
__device__ __forceinline__ Place place(const StoreParams& p, uint32_t u, const Divider& per_token, const Divider& per_row, int unit, int& i) {
    const uint32_t tok = quotient(u, per_token), in = u - tok * per_token.d, head = quotient(in, per_row), c = in - head * per_row.d;
    while (static_cast<int>(tok) >= p.cu[i + 1]) ++i;
    const int64_t row = p.row[i] + static_cast<int64_t>(head) * p.cap[i] + (static_cast<int>(tok) - p.cu[i]);
    return Place{(static_cast<int64_t>(p.token0) * per_token.d) + u, (row * per_row.d + c) * unit};
}
// The request of the block's first unit.
__device__ __forceinline__ int first_request(const StoreParams& p, uint32_t tok) {
    int lo = 0, hi = p.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.cu[mid] <= static_cast<int>(tok)) lo = mid; else hi = mid;
    }
    return lo;
}

template <int DTYPE, int FORMAT, bool PACK>
__global__ void __launch_bounds__(kThreads) store_kernel(const __grid_constant__ StoreParams p, const Divider per_token, const Divider per_row) {
    using E = Elem<DTYPE>;
    using F = Format<FORMAT>;
    constexpr int ES = E::kBytes / 16;               // bytes of an element
    const int a = blockIdx.y;
    const uint32_t units = static_cast<uint32_t>(p.cu[p.n]) * per_token.d;
    const uint32_t u0 = blockIdx.x * (kThreads * kUnits);
    int i = first_request(p, quotient(u0, per_token));
    uint8_t* pool = static_cast<uint8_t*>(p.pool) + (p.row0 + a * p.rows_per_array) * p.head_dim * ES;
    const int64_t array = static_cast<int64_t>(a) * p.store_tokens * per_token.d;
    uint8_t* codes = static_cast<uint8_t*>(p.codes) + array * F::kBytes;
    const int lanes = p.group >> 4, shift = __ffs(lanes) - 1;          // a power of two that divides a row's units
    float* scales = p.scales + (array >> shift);
    const float2 own = DTYPE == ODMA_DTYPE_FP8_E4M3 ? p.scale[a] : make_float2(1.f, 1.f);
    Place at[kUnits];
    bool in[kUnits];
    Words<E::kBytes> x[kUnits];
    Words<F::kBytes> c[kUnits];
    float scale[kUnits];
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        const uint32_t u = u0 + k * kThreads + threadIdx.x;
        in[k] = u < units;
        if (!in[k]) continue;
        at[k] = place(p, u, per_token, per_row, 16, i);
        if (PACK) {
            load(pool + at[k].slab * ES, x[k]);
        } else {
            load(codes + at[k].store * F::kBytes, c[k]);
            scale[k] = __ldg(scales + (at[k].store >> shift));
        }
    }
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        float f[16];
        if (PACK) {
            // (threads without a unit take part in the shuffles: units end with a row, so no group is shared with them)
            uint32_t top = in[k] ? E::top(x[k]) : 0u;
            for (int o = 1; o < lanes; o <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
            if (!in[k]) continue;
            const float most = E::value(top, own.x);
            float s, inv;
            if (top >= E::kInf) {                    // an infinity or a NaN: the group reads back as NaN
                s = NAN;
                inv = 0.f;
            } else if (most < 7.888609052210118e-31f) {      // 2^-100: as good as zero, and 1 / scale stays finite
                s = inv = 0.f;
            } else {
                s = __fdiv_rn(most, F::kTop);
                inv = __fdiv_rn(1.f, s);
            }
            E::floats(x[k], own.x, f);
            if (top >= E::kInf)
#pragma unroll
                for (int e = 0; e < 16; ++e) f[e] = 0.f;
            F::pack(f, inv, c[k]);
            store(codes + at[k].store * F::kBytes, c[k]);
            if ((at[k].store & (lanes - 1)) == 0) __stcs(scales + (at[k].store >> shift), s);
        } else {
            if (!in[k]) continue;
            F::floats(c[k], scale[k], f);
            E::pack(f, own.y, x[k]);
            store(pool + at[k].slab * ES, x[k]);
        }
    }
}

// Rows as they are, in units of 16 bytes.
template <bool PACK>
__global__ void __launch_bounds__(kThreads) store_raw_kernel(const __grid_constant__ StoreParams p, const Divider per_token, const Divider per_row) {
    const int a = blockIdx.y;
    const uint32_t units = static_cast<uint32_t>(p.cu[p.n]) * per_token.d, u0 = blockIdx.x * (kThreads * kUnits);
    int i = first_request(p, quotient(u0, per_token));
    uint4* pool = static_cast<uint4*>(p.pool) + (p.row0 + a * p.rows_per_array) * per_row.d;
    uint4* codes = static_cast<uint4*>(p.codes) + static_cast<int64_t>(a) * p.store_tokens * per_token.d;
    Place at[kUnits];
    uint4 x[kUnits];
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        const uint32_t u = u0 + k * kThreads + threadIdx.x;
        if (u >= units) continue;
        at[k] = place(p, u, per_token, per_row, 1, i);
        x[k] = __ldcs(PACK ? pool + at[k].slab : codes + at[k].store);
    }
#pragma unroll
    for (int k = 0; k < kUnits; ++k)
        if (u0 + k * kThreads + threadIdx.x < units) __stcs(PACK ? codes + at[k].store : pool + at[k].slab, x[k]);
}

template <int DTYPE, int FORMAT>
void launch_t(const StoreParams& p, dim3 grid, const Divider& per_token, const Divider& per_row, bool pack, cudaStream_t stream) {
    if (pack)
        store_kernel<DTYPE, FORMAT, true><<<grid, kThreads, 0, stream>>>(p, per_token, per_row);
    else
        store_kernel<DTYPE, FORMAT, false><<<grid, kThreads, 0, stream>>>(p, per_token, per_row);
}
template <int DTYPE>
cudaError_t launch_f(const StoreParams& p, int format, dim3 grid, const Divider& per_token, const Divider& per_row, bool pack, cudaStream_t stream) {
    switch (format) {
        case ODMA_STORE_E4M3: launch_t<DTYPE, ODMA_STORE_E4M3>(p, grid, per_token, per_row, pack, stream); break;
        case ODMA_STORE_INT8: launch_t<DTYPE, ODMA_STORE_INT8>(p, grid, per_token, per_row, pack, stream); break;
        case ODMA_STORE_INT4: launch_t<DTYPE, ODMA_STORE_INT4>(p, grid, per_token, per_row, pack, stream); break;
        default: return cudaErrorInvalidValue;
    }
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_store(const StoreParams& p, int format, int dtype, bool pack, cudaStream_t stream) {
    const int es = dtype == ODMA_DTYPE_F32 ? 4 : dtype == ODMA_DTYPE_BF16 ? 2 : 1;
    const uint32_t row = static_cast<uint32_t>(format == ODMA_STORE_RAW ? p.head_dim * es / 16 : p.head_dim / 16);
    const Divider per_row = divider(row), per_token = divider(row * p.kv_heads);
    const uint64_t units = static_cast<uint64_t>(p.cu[p.n]) * per_token.d;
    if (units == 0) return cudaSuccess;
    const dim3 grid(static_cast<unsigned>((units + kThreads * kUnits - 1) / (kThreads * kUnits)), static_cast<unsigned>(p.arrays));
    if (format == ODMA_STORE_RAW) {
        if (pack)
            store_raw_kernel<true><<<grid, kThreads, 0, stream>>>(p, per_token, per_row);
        else
            store_raw_kernel<false><<<grid, kThreads, 0, stream>>>(p, per_token, per_row);
        return cudaGetLastError();
    }
    switch (dtype) {
        case ODMA_DTYPE_F32: return launch_f<ODMA_DTYPE_F32>(p, format, grid, per_token, per_row, pack, stream);
        case ODMA_DTYPE_BF16: return launch_f<ODMA_DTYPE_BF16>(p, format, grid, per_token, per_row, pack, stream);
        case ODMA_DTYPE_FP8_E4M3: return launch_f<ODMA_DTYPE_FP8_E4M3>(p, format, grid, per_token, per_row, pack, stream);
    }
    return cudaErrorInvalidValue;
}

}  // namespace odma
