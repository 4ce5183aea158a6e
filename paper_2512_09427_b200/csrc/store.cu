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
// token lie side by side, and meet whole rows of a slab.  A group's maximum goes through log2(G / 16) shuffles.  12 requests
// of 8,191 tokens in all, 28 layers of 4 heads of 128, bf16 <-> E4M3 (712 MB): out 119 us (6.0 TB/s), back 111 us (6.4 TB/s);
// 5,001 tokens to 4 bits and back (753 MB): 129 us; raw rows (939 MB) 143 us either way (6.55 TB/s).  8-bit pools move half as
// much for as many conversions, and the issue slots fill up: 8,191 tokens out to 4 bits 127 us (3.0 TB/s, 87 % of the slots), to 8
// bits 129 us (85 %), 8 bits back 100 us (75 %).  Out, the quantising counts too: 3 units of 128 threads 119 us, 2 or 4
// of them 124 and 122, 4 of 256 127; two 16-byte loads per unit instead of one of 32 bytes 129.
#include "device_utils.cuh"
#include "odma.h"

namespace odma {
namespace {

using namespace dev;

constexpr int kThreads = 128;
constexpr int kUnits = 3;                            // units of 16 elements per thread

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
// Loads and stores of up to 32 bytes in one instruction: a warp's then meet whole sectors.  Nothing is read twice.
__device__ __forceinline__ void load(const void* p, Words<16>& x) {
    const uint4 v = __ldcs(static_cast<const uint4*>(p));
    x.w[0] = v.x, x.w[1] = v.y, x.w[2] = v.z, x.w[3] = v.w;
}
__device__ __forceinline__ void load(const void* p, Words<8>& x) {
    const uint2 v = __ldcs(static_cast<const uint2*>(p));
    x.w[0] = v.x, x.w[1] = v.y;
}
__device__ __forceinline__ void load8(const void* p, uint32_t* w) {
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p));
}
__device__ __forceinline__ void load(const void* p, Words<32>& x) { load8(p, x.w); }
__device__ __forceinline__ void load(const void* p, Words<64>& x) {
    load8(p, x.w);
    load8(static_cast<const uint8_t*>(p) + 32, x.w + 8);
}
__device__ __forceinline__ void store(void* p, const Words<8>& x) { __stcs(static_cast<uint2*>(p), make_uint2(x.w[0], x.w[1])); }
__device__ __forceinline__ void store(void* p, const Words<16>& x) { __stcs(static_cast<uint4*>(p), make_uint4(x.w[0], x.w[1], x.w[2], x.w[3])); }
__device__ __forceinline__ void store(void* p, const Words<32>& x) { store8(p, x.w); }
__device__ __forceinline__ void store(void* p, const Words<64>& x) {
    store8(p, x.w);
    store8(static_cast<uint8_t*>(p) + 32, x.w + 8);
}

// Pair i of f times `by`, each product rounded to fp32.
__device__ __forceinline__ float2 times(const float (&f)[16], int i, float by) {
    return mul2(make_float2(f[2 * i], f[2 * i + 1]), make_float2(by, by));
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
        for (int i = 0; i < 4; ++i) {
            const float2 a = times(f, 2 * i, inv), b = times(f, 2 * i + 1, inv);
            x.w[i] = pack_e4m3(a.x, a.y) | pack_e4m3(b.x, b.y) << 16;
        }
    }
};

// ---- the store's formats

constexpr float kMagic = 12582912.f;                 // 1.5 * 2^23: adding it rounds to the nearest whole number, ties to even,
                                                     // which then stands in the low bits
// (one at a time: as a pair, the sum would be contracted with the product in front of it)
__device__ __forceinline__ uint32_t rounded(float x, float magic) { return __float_as_uint(__fadd_rn(x, magic)); }

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
            const float2 a = times(f, 2 * i, inv), b = times(f, 2 * i + 1, inv);
            c.w[i] = __byte_perm(__byte_perm(rounded(a.x, kMagic), rounded(a.y, kMagic), 0x0040),
                                 __byte_perm(rounded(b.x, kMagic), rounded(b.y, kMagic), 0x0040), 0x5410);
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
    // Numbers from 1 to 15 (8 more than meant), each with the constant bits of kMagic above it: shifted and added up, these
    // make one constant, and flipping every nibble's first bit takes the 8 back.
    __device__ static void pack(const float (&f)[16], float inv, Words<8>& c) {
        constexpr uint32_t kBits = 0x4B400000u, kAll = kBits * 0x11111111u;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t w = 0;
#pragma unroll
            for (int k = 3; k >= 0; --k) {
                const float2 a = times(f, 4 * i + k, inv);
                w = (w << 4) + rounded(a.y, kMagic + 8.f);
                w = (w << 4) + rounded(a.x, kMagic + 8.f);
            }
            c.w[i] = (w - kAll) ^ 0x88888888u;
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

// Units of an array of the launch, tokens in order: unit `in` of token `tok` is element 16 c of KV head `head`.  A block
// takes kUnits runs of `step` tokens, a thread the same unit of each where a token has no more units than the block threads
// (`step` is 0 where it has: every unit is worked out by itself).
struct Place {
    int64_t store, slab;                             // unit of the store's array, and of the pool's
};
struct Run {
    const StoreParams& p;
    const Divider &per_token, &per_row;
    uint32_t u0, units, stride, tok, in, head, c;
    int i;                                           // the request of the last unit asked for
    bool mine;

    __device__ __forceinline__ Run(const StoreParams& params, const Divider& token, const Divider& row, uint32_t step)
        : p(params), per_token(token), per_row(row) {
        stride = step ? step * token.d : kThreads;
        u0 = blockIdx.x * (stride * kUnits) + threadIdx.x;
        units = static_cast<uint32_t>(p.cu[p.n]) * token.d;
        mine = threadIdx.x < stride;
        split(u0);
        int lo = 0, hi = p.n;                        // the last request that begins at the token or in front of it
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (p.cu[mid] <= static_cast<int>(tok)) lo = mid; else hi = mid;
        }
        i = lo;
    }
    __device__ __forceinline__ void split(uint32_t u) {
        tok = quotient(u, per_token);
        in = u - tok * per_token.d;
        head = quotient(in, per_row);
        c = in - head * per_row.d;
    }
    __device__ __forceinline__ bool has(int k) const { return mine && u0 + k * stride < units; }
    __device__ __forceinline__ Place at(int k, uint32_t step) {
        if (k > 0) {
            if (step)
                tok += step;
            else
                split(u0 + k * stride);
        }
        while (static_cast<int>(tok) >= p.cu[i + 1]) ++i;
        const int64_t row = p.row[i] + static_cast<int64_t>(head) * p.cap[i] + (static_cast<int>(tok) - p.cu[i]);
        return Place{static_cast<int64_t>(p.token0) * per_token.d + (u0 + k * stride), row * per_row.d + c};
    }
};

template <int DTYPE, int FORMAT, bool PACK>
__global__ void __launch_bounds__(kThreads) store_kernel(const __grid_constant__ StoreParams p, const __grid_constant__ Divider per_token,
                                                        const __grid_constant__ Divider per_row, uint32_t step) {
    using E = Elem<DTYPE>;
    using F = Format<FORMAT>;
    constexpr int ES = E::kBytes / 16;               // bytes of an element
    const int a = blockIdx.y;
    Run run(p, per_token, per_row, step);
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
        in[k] = run.has(k);
        if (!in[k]) continue;
        at[k] = run.at(k, step);
        if (PACK) {
            load(pool + at[k].slab * E::kBytes, x[k]);
        } else {
            load(codes + at[k].store * F::kBytes, c[k]);
            scale[k] = __ldg(scales + (at[k].store >> shift));
        }
    }
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        float f[16];
        if (PACK) {
            // (threads without a unit take part in the shuffles; runs of units are whole tokens, or begin at a multiple of
            // a warp's threads, so no group is shared with them)
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
                inv = __frcp_rn(s);
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
            store(pool + at[k].slab * E::kBytes, x[k]);
        }
    }
}

// Rows as they are, in units of 16 bytes.
template <bool PACK>
__global__ void __launch_bounds__(kThreads) store_raw_kernel(const __grid_constant__ StoreParams p, const __grid_constant__ Divider per_token,
                                                            const __grid_constant__ Divider per_row, uint32_t step) {
    const int a = blockIdx.y;
    Run run(p, per_token, per_row, step);
    uint4* pool = static_cast<uint4*>(p.pool) + (p.row0 + a * p.rows_per_array) * per_row.d;
    uint4* codes = static_cast<uint4*>(p.codes) + static_cast<int64_t>(a) * p.store_tokens * per_token.d;
    Place at[kUnits];
    uint4 x[kUnits];
#pragma unroll
    for (int k = 0; k < kUnits; ++k) {
        if (!run.has(k)) continue;
        at[k] = run.at(k, step);
        x[k] = __ldcs(PACK ? pool + at[k].slab : codes + at[k].store);
    }
#pragma unroll
    for (int k = 0; k < kUnits; ++k)
        if (run.has(k)) __stcs(PACK ? codes + at[k].store : pool + at[k].slab, x[k]);
}

template <int DTYPE, int FORMAT>
void launch_t(const StoreParams& p, dim3 grid, const Divider& per_token, const Divider& per_row, uint32_t step, bool pack, cudaStream_t stream) {
    if (pack)
        store_kernel<DTYPE, FORMAT, true><<<grid, kThreads, 0, stream>>>(p, per_token, per_row, step);
    else
        store_kernel<DTYPE, FORMAT, false><<<grid, kThreads, 0, stream>>>(p, per_token, per_row, step);
}
template <int DTYPE>
cudaError_t launch_f(const StoreParams& p, int format, dim3 grid, const Divider& per_token, const Divider& per_row, uint32_t step, bool pack, cudaStream_t stream) {
    switch (format) {
        case ODMA_STORE_E4M3: launch_t<DTYPE, ODMA_STORE_E4M3>(p, grid, per_token, per_row, step, pack, stream); break;
        case ODMA_STORE_INT8: launch_t<DTYPE, ODMA_STORE_INT8>(p, grid, per_token, per_row, step, pack, stream); break;
        case ODMA_STORE_INT4: launch_t<DTYPE, ODMA_STORE_INT4>(p, grid, per_token, per_row, step, pack, stream); break;
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
    const uint32_t step = per_token.d <= kThreads ? kThreads / per_token.d : 0;
    const uint64_t block = static_cast<uint64_t>(step ? step * per_token.d : kThreads) * kUnits;
    const dim3 grid(static_cast<unsigned>((units + block - 1) / block), static_cast<unsigned>(p.arrays));
    if (format == ODMA_STORE_RAW) {
        if (pack)
            store_raw_kernel<true><<<grid, kThreads, 0, stream>>>(p, per_token, per_row, step);
        else
            store_raw_kernel<false><<<grid, kThreads, 0, stream>>>(p, per_token, per_row, step);
        return cudaGetLastError();
    }
    switch (dtype) {
        case ODMA_DTYPE_F32: return launch_f<ODMA_DTYPE_F32>(p, format, grid, per_token, per_row, step, pack, stream);
        case ODMA_DTYPE_BF16: return launch_f<ODMA_DTYPE_BF16>(p, format, grid, per_token, per_row, step, pack, stream);
        case ODMA_DTYPE_FP8_E4M3: return launch_f<ODMA_DTYPE_FP8_E4M3>(p, format, grid, per_token, per_row, step, pack, stream);
    }
    return cudaErrorInvalidValue;
}

}  // namespace odma
