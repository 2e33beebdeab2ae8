// Microscaled messages: what K workers send at a synchronization, in 4 or 8
// bits an element.  A row is one worker's difference from the model that all
// of them share; blocks of 32 of its elements share a power of two.
//
//   adpsgd_mx_quantize    d = (x - base) + residual, rounded to the format; residual' = d - d_sent
//   adpsgd_mx_dequantize  y = base + d_sent
//   adpsgd_mx_average     base' = base + mean_k d_sent, broadcast to x, and every tensor's variance
//   adpsgd_mx_product     C[j][k] = sum_i a_j,i b_k,i for every tensor
//
// Every call is asynchronous, allocates nothing and keeps nothing, so that it
// can be captured into a graph.
//
// Tensors and partial sums: a block takes a chunk of consecutive elements,
// whatever tensors begin in it, and leaves one partial sum for each (chunk,
// tensor) pair that meet.  Walking along the row, each step to the next pair
// moves on by one chunk or by one tensor, so c + tau numbers the pairs without
// a table: no plan has to be built before a call.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <initializer_list>
#include <string>
#include <type_traits>

#include "adpsgd.h"
#include "common.hpp"

namespace adpsgd {
namespace {

constexpr int kThreads = 256;
constexpr int kMxBlock = 32;           // elements that share a scale
constexpr int32_t kMaxK = 65536;
constexpr int32_t kMaxT = 1 << 24;
constexpr int32_t kMaxProductK = 256;
// Blocks a launch has at most; the kernels stride over the rest.  A multiple of
// 8, so that a block's chunks stay on its XCD.
constexpr uint32_t kMaxGrid = 1u << 22;
constexpr int64_t kMaxPieces = (int64_t(1) << 31) - 1;

// Rows need not be 16-byte aligned: the hardware takes a 16-byte access at any
// multiple of four.
typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float v4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef int i8v __attribute__((ext_vector_type(8)));
typedef short s2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));

// ---- formats ---------------------------------------------------------------
// F = 0: E2M1 (two elements a byte, the even one in the low half), 1: E4M3.
// Code: the codes of a float4 group, as loaded and stored by a lane.
template <int F>
struct Fmt;
template <>
struct Fmt<ADPSGD_MX_E2M1> {
    using Code = uint16_t;
    static constexpr int kTopExp = 2;               // the largest number is 1.5 * 2^2
    static constexpr uint32_t kTopMan = 0x400000;
    static constexpr float kMost = 0x1.8p+127f;     // the largest of its numbers that fp32 holds
    static __device__ uint32_t encode(f4 v, float s) {
        uint32_t r = 0;
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v.x, v.y, s, 0);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v.z, v.w, s, 1);
    }
    static __device__ f4 decode(uint32_t c, float s) {
        const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 0);
        const f2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 1);
        return f4{a.x, a.y, b.x, b.y};
    }
};
template <>
struct Fmt<ADPSGD_MX_E4M3> {
    using Code = uint32_t;
    static constexpr int kTopExp = 8;               // 1.75 * 2^8
    static constexpr uint32_t kTopMan = 0x600000;
    static constexpr float kMost = 0x1.ep+127f;
    static __device__ uint32_t encode(f4 v, float s) {
        s2v r = {0, 0};
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, v.x, v.y, s, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, v.z, v.w, s, true);
        return __builtin_bit_cast(uint32_t, r);
    }
    static __device__ f4 decode(uint32_t c, float s) {
        const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, s, false);
        const f2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, s, true);
        return f4{a.x, a.y, b.x, b.y};
    }
};

// 2^(byte - 127) as the conversions take it: they read the exponent field
// (255: NaN for every element).  Byte 0 is a subnormal number.
__device__ __forceinline__ float scale_of(uint32_t byte) {
    const uint32_t b = byte << 23;
    return __uint_as_float(b > 0x400000u ? b : 0x400000u);
}

// The largest of the 8 lanes that hold a block (unsigned compare: of magnitudes'
// bits, so that a NaN is the largest).
__device__ __forceinline__ uint32_t max_of_8_lanes(uint32_t v) {
    auto other = [&](auto ctrl) {
        return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xf, 0xf, true);
    };
    uint32_t o = other(std::integral_constant<int, 0xB1>{});   // quad_perm 1,0,3,2
    v = o > v ? o : v;
    o = other(std::integral_constant<int, 0x4E>{});            // quad_perm 2,3,0,1
    v = o > v ? o : v;
    o = other(std::integral_constant<int, 0x141>{});           // mirrored halves of 16 lanes
    return o > v ? o : v;
}

// The last tensor that begins at or before element e (empty ones before it are
// passed over), by all lanes of a wave: 64 offsets at a time.
__device__ __forceinline__ int32_t tensor_at(const int64_t *off, int32_t T, int64_t e) {
    int32_t lo = 0, n = T;
    const int lane = threadIdx.x & 63;
    while (n > 1) {
        const int32_t step = (n + 63) / 64;
        const int64_t i = (int64_t)lane * step;
        const uint64_t before = __ballot(i < n && off[lo + (i < n ? i : 0)] <= e);
        const int32_t hits = __popcll(before);
        const int32_t at = (hits > 0 ? hits - 1 : 0) * step;
        lo += at;
        n = n - at < step ? n - at : step;
    }
    return lo;
}

// A sum over the block's threads, in the same order every time; valid in thread 0.
__device__ __forceinline__ double block_sum(double v, double *lds) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double t = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < kThreads / 64; ++w) t += lds[w];
    __syncthreads();
    return t;
}

__device__ __forceinline__ f4 load4(const float *p, int64_t e, int64_t P) {
    if (e + 4 <= P) return *reinterpret_cast<const f4 *>(p + e);
    f4 v = {0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < 4; ++j)
        if (e + j < P) v[j] = p[e + j];
    return v;
}
__device__ __forceinline__ void store4(float *p, int64_t e, int64_t P, f4 v) {
    if (e + 4 <= P) {
        *reinterpret_cast<f4 *>(p + e) = v;
        return;
    }
    for (int j = 0; j < 4; ++j)
        if (e + j < P) p[e + j] = v[j];
}

// ---- quantize, dequantize ---------------------------------------------------
// Blocks are dealt to the XCDs round-robin: the K rows' blocks of one piece of
// the row follow one another on one XCD, whose L2 then holds base for them.
struct RowGrid {
    uint32_t K;
    uint32_t pieces;       // of a row
    uint32_t blocks;       // virtual blocks of the launch
    uint32_t spread;       // 8: pieces dealt to XCDs; 1: too few pieces for that
};
RowGrid row_grid(int32_t K, int64_t P, int64_t piece) {
    RowGrid g;
    g.K = (uint32_t)K;
    g.pieces = (uint32_t)((P + piece - 1) / piece);
    g.spread = g.pieces >= 8 ? 8 : 1;
    g.blocks = (g.pieces + g.spread - 1) / g.spread * g.spread * g.K;
    return g;
}
__device__ __forceinline__ bool row_piece(const RowGrid &g, uint32_t b, uint32_t *k, uint32_t *piece) {
    const uint32_t s = b / g.spread;
    *k = s % g.K;
    *piece = s / g.K * g.spread + b % g.spread;
    return *piece < g.pieces;
}

struct QuantizeParams {
    const float *x;
    const float *base;
    const float *r_in;
    float *r_out;
    uint8_t *codes;
    uint8_t *scales;
    int64_t x_ld, r_ld, code_ld, scale_ld;
    int64_t P;
    RowGrid g;
};

// One lane holds four elements of a block, eight lanes a block.  Elements past
// the row's end count as zero and are sent as such.
template <int F, int NU>
__global__ void __launch_bounds__(kThreads) k_mx_quantize(QuantizeParams p) {
    using Code = typename Fmt<F>::Code;
    const int64_t padded = (p.P + kMxBlock - 1) / kMxBlock * kMxBlock;
    for (uint32_t b = blockIdx.x; b < p.g.blocks; b += gridDim.x) {
        uint32_t k, piece;
        if (!row_piece(p.g, b, &k, &piece)) continue;
        const int64_t e0 = (int64_t)piece * (kThreads * 4 * NU) + threadIdx.x * 4;
        const float *x = p.x + k * p.x_ld;
        f4 d[NU];
#pragma unroll
        for (int u = 0; u < NU; ++u) d[u] = load4(x, e0 + u * (kThreads * 4), p.P);
        if (p.base) {
#pragma unroll
            for (int u = 0; u < NU; ++u) d[u] -= load4(p.base, e0 + u * (kThreads * 4), p.P);
        }
        if (p.r_in) {
#pragma unroll
            for (int u = 0; u < NU; ++u) d[u] += load4(p.r_in + k * p.r_ld, e0 + u * (kThreads * 4), p.P);
        }
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const int64_t e = e0 + u * (kThreads * 4);
            if (e >= padded) continue;          // (whole blocks: the lanes of one agree)
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t a = __float_as_uint(d[u][j]) & 0x7fffffffu;
                m = a > m ? a : m;
            }
            m = max_of_8_lanes(m);
            // the least power of two that holds the largest element
            const int32_t s = (int32_t)(m >> 23) - Fmt<F>::kTopExp + ((m & 0x7fffffu) > Fmt<F>::kTopMan ? 1 : 0);
            const bool bad = m >= 0x7f800000u;   // a NaN or an infinity: nothing of the block can be sent
            const uint32_t byte = bad ? 255u : (uint32_t)(s > 0 ? s : 0);
            f4 v = d[u];
            if (bad) v = f4{0.f, 0.f, 0.f, 0.f};
            else if (byte == 255u - Fmt<F>::kTopExp) {     // (the next number up would be 2^128)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = fminf(fmaxf(v[j], -Fmt<F>::kMost), Fmt<F>::kMost);
            }
            const float scale = bad ? 1.f : scale_of(byte);
            const uint32_t c = Fmt<F>::encode(v, scale);
            *reinterpret_cast<Code *>(p.codes + k * p.code_ld + (e >> 2) * sizeof(Code)) = (Code)c;
            if ((threadIdx.x & 7) == 0) p.scales[k * p.scale_ld + (e >> 5)] = (uint8_t)byte;
            if (p.r_out && e < p.P) store4(p.r_out + k * p.r_ld, e, p.P, (bad ? v : d[u]) - Fmt<F>::decode(c, scale));
        }
    }
}

struct DequantizeParams {
    const uint8_t *codes;
    const uint8_t *scales;
    const float *base;
    float *y;
    int64_t y_ld, code_ld, scale_ld;
    int64_t P;
    RowGrid g;
};

template <int F, int NU>
__global__ void __launch_bounds__(kThreads) k_mx_dequantize(DequantizeParams p) {
    using Code = typename Fmt<F>::Code;
    for (uint32_t b = blockIdx.x; b < p.g.blocks; b += gridDim.x) {
        uint32_t k, piece;
        if (!row_piece(p.g, b, &k, &piece)) continue;
        const int64_t e0 = (int64_t)piece * (kThreads * 4 * NU) + threadIdx.x * 4;
        uint32_t c[NU], s[NU];
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const int64_t e = e0 + u * (kThreads * 4);
            if (e >= p.P) continue;
            c[u] = *reinterpret_cast<const Code *>(p.codes + k * p.code_ld + (e >> 2) * sizeof(Code));
            s[u] = p.scales[k * p.scale_ld + (e >> 5)];
        }
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const int64_t e = e0 + u * (kThreads * 4);
            if (e >= p.P) continue;
            f4 v = Fmt<F>::decode(c[u], scale_of(s[u]));
            if (p.base) v = load4(p.base, e, p.P) + v;
            store4(p.y + k * p.y_ld, e, p.P, v);
        }
    }
}

// ---- average ----------------------------------------------------------------
struct AverageParams {
    const uint8_t *codes;
    const uint8_t *scales;
    const float *base;
    float *base_out;
    float *x;
    const int64_t *off;
    double *partials;      // [chunks + T]
    int64_t x_ld, code_ld, scale_ld;
    int64_t P;
    uint32_t chunks;
    int32_t K, T;
};

// Sums in 64 bits: of numbers with at most four significant bits the sums over
// the workers, s1 of d and s2 of d^2, are exact unless their scales are 2^40
// apart, so K s2 - s1^2 = K sum_k (d_k - mean)^2 loses nothing where the
// workers agree, and one pass over the rows is enough.
template <int F, int NU>
__global__ void __launch_bounds__(kThreads) k_mx_average(AverageParams p) {
    using Code = typename Fmt<F>::Code;
    __shared__ double lds[kThreads / 64];
    const double inv = 1.0 / (double)p.K;
    for (uint32_t c = blockIdx.x; c < p.chunks; c += gridDim.x) {
        const int64_t c0 = (int64_t)c * (kThreads * 4 * NU);
        const int64_t c1 = c0 + kThreads * 4 * NU < p.P ? c0 + kThreads * 4 * NU : p.P;
        const int64_t e0 = c0 + threadIdx.x * 4;
        double s1[NU][4] = {}, s2[NU][4] = {};
        for (int32_t k = 0; k < p.K; ++k) {
            const uint8_t *codes = p.codes + k * p.code_ld, *scales = p.scales + k * p.scale_ld;
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                const int64_t e = e0 + u * (kThreads * 4);
                if (e >= p.P) continue;
                const f4 v = Fmt<F>::decode(*reinterpret_cast<const Code *>(codes + (e >> 2) * sizeof(Code)),
                                            scale_of(scales[e >> 5]));
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const double d = v[j];
                    s1[u][j] += d;
                    s2[u][j] = fma(d, d, s2[u][j]);
                }
            }
        }
        double all = 0.0;
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const int64_t e = e0 + u * (kThreads * 4);
            if (e >= p.P) continue;
            f4 v = {0.f, 0.f, 0.f, 0.f};
            if (p.base) v = load4(p.base, e, p.P);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] = (float)((double)v[j] + s1[u][j] * inv);
                double q = (double)p.K * s2[u][j] - s1[u][j] * s1[u][j];
                q = e + j < p.P ? (q < 0.0 ? 0.0 : q) : 0.0;    // (a NaN stays)
                s2[u][j] = q;
                all += q;
            }
            if (p.base_out) store4(p.base_out, e, p.P, v);
            if (p.x)
                for (int32_t k = 0; k < p.K; ++k) store4(p.x + k * p.x_ld, e, p.P, v);
        }
        int32_t tau = tensor_at(p.off, p.T, c0);
        if (p.off[tau + 1] >= c1) {
            all = block_sum(all, lds);
            if (threadIdx.x == 0) p.partials[(int64_t)c + tau] = all;
            continue;
        }
        for (; tau < p.T && p.off[tau] < c1; ++tau) {
            const int64_t lo = p.off[tau], hi = p.off[tau + 1];
            if (hi <= lo || hi <= c0) continue;
            double part = 0.0;
#pragma unroll
            for (int u = 0; u < NU; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int64_t e = e0 + u * (kThreads * 4) + j;
                    if (e >= lo && e < hi) part += s2[u][j];
                }
            part = block_sum(part, lds);
            if (threadIdx.x == 0) p.partials[(int64_t)c + tau] = part;
        }
    }
}

// One block per tensor: the sum of its chunks' partial sums over K^2.
__global__ void __launch_bounds__(kThreads) k_mx_variance(const int64_t *off, const double *partials, int64_t chunk,
                                                          int64_t P, int32_t T, double k2, double *var) {
    __shared__ double lds[kThreads / 64];
    for (int32_t tau = blockIdx.x; tau < T; tau += gridDim.x) {
        const int64_t lo = off[tau] > 0 ? off[tau] : 0, hi = off[tau + 1] < P ? off[tau + 1] : P;
        double s = 0.0;
        if (hi > lo) {
            const int64_t last = (hi - 1) / chunk;
            for (int64_t c = lo / chunk + threadIdx.x; c <= last; c += kThreads) s += partials[c + tau];
        }
        s = block_sum(s, lds);
        if (threadIdx.x == 0) var[tau] = s / k2;
    }
}

// ---- product ----------------------------------------------------------------
// Rows of the two operands are the rows and columns of C, the elements are the
// contraction, on 16x16 tiles.  A lane holds one row (lane mod 16) and, of
// every 512 elements, each fourth 16-byte unit (lane / 16).  Which elements
// share a matrix instruction does not matter to the sum, only that both
// operands agree.
//   E2M1: a unit is a block; the scaled 16x16x128 instruction multiplies the
//         codes and applies both scales; its sums are rounded as fp32.
//   E4M3: the 8-bit instructions drop products 2^-15 below the largest of
//         their sum, so the codes are converted to bf16, exactly and with
//         their scales (an element below 2^-126 becomes zero), for the bf16 instruction.
constexpr int kSuper = 512;

struct ProductParams {
    const uint8_t *ac, *as, *bc, *bs;
    const int64_t *off;
    float *partials;       // [chunks + T][K][K]
    int64_t code_ld, scale_ld;    // of a
    int64_t b_code_ld, b_scale_ld;
    int64_t P;
    int64_t chunk;         // elements, a multiple of 4 kSuper
    uint32_t chunks;
    int32_t K, T;
};

// Keep the elements of 16-byte unit [first, first + n) that lie in [lo, hi).
template <int F>
__device__ __forceinline__ void mask_unit(u4 &v, uint32_t &scale, int64_t first, int64_t lo, int64_t hi) {
    constexpr int n = F == ADPSGD_MX_E2M1 ? 32 : 16, bits = 128 / n, per = 32 / bits;
    int64_t a = lo - first, b = hi - first;
    a = a < 0 ? 0 : a;
    b = b > n ? n : b;
    if (a >= b) {
        v = u4{0, 0, 0, 0};
        scale = 127;       // (nothing here is this tensor's, a NaN scale neither)
        return;
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        uint32_t m = 0;
        for (int j = 0; j < per; ++j)
            if (w * per + j >= a && w * per + j < b) m |= ((bits == 4 ? 0xfu : 0xffu) << (bits * j));
        v[w] &= m;
    }
}

// A unit of E4M3 codes as two operands of the bf16 instruction.
__device__ __forceinline__ void bf16_of(const u4 &v, uint32_t byte, bf8v *out) {
    const float s = scale_of(byte);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        u4 o;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const uint32_t c = v[2 * h + w];
            o[2 * w] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, s, false));
            o[2 * w + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, s, true));
        }
        out[h] = __builtin_bit_cast(bf8v, o);
    }
}

// One 16-byte unit of NT tiles of 16 rows, and its scale.
template <int F, int NT>
struct Unit {
    u4 code[NT];
    uint32_t scale[NT];
};

// Scale bytes of a superblock's units j of this lane, out of the row's 16.
template <int F>
__device__ __forceinline__ uint32_t unit_scale(const u4 &bytes, int j) {
    const int q = (threadIdx.x & 63) >> 4;
    if constexpr (F == ADPSGD_MX_E2M1) return (bytes[j] >> (8 * q)) & 0xff;
    else return (bytes[j >> 1] >> (16 * (j & 1) + 8 * (q >> 1))) & 0xff;
}

template <int F>
__device__ __forceinline__ v4 multiply(const u4 &a, uint32_t sa, const u4 &b, uint32_t sb, v4 acc) {
    if constexpr (F == ADPSGD_MX_E2M1) {
        const i8v x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
        const i8v y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, acc, 4, 4, 0, (int)sa, 0, (int)sb);
    } else {
        bf8v x[2], y[2];
        bf16_of(a, sa, x);
        bf16_of(b, sb, y);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[0], y[0], acc, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[1], y[1], acc, 0, 0, 0);
    }
}

// Groups of 16 NT rows that a block of the grid's second axis multiplies.
enum { kDiagonal = 0, kAbove = 1, kEvery = 2 };

// NT: tiles of 16 rows of an operand that a wave holds at once.  kDiagonal: a
// group with itself (b is a), tiles below the diagonal left out; kAbove: the
// pairs of groups I < J (b is a); kEvery: all pairs.
template <int F, int NT, int Pairs>
__global__ void __launch_bounds__(kThreads) k_mx_product(ProductParams p) {
    constexpr bool kOne = Pairs == kDiagonal;
    constexpr int kUnits = F == ADPSGD_MX_E2M1 ? 4 : 8;   // a lane's units of a superblock
    constexpr int kUnitElems = F == ADPSGD_MX_E2M1 ? 32 : 16;
    __shared__ float lds[kThreads / 64][256];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t units = (p.P + kMxBlock - 1) / kMxBlock * (kMxBlock / kUnitElems);
    const int32_t groups = (p.K + 16 * NT - 1) / (16 * NT);
    int32_t I = blockIdx.y, J = blockIdx.y;
    if (Pairs == kEvery) {
        I = blockIdx.y / groups;
        J = blockIdx.y % groups;
    } else if (Pairs == kAbove) {
        I = 0;
        while (J >= groups - 1 - I) {
            J -= groups - 1 - I;
            ++I;
        }
        J += I + 1;
    }
    // this lane's rows; those past K repeat the last one: their part of C is not kept
    const uint8_t *ac[NT], *as[NT], *bc[NT], *bs[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        int32_t r = (I * NT + t) * 16 + (lane & 15);
        r = r < p.K ? r : p.K - 1;
        ac[t] = p.ac + r * p.code_ld;
        as[t] = p.as + r * p.scale_ld;
        r = (J * NT + t) * 16 + (lane & 15);
        r = r < p.K ? r : p.K - 1;
        bc[t] = p.bc + r * p.b_code_ld;
        bs[t] = p.bs + r * p.b_scale_ld;
    }
    for (uint32_t c = blockIdx.x; c < p.chunks; c += gridDim.x) {
        const int64_t c0 = (int64_t)c * p.chunk;
        const int64_t c1 = c0 + p.chunk < p.P ? c0 + p.chunk : p.P;
        for (int32_t tau = tensor_at(p.off, p.T, c0); tau < p.T && p.off[tau] < c1; ++tau) {
            int64_t lo = p.off[tau], hi = p.off[tau + 1];
            lo = lo > c0 ? lo : c0;
            hi = hi < c1 ? hi : c1;
            if (hi <= lo) continue;
            v4 acc[NT][NT];
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = v4{0.f, 0.f, 0.f, 0.f};
            for (int64_t sb = lo / kSuper + wave; sb * kSuper < hi; sb += kThreads / 64) {
                const bool edge = sb * kSuper < lo || (sb + 1) * kSuper > hi;
                u4 sa[NT], sbb[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    sa[t] = *reinterpret_cast<const u4 *>(as[t] + sb * 16);
                    if (!kOne) sbb[t] = *reinterpret_cast<const u4 *>(bs[t] + sb * 16);
                }
#pragma unroll
                for (int j = 0; j < kUnits; ++j) {
                    const int64_t at = sb * (4 * kUnits) + 4 * j + (lane >> 4);
                    const int64_t u = at < units ? at : units - 1;
                    Unit<F, NT> a, b;
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        a.code[t] = *reinterpret_cast<const u4 *>(ac[t] + u * 16);
                        a.scale[t] = unit_scale<F>(sa[t], j);
                        if (!kOne) {
                            b.code[t] = *reinterpret_cast<const u4 *>(bc[t] + u * 16);
                            b.scale[t] = unit_scale<F>(sbb[t], j);
                        }
                        if (edge) {
                            mask_unit<F>(a.code[t], a.scale[t], at * kUnitElems, lo, hi);
                            if (!kOne) mask_unit<F>(b.code[t], b.scale[t], at * kUnitElems, lo, hi);
                        }
                    }
                    const Unit<F, NT> &o = kOne ? a : b;
#pragma unroll
                    for (int i = 0; i < NT; ++i)
#pragma unroll
                        for (int t = kOne ? i : 0; t < NT; ++t)
                            acc[i][t] = multiply<F>(a.code[i], a.scale[i], o.code[t], o.scale[t], acc[i][t]);
                }
            }
            // the four waves' tiles, summed, into the pair's partial sum
            float *out = p.partials + ((int64_t)c + tau) * p.K * p.K;
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = kOne ? i : 0; j < NT; ++j) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) lds[wave][(4 * (lane >> 4) + r) * 16 + (lane & 15)] = acc[i][j][r];
                    __syncthreads();
                    const int32_t row = (I * NT + i) * 16 + (int32_t)threadIdx.x / 16;
                    const int32_t col = (J * NT + j) * 16 + (int32_t)threadIdx.x % 16;
                    double s = 0.0;
                    for (int w = 0; w < kThreads / 64; ++w) s += lds[w][threadIdx.x];
                    if (row < p.K && col < p.K) out[(int64_t)row * p.K + col] = (float)s;
                    __syncthreads();
                }
        }
    }
}

// The tensors' sums of their chunks' partial sums; where b is a, tiles below
// the diagonal are the transposed ones above it.
__global__ void __launch_bounds__(kThreads) k_mx_product_sum(const int64_t *off, const float *partials, int64_t chunk,
                                                             int64_t P, int32_t K, int32_t T, int same, float *out) {
    const int64_t n = (int64_t)K * K;
    for (int32_t tau = blockIdx.x; tau < T; tau += gridDim.x) {
        const int64_t lo = off[tau] > 0 ? off[tau] : 0, hi = off[tau + 1] < P ? off[tau + 1] : P;
        const int64_t i = (int64_t)blockIdx.y * kThreads + threadIdx.x;
        if (i >= n) continue;
        const int32_t row = (int32_t)(i / K), col = (int32_t)(i % K);
        const int64_t at = same && row / 16 > col / 16 ? (int64_t)col * K + row : i;
        double s = 0.0;
        if (hi > lo)
            for (int64_t c = lo / chunk; c <= (hi - 1) / chunk; ++c) s += partials[(c + tau) * n + at];
        out[tau * n + i] = (float)s;
    }
}

}  // namespace
}  // namespace adpsgd

using namespace adpsgd;

namespace {

struct Bytes {
    int64_t codes, scales;      // of a row
};
Bytes row_bytes(int32_t format, int64_t P) {
    const int64_t blocks = (P + kMxBlock - 1) / kMxBlock;
    return {blocks * (format == ADPSGD_MX_E2M1 ? 16 : 32), blocks};
}

bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
bool aligned4(const void *p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

// Rows of device memory that a call reads or writes (ptr NULL: none).
struct Rows {
    const char *name;
    const void *ptr;
    int64_t rows, stride, bytes;      // stride and length of a row in bytes
};
Rows floats(const char *name, const float *p, int64_t rows, int64_t ld, int64_t P) {
    return {name, p, rows, 4 * ld, 4 * P};
}
Rows code_rows(const adpsgd_mx_rows *r) {
    return {"codes", r->codes, r->K, r->code_stride, row_bytes(r->format, r->P).codes};
}
Rows scale_rows(const adpsgd_mx_rows *r) {
    return {"scales", r->scales, r->K, r->scale_stride, row_bytes(r->format, r->P).scales};
}

// Both sets of rows ascend in memory, so two steps through them find a common byte.
bool overlap(const Rows &a, const Rows &b) {
    if (!a.ptr || !b.ptr) return false;
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a.ptr), pb = reinterpret_cast<uintptr_t>(b.ptr);
    const uintptr_t ea = pa + (uintptr_t)((a.rows - 1) * a.stride + a.bytes);
    const uintptr_t eb = pb + (uintptr_t)((b.rows - 1) * b.stride + b.bytes);
    if (ea <= pb || eb <= pa) return false;
    for (int64_t i = 0, j = 0; i < a.rows && j < b.rows;) {
        const uintptr_t x = pa + (uintptr_t)(i * a.stride), y = pb + (uintptr_t)(j * b.stride);
        if (x + (uintptr_t)a.bytes <= y) ++i;
        else if (y + (uintptr_t)b.bytes <= x) ++j;
        else return true;
    }
    return false;
}

int check_apart(const Rows &out, std::initializer_list<Rows> others) {
    for (const Rows &r : others)
        if (overlap(out, r))
            return fail(ADPSGD_EINVAL, std::string(out.name) + " and " + r.name + " overlap");
    return ADPSGD_OK;
}

int check_rows(const adpsgd_mx_rows *r, const char *name) {
    const std::string n(name);
    if (!r) return fail(ADPSGD_EINVAL, n + " is NULL");
    if (r->format != ADPSGD_MX_E2M1 && r->format != ADPSGD_MX_E4M3)
        return fail(ADPSGD_EINVAL, n + ".format must be ADPSGD_MX_E2M1 or ADPSGD_MX_E4M3");
    if (r->K < 1 || r->K > kMaxK) return fail(ADPSGD_EINVAL, "K must be in [1, 65536]");
    if (r->P < 0 || (r->P + 3) / 4 > (int64_t(1) << 32)) return fail(ADPSGD_EINVAL, "P must be >= 0 with P/4 below 2^32");
    if ((r->P + 1023) / 1024 * r->K > kMaxPieces) return fail(ADPSGD_EINVAL, "K * P must be below 2^41");
    const Bytes need = row_bytes(r->format, r->P);
    if (r->code_stride < need.codes || r->code_stride % 16 != 0)
        return fail(ADPSGD_EINVAL, n + ".code_stride must be a multiple of 16 and hold a row (" +
                                       std::to_string(need.codes) + " bytes)");
    if (r->scale_stride < need.scales || r->scale_stride % 16 != 0)
        return fail(ADPSGD_EINVAL, n + ".scale_stride must be a multiple of 16 and hold a row (" +
                                       std::to_string(need.scales) + " bytes)");
    if (r->P > 0 && (!r->codes || !r->scales || !aligned16(r->codes) || !aligned16(r->scales)))
        return fail(ADPSGD_EINVAL, n + ".codes and .scales must be non-NULL and 16-byte aligned");
    return ADPSGD_OK;
}

// The row stride of a float array (0 means P).
int check_ld(int64_t stride, int64_t P, const char *name, int64_t *ld) {
    if (stride < 0 || (stride > 0 && stride < P))
        return fail(ADPSGD_EINVAL, std::string(name) + " must be 0 or >= P");
    *ld = stride > 0 ? stride : P;
    return ADPSGD_OK;
}

int check_float(const float *p, bool needed, const char *name) {
    if ((needed && !p) || !aligned4(p))
        return fail(ADPSGD_EINVAL, std::string(name) + (needed ? " must be non-NULL and 4-byte aligned" : " must be 4-byte aligned"));
    return ADPSGD_OK;
}

int check_tensors(int32_t T, const int64_t *off) {
    if (T < 1 || T > kMaxT) return fail(ADPSGD_EINVAL, "T must be in [1, 2^24]");
    if (!off || reinterpret_cast<uintptr_t>(off) % 8 != 0)
        return fail(ADPSGD_EINVAL, "tensor_offsets must be non-NULL and 8-byte aligned");
    return ADPSGD_OK;
}

int check_workspace(const void *ws, size_t have, size_t need) {
    if (need > 0 && (!ws || reinterpret_cast<uintptr_t>(ws) % 256 != 0))
        return fail(ADPSGD_EINVAL, "workspace must be non-NULL and 256-byte aligned");
    if (have < need) return fail(ADPSGD_EINVAL, "workspace needs " + std::to_string(need) + " bytes");
    return ADPSGD_OK;
}

int launched(const char *what) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(ADPSGD_EDEVICE, std::string(what) + ": " + hipGetErrorString(e));
    return ok();
}

uint32_t grid_for(uint64_t blocks) { return (uint32_t)(blocks < kMaxGrid ? blocks : kMaxGrid); }

// Four groups a lane keep more loads in flight; one spreads a small problem
// over more of the chip.
bool four_groups(int64_t elements) { return elements >= int64_t(1) << 22; }

int64_t average_chunk(int64_t P) {
    return kThreads * 4 * (four_groups(P) ? 4 : 1);
}

// Elements of a product block: 2048 blocks of whole superblocks for each wave,
// at most 16384 elements (of which fp32 sums are taken) for one wave.
int64_t product_chunk(int64_t P) {
    const int64_t step = 4 * kSuper;
    int64_t n = (P / 2048 + step - 1) / step * step;
    n = n < step ? step : n;
    return n > 65536 ? 65536 : n;
}

}  // namespace

extern "C" int64_t adpsgd_mx_code_stride(int32_t format, int64_t P) {
    if ((format != ADPSGD_MX_E2M1 && format != ADPSGD_MX_E4M3) || P <= 0) return 0;
    const int64_t n = (row_bytes(format, P).codes + 255) / 256;
    return 256 * (n + 1 - n % 2);
}

extern "C" int64_t adpsgd_mx_scale_stride(int64_t P) {
    if (P <= 0) return 0;
    const int64_t n = (row_bytes(ADPSGD_MX_E2M1, P).scales + 255) / 256;
    return 256 * (n + 1 - n % 2);
}

extern "C" int adpsgd_mx_quantize(const adpsgd_mx_rows *out, const float *x, int64_t x_stride, const float *base,
                                  const float *residual_in, float *residual_out, int64_t residual_stride, void *stream) {
    if (int rc = check_rows(out, "out")) return rc;
    const int64_t P = out->P;
    QuantizeParams p{};
    if (int rc = check_ld(x_stride, P, "x_stride", &p.x_ld)) return rc;
    if (int rc = check_ld(residual_stride, P, "residual_stride", &p.r_ld)) return rc;
    if (int rc = check_float(x, P > 0, "x")) return rc;
    if (int rc = check_float(base, false, "base")) return rc;
    if (int rc = check_float(residual_in, false, "residual_in")) return rc;
    if (int rc = check_float(residual_out, false, "residual_out")) return rc;
    if (P == 0) return ok();
    const int64_t K = out->K;
    const Rows r_x = floats("x", x, K, p.x_ld, P), r_base = floats("base", base, 1, P, P);
    const Rows r_in = floats("residual_in", residual_in != residual_out ? residual_in : nullptr, K, p.r_ld, P);
    const Rows r_out = floats("residual_out", residual_out, K, p.r_ld, P);
    if (int rc = check_apart(r_out, {r_x, r_base, r_in})) return rc;
    if (int rc = check_apart(code_rows(out), {r_x, r_base, floats("residual_in", residual_in, K, p.r_ld, P), r_out})) return rc;
    if (int rc = check_apart(scale_rows(out), {r_x, r_base, floats("residual_in", residual_in, K, p.r_ld, P), r_out, code_rows(out)}))
        return rc;
    p.x = x;
    p.base = base;
    p.r_in = residual_in;
    p.r_out = residual_out;
    p.codes = static_cast<uint8_t *>(out->codes);
    p.scales = static_cast<uint8_t *>(out->scales);
    p.code_ld = out->code_stride;
    p.scale_ld = out->scale_stride;
    p.P = P;
    const bool four = four_groups(out->K * P);
    p.g = row_grid(out->K, P, kThreads * 4 * (four ? 4 : 1));
    const dim3 grid(grid_for(p.g.blocks)), block(kThreads);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (out->format == ADPSGD_MX_E2M1) {
        if (four) k_mx_quantize<ADPSGD_MX_E2M1, 4><<<grid, block, 0, st>>>(p);
        else k_mx_quantize<ADPSGD_MX_E2M1, 1><<<grid, block, 0, st>>>(p);
    } else {
        if (four) k_mx_quantize<ADPSGD_MX_E4M3, 4><<<grid, block, 0, st>>>(p);
        else k_mx_quantize<ADPSGD_MX_E4M3, 1><<<grid, block, 0, st>>>(p);
    }
    return launched("quantize launch");
}

extern "C" int adpsgd_mx_dequantize(const adpsgd_mx_rows *rows, const float *base, float *y, int64_t y_stride,
                                    void *stream) {
    if (int rc = check_rows(rows, "rows")) return rc;
    const int64_t P = rows->P;
    DequantizeParams p{};
    if (int rc = check_ld(y_stride, P, "y_stride", &p.y_ld)) return rc;
    if (int rc = check_float(base, false, "base")) return rc;
    if (int rc = check_float(y, P > 0, "y")) return rc;
    if (P == 0) return ok();
    if (int rc = check_apart(floats("y", y, rows->K, p.y_ld, P),
                             {floats("base", base, 1, P, P), code_rows(rows), scale_rows(rows)}))
        return rc;
    p.codes = static_cast<const uint8_t *>(rows->codes);
    p.scales = static_cast<const uint8_t *>(rows->scales);
    p.base = base;
    p.y = y;
    p.code_ld = rows->code_stride;
    p.scale_ld = rows->scale_stride;
    p.P = P;
    const bool four = four_groups(rows->K * P);
    p.g = row_grid(rows->K, P, kThreads * 4 * (four ? 4 : 1));
    const dim3 grid(grid_for(p.g.blocks)), block(kThreads);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (rows->format == ADPSGD_MX_E2M1) {
        if (four) k_mx_dequantize<ADPSGD_MX_E2M1, 4><<<grid, block, 0, st>>>(p);
        else k_mx_dequantize<ADPSGD_MX_E2M1, 1><<<grid, block, 0, st>>>(p);
    } else {
        if (four) k_mx_dequantize<ADPSGD_MX_E4M3, 4><<<grid, block, 0, st>>>(p);
        else k_mx_dequantize<ADPSGD_MX_E4M3, 1><<<grid, block, 0, st>>>(p);
    }
    return launched("dequantize launch");
}

extern "C" size_t adpsgd_mx_average_workspace(int32_t K, int64_t P, int32_t T) {
    if (K < 1 || K > kMaxK || P < 0 || (P + 3) / 4 > (int64_t(1) << 32) || T < 1 || T > kMaxT) return 0;
    const int64_t chunk = average_chunk(P);
    return sizeof(double) * (size_t)((P + chunk - 1) / chunk + T);
}

extern "C" int adpsgd_mx_average(const adpsgd_mx_rows *rows, int32_t T, const int64_t *tensor_offsets,
                                 const float *base, float *base_out, float *x, int64_t x_stride, double *var,
                                 void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = check_rows(rows, "rows")) return rc;
    const int64_t P = rows->P;
    AverageParams p{};
    if (int rc = check_tensors(T, tensor_offsets)) return rc;
    if (int rc = check_ld(x_stride, P, "x_stride", &p.x_ld)) return rc;
    if (int rc = check_float(base, false, "base")) return rc;
    if (int rc = check_float(base_out, false, "base_out")) return rc;
    if (int rc = check_float(x, false, "x")) return rc;
    if (!var || reinterpret_cast<uintptr_t>(var) % 8 != 0)
        return fail(ADPSGD_EINVAL, "var must be non-NULL and 8-byte aligned");
    if (int rc = check_workspace(workspace, workspace_bytes, adpsgd_mx_average_workspace(rows->K, P, T))) return rc;
    if (P > 0) {
        const Rows r_x = floats("x", x, rows->K, p.x_ld, P), r_out = floats("base_out", base_out, 1, P, P);
        const Rows codes = code_rows(rows), scales = scale_rows(rows);
        if (int rc = check_apart(r_x, {floats("base", base, 1, P, P), r_out, codes, scales})) return rc;
        if (int rc = check_apart(r_out, {floats("base", base != base_out ? base : nullptr, 1, P, P), codes, scales}))
            return rc;
    }
    p.codes = static_cast<const uint8_t *>(rows->codes);
    p.scales = static_cast<const uint8_t *>(rows->scales);
    p.base = base;
    p.base_out = base_out;
    p.x = x;
    p.off = tensor_offsets;
    p.partials = static_cast<double *>(workspace);
    p.code_ld = rows->code_stride;
    p.scale_ld = rows->scale_stride;
    p.P = P;
    const int64_t chunk = average_chunk(P);
    p.chunks = (uint32_t)((P + chunk - 1) / chunk);
    p.K = rows->K;
    p.T = T;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (P > 0) {
        const dim3 grid(grid_for(p.chunks)), block(kThreads);
        if (rows->format == ADPSGD_MX_E2M1) {
            if (four_groups(P)) k_mx_average<ADPSGD_MX_E2M1, 4><<<grid, block, 0, st>>>(p);
            else k_mx_average<ADPSGD_MX_E2M1, 1><<<grid, block, 0, st>>>(p);
        } else {
            if (four_groups(P)) k_mx_average<ADPSGD_MX_E4M3, 4><<<grid, block, 0, st>>>(p);
            else k_mx_average<ADPSGD_MX_E4M3, 1><<<grid, block, 0, st>>>(p);
        }
        if (int rc = launched("average launch")) return rc;
    }
    k_mx_variance<<<grid_for((uint64_t)T), kThreads, 0, st>>>(tensor_offsets, p.partials, chunk, P, T,
                                                              (double)rows->K * rows->K, var);
    return launched("variance launch");
}

extern "C" size_t adpsgd_mx_product_workspace(int32_t K, int64_t P, int32_t T) {
    if (K < 1 || K > kMaxProductK || P < 0 || (P + 3) / 4 > (int64_t(1) << 32) || T < 1 || T > kMaxT) return 0;
    const int64_t chunk = product_chunk(P);
    return sizeof(float) * (size_t)((P + chunk - 1) / chunk + T) * K * K;
}

namespace {

template <int F, int NT>
void launch_product(const ProductParams &p, bool same, hipStream_t st) {
    const int32_t groups = (p.K + 16 * NT - 1) / (16 * NT);
    const uint32_t x = grid_for(p.chunks);
    if (!same) {
        k_mx_product<F, NT, kEvery><<<dim3(x, groups * groups), kThreads, 0, st>>>(p);
        return;
    }
    k_mx_product<F, NT, kDiagonal><<<dim3(x, groups), kThreads, 0, st>>>(p);
    if constexpr (NT == 4)
        if (groups > 1) k_mx_product<F, NT, kAbove><<<dim3(x, groups * (groups - 1) / 2), kThreads, 0, st>>>(p);
}

template <int F>
void launch_product(const ProductParams &p, bool same, hipStream_t st) {
    if (p.K <= 16) launch_product<F, 1>(p, same, st);
    else if (p.K <= 32) launch_product<F, 2>(p, same, st);
    else launch_product<F, 4>(p, same, st);
}

}  // namespace

extern "C" int adpsgd_mx_product(const adpsgd_mx_rows *a, const adpsgd_mx_rows *b, int32_t T,
                                 const int64_t *tensor_offsets, float *out, void *workspace, size_t workspace_bytes,
                                 void *stream) {
    if (int rc = check_rows(a, "a")) return rc;
    const bool same = !b || b == a || (b->codes == a->codes && b->scales == a->scales);
    if (b) {
        if (int rc = check_rows(b, "b")) return rc;
        if (b->format != a->format || b->K != a->K || b->P != a->P ||
            (same && (b->code_stride != a->code_stride || b->scale_stride != a->scale_stride)))
            return fail(ADPSGD_EINVAL, "a and b must have the same format, K and P");
    } else {
        b = a;
    }
    if (a->K > kMaxProductK) return fail(ADPSGD_EINVAL, "K must be in [1, 256]");
    if (int rc = check_tensors(T, tensor_offsets)) return rc;
    if (int rc = check_float(out, true, "out")) return rc;
    const int64_t P = a->P;
    if (int rc = check_workspace(workspace, workspace_bytes, adpsgd_mx_product_workspace(a->K, P, T))) return rc;
    ProductParams p{};
    p.ac = static_cast<const uint8_t *>(a->codes);
    p.as = static_cast<const uint8_t *>(a->scales);
    p.bc = static_cast<const uint8_t *>(b->codes);
    p.bs = static_cast<const uint8_t *>(b->scales);
    p.off = tensor_offsets;
    p.partials = static_cast<float *>(workspace);
    p.code_ld = a->code_stride;
    p.scale_ld = a->scale_stride;
    p.b_code_ld = b->code_stride;
    p.b_scale_ld = b->scale_stride;
    p.P = P;
    p.chunk = product_chunk(P);
    p.chunks = (uint32_t)((P + p.chunk - 1) / p.chunk);
    p.K = a->K;
    p.T = T;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (P > 0) {
        if (a->format == ADPSGD_MX_E2M1) launch_product<ADPSGD_MX_E2M1>(p, same, st);
        else launch_product<ADPSGD_MX_E4M3>(p, same, st);
        if (int rc = launched("product launch")) return rc;
    }
    const uint32_t per = (uint32_t)(((int64_t)a->K * a->K + kThreads - 1) / kThreads);
    k_mx_product_sum<<<dim3(grid_for((uint64_t)T), per), kThreads, 0, st>>>(tensor_offsets, p.partials, p.chunk, P,
                                                                            a->K, T, same, out);
    return launched("product sum launch");
}
