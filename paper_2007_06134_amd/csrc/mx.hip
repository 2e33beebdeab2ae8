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
constexpr uint32_t kMaxGrid = 1u << 23;
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
        for (uint32_t w = 0; w < blockDim.x / 64; ++w) t += lds[w];
    __syncthreads();
    return t;
}

// A float4 group of a row.  NT: past the caches, for rows that they would not
// keep.  Full: the caller knows that the group ends by the row's end.
template <bool NT, bool Full>
__device__ __forceinline__ f4 load4(const float *p, int64_t e, int64_t P) {
    if (Full || e + 4 <= P) {
        if constexpr (NT) return __builtin_nontemporal_load(reinterpret_cast<const f4 *>(p + e));
        return *reinterpret_cast<const f4 *>(p + e);
    }
    f4 v = {0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < 4; ++j)
        if (e + j < P) v[j] = p[e + j];
    return v;
}
template <bool NT, bool Full>
__device__ __forceinline__ void store4(float *p, int64_t e, int64_t P, f4 v) {
    if (Full || e + 4 <= P) {
        if constexpr (NT) __builtin_nontemporal_store(v, reinterpret_cast<f4 *>(p + e));
        else *reinterpret_cast<f4 *>(p + e) = v;
        return;
    }
    for (int j = 0; j < 4; ++j)
        if (e + j < P) p[e + j] = v[j];
}

// ---- quantize, dequantize ---------------------------------------------------
// A wave takes pieces of kPiece elements of one row, the kilobyte that its
// lanes' float4 groups are.  Blocks are dealt to the XCDs round-robin, and so
// are a row's pieces; an XCD takes `run` of its pieces of one row, then the
// same pieces of the next row, so that base comes from memory once and from
// that XCD's L2 for the other rows.
constexpr int kPiece = 256;
struct RowGrid {
    uint32_t K;
    uint32_t slots;        // of a row: groups of spread NU pieces
    uint32_t blocks;       // virtual blocks of the launch
    uint32_t spread;       // 8: pieces dealt to XCDs; 1: too few pieces for that
    uint32_t run;
};
RowGrid row_grid(int32_t K, int64_t P, int nu) {
    RowGrid g;
    const int64_t pieces = (P + kPiece - 1) / kPiece;
    g.K = (uint32_t)K;
    g.spread = pieces >= 8 ? 8 : 1;
    g.slots = (uint32_t)((pieces + g.spread * nu - 1) / (g.spread * nu));
    g.run = g.slots >= 128u / nu ? 32u / nu : 1;
    g.blocks = (g.slots + g.run - 1) / g.run * g.run * g.spread * g.K;
    return g;
}
// Block b's row and first piece (its further ones lie spread apart).
__device__ __forceinline__ bool row_piece(const RowGrid &g, int nu, uint32_t b, uint32_t *k, uint32_t *piece) {
    const uint32_t s = b / g.spread, run = s / g.run;
    *k = run % g.K;
    const uint32_t slot = run / g.K * g.run + s % g.run;
    *piece = slot * nu * g.spread + b % g.spread;
    return slot < g.slots;
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
template <int F, bool NT, bool Full>
__device__ __forceinline__ void quantize_piece(const QuantizeParams &p, uint32_t k, int64_t e) {
    using Code = typename Fmt<F>::Code;
    f4 d = load4<NT, Full>(p.x + k * p.x_ld, e, p.P);
    f4 b = {0.f, 0.f, 0.f, 0.f}, r = {0.f, 0.f, 0.f, 0.f};
    if (p.base) b = load4<false, Full>(p.base, e, p.P);
    if (p.r_in) r = load4<NT, Full>(p.r_in + k * p.r_ld, e, p.P);
    if (p.base) d -= b;
    if (p.r_in) d += r;
    // (lanes of one block are all past the padded row's end or none is)
    if (!Full && e >= (p.P + kMxBlock - 1) / kMxBlock * kMxBlock) return;
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t a = __float_as_uint(d[j]) & 0x7fffffffu;
        m = a > m ? a : m;
    }
    m = max_of_8_lanes(m);
    // the least power of two that holds the largest element
    const int32_t s = (int32_t)(m >> 23) - Fmt<F>::kTopExp + ((m & 0x7fffffu) > Fmt<F>::kTopMan ? 1 : 0);
    uint32_t byte = (uint32_t)(s > 0 ? s : 0);
    f4 v = d;
    float scale = scale_of(byte);
    if (m >= __float_as_uint(Fmt<F>::kMost)) {
        if (m >= 0x7f800000u) {      // a NaN or an infinity: nothing of the block can be sent
            byte = 255;
            scale = 1.f;
            d = v = f4{0.f, 0.f, 0.f, 0.f};
        } else {                     // the format's next number is 2^128
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = fminf(fmaxf(v[j], -Fmt<F>::kMost), Fmt<F>::kMost);
        }
    }
    const uint32_t c = Fmt<F>::encode(v, scale);
    *reinterpret_cast<Code *>(p.codes + k * p.code_ld + (e >> 2) * sizeof(Code)) = (Code)c;
    if ((threadIdx.x & 7) == 0) p.scales[k * p.scale_ld + (e >> 5)] = (uint8_t)byte;
    if (p.r_out && (Full || e < p.P))
        store4<NT, Full>(p.r_out + k * p.r_ld, e, p.P, d - Fmt<F>::decode(c, scale));
}

template <int F, bool NT>
__global__ void __launch_bounds__(64) k_mx_quantize(QuantizeParams p) {
    for (uint32_t b = blockIdx.x; b < p.g.blocks; b += gridDim.x) {
        uint32_t k, piece;
        if (!row_piece(p.g, 1, b, &k, &piece)) continue;
        const int64_t e0 = (int64_t)piece * kPiece, e = e0 + threadIdx.x * 4;
        if (e0 + kPiece <= p.P) quantize_piece<F, NT, true>(p, k, e);
        else quantize_piece<F, NT, false>(p, k, e);
    }
}

struct DequantizeParams {
    const uint8_t *codes;
    const uint8_t *scales;
    const float *base;
    float *y;
    int64_t y_ld, code_ld, scale_ld;
    int64_t P;
    int32_t K;
    uint32_t groups, blocks, spread;
};

// A block takes a chunk of the elements of up to kReadRows rows: base is loaded
// once for them.
constexpr int kReadRows = 4;
constexpr int kReadChunk = kThreads * 4;
template <int F, bool NT, bool Full>
__device__ __forceinline__ void dequantize_chunk(const DequantizeParams &p, int32_t k0, int64_t e) {
    using Code = typename Fmt<F>::Code;
    const int64_t at = Full || e < p.P ? e : (p.P - 1) / 4 * 4;
    uint32_t c[kReadRows], s[kReadRows];
    f4 b = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kReadRows; ++i) {
        if (k0 + i >= p.K) break;
        c[i] = *reinterpret_cast<const Code *>(p.codes + (k0 + i) * p.code_ld + (at >> 2) * sizeof(Code));
        s[i] = p.scales[(k0 + i) * p.scale_ld + (at >> 5)];
    }
    if (p.base) b = load4<false, Full>(p.base, e, p.P);
#pragma unroll
    for (int i = 0; i < kReadRows; ++i) {
        if (k0 + i >= p.K) break;
        f4 v = Fmt<F>::decode(c[i], scale_of(s[i]));
        if (p.base) v = b + v;
        store4<NT, Full>(p.y + (k0 + i) * p.y_ld, e, p.P, v);
    }
}

template <int F, bool NT>
__global__ void __launch_bounds__(kThreads) k_mx_dequantize(DequantizeParams p) {
    for (uint32_t b = blockIdx.x; b < p.blocks; b += gridDim.x) {
        // the groups of rows of one chunk follow one another on one XCD
        const uint32_t s = b / p.spread;
        const int32_t k0 = (int32_t)(s % p.groups) * kReadRows;
        const int64_t c0 = (int64_t)(s / p.groups * p.spread + b % p.spread) * kReadChunk;
        if (c0 >= p.P) continue;
        if (c0 + kReadChunk <= p.P) dequantize_chunk<F, NT, true>(p, k0, c0 + threadIdx.x * 4);
        else dequantize_chunk<F, NT, false>(p, k0, c0 + threadIdx.x * 4);
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
constexpr int kRowsAtOnce = 8;     // rows whose codes are in flight together
constexpr int kAverageGroups = 2;  // float4 groups of a lane in a large problem

template <int F, int NU, bool NT, bool Full>
__device__ __forceinline__ void average_chunk(const AverageParams &p, int64_t c0, int64_t c1, double s2[NU][4],
                                              int32_t *tau, double *all) {
    using Code = typename Fmt<F>::Code;
    const int64_t e0 = c0 + threadIdx.x * 4;
    double s1[NU][4] = {};
    int64_t at[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        at[u] = e0 + u * (kThreads * 4);
        if (!Full && at[u] >= p.P) at[u] = (p.P - 1) / 4 * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) s2[u][j] = 0.0;
    }
    f4 b[NU];
    for (int32_t k0 = 0; k0 < p.K; k0 += kRowsAtOnce) {
        uint32_t c[kRowsAtOnce][NU], s[kRowsAtOnce][NU];
#pragma unroll
        for (int i = 0; i < kRowsAtOnce; ++i) {
            if (k0 + i >= p.K) break;
            const uint8_t *codes = p.codes + (k0 + i) * p.code_ld, *scales = p.scales + (k0 + i) * p.scale_ld;
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                c[i][u] = *reinterpret_cast<const Code *>(codes + (at[u] >> 2) * sizeof(Code));
                s[i][u] = scales[at[u] >> 5];
            }
        }
        if (k0 == 0) {     // the rest that has to come from memory, behind the first rows
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                b[u] = f4{0.f, 0.f, 0.f, 0.f};
                if (p.base) b[u] = load4<false, Full>(p.base, e0 + u * (kThreads * 4), p.P);
            }
            *tau = tensor_at(p.off, p.T, c0);
        }
#pragma unroll
        for (int i = 0; i < kRowsAtOnce; ++i) {
            if (k0 + i >= p.K) break;
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                const f4 v = Fmt<F>::decode(c[i][u], scale_of(s[i][u]));
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const double d = v[j];
                    s1[u][j] += d;
                    s2[u][j] = fma(d, d, s2[u][j]);
                }
            }
        }
    }
    const double inv = 1.0 / (double)p.K;
    *all = 0.0;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        const int64_t e = e0 + u * (kThreads * 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            b[u][j] = (float)((double)b[u][j] + s1[u][j] * inv);
            double q = (double)p.K * s2[u][j] - s1[u][j] * s1[u][j];
            q = Full || e + j < c1 ? (q < 0.0 ? 0.0 : q) : 0.0;    // (a NaN stays)
            s2[u][j] = q;
            *all += q;
        }
        if (p.base_out) store4<NT, Full>(p.base_out, e, p.P, b[u]);
        if (p.x)
            for (int32_t k = 0; k < p.K; ++k) store4<NT, Full>(p.x + k * p.x_ld, e, p.P, b[u]);
    }
}

template <int F, int NU, bool NT>
__global__ void __launch_bounds__(kThreads) k_mx_average(AverageParams p) {
    __shared__ double lds[kThreads / 64];
    constexpr int kChunk = kThreads * 4 * NU;
    for (uint32_t c = blockIdx.x; c < p.chunks; c += gridDim.x) {
        const int64_t c0 = (int64_t)c * kChunk, c1 = c0 + kChunk < p.P ? c0 + kChunk : p.P;
        double q[NU][4], all;
        int32_t tau;
        if (c0 + kChunk <= p.P) average_chunk<F, NU, NT, true>(p, c0, c1, q, &tau, &all);
        else average_chunk<F, NU, NT, false>(p, c0, c1, q, &tau, &all);
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
                    const int64_t e = c0 + threadIdx.x * 4 + u * (kThreads * 4) + j;
                    if (e >= lo && e < hi) part += q[u][j];
                }
            part = block_sum(part, lds);
            if (threadIdx.x == 0) p.partials[(int64_t)c + tau] = part;
        }
    }
}

// One block per tensor: the sum of its chunks' partial sums over K^2.
__global__ void __launch_bounds__(1024) k_mx_variance(const int64_t *off, const double *partials, int64_t chunk,
                                                      int64_t P, int32_t T, double k2, double *var) {
    __shared__ double lds[16];
    for (int32_t tau = blockIdx.x; tau < T; tau += gridDim.x) {
        const int64_t lo = off[tau] > 0 ? off[tau] : 0, hi = off[tau + 1] < P ? off[tau + 1] : P;
        double s = 0.0;
        if (hi > lo) {
            const int64_t last = (hi - 1) / chunk;
            // (threads past a short tensor's chunks add nothing)
            double t[4] = {};
            int64_t c = lo / chunk + threadIdx.x;
            for (; c + 3 * (int64_t)blockDim.x <= last; c += 4 * (int64_t)blockDim.x)
                for (int i = 0; i < 4; ++i) t[i] += partials[c + i * (int64_t)blockDim.x + tau];
            for (; c <= last; c += blockDim.x) t[0] += partials[c + tau];
            s = (t[0] + t[1]) + (t[2] + t[3]);
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
// Where K <= 8, the 16 rows of the tile are 16 / R stretches of 512 elements of
// R = 1, 2, 4 or 8 workers: products of different stretches come out too and
// are left out.
constexpr int kSuper = 512;

struct ProductParams {
    const uint8_t *ac, *as, *bc, *bs;
    const int64_t *off;
    float *partials;       // [chunks + T][K][K]
    int64_t code_ld, scale_ld;    // of a
    int64_t b_code_ld, b_scale_ld;
    int64_t P;
    int64_t chunk;         // elements, a multiple of 4 stretches kSuper
    uint32_t chunks;
    int32_t K, T;
    int32_t R, stretches;  // 16 and 1 where K > 8
};

// Bits of the elements [a, b) of 32 / bits elements from w * (32 / bits) on.
template <int bits>
__device__ __forceinline__ uint32_t element_mask(int a, int b, int w) {
    constexpr int per = 32 / bits;
    a -= w * per;
    b -= w * per;
    a = a < 0 ? 0 : (a > per ? per : a);
    b = b < 0 ? 0 : (b > per ? per : b);
    return (uint32_t)((1ull << (bits * b)) - 1) & ~(uint32_t)((1ull << (bits * a)) - 1);
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

// The scale byte of this lane's unit j, out of the 16 of its 512 elements.
template <int F>
__device__ __forceinline__ uint32_t unit_scale(const u4 &bytes, int j) {
    const int q = (threadIdx.x & 63) >> 4;
    if constexpr (F == ADPSGD_MX_E2M1) return (bytes[j] >> (8 * q)) & 0xff;
    else return (bytes[j >> 1] >> (16 * (j & 1) + 8 * (q >> 1))) & 0xff;
}

// acc += the products of unit a's tiles with unit o's (One: o is a, and the
// tiles below the diagonal are left out).
template <int F, int NT, bool One>
__device__ __forceinline__ void multiply(const u4 *a, const uint32_t *sa, const u4 *o, const uint32_t *so,
                                         v4 (&acc)[NT][NT]) {
    if constexpr (F == ADPSGD_MX_E2M1) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const i8v x = {(int)a[i][0], (int)a[i][1], (int)a[i][2], (int)a[i][3], 0, 0, 0, 0};
#pragma unroll
            for (int t = One ? i : 0; t < NT; ++t) {
                const i8v y = {(int)o[t][0], (int)o[t][1], (int)o[t][2], (int)o[t][3], 0, 0, 0, 0};
                acc[i][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, acc[i][t], 4, 4, 0, (int)sa[i], 0,
                                                                             (int)so[t]);
            }
        }
    } else {
        bf8v x[NT][2], y[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            bf16_of(a[t], sa[t], x[t]);
            if (!One) bf16_of(o[t], so[t], y[t]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int t = One ? i : 0; t < NT; ++t)
                    acc[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[i][h], One ? x[t][h] : y[t][h], acc[i][t], 0, 0, 0);
    }
}

// One operand's rows as a lane holds them.
template <int NT>
struct Lanes {
    const uint8_t *codes[NT], *scales[NT];
    __device__ __forceinline__ void point(const uint8_t *c, const uint8_t *s, int64_t code_ld, int64_t scale_ld,
                                          int32_t row0, int32_t R, int32_t K) {
        const int r = threadIdx.x & 15;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            // (rows past K repeat the last one: their part of C is not kept)
            int32_t k = NT == 1 ? row0 + r % R : row0 + t * 16 + r;
            k = k < K ? k : K - 1;
            codes[t] = c + k * code_ld;
            scales[t] = s + k * scale_ld;
        }
    }
};

// The products of 512 elements of each of the tile's rows; stretch: this lane's
// first element over 512.  Edge: part of them is not in [lo, hi).
template <int F, int NT, bool One, bool Edge>
__device__ __forceinline__ void product_super(const Lanes<NT> &A, const Lanes<NT> &B, int64_t stretch, int64_t lo,
                                              int64_t hi, int64_t P, v4 (&acc)[NT][NT]) {
    constexpr int kUnits = F == ADPSGD_MX_E2M1 ? 4 : 8;         // a lane's units of 512 elements
    constexpr int kBits = F == ADPSGD_MX_E2M1 ? 4 : 8, n = 128 / kBits;
    const int q = (threadIdx.x & 63) >> 4;
    int64_t st = stretch, last = 0;
    if (Edge) {      // stay inside the rows: what is read again is masked
        const int64_t top = (P - 1) / kSuper;
        st = st < top ? st : top;
        last = (P + kMxBlock - 1) / kMxBlock * (kMxBlock / n) - 1;
    }
    // units in flight together: what the registers hold
    constexpr int kFly = NT == 1 ? kUnits : NT == 2 ? 4 : 2;
    u4 sa[NT], sb[NT], a[kFly][NT], b[kFly][NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        sa[t] = *reinterpret_cast<const u4 *>(A.scales[t] + st * 16);
        if (!One) sb[t] = *reinterpret_cast<const u4 *>(B.scales[t] + st * 16);
    }
    int from = 0, to = kSuper;
    if (Edge) {
        const int64_t e = stretch * kSuper;
        from = lo <= e ? 0 : (lo - e < kSuper ? (int)(lo - e) : kSuper);
        to = hi - e >= kSuper ? kSuper : (hi > e ? (int)(hi - e) : 0);
    }
#pragma unroll
    for (int j0 = 0; j0 < kUnits; j0 += kFly) {
#pragma unroll
        for (int j = 0; j < kFly; ++j) {
            int64_t u = st * (4 * kUnits) + 4 * (j0 + j) + q;
            if (Edge) u = u < last ? u : last;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                a[j][t] = *reinterpret_cast<const u4 *>(A.codes[t] + u * 16);
                if (!One) b[j][t] = *reinterpret_cast<const u4 *>(B.codes[t] + u * 16);
            }
        }
#pragma unroll
        for (int j = 0; j < kFly; ++j) {
            uint32_t ba[NT], bb[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                ba[t] = unit_scale<F>(sa[t], j0 + j);
                if (!One) bb[t] = unit_scale<F>(sb[t], j0 + j);
            }
            if (Edge) {
                const int first = (4 * (j0 + j) + q) * n;
                const bool none = first >= to || first + n <= from;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint32_t m = none ? 0u : element_mask<kBits>(from - first, to - first, w);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        a[j][t][w] &= m;
                        if (!One) b[j][t][w] &= m;
                    }
                }
                // (none of this tensor's elements: neither is a NaN scale its own)
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    ba[t] = none ? 127u : ba[t];
                    if (!One) bb[t] = none ? 127u : bb[t];
                }
            }
            multiply<F, NT, One>(a[j], ba, One ? a[j] : b[j], One ? ba : bb, acc);
        }
        if (kFly < kUnits) __builtin_amdgcn_sched_barrier(0);
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
    constexpr int kWaves = kThreads / 64;
    __shared__ float lds[kWaves][NT * NT][256];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
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
    Lanes<NT> A, B;
    A.point(p.ac, p.as, p.code_ld, p.scale_ld, I * 16 * NT, p.R, p.K);
    if (!kOne) B.point(p.bc, p.bs, p.b_code_ld, p.b_scale_ld, J * 16 * NT, p.R, p.K);
    const int32_t stretches = NT == 1 ? p.stretches : 1;
    const int32_t mine = NT == 1 ? (lane & 15) / p.R : 0;
    const int64_t super = (int64_t)stretches * kSuper;
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
            for (int64_t sb = lo / super + wave; sb * super < hi; sb += kWaves) {
                const int64_t stretch = sb * stretches + mine;
                if (sb * super >= lo && (sb + 1) * super <= hi)
                    product_super<F, NT, kOne, false>(A, B, stretch, lo, hi, p.P, acc);
                else
                    product_super<F, NT, kOne, true>(A, B, stretch, lo, hi, p.P, acc);
            }
            // the waves' tiles (and the stretches' parts of one), summed, into the pair's partial sum
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = kOne ? i : 0; j < NT; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        lds[wave][i * NT + j][(4 * (lane >> 4) + r) * 16 + (lane & 15)] = acc[i][j][r];
            __syncthreads();
            float *out = p.partials + ((int64_t)c + tau) * p.K * p.K;
            const int32_t row = (int32_t)threadIdx.x / 16, col = (int32_t)threadIdx.x % 16;
            if (NT == 1) {
                if (I * 16 + row < p.K && J * 16 + col < p.K && row < p.R && col < p.R) {
                    double s = 0.0;
                    for (int w = 0; w < kWaves; ++w)
                        for (int g = 0; g < stretches; ++g) s += lds[w][0][(g * p.R + row) * 16 + g * p.R + col];
                    out[row * p.K + col] = (float)s;
                }
            } else {
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int j = kOne ? i : 0; j < NT; ++j) {
                        const int32_t y = (I * NT + i) * 16 + row, x = (J * NT + j) * 16 + col;
                        double s = 0.0;
                        for (int w = 0; w < kWaves; ++w) s += lds[w][i * NT + j][threadIdx.x];
                        if (y < p.K && x < p.K) out[(int64_t)y * p.K + x] = (float)s;
                    }
            }
            __syncthreads();
        }
    }
}

// The tensors' sums of their chunks' partial sums, in 64 bits, by lanes of
// `outs` entries: blockDim / outs of them share a tensor's chunks.  Where b is a,
// tiles below the diagonal are the transposed ones above it.
__global__ void __launch_bounds__(1024) k_mx_product_sum(const int64_t *off, const float *partials, int64_t chunk,
                                                         int64_t P, int32_t K, int32_t T, int same, int32_t outs,
                                                         float *out) {
    __shared__ double lds[1024];
    const int64_t n = (int64_t)K * K;
    const int32_t share = blockDim.x / outs, part = threadIdx.x / outs;
    const int64_t i = (int64_t)blockIdx.y * outs + threadIdx.x % outs;
    const int32_t row = (int32_t)(i / K), col = (int32_t)(i % K);
    const float *from = partials + (same && row / 16 > col / 16 ? (int64_t)col * K + row : i);
    for (int32_t tau = blockIdx.x; tau < T; tau += gridDim.x) {
        const int64_t lo = off[tau] > 0 ? off[tau] : 0, hi = off[tau + 1] < P ? off[tau + 1] : P;
        double s[4] = {};
        if (hi > lo && i < n) {
            const int64_t last = (hi - 1) / chunk;
            int64_t c = lo / chunk + part;
            for (; c + 3 * (int64_t)share <= last; c += 4 * (int64_t)share)
                for (int u = 0; u < 4; ++u) s[u] += from[(c + u * (int64_t)share + tau) * n];
            for (; c <= last; c += share) s[0] += from[(c + tau) * n];
        }
        lds[threadIdx.x] = (s[0] + s[1]) + (s[2] + s[3]);
        __syncthreads();
        if (part == 0 && i < n) {
            double t = 0.0;
            for (int32_t w = 0; w < share; ++w) t += lds[w * outs + threadIdx.x];
            out[tau * n + i] = (float)t;
        }
        __syncthreads();
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

// fp32 rows beyond the 256 MB last-level cache go past it.
bool past_cache(int64_t K, int64_t P) { return (double)K * (double)P * 4.0 > 256e6; }

// Several groups a lane for long rows (half the blocks' fixed work), one where
// that would leave compute units without a block.
bool long_rows(int64_t P) { return P >= int64_t(1) << 22; }

int64_t average_chunk_elements(int64_t P) { return kThreads * 4 * (long_rows(P) ? kAverageGroups : 1); }

// Workers of a tile where several stretches share it.
int32_t tile_workers(int32_t K) { return K > 8 ? 16 : K > 4 ? 8 : K > 2 ? 4 : K; }

// Elements of a product block: 2048 blocks of a whole tile for each wave, at
// most 16384 elements (of which fp32 sums are taken) for one wave.
int64_t product_chunk(int32_t K, int64_t P) {
    const int64_t step = 4 * kSuper * (16 / tile_workers(K));
    const int64_t n = (P / 2048 + step - 1) / step * step;
    return n < step ? step : n > 65536 ? 65536 : n;
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
    p.g = row_grid(out->K, P, 1);
    const dim3 grid(grid_for(p.g.blocks)), block(64);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const bool nt = past_cache(out->K, P);
    if (out->format == ADPSGD_MX_E2M1) {
        if (nt) k_mx_quantize<ADPSGD_MX_E2M1, true><<<grid, block, 0, st>>>(p);
        else k_mx_quantize<ADPSGD_MX_E2M1, false><<<grid, block, 0, st>>>(p);
    } else {
        if (nt) k_mx_quantize<ADPSGD_MX_E4M3, true><<<grid, block, 0, st>>>(p);
        else k_mx_quantize<ADPSGD_MX_E4M3, false><<<grid, block, 0, st>>>(p);
    }
    return launched("quantize launch");
}

namespace {

template <int F>
void launch_dequantize(DequantizeParams &p, int32_t K, hipStream_t st) {
    p.K = K;
    p.groups = (uint32_t)((K + kReadRows - 1) / kReadRows);
    const uint32_t chunks = (uint32_t)((p.P + kReadChunk - 1) / kReadChunk);
    p.spread = chunks >= 8 ? 8 : 1;
    p.blocks = (chunks + p.spread - 1) / p.spread * p.spread * p.groups;
    if (past_cache(K, p.P)) k_mx_dequantize<F, true><<<grid_for(p.blocks), kThreads, 0, st>>>(p);
    else k_mx_dequantize<F, false><<<grid_for(p.blocks), kThreads, 0, st>>>(p);
}

template <int F>
void launch_average(const AverageParams &p, hipStream_t st) {
    const bool nt = past_cache(p.K, p.P), several = long_rows(p.P);
    const uint32_t grid = grid_for(p.chunks);
    if (several && nt) k_mx_average<F, kAverageGroups, true><<<grid, kThreads, 0, st>>>(p);
    else if (several) k_mx_average<F, kAverageGroups, false><<<grid, kThreads, 0, st>>>(p);
    else if (nt) k_mx_average<F, 1, true><<<grid, kThreads, 0, st>>>(p);
    else k_mx_average<F, 1, false><<<grid, kThreads, 0, st>>>(p);
}

}  // namespace

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
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (rows->format == ADPSGD_MX_E2M1) launch_dequantize<ADPSGD_MX_E2M1>(p, rows->K, st);
    else launch_dequantize<ADPSGD_MX_E4M3>(p, rows->K, st);
    return launched("dequantize launch");
}

extern "C" size_t adpsgd_mx_average_workspace(int32_t K, int64_t P, int32_t T) {
    if (K < 1 || K > kMaxK || P < 0 || (P + 3) / 4 > (int64_t(1) << 32) || T < 1 || T > kMaxT) return 0;
    const int64_t chunk = average_chunk_elements(P);
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
    const int64_t chunk = average_chunk_elements(P);
    p.chunks = (uint32_t)((P + chunk - 1) / chunk);
    p.K = rows->K;
    p.T = T;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (P > 0) {
        if (rows->format == ADPSGD_MX_E2M1) launch_average<ADPSGD_MX_E2M1>(p, st);
        else launch_average<ADPSGD_MX_E4M3>(p, st);
        if (int rc = launched("average launch")) return rc;
    }
    k_mx_variance<<<grid_for((uint64_t)T), p.chunks > 4096 ? 1024 : kThreads, 0, st>>>(tensor_offsets, p.partials, chunk, P, T,
                                                              (double)rows->K * rows->K, var);
    return launched("variance launch");
}

extern "C" size_t adpsgd_mx_product_workspace(int32_t K, int64_t P, int32_t T) {
    if (K < 1 || K > kMaxProductK || P < 0 || (P + 3) / 4 > (int64_t(1) << 32) || T < 1 || T > kMaxT) return 0;
    const int64_t chunk = product_chunk(K, P);
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
    p.chunk = product_chunk(a->K, P);
    p.chunks = (uint32_t)((P + p.chunk - 1) / p.chunk);
    p.K = a->K;
    p.T = T;
    p.R = tile_workers(a->K);
    p.stretches = 16 / p.R;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (P > 0) {
        if (a->format == ADPSGD_MX_E2M1) launch_product<ADPSGD_MX_E2M1>(p, same, st);
        else launch_product<ADPSGD_MX_E4M3>(p, same, st);
        if (int rc = launched("product launch")) return rc;
    }
    // a block for each tensor and 64 entries; many threads to an entry where a tensor may have many chunks
    const int64_t n = (int64_t)a->K * a->K;
    int32_t outs = 1;
    while (outs < 64 && outs < n) outs *= 2;
    const uint32_t threads = (int64_t)p.chunks > 8 * (int64_t)T ? 1024 : kThreads;
    k_mx_product_sum<<<dim3(grid_for((uint64_t)T), (uint32_t)((n + outs - 1) / outs)), threads, 0, st>>>(
        tensor_offsets, p.partials, p.chunk, P, a->K, T, same, outs, out);
    return launched("product sum launch");
}
