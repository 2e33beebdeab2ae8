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

#include <rocprofiler-sdk-roctx/roctx.h>

#include <algorithm>
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
constexpr int64_t kMaxP = int64_t(1) << 34;
constexpr int32_t kMaxT = 1 << 24;
constexpr int32_t kMaxProductK = 256;
constexpr int64_t kMaxStride = int64_t(1) << 44;   // K rows of this many floats still have 63-bit addresses
// Blocks a launch has at most; the kernels stride over the rest.  A multiple of
// 8, so that a block's chunks stay on its XCD.
constexpr uint32_t kMaxGrid = 1u << 23;
constexpr int64_t kMaxPieces = (int64_t(1) << 31) - 1;   // of K rows (with what padding adds, a 32-bit block number)

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

// The same numbers in 64 bits, where none is too large (those of rows from elsewhere may
// be 2^128 and more, which decode makes infinite: from scale byte kFarByte on).
template <int F>
constexpr uint32_t kFarByte = 254 - Fmt<F>::kTopExp + 1;
struct Wide {
    double v[4];
};
template <int F>
__device__ __forceinline__ Wide decode_wide(uint32_t c, uint32_t byte) {
    const f4 v = Fmt<F>::decode(c, 1.f);
    const uint64_t s = byte == 255 ? 0x7ff8ull << 48 : (uint64_t)(byte + 1023 - 127) << 52;
    Wide w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w.v[j] = (double)v[j] * __builtin_bit_cast(double, s);
    return w;
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

// Where tensors near element e begin: lane i gets tensor *from + i's first element (past
// the last tensor P), the last one to begin by e being among the first 63.  By all
// lanes of a wave, 64 offsets at a time.
__device__ __forceinline__ int64_t offsets_near(const int64_t *off, int32_t T, int64_t e, int32_t *from) {
    int32_t lo = 0, n = T;
    const int lane = threadIdx.x & 63;
    while (n > 63) {
        const int32_t step = (n + 63) / 64;
        const int64_t i = (int64_t)lane * step;
        const uint64_t before = __ballot(i < n && off[lo + (i < n ? i : 0)] <= e);
        const int32_t hits = __popcll(before);
        const int32_t at = (hits > 0 ? hits - 1 : 0) * step;
        lo += at;
        n = n - at < step ? n - at : step;
    }
    *from = __builtin_amdgcn_readfirstlane(lo);
    return off[*from + lane < T ? *from + lane : T];
}

// Element boundaries counted from c0 in 32 bits; -1 and kFar stand for all before it
// and all far behind a chunk.
constexpr int32_t kFar = 1 << 30;
__device__ __forceinline__ int32_t boundary_from(int64_t off, int64_t c0) {
    int64_t v = (int64_t)((uint64_t)off - (uint64_t)c0);
    // (a loaded offset is waited for here: where it is used all stores so far would be, too)
    asm volatile("" : "+v"(v));
    return v < 0 ? -1 : v < kFar ? (int32_t)v : kFar;
}

// The last of the tensors from ... from + 62 that begins at or before the element that
// lane i's bound of tensor from + i is counted from (else the first).
__device__ __forceinline__ int32_t begun(int32_t bound, int32_t from, int32_t T) {
    const int lane = threadIdx.x & 63;
    const int32_t hits = __popcll(__ballot(lane < 63 && from + lane < T && bound <= 0));
    return hits > 0 ? hits - 1 : 0;
}

// A sum over the wave's lanes, in the same order every time.
__device__ __forceinline__ double wave_sum(double v) {
    auto add = [&](auto ctrl) {
        const uint64_t b = __builtin_bit_cast(uint64_t, v);
        constexpr int c = decltype(ctrl)::value;
        const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, c, 0xf, 0xf, true);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), c, 0xf, 0xf, true);
        v += __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
    };
    add(std::integral_constant<int, 0xB1>{});    // quad_perm 1,0,3,2
    add(std::integral_constant<int, 0x4E>{});    // quad_perm 2,3,0,1
    add(std::integral_constant<int, 0x141>{});   // mirrored halves of 16 lanes
    add(std::integral_constant<int, 0x140>{});   // mirrored 16 lanes
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

// A sum over the block's threads, in the same order every time; valid in thread 0.
__device__ __forceinline__ double block_sum(double v, double *lds) {
    v = wave_sum(v);
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
// (K = 8, P = 138M with residuals: 2.24-2.29 ms; 2.48 ms with blocks of 8 KB of a row,
// 2.72 ms with 16 KB.)
constexpr int kPiece = 256;
struct RowGrid {
    uint32_t K;
    uint32_t slots;        // of a row: groups of `spread` pieces
    uint32_t blocks;       // virtual blocks of the launch
    uint32_t spread;       // 8: pieces dealt to XCDs; 1: too few pieces for that
    uint32_t run;
};
RowGrid row_grid(int32_t K, int64_t P) {
    RowGrid g;
    const int64_t pieces = (P + kPiece - 1) / kPiece;
    g.K = (uint32_t)K;
    g.spread = pieces >= 8 ? 8 : 1;
    g.slots = (uint32_t)((pieces + g.spread - 1) / g.spread);
    g.run = g.slots >= 128 ? 32 : 1;
    g.blocks = (g.slots + g.run - 1) / g.run * g.run * g.spread * g.K;
    return g;
}
// Block b's row and piece.
__device__ __forceinline__ bool row_piece(const RowGrid &g, uint32_t b, uint32_t *k, uint32_t *piece) {
    const uint32_t s = b / g.spread, run = s / g.run;
    *k = run % g.K;
    const uint32_t slot = run / g.K * g.run + s % g.run;
    *piece = slot * g.spread + b % g.spread;
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
        if (!row_piece(p.g, b, &k, &piece)) continue;
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
    uint32_t groups, chunks;     // of R rows, of kReadChunk elements
    bool together;
};

// A block takes a chunk of the elements of up to R rows.  The fewer rows are
// written at a time the faster, but each group of R loads base again.  Times in
// us at K = 8, P = 138M without and with base, K = 16, P = 25.6M (8 bits) without
// and with:
//   R = 2, a group of rows after another                  862, 1159, 327, 413
//   R = 4, a group of rows after another                  899, 1045, 356, 378
//   R = 4, the groups of one chunk together on one XCD    911, 1001, 374, 389
// So two rows without base, and four with it: together where base is too
// large to be kept by the cache from one group to the next.
constexpr int kReadChunk = kThreads * 4;
template <int F, int R, bool NT, bool Full>
__device__ __forceinline__ void dequantize_chunk(const DequantizeParams &p, int32_t k0, int64_t e) {
    using Code = typename Fmt<F>::Code;
    const int64_t at = Full || e < p.P ? e : (p.P - 1) / 4 * 4;
    uint32_t c[R], s[R];
    f4 b = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (k0 + i >= p.K) break;
        c[i] = *reinterpret_cast<const Code *>(p.codes + (k0 + i) * p.code_ld + (at >> 2) * sizeof(Code));
        s[i] = p.scales[(k0 + i) * p.scale_ld + (at >> 5)];
    }
    if (p.base) b = load4<false, Full>(p.base, e, p.P);
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (k0 + i >= p.K) break;
        f4 v = Fmt<F>::decode(c[i], scale_of(s[i]));
        if (p.base) {
            v = b + v;
            if (s[i] >= kFarByte<F>) {      // (a sum that 64 bits do not hold is no tie in 24: rounded as once)
                const Wide w = decode_wide<F>(c[i], s[i]);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = (float)((double)b[j] + w.v[j]);
            }
        }
        store4<NT, Full>(p.y + (k0 + i) * p.y_ld, e, p.P, v);
    }
}

template <int F, int R, bool NT>
__global__ void __launch_bounds__(kThreads) k_mx_dequantize(DequantizeParams p) {
    for (uint32_t b = blockIdx.x; b < p.groups * p.chunks; b += gridDim.x) {
        uint32_t group = b / p.chunks, chunk = b % p.chunks;
        if (p.together) {                     // (chunks is a multiple of 8)
            group = b / 8 % p.groups;
            chunk = b / 8 / p.groups * 8 + b % 8;
        }
        const int64_t c0 = (int64_t)chunk * kReadChunk;
        if (c0 >= p.P) continue;
        if (c0 + kReadChunk <= p.P) dequantize_chunk<F, R, NT, true>(p, group * R, c0 + threadIdx.x * 4);
        else dequantize_chunk<F, R, NT, false>(p, group * R, c0 + threadIdx.x * 4);
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
    double inv_k;
};

// Sums in 64 bits, s1 of d and s2 of d^2 over the workers, so that one pass over the rows is enough:
// numbers have at most four significant bits.  Either an element's are equal for all workers, and K s2 and s1^2
// come out the same; or two of them differ by a sixteenth of the largest, and K s2 - s1^2 = K sum_k (d_k - mean)^2
// is at least s2 / 512, of which the roundings of the sums (none where the blocks' scales are alike: 12 (E2M1) or
// 2^18 (E4M3) steps at most, squared, in 53 bits) are K^2 2^-44 at most.
// What bounds it is the writing of K rows: at K = 8, P = 138M 1.08 ms, 5.6 TB/s.
// The codes of eight rows are loaded before any is used (a row at a time: 1.72 ms), of
// sixteen where a lane has one group of each (us, and with eight: K = 32, P = 1.2M, 8 bits 47.6 and 49.0, 4 bits
// 41.8 and 43.1; K = 64, P = 65K 15.6 and 16.8; K = 100, P = 1M 89.7 and 91.1; 49.2 with 32 in the first).
constexpr int kAverageGroups = 2;  // float4 groups of a lane in a large problem

template <int F, int NU, bool NT, bool Full>
__device__ __forceinline__ void average_chunk(const AverageParams &p, int64_t c0, int64_t c1, double s2[NU][4],
                                              int32_t *from, int32_t *bound) {
    using Code = typename Fmt<F>::Code;
    constexpr int kRowsAtOnce = NU == 1 ? 16 : 8;     // whose codes are in flight together
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
    int64_t edge = 0;
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
            edge = offsets_near(p.off, p.T, c0, from);
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
    *bound = boundary_from(edge, c0);
    // Numbers of 2^128 and more are infinite as fp32, their sums need not be: where one is not
    // finite the wave reads its rows again, in 64 bits.  (Ordinary rows pay one addition an element;
    // K = 8, P = 138M 1085 us, 1086 without.)
    double most = 0.0;
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) most += s2[u][j];
    if (__any(!(most < __builtin_inf()))) {
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            int64_t place = c0 + u * (kThreads * 4) + threadIdx.x * 4;
            if (!Full && place >= p.P) place = (p.P - 1) / 4 * 4;
#pragma unroll
            for (int j = 0; j < 4; ++j) s1[u][j] = s2[u][j] = 0.0;
#pragma unroll 1
            for (int32_t k = 0; k < p.K; ++k) {
                const Wide w = decode_wide<F>(*reinterpret_cast<const Code *>(p.codes + k * p.code_ld + (place >> 2) * sizeof(Code)),
                                              p.scales[k * p.scale_ld + (place >> 5)]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s1[u][j] += w.v[j];
                    s2[u][j] = fma(w.v[j], w.v[j], s2[u][j]);
                }
            }
        }
    }
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        const int64_t e = e0 + u * (kThreads * 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            b[u][j] = (float)((double)b[u][j] + s1[u][j] * p.inv_k);
            double q = (double)p.K * s2[u][j] - s1[u][j] * s1[u][j];
            q = Full || e + j < c1 ? (q < 0.0 ? 0.0 : q) : 0.0;    // (a NaN stays)
            s2[u][j] = q;
        }
        if (p.base_out) store4<NT, Full>(p.base_out, e, p.P, b[u]);
        if (p.x)
            for (int32_t k = 0; k < p.K; ++k) store4<NT, Full>(p.x + k * p.x_ld, e, p.P, b[u]);
    }
}

// Where several tensors meet a chunk, its squares go to LDS and each wave sums every
// fourth tensor's (K = 8, P = 1.2M in 400 tensors: 17.0 us; 22.4 where the whole block
// sums one tensor's after the other).
template <int F, int NU, bool NT>
__global__ void __launch_bounds__(kThreads) k_mx_average(AverageParams p) {
    constexpr int kChunk = kThreads * 4 * NU;
    __shared__ double lds[kChunk];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    for (uint32_t c = blockIdx.x; c < p.chunks; c += gridDim.x) {
        const int64_t c0 = (int64_t)c * kChunk, c1 = c0 + kChunk < p.P ? c0 + kChunk : p.P;
        const int32_t size = (int32_t)(c1 - c0);
        double q[NU][4];
        int32_t from, bound;       // lane i: where tensor from + i begins
        if (c0 + kChunk <= p.P) average_chunk<F, NU, NT, true>(p, c0, c1, q, &from, &bound);
        else average_chunk<F, NU, NT, false>(p, c0, c1, q, &from, &bound);
        double *partials = p.partials + (int64_t)c;
        const int32_t first = begun(bound, from, p.T);
        if (__builtin_amdgcn_readlane(bound, first + 1) >= size) {
            double all = 0.0;
#pragma unroll
            for (int u = 0; u < NU; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) all += q[u][j];
            all = block_sum(all, lds);
            if (threadIdx.x == 0) partials[from + first] = all;
            continue;
        }
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) lds[u * (kThreads * 4) + threadIdx.x * 4 + j] = q[u][j];
        __syncthreads();
        for (int turn = wave;;) {
            // the tensors among from ... from + 62 that hold some of the chunk
            const int32_t end_of = __shfl_down(bound, 1, 64);
            uint64_t some = __ballot(lane < 63 && from + lane < p.T && bound < end_of && end_of > 0 && bound < size);
            for (; some; some &= some - 1, ++turn) {
                if (turn % (kThreads / 64) != 0) continue;
                const int i = __ffsll((unsigned long long)some) - 1;
                const int32_t begin = __builtin_amdgcn_readlane(bound, i), end = __builtin_amdgcn_readlane(bound, i + 1);
                const int32_t lo = begin > 0 ? begin : 0, hi = end < size ? end : size;
                double part = 0.0;
                for (int32_t e = lo + lane; e < hi; e += 64) part += lds[e];
                part = wave_sum(part);
                if (lane == 0) partials[from + i] = part;
            }
            const int32_t reached = __builtin_amdgcn_readlane(bound, 63);
            if (reached >= size || from + 63 >= p.T) break;
            // on at tensor from + 63, or past any number of empty ones
            int32_t next;
            const int64_t off = offsets_near(p.off, p.T, c0 + (reached > 0 ? reached : 0), &next);
            if (next >= from + 63) {
                from = next;
                bound = boundary_from(off, c0);
            } else {
                from += 63;
                bound = boundary_from(p.off[from + lane < p.T ? from + lane : p.T], c0);
            }
        }
        __syncthreads();
    }
}

// Partial sums that a thread has on the way at once: few threads share a tensor's,
// and waiting for each would take longer than reading them.
constexpr int kBatch = 16;

// One block per tensor: the sum of its chunks' partial sums over K^2.
__global__ void __launch_bounds__(1024) k_mx_variance(const int64_t *off, const double *partials, int64_t chunk,
                                                      int64_t P, int32_t T, double k2, double *var) {
    __shared__ double lds[16];
    for (int32_t tau = blockIdx.x; tau < T; tau += gridDim.x) {
        const int64_t lo = off[tau] > 0 ? off[tau] : 0, hi = off[tau + 1] < P ? off[tau + 1] : P;
        double s = 0.0;
        if (hi > lo) {
            const int64_t last = (hi - 1) / chunk;
            for (int64_t c = lo / chunk + threadIdx.x; c <= last; c += kBatch * (int64_t)blockDim.x) {
                double v[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {     // (loads without branches; past the end c's again)
                    const int64_t at = c + i * (int64_t)blockDim.x;
                    v[i] = partials[(at <= last ? at : c) + tau];
                }
#pragma unroll
                for (int i = 0; i < kBatch; ++i) s += c + i * (int64_t)blockDim.x <= last ? v[i] : 0.0;
            }
        }
        s = block_sum(s, lds);
        if (threadIdx.x == 0) var[tau] = s / k2;
    }
}

// ---- product ----------------------------------------------------------------
// Rows of the two operands are the rows and columns of C, the elements are the
// contraction, on 16x16 tiles.  Which elements share a matrix instruction does
// not matter to the sum, only that both operands agree.
//   E2M1: a 16-byte unit is a block; the scaled 16x16x128 instruction multiplies
//         the codes and applies both scales; its sums are rounded as fp32.
//   E4M3: the 8-bit instructions drop products 2^-13 below the largest of
//         their sum, so the codes are converted to bf16, exactly and with
//         their scales (an element below 2^-126 is rounded to bf16's subnormal
//         numbers), for the bf16 instruction.
// A lane of these instructions holds one row (lane mod 16), but lanes that load
// 16 bytes of a row each cost an access of the vector cache each.  So four lanes
// load 64 consecutive bytes of a row, a quarter of the accesses (K = 8, P = 138M:
// 11 million, not 43), and the units change lanes through the wave's own part of
// LDS, units of a row rotated by the row over 4, so that neither side meets bank
// conflicts (K = 32, P = 20M: 72 us, 81 us without).  What bounds it is reading the
// rows: at K = 8, P = 138M 99-104 us, 5.6-5.9 TB/s.
// Where K <= 8, the 16 rows of the tile are 16 / R stretches of R = 1, 2, 4 or 8
// workers: products of different stretches come out too and are left out.
// Masks come from a table in LDS (three instructions a register of codes; from shifts
// a dozen: 400 tensors of 32 workers 23 us, 20 us from the table).
constexpr int kSuper = 512;
constexpr int kProductWaves = kThreads / 64;

struct ProductParams {
    const uint8_t *ac, *as, *bc, *bs;
    const int64_t *off;
    float *partials;       // [chunks + T][K][K]
    float *out;            // [T][K][K]
    int64_t code_ld, scale_ld;    // of a
    int64_t b_code_ld, b_scale_ld;
    int64_t P;
    int64_t chunk;         // a wave's elements, a multiple of stretches kSuper
    uint32_t blocks;       // of kProductWaves chunks
    uint32_t pairs;        // of groups of rows
    int32_t K, T;
    int32_t R, stretches;  // 16 and 1 where K > 8 (and where P is small)
    int32_t log_r;         // R = 2^log_r
};

// The lowest n bits, n in [0, 32].
__device__ __forceinline__ uint32_t low_bits(int n) { return n > 0 ? 0xffffffffu >> (32 - n) : 0u; }

// A unit's masks: entry t's lowest t elements are set, by a block's first threads.
template <int F>
struct Masks {
    static constexpr int kBits = F == ADPSGD_MX_E2M1 ? 4 : 8, kUnit = 128 / kBits;     // elements
    u4 low[kUnit + 1];
    __device__ __forceinline__ void make() {
        const int t = threadIdx.x;
        if (t > kUnit) return;
        u4 m;
        for (int i = 0; i < 4; ++i) {
            const int n = t * kBits - 32 * i;
            m[i] = low_bits(n < 32 ? n : 32);
        }
        low[t] = m;
    }
    // of the first n elements
    __device__ __forceinline__ u4 first(int n) const { return low[n < 0 ? 0 : n > kUnit ? kUnit : n]; }
};

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

// Between what a wave's lanes write to LDS and what its other lanes read there, both ways.  The
// hardware takes a wave's LDS operations in order, so it needs no instruction (as many with it as
// without); it is the compiler that may not move one past another.
__device__ __forceinline__ void lds_turn() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// 256 bytes of codes, kElems elements, of each row of a wave's tiles in LDS.
template <int TILES>
struct WaveLds {
    u4 code[TILES][4][64];
    uint32_t scale[TILES][64];
};

// The loads of a wave: lane l takes row l / 4 of each tile.
template <int F, int NT>
struct Fetch {
    static constexpr int kElems = F == ADPSGD_MX_E2M1 ? 512 : 256;
    static constexpr int kScaleBytes = kElems / 128;      // a lane's part of a row's kElems / 32
    const uint8_t *codes[NT], *scales[NT];
    u4 code[NT][4];
    uint32_t scale[NT];

    __device__ __forceinline__ void point(const uint8_t *c, const uint8_t *s, int64_t code_ld, int64_t scale_ld,
                                          int32_t row0, int32_t R, int32_t K) {
        const int lane = threadIdx.x & 63, r = lane >> 2;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            // (rows past K repeat the last one: their part of C is not kept)
            int32_t k = NT == 1 ? row0 + r % R : row0 + t * 16 + r;
            k = k < K ? k : K - 1;
            codes[t] = c + k * code_ld + ((lane & 3) ^ (lane >> 4)) * 16;
            scales[t] = s + k * scale_ld + (lane & 3) * kScaleBytes;
        }
    }
    // stretch: the lane's row's first element over kElems.  Inside: they all exist;
    // else units past the row's end are loaded from inside it (and masked later).
    template <bool Inside>
    __device__ __forceinline__ void load(int64_t stretch, int64_t P) {
        const int lane = threadIdx.x & 63;
        int64_t st = stretch, last = 0;
        if (!Inside) {
            const int64_t top = (P - 1) / kElems;
            st = st < top ? st : top;
            last = (P + kMxBlock - 1) / kMxBlock * (512 / kElems) - 1 - st * 16 - ((lane & 3) ^ (lane >> 4));
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if constexpr (kScaleBytes == 4) scale[t] = *reinterpret_cast<const uint32_t *>(scales[t] + st * 16);
            else scale[t] = *reinterpret_cast<const uint16_t *>(scales[t] + st * 8);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                int64_t u = 4 * j;
                if (!Inside) u = u < last ? u : last;
                code[t][j] = *reinterpret_cast<const u4 *>(codes[t] + st * 256 + u * 16);
            }
        }
    }
    template <int TILES>
    __device__ __forceinline__ void stash(WaveLds<TILES> &to, int tile0) const {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int j = 0; j < 4; ++j) to.code[tile0 + t][j][lane] = code[t][j];
            to.scale[tile0 + t][lane] = scale[t];
        }
    }
};

// acc += the products of the elements [from, to) of the rows' kElems (Masked) or of
// all.  Lane (row r = lane mod 16, q = lane / 16) takes unit 4 q + j of its row in
// step j; only `units` consecutive ones from unit0 on hold any (both the same in all
// lanes; of several rows' units in line).
template <int F, int NT, bool One, bool Masked>
__device__ __forceinline__ void multiply_super(const WaveLds<One ? NT : 2 * NT> &w, const Masks<F> &masks, int from,
                                               int to, int unit0, int units, v4 (&acc)[NT][NT]) {
    constexpr int TILES = One ? NT : 2 * NT, n = Masks<F>::kUnit;
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
    uint32_t scale[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) scale[t] = w.scale[t][4 * r + q];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (Masked && ((j - unit0) & 3) >= units) continue;
        u4 code[TILES];
        uint32_t byte[TILES];
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            code[t] = w.code[t][q][4 * r + (j ^ (r >> 2))];
            byte[t] = (F == ADPSGD_MX_E2M1 ? scale[t] >> (8 * j) : scale[t] >> (8 * (j >> 1))) & 0xff;
        }
        if (Masked) {
            const int first = (4 * q + j) * n;
            const bool none = first >= to || first + n <= from;
            const u4 m = masks.first(to - first) & ~masks.first(from - first);
#pragma unroll
            for (int t = 0; t < TILES; ++t) code[t] &= m;
            // (none of this tensor's elements: neither is a NaN scale its own)
#pragma unroll
            for (int t = 0; t < TILES; ++t) byte[t] = none ? 127u : byte[t];
        }
        multiply<F, NT, One>(code, byte, code + (One ? 0 : NT), byte + (One ? 0 : NT), acc);
        // one step's masked or converted operands at a time
        if (Masked || F == ADPSGD_MX_E4M3) __builtin_amdgcn_sched_barrier(0);
    }
}

// Which groups of 16 NT rows are multiplied: one group with itself (b is a), the pairs
// of groups I <= J (b is a), all pairs.
enum { kOneGroup = 0, kUpper = 1, kEvery = 2 };

// A wave walks through its chunk, 256 bytes of each row at a time, with the
// tensors that meet it: their boundaries mask the elements in registers, and
// where a tensor ends (or the chunk does) the accumulators are left as its
// partial sum, or as its result if all of it lies in the chunk.  Where a whole
// block's elements are one tensor's (the rule for long tensors), its four waves
// leave one partial sum.
//
// NT: tiles of 16 rows of an operand that a wave holds at once (of one group, those
// below the diagonal are left out).  The pairs of groups of the same elements follow each
// other on one XCD, whose L2 gives the rows to all but the first (K = 256, P = 4M, groups of 32, 430 us,
// 767 with the pairs apart; two sets of 128, P = 5M 232 and 359).
template <int F, int NT, int Pairs>
__global__ void __launch_bounds__(kThreads) k_mx_product(ProductParams p) {
    constexpr bool kOne = Pairs == kOneGroup;
    constexpr bool kPacked = NT == 1;         // (a tile may hold several stretches)
    constexpr int TILES = kOne ? NT : 2 * NT, kElems = Fetch<F, NT>::kElems;
    __shared__ WaveLds<TILES> shared[kProductWaves];
    __shared__ float parts[kPacked ? kProductWaves * 256 : 1];
    __shared__ Masks<F> masks;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    WaveLds<TILES> &mine = shared[wave];
    const int32_t groups = (p.K + 16 * NT - 1) / (16 * NT);
    const uint32_t pair = blockIdx.x / 8 % p.pairs, b = blockIdx.x / 8 / p.pairs * 8 + blockIdx.x % 8;
    if (b >= p.blocks) return;
    int32_t I = 0, J = 0;
    if (Pairs == kEvery) {
        I = pair / groups;
        J = pair % groups;
    } else if (Pairs == kUpper) {
        for (J = pair; J >= groups - I; ++I) J -= groups - I;
        J += I;
    }
    Fetch<F, NT> a, o;
    a.point(p.ac, p.as, p.code_ld, p.scale_ld, I * 16 * NT, p.R, p.K);
    if (!kOne) o.point(p.bc, p.bs, p.b_code_ld, p.b_scale_ld, J * 16 * NT, p.R, p.K);
    const int32_t stretches = kPacked ? p.stretches : 1;
    const int32_t fetched = kPacked ? (lane >> 2) / p.R : 0, held = kPacked ? (lane & 15) / p.R : 0;   // stretch of a lane's row
    const int64_t super = (int64_t)stretches * kElems;

    v4 acc[NT][NT];
    auto clear = [&] {
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = v4{0.f, 0.f, 0.f, 0.f};
    };
    // Two levels of fp32 sums: acc over 256 bytes of each row and total of those.  (Error against 64 bits in 8 bits at
    // K = 16, P = 25.6M 3.1e-8 of the result, 5.5e-7 with one level; in 4 bits, whose sums are exact only where
    // scales are alike, 3.0e-7 and 5.2e-7 of 48 workers' blocks of many sizes, 1.1e-7 and 3.8e-6 of small products
    // beside a large one, K = 70.  4 bits, us, and with one level: K = 8, P = 138M 106 and 106, K = 32, P = 20M 72
    // and 72, K = 33, P = 20M 83 and 79, K = 64, P = 5M 42 and 42, K = 256, P = 4.3M 405 and 400.)
    // A piece of less than that before or behind a tensor's whole ones is a level by itself,
    // but of three or four tiles of 4 bits joins its neighbour's (K = 100, P = 5M in 10 tensors 131 us, 139 by itself).
    constexpr bool kPieces = F == ADPSGD_MX_E4M3 || NT <= 2;
    v4 total[NT][NT];
    auto each = [&](auto f) {
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int j = kOne ? i : 0; j < NT; ++j) f(i, j);
    };
    auto level = [&] {
        each([&](int i, int j) {
            total[i][j] += acc[i][j];
            acc[i][j] = v4{0.f, 0.f, 0.f, 0.f};
        });
    };
    auto join = [&] {
        each([&](int i, int j) {
            if (kPieces) acc[i][j] = total[i][j];
            else acc[i][j] += total[i][j];
            total[i][j] = v4{0.f, 0.f, 0.f, 0.f};
        });
    };
    each([&](int i, int j) { total[i][j] = v4{0.f, 0.f, 0.f, 0.f}; });
    auto park = [&](float *at) {
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int j = kOne ? i : 0; j < NT; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    at[(i * NT + j) * 256 + (4 * (lane >> 4) + r) * 16 + (lane & 15)] = acc[i][j][r];
    };
    // Entry (y, x) of a K x K matrix; mirrored where b is a and tile (x, y) is not computed.
    auto put = [&](float *out, bool mirror, int32_t y, int32_t x, float v) {
        if (y >= p.K || x >= p.K) return;
        out[(int64_t)y * p.K + x] = v;
        if (Pairs != kEvery && mirror && y / 16 != x / 16) out[(int64_t)x * p.K + y] = v;
    };
    // One wave's accumulators to out.  (The addresses are worked out here each
    // time: kept across the loops they would take more registers than the rest.)
    auto leave = [&](float *out, bool mirror) {
        int l = lane;
        asm volatile("" : "+v"(l));
        if (kPacked && stretches > 1) {      // the stretches' parts of the tile, summed
            float *at = parts + wave * 256;
            park(at);
            lds_turn();
            for (int e = l; e < p.R * p.R; e += 64) {
                const int32_t row = e >> p.log_r, col = e & (p.R - 1);
                double s = 0.0;
                for (int g = 0; g < stretches; ++g) s += at[(g * p.R + row) * 16 + g * p.R + col];
                put(out, mirror, row, col, (float)s);
            }
            lds_turn();
            return;
        }
        // (32-bit indexes from a scalar base; most matrices fill their tiles)
        const uint32_t K = (uint32_t)p.K, y0 = I * 16 * NT + 4 * (l >> 4), x0 = J * 16 * NT + (l & 15), at = y0 * K + x0;
        const bool whole = (uint32_t)((I + 1) * 16 * NT) <= K && (uint32_t)((J + 1) * 16 * NT) <= K;
        auto store = [&](auto inside) {
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = kOne ? i : 0; j < NT; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if (!decltype(inside)::value && (y0 + 16 * i + r >= K || x0 + 16 * j >= K)) continue;
                        out[at + (16 * i + r) * K + 16 * j] = acc[i][j][r];
                        if (Pairs != kEvery && mirror && (Pairs == kUpper ? I != J : i != j))
                            out[(x0 + 16 * j) * K + y0 + 16 * i + r] = acc[i][j][r];
                    }
        };
        if (whole) store(std::true_type{});
        else store(std::false_type{});
    };
    const int64_t n = (int64_t)p.K * p.K;
    masks.make();
    __syncthreads();
    const int64_t c = (int64_t)b * kProductWaves + wave;           // this wave's chunk
    const int64_t b0 = (int64_t)b * kProductWaves * p.chunk, b1 = b0 + kProductWaves * p.chunk;
    const int64_t c0 = c * p.chunk, c1 = c0 + p.chunk < p.P ? c0 + p.chunk : p.P;
    int64_t s0 = c0;
    a.template load<false>(s0 / kElems + fetched, p.P);
    if (!kOne) o.template load<false>(s0 / kElems + fetched, p.P);
    int32_t from;                  // lane i: where tensor from + i begins
    int64_t edge = offsets_near(p.off, p.T, b0, &from);
    clear();
    int32_t bound = boundary_from(edge, b0), tau = from + begun(bound, from, p.T);
    if (__builtin_amdgcn_readlane(bound, tau - from) <= 0 && __builtin_amdgcn_readlane(bound, tau - from + 1) >= b1 - b0 &&
        b1 <= p.P) {
        while (s0 < c1) {
            lds_turn();
            a.stash(mine, 0);
            if (!kOne) o.stash(mine, NT);
            lds_turn();
            s0 += super;
            if (s0 < c1) {      // (on their way while these are multiplied)
                a.template load<true>(s0 / kElems + fetched, p.P);
                if (!kOne) o.template load<true>(s0 / kElems + fetched, p.P);
            }
            multiply_super<F, NT, kOne, false>(mine, masks, 0, kElems, 0, 16, acc);
            level();
        }
        join();
        lds_turn();
        float *at = kPacked ? parts : reinterpret_cast<float *>(shared);
        constexpr int kStride = kPacked ? 256 : sizeof(WaveLds<TILES>) / sizeof(float);   // of waves
        park(at + wave * kStride);
        __syncthreads();
        float *out = p.partials + ((int64_t)b * kProductWaves + tau) * n;
        int thread = threadIdx.x;
        asm volatile("" : "+v"(thread));
        const int32_t row = thread / 16, col = thread % 16;
        if (!kPacked || (row < p.R && col < p.R)) {
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = kOne ? i : 0; j < NT; ++j) {
                    double s = 0.0;
                    for (int w = 0; w < kProductWaves; ++w)
                        for (int g = 0; g < stretches; ++g)
                            s += at[w * kStride + (i * NT + j) * 256 + (g * p.R + row) * 16 + g * p.R + col];
                    put(out, false, (I * NT + i) * 16 + row, (J * NT + j) * 16 + col, (float)s);
                }
        }
        return;
    }
    if (c0 >= p.P) return;
    // From here on elements are counted from c0, in 32 bits (scalar ones: an int64 compare takes
    // vector instructions).  64 boundaries at a time, lane i that of tensor from + i.
    auto boundary = [&](int32_t i) { return boundary_from(p.off[i + lane < p.T ? i + lane : p.T], c0); };
    bound = boundary_from(edge, c0);
    for (;;) {                     // the last tensor that begins by c0
        tau = from + begun(bound, from, p.T);
        if (tau < from + 62) break;
        from = tau;
        bound = boundary(from);
        if (__builtin_amdgcn_readlane(bound, 1) > 0) break;
    }
    const int32_t span = (int32_t)super, size = (int32_t)(c1 - c0);
    bool open = false;             // acc holds something of tensor tau
    for (int32_t at = 0; at < size;) {
        const int32_t next = at + span < size ? at + span : size;
        lds_turn();
        a.stash(mine, 0);
        if (!kOne) o.stash(mine, NT);
        lds_turn();
        if (next < size) {
            a.template load<false>((c0 + next) / kElems + fetched, p.P);
            if (!kOne) o.template load<false>((c0 + next) / kElems + fetched, p.P);
        }
        while (tau < p.T) {
            if (tau - from == 63) {
                from = tau;
                bound = boundary(from);
            }
            const int32_t begin = __builtin_amdgcn_readlane(bound, tau - from);
            const int32_t end = __builtin_amdgcn_readlane(bound, tau - from + 1);
            if (begin >= next) break;
            if (end <= begin) {          // past the empty ones among the 64
                const uint64_t more = __ballot(bound > begin) & ~((uint64_t(2) << (tau - from)) - 1);
                tau = more ? from + __ffsll((unsigned long long)more) - 2 : from + 63;
                continue;
            }
            const int32_t lo = begin > at ? begin : at, hi = end < next ? end : next;
            if (hi > lo) {
                open = true;
                if (hi - lo == span) {
                    multiply_super<F, NT, kOne, false>(mine, masks, 0, kElems, 0, 16, acc);
                    level();
                } else {
                    // what of this lane's row is the tensor's
                    const int first = at + held * kElems, f = lo - first, t = hi - first;
                    const int unit0 = (lo - at) / Masks<F>::kUnit, units = (hi - at - 1) / Masks<F>::kUnit - unit0 + 1;
                    multiply_super<F, NT, kOne, true>(mine, masks, f < 0 ? 0 : f, t > kElems ? kElems : t, unit0, units, acc);
                    if (kPieces) level();
                }
            }
            if (end > next) break;
            if (open) {
                join();
                if (begin >= 0) leave(p.out + tau * n, true);        // (all of it was here)
                else leave(p.partials + (c + tau) * n, false);
                clear();
                open = false;
            }
            ++tau;
        }
        at = next;
    }
    if (open) {
        join();
        leave(p.partials + (c + tau) * n, false);
    }
}

// The tensors' sums of the partial sums that k_mx_product left, in 64 bits, by
// lanes of `outs` entries: blockDim / outs of them share a tensor's.  Where b is a,
// tiles below the diagonal are the transposed ones above it.
__global__ void __launch_bounds__(1024) k_mx_product_sum(const int64_t *off, const float *partials, int64_t chunk,
                                                         int64_t P, int32_t K, int32_t T, int same, int32_t outs,
                                                         float *out) {
    __shared__ double lds[1024];
    const int64_t n = (int64_t)K * K, block = chunk * kProductWaves;
    const int32_t share = blockDim.x / outs, part = threadIdx.x / outs;
    const int64_t i = (int64_t)blockIdx.y * outs + threadIdx.x % outs;
    const int32_t row = (int32_t)(i / K), col = (int32_t)(i % K);
    const float *from = partials + (same && row / 16 > col / 16 ? (int64_t)col * K + row : i);
    for (int32_t tau = blockIdx.x; tau < T; tau += gridDim.x) {
        const int64_t lo = off[tau] > 0 ? off[tau] : 0, hi = off[tau + 1] < P ? off[tau + 1] : P;
        if (hi > lo && lo / chunk == (hi - 1) / chunk) continue;      // (one chunk: out has it)
        double s = 0.0;
        if (hi > lo && i < n) {
            // chunks before the tensor's whole blocks, one of each of those, chunks behind them
            const int64_t first = lo / chunk, end = (hi - 1) / chunk + 1;
            const int64_t b0 = (lo + block - 1) / block, b1 = hi / block;
            auto add = [&](int64_t c, int64_t count, int32_t step) {
                const float *at = from + (c + tau) * n;
                const int64_t ld = step * n;
                int32_t m = part;
                for (; m + (kBatch - 1) * share < count; m += kBatch * share) {
                    float v[kBatch];
#pragma unroll
                    for (int u = 0; u < kBatch; ++u) v[u] = at[(int64_t)(m + u * share) * ld];
#pragma unroll
                    for (int u = 0; u < kBatch; ++u) s += (double)v[u];
                }
                for (; m < count; m += 4 * share) {      // (loads without branches; past the end m's again)
                    float v[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) v[u] = at[(int64_t)(m + u * share < count ? m + u * share : m) * ld];
#pragma unroll
                    for (int u = 0; u < 4; ++u) s += m + u * share < count ? (double)v[u] : 0.0;
                }
            };
            if (b1 > b0) {
                add(first, b0 * kProductWaves - first, 1);
                add(b0 * kProductWaves, b1 - b0, kProductWaves);
                add(b1 * kProductWaves, end - b1 * kProductWaves, 1);
            } else {
                add(first, end - first, 1);
            }
        }
        lds[threadIdx.x] = s;
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
    if (r->P < 0 || r->P > kMaxP) return fail(ADPSGD_EINVAL, "P must be in [0, 2^34]");
    if ((r->P + kPiece - 1) / kPiece > kMaxPieces / r->K) return fail(ADPSGD_EINVAL, "K * P must be below 2^39");
    const Bytes need = row_bytes(r->format, r->P);
    if (r->code_stride < need.codes || r->code_stride % 16 != 0 || r->code_stride > kMaxStride)
        return fail(ADPSGD_EINVAL, n + ".code_stride must be a multiple of 16, at most 2^44 and hold a row (" +
                                       std::to_string(need.codes) + " bytes)");
    if (r->scale_stride < need.scales || r->scale_stride % 16 != 0 || r->scale_stride > kMaxStride)
        return fail(ADPSGD_EINVAL, n + ".scale_stride must be a multiple of 16, at most 2^44 and hold a row (" +
                                       std::to_string(need.scales) + " bytes)");
    if (r->P > 0 && (!r->codes || !r->scales || !aligned16(r->codes) || !aligned16(r->scales)))
        return fail(ADPSGD_EINVAL, n + ".codes and .scales must be non-NULL and 16-byte aligned");
    return ADPSGD_OK;
}

// The row stride of a float array (0 means P).
int check_ld(int64_t stride, int64_t P, const char *name, int64_t *ld) {
    if (stride < 0 || (stride > 0 && stride < P) || stride > kMaxStride)
        return fail(ADPSGD_EINVAL, std::string(name) + " must be 0 or >= P, and at most 2^44");
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

struct Range {
    explicit Range(const char *name) { roctxRangePushA(name); }
    ~Range() { roctxRangePop(); }
};

int launched(const char *what) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(ADPSGD_EDEVICE, std::string(what) + ": " + hipGetErrorString(e));
    return ok();
}

uint32_t grid_for(uint64_t blocks) { return (uint32_t)(blocks < kMaxGrid ? blocks : kMaxGrid); }

// Rows of fp32 that would take most of the 256 MB last-level cache go past it
// (quantize at K = 8, P = 4M with residuals in and out, 384 MB: 66 us, 75 us
// through it); smaller ones may well be in it (average at K = 32, P = 1.2M,
// 154 MB, of a model just worked on: 41 us, 50 us past it).
bool past_cache(int64_t K, int64_t P, int arrays) { return (double)K * (double)P * 4.0 * arrays > 192e6; }

// Several groups a lane for long rows (half the blocks' fixed work), one where
// that would leave compute units without a block.
bool long_rows(int64_t P) { return P >= int64_t(1) << 22; }

int64_t average_chunk_elements(int64_t P) { return kThreads * 4 * (long_rows(P) ? kAverageGroups : 1); }

// Rows of a tile that a stretch takes: as many as there are workers, or more (the last
// one repeated) where that few elements for so many stretches would make fewer than
// 512 waves: K = 2, P = 1.2M in 400 tensors 22.5 us in 293 waves, 15.7 in 1172.
int32_t tile_workers(int32_t K, int64_t P) {
    int32_t R = K > 8 ? 16 : K > 4 ? 8 : K > 2 ? 4 : K;
    while (R < 16 && P < 512 * kSuper * (16 / R)) R *= 2;
    return R;
}

// Elements of a product's wave: of as many waves as the compute units hold evenly, four to
// a block and 256 blocks a step (us, with this many waves a unit).  20 of the kernels for
// up to 16 workers (K = 8, P = 138M: 105; 108 with 32; K = 16, P = 25.6M, 8 bits: 82, 88
// with 32, 87 with 16), 8 for up to 32 (K = 24, P = 5M: 25; 28 with 12, 33 with 13; K = 32, P =
// 20M: 72, 74 with 12, 83 with 13; many small tensors are better off with 8 than 4, K = 32, P = 1.2M in
// 400 tensors 19.3 and 21.6, a single one with 4, K = 24, P = 5M 25 and 22.5), 4 for up to 64 (K = 64, P =
// 5M: 42; 54 with 2, 55 with 5, 49 with 8), and a whole number of fours where more are
// needed (two sets of 40, P = 20M: 169 with 8, 210 with 5).  More workers fill the units
// with pairs of groups: fewer waves, so that the K x K partial sums come to 8 MB.
// No wave takes less than its partial sums outweigh, nor more than 16384 elements of a
// row (of which fp32 sums are taken): rows longer than 16384 waves hold have P K^2 / 4096 bytes of
// partial sums (K = 256, P = 2^22: 67 MB), of which blocks inside one tensor write and read a quarter.
int64_t product_chunk(int32_t K, int64_t P) {
    const int64_t super = kSuper * (16 / tile_workers(K, P)), most = 32;
    const int64_t supers = (P + super - 1) / super, least = (15 * (int64_t)K + super - 1) / super;
    int64_t waves = K <= 16 ? 5120 : K <= 32 ? 2048 : K <= 64 ? 1024 : (int64_t(1) << 21) / ((int64_t)K * K);
    if (K <= 64 && supers > most * waves) waves = (supers + most * 1024 - 1) / (most * 1024) * 1024;
    return super * std::min<int64_t>(most, std::max<int64_t>(least, (supers + waves - 1) / waves));
}

int64_t product_blocks(int32_t K, int64_t P) {
    const int64_t block = product_chunk(K, P) * kProductWaves;
    return (P + block - 1) / block;
}

}  // namespace

extern "C" int64_t adpsgd_mx_code_stride(int32_t format, int64_t P) {
    if ((format != ADPSGD_MX_E2M1 && format != ADPSGD_MX_E4M3) || P <= 0 || P > kMaxP) return 0;
    const int64_t n = (row_bytes(format, P).codes + 255) / 256;
    return 256 * (n + 1 - n % 2);
}

extern "C" int64_t adpsgd_mx_scale_stride(int64_t P) {
    if (P <= 0 || P > kMaxP) return 0;
    const int64_t n = (row_bytes(ADPSGD_MX_E2M1, P).scales + 255) / 256;
    return 256 * (n + 1 - n % 2);
}

extern "C" int adpsgd_mx_quantize(const adpsgd_mx_rows *out, const float *x, int64_t x_stride, const float *base,
                                  const float *residual_in, float *residual_out, int64_t residual_stride, void *stream) {
    Range range_("adpsgd_mx_quantize");
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
    p.g = row_grid(out->K, P);
    const dim3 grid(grid_for(p.g.blocks)), block(64);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const bool nt = past_cache(out->K, P, 1 + (residual_in != nullptr) + (residual_out && residual_out != residual_in));
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

template <int F, int R>
void launch_dequantize(DequantizeParams &p, bool nt, hipStream_t st) {
    p.groups = (uint32_t)((p.K + R - 1) / R);
    const uint32_t grid = grid_for((uint64_t)p.groups * p.chunks);
    if (nt) k_mx_dequantize<F, R, true><<<grid, kThreads, 0, st>>>(p);
    else k_mx_dequantize<F, R, false><<<grid, kThreads, 0, st>>>(p);
}

template <int F>
void launch_dequantize(DequantizeParams &p, hipStream_t st) {
    p.chunks = (uint32_t)((p.P + kReadChunk - 1) / kReadChunk);
    p.together = p.base && past_cache(1, p.P, 1);
    if (p.together) p.chunks = (p.chunks + 7) / 8 * 8;
    const bool nt = past_cache(p.K, p.P, 1);
    if (p.base && p.K > 2) launch_dequantize<F, 4>(p, nt, st);
    else launch_dequantize<F, 2>(p, nt, st);
}

template <int F>
void launch_average(const AverageParams &p, hipStream_t st) {
    const bool nt = past_cache(p.K, p.P, 1), several = long_rows(p.P);
    const uint32_t grid = grid_for(p.chunks);
    if (several && nt) k_mx_average<F, kAverageGroups, true><<<grid, kThreads, 0, st>>>(p);
    else if (several) k_mx_average<F, kAverageGroups, false><<<grid, kThreads, 0, st>>>(p);
    else if (nt) k_mx_average<F, 1, true><<<grid, kThreads, 0, st>>>(p);
    else k_mx_average<F, 1, false><<<grid, kThreads, 0, st>>>(p);
}

}  // namespace

extern "C" int adpsgd_mx_dequantize(const adpsgd_mx_rows *rows, const float *base, float *y, int64_t y_stride,
                                    void *stream) {
    Range range_("adpsgd_mx_dequantize");
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
    p.K = rows->K;
    p.y = y;
    p.code_ld = rows->code_stride;
    p.scale_ld = rows->scale_stride;
    p.P = P;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (rows->format == ADPSGD_MX_E2M1) launch_dequantize<ADPSGD_MX_E2M1>(p, st);
    else launch_dequantize<ADPSGD_MX_E4M3>(p, st);
    return launched("dequantize launch");
}

extern "C" size_t adpsgd_mx_average_workspace(int32_t K, int64_t P, int32_t T) {
    if (K < 1 || K > kMaxK || P < 0 || P > kMaxP || T < 1 || T > kMaxT) return 0;
    const int64_t chunk = average_chunk_elements(P);
    return sizeof(double) * (size_t)((P + chunk - 1) / chunk + T);
}

extern "C" int adpsgd_mx_average(const adpsgd_mx_rows *rows, int32_t T, const int64_t *tensor_offsets,
                                 const float *base, float *base_out, float *x, int64_t x_stride, double *var,
                                 void *workspace, size_t workspace_bytes, void *stream) {
    Range range_("adpsgd_mx_average");
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
    p.inv_k = 1.0 / rows->K;
    p.K = rows->K;
    p.T = T;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (P > 0) {
        if (rows->format == ADPSGD_MX_E2M1) launch_average<ADPSGD_MX_E2M1>(p, st);
        else launch_average<ADPSGD_MX_E4M3>(p, st);
        if (int rc = launched("average launch")) return rc;
    }
    // more threads where a tensor may have many partial sums (a launch has less than 2^32 threads)
    const int threads = p.chunks > 4096 && T < 1 << 16 ? 1024 : kThreads;
    k_mx_variance<<<grid_for((uint64_t)T), threads, 0, st>>>(tensor_offsets, p.partials, chunk, P, T,
                                                             (double)rows->K * rows->K, var);
    return launched("variance launch");
}

extern "C" size_t adpsgd_mx_product_workspace(int32_t K, int64_t P, int32_t T) {
    if (K < 1 || K > kMaxProductK || P < 0 || P > kMaxP || T < 1 || T > kMaxT) return 0;
    return sizeof(float) * (size_t)(product_blocks(K, P) * kProductWaves + T) * K * K;
}

namespace {

// Groups of rows by K: the more a wave holds, the fewer times the rows are loaded, but
// the fewer waves a compute unit holds.  us, b is a, E2M1 (in brackets E4M3): K = 64, P = 5M 61 (105) as groups of
// 32, 42 (69) as one of 64; K = 33, P = 20M 141 as groups of 32, 103 as one of 64, 83 as one of
// 48; K = 100 as groups of 32 and of 48 P = 5M 142 and 128 (287 and 269), P = 0.5M 25 and 32; K = 256
// P = 4.3M 478 and 405 (903 and 802), P = 0.5M 64 and 63.  Two operands: K = 40, P = 5M 64 as groups of
// 32, 47 as one of 48; K = 70 130 as nine pairs of 32, 118 as four of 48; K = 64 88 (162) as
// two groups of 32, 109 (195) as two of 48.
template <int F, int NT, int Pairs>
void launch_product(ProductParams &p, uint32_t pairs, hipStream_t st) {
    p.pairs = pairs;
    k_mx_product<F, NT, Pairs><<<(p.blocks + 7) / 8 * 8 * pairs, kThreads, 0, st>>>(p);
}

template <int F>
void launch_product(ProductParams &p, bool same, hipStream_t st) {
    const uint32_t by32 = (p.K + 31) / 32, by48 = (p.K + 47) / 48;
    if (!same) {
        if (p.K <= 16) launch_product<F, 1, kEvery>(p, 1, st);
        else if (by48 < by32) launch_product<F, 3, kEvery>(p, by48 * by48, st);
        else launch_product<F, 2, kEvery>(p, by32 * by32, st);
        return;
    }
    if (p.K <= 16) launch_product<F, 1, kOneGroup>(p, 1, st);
    else if (p.K <= 32) launch_product<F, 2, kOneGroup>(p, 1, st);
    else if (p.K <= 48) launch_product<F, 3, kOneGroup>(p, 1, st);
    else if (p.K <= 64) launch_product<F, 4, kOneGroup>(p, 1, st);
    else if (long_rows(p.P)) launch_product<F, 3, kUpper>(p, by48 * (by48 + 1) / 2, st);
    else launch_product<F, 2, kUpper>(p, by32 * (by32 + 1) / 2, st);
}

}  // namespace

extern "C" int adpsgd_mx_product(const adpsgd_mx_rows *a, const adpsgd_mx_rows *b, int32_t T,
                                 const int64_t *tensor_offsets, float *out, void *workspace, size_t workspace_bytes,
                                 void *stream) {
    Range range_("adpsgd_mx_product");
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
    p.out = out;
    p.code_ld = a->code_stride;
    p.scale_ld = a->scale_stride;
    p.b_code_ld = b->code_stride;
    p.b_scale_ld = b->scale_stride;
    p.P = P;
    p.chunk = product_chunk(a->K, P);
    p.blocks = (uint32_t)product_blocks(a->K, P);
    p.K = a->K;
    p.T = T;
    p.R = tile_workers(a->K, P);
    p.stretches = 16 / p.R;
    while (1 << p.log_r < p.R) ++p.log_r;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (P > 0) {
        if (a->format == ADPSGD_MX_E2M1) launch_product<ADPSGD_MX_E2M1>(p, same, st);
        else launch_product<ADPSGD_MX_E4M3>(p, same, st);
        if (int rc = launched("product launch")) return rc;
    }
    // A block for each tensor and `outs` entries; more threads to an entry the more partial sums a
    // tensor has, and fewer entries a block where they are many (K = 64, P = 5M in one tensor 42 us in
    // all, 51 with 128 entries a block; K = 32, P = 1.2M in 100 tensors, 11 partial sums each, 18 and 16.5).
    const int64_t n = (int64_t)a->K * a->K, items = (int64_t)p.blocks * kProductWaves / T;
    int32_t outs = 1, share = 1;
    while (outs < (items > 16 ? 16 : 128) && outs < n) outs *= 2;
    while (outs * share < 1024 && share * 8 < items) share *= 2;
    const uint32_t threads = (uint32_t)(outs * share);
    k_mx_product_sum<<<dim3(grid_for((uint64_t)T), (uint32_t)((n + outs - 1) / outs)), threads, 0, st>>>(
        tensor_offsets, p.partials, p.chunk, P, a->K, T, same, outs, out);
    return launched("product sum launch");
}
