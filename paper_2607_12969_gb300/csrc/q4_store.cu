// q4_store.cu -- matrices of 4-bit codes with a scale per row and group of columns:
// rounding and widening (lrc_q4_round, lrc_q4_widen).
//
// What[i][c] = s (q - z).  The codes' layout is the one include/lrc.h states:
// 64-byte blocks of 128 columns, column 32 j + 8 t + e in word 4 t + j.
#include <math.h>

#include <type_traits>

#include "q4.cuh"

namespace lrc {
namespace {

using namespace q4;

constexpr float kSeventh = 0.14285714285714285f;      // binary32 next to 1/7
constexpr float kFifteenth = 0.06666666666666667f;    // and to 1/15

// Bit position of column e of a word.
__device__ __forceinline__ int nibble_shift(int e) { return 2 * e + (e & 1) * 14; }

template <typename S> __device__ __forceinline__ float largest();
template <> __device__ __forceinline__ float largest<float>() { return 3.402823466e38f; }
template <> __device__ __forceinline__ float largest<__half>() { return 65504.f; }
template <> __device__ __forceinline__ float largest<bf16>() { return 3.3895313892515355e38f; }

__device__ __forceinline__ float src_f32(double x) { return (float)x; }
template <typename T> __device__ __forceinline__ float src_f32(T x) { return el::to_f32(x); }

// Rounding goes over pieces of kPieceRows rows and 512 columns, widening of 256, a
// block each; a warp takes every eighth row.  The scales of a piece pass through shared
// memory: in memory the rows are side by side, not the groups.
constexpr int kPieceRows = 32, kRoundCols = 512, kPieceCols = 256;

__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float min_nan(float a, float b) {
    float d;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// Eight elements of a row from column c on, zeros from n on.
template <typename W>
union Eight {
    uint4 q[sizeof(W) / 2];
    W e[8];
    __device__ __forceinline__ Eight() {}
    __device__ __forceinline__ void load(const W* row, int64_t c, int64_t n, bool whole16) {
        if (whole16 && c + 8 <= n) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(W) / 2; ++i) q[i] = __ldcs(reinterpret_cast<const uint4*>(row + c) + i);
        } else {
#pragma unroll
            for (int i = 0; i < (int)sizeof(W) / 2; ++i) q[i] = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i < n) e[i] = row[c + i];
        }
    }
};

// Sixteen 16-bit elements from an address that is only aligned to theirs, of the three
// whole 16 bytes around them (which are the row's: eight more elements on both sides).
template <typename W>
__device__ __forceinline__ void load_between(const W* at, Eight<W> (&v)[2]) {
    const uint32_t past = (uint32_t)(reinterpret_cast<uintptr_t>(at) & 15u);
    const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(at) - past);
    const uint4 a = __ldcs(p), b = __ldcs(p + 1), c = __ldcs(p + 2);
    uint32_t w[12] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w, c.x, c.y, c.z, c.w};
#pragma unroll
    for (int i = 0; i < 10; ++i) w[i] = past & 8u ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 9; ++i) w[i] = past & 4u ? w[i + 1] : w[i];
    uint32_t u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = __funnelshift_r(w[i], w[i + 1], (past & 2u) * 8u);
    v[0].q[0] = make_uint4(u[0], u[1], u[2], u[3]);
    v[1].q[0] = make_uint4(u[4], u[5], u[6], u[7]);
}

// Of two 16-bit numbers each, the larger ones; NaN where one is.
template <typename W> __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b);
template <> __device__ __forceinline__ uint32_t max2<__half>(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
template <> __device__ __forceinline__ uint32_t max2<bf16>(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
template <typename W> __device__ __forceinline__ float half_of(uint32_t pair, int which) {
    union {
        uint16_t u;
        W v;
    } x;
    x.u = (uint16_t)(which ? pair >> 16 : pair);
    return el::to_f32(x.v);
}

// Least and largest element of a group of kLanes lanes, 0 among them (ZEROS), or
// (hi) the largest magnitude.  16-bit elements two at a time, least ones negated.
template <typename W, bool ZEROS, int kLanes>
__device__ __forceinline__ void range_of(const Eight<W> (&v)[2], float& lo, float& hi) {
    lo = hi = 0.f;
    if constexpr (sizeof(W) == 2) {
        uint32_t up = 0, down = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t p[4] = {v[h].q[0].x, v[h].q[0].y, v[h].q[0].z, v[h].q[0].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                up = max2<W>(up, ZEROS ? p[i] : p[i] & 0x7fff7fffu);
                if (ZEROS) down = max2<W>(down, p[i] ^ 0x80008000u);
            }
        }
        // (ZEROS) the halves of each joined, then one of each a half
        if (ZEROS) up = max2<W>(__byte_perm(up, down, 0x5410), __byte_perm(up, down, 0x7632));
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) up = max2<W>(up, __shfl_xor_sync(0xffffffffu, up, o));
        hi = half_of<W>(up, 0);
        if (ZEROS) lo = -half_of<W>(up, 1);
        else hi = max_nan(hi, half_of<W>(up, 1));
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float w = src_f32(v[h].e[e]);
                if (ZEROS) lo = min_nan(lo, w);
                hi = max_nan(hi, ZEROS ? w : fabsf(w));
            }
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) {
            if (ZEROS) lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
            hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        }
    }
}

// A thread rounds sixteen consecutive columns, two words of codes; group / 16
// neighbouring lanes share a scale.  Adding 1.5 * 2^23 rounds to an integer, ties to
// even; codes are kept in range and put together with binary32 instructions, whose
// pipe has room where that of minima, shifts and masks has half the rate.  Bound by
// instructions, and HBM: 16384 x 8192 of bfloat16 with zero codes 65 us, 5.2 TB/s of
// 6.8; of binary32 95 us, 6.4 TB/s.  Eight columns a thread, with a range and a scale
// formed twice as often, 97 us (87 with four rows' loads at once; with sixteen columns
// that gains nothing).
// ANY: rows of 16-bit elements that start anywhere (16383 x 8191 to codes and back 188
// us; element by element 244).  whole16: all start on 16 bytes.  Wider elements whose
// rows do not go one by one: 16383 x 8191 of binary32 242 us.  binary64 252 us.
template <typename W, typename S, int GROUP, bool ZEROS, bool ANY>
__global__ void __launch_bounds__(256)
q4_round_kernel(const W* __restrict__ src, int64_t m, int64_t n, int64_t ldw, bool whole16, uint32_t* __restrict__ Q,
                S* __restrict__ scales, uint8_t* __restrict__ zeros, int64_t blocks, int64_t pieces, int64_t ldm) {
    constexpr int kGroups = kRoundCols / GROUP, kLanes = GROUP / 16;
    __shared__ S sh_s[kGroups][kPieceRows];
    __shared__ uint8_t sh_z[kGroups][kPieceRows];
    const int64_t r0 = blockIdx.x / pieces * kPieceRows, piece = blockIdx.x % pieces;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t c0 = piece * kRoundCols + lane * 16, block = piece * 4 + (lane >> 3);
    const int chunk = (lane & 7) * 2;                        // of the block of 128 columns: 4 j + t
    const int64_t word_at = block * 16 + (chunk & 3) * 4 + (chunk >> 2);
    tc::pdl_wait();
    tc::pdl_trigger();
#pragma unroll
    for (int i = 0; i < kPieceRows / 8; ++i) {
        const int r = warp + 8 * i;
        const int64_t row = r0 + r;
        if (row >= m) break;
        Eight<W> v[2];
        if (ANY && c0 >= 8 && c0 + 24 <= n) {
            load_between(src + row * ldw + c0, v);
        } else {
            v[0].load(src + row * ldw, c0, n, !ANY && whole16);
            v[1].load(src + row * ldw, c0 + 8, n, !ANY && whole16);
        }
        float lo, hi;
        range_of<W, ZEROS, kLanes>(v, lo, hi);
        const bool bad = !(hi <= 3.402823466e38f) || !(lo >= -3.402823466e38f);
        const float wide = ZEROS ? __fmul_rn(__fsub_rn(hi, lo), kFifteenth) : __fmul_rn(hi, kSeventh);
        S stored = el::from_f32<S>(fminf(wide, largest<S>()));
        const float s = el::to_f32(stored);
        const bool none = s < 1.17549435e-38f;
        const float inv = none ? 0.f : __frcp_rn(s);
        if (none) stored = el::from_f32<S>(0.f);
        float z = 8.f;
        if (ZEROS) z = fminf(fmaxf(rintf(__fmul_rn(-lo, inv)), 0.f), 15.f);
        if (bad) {
            stored = el::from_f32<S>(__int_as_float(0x7fffffff));
            z = 8.f;
        }
        // t + 1.5 * 2^23 = the integer next to t, and that; what follows is exact: its
        // sum with z over 16 kept in 0 ... 1, and 15 / 16 less that, not below 0, is
        // (15 - code) / 16.  Even columns' codes are the word's low half, from 2^23 on.
        const float shift = fmaf(z, 0.0625f, -786432.f);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float half[2] = {8388608.f + 65535.f, 8388608.f + 65535.f}, place = -16.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float t = __fadd_rn(__fmul_rn(src_f32(v[h].e[e]), inv), 12582912.f);
                const float rest = __saturatef(0.9375f - __saturatef(fmaf(t, 0.0625f, shift)));
                half[e & 1] = fmaf(rest, place, half[e & 1]);
                if (e & 1) place *= 16.f;
            }
            uint32_t word = __byte_perm(__float_as_uint(half[0]), __float_as_uint(half[1]), 0x5410);
            if (bad) word = 0x88888888u;
            if (block < blocks) Q[row * blocks * 16 + word_at + 4 * h] = word;
        }
        if (lane % kLanes == 0) {
            sh_s[lane / kLanes][r] = stored;
            if (ZEROS) sh_z[lane / kLanes][r] = (uint8_t)(int)z;
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < kGroups * kPieceRows; e += 256) {
        const int64_t g = piece * kGroups + e / kPieceRows, row = r0 + e % kPieceRows;
        if (g * GROUP < n && row < m) {
            scales[g * ldm + row] = sh_s[e / kPieceRows][e % kPieceRows];
            if (ZEROS) zeros[g * ldm + row] = sh_z[e / kPieceRows][e % kPieceRows];
        }
    }
}

template <typename D> __device__ __forceinline__ D wide(float s, int q) { return el::from_f32<D>(__fmul_rn(s, (float)q)); }
template <> __device__ __forceinline__ double wide<double>(float s, int q) { return (double)s * (double)q; }

// Widening, VEC columns a lane at a time: 16 bytes, or one element where the rows of
// dst start anywhere.  16384 x 8192 to binary32 with zero codes, bound by the writes:
// 103 us, 5.9 TB/s (92 right after the rounding).
template <typename S, typename D, int VEC>
__global__ void __launch_bounds__(256)
q4_widen_kernel(const uint32_t* __restrict__ Q, const S* __restrict__ scales, const uint8_t* __restrict__ zeros,
                int group, int64_t m, int64_t n, int64_t blocks, int64_t pieces, int64_t ldm, D* __restrict__ dst,
                int64_t ld) {
    __shared__ float sh_s[kPieceCols / 32][kPieceRows];
    __shared__ int sh_z[kPieceCols / 32][kPieceRows];
    const int64_t r0 = blockIdx.x / pieces * kPieceRows, piece = blockIdx.x % pieces;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, groups = kPieceCols / group;
    tc::pdl_wait();
    tc::pdl_trigger();
    for (int e = threadIdx.x; e < groups * kPieceRows; e += 256) {
        const int64_t g = piece * groups + e / kPieceRows, row = r0 + e % kPieceRows;
        if (g * group < n && row < m) {
            sh_s[e / kPieceRows][e % kPieceRows] = el::to_f32(scales[g * ldm + row]);
            sh_z[e / kPieceRows][e % kPieceRows] = zeros ? (int)zeros[g * ldm + row] : 8;
        }
    }
    __syncthreads();
    const int shift_of_group = group == 32 ? 5 : group == 64 ? 6 : 7;
#pragma unroll
    for (int i = 0; i < kPieceRows / 8; ++i) {
        const int r = warp + 8 * i;
        const int64_t row = r0 + r;
        if (row >= m) break;
#pragma unroll
        for (int k = 0; k < kPieceCols / (32 * VEC); ++k) {
            const int cp = k * 32 * VEC + lane * VEC;        // column of the piece
            const int64_t c = piece * kPieceCols + cp;
            if (c >= n) continue;
            const int chunk = (cp & 127) >> 3;
            const uint32_t word =
                __ldg(Q + (row * blocks + piece * 2 + (cp >> 7)) * 16 + (chunk & 3) * 4 + (chunk >> 2));
            const float s = sh_s[cp >> shift_of_group][r];
            const int z = sh_z[cp >> shift_of_group][r];
            union {
                uint4 q;
                D e[VEC];
            } u;
#pragma unroll
            for (int e = 0; e < VEC; ++e) u.e[e] = wide<D>(s, (int)((word >> nibble_shift((cp & 7) + e)) & 15u) - z);
            D* to = dst + row * ld + c;
            if (VEC > 1 && c + VEC <= n) {
                __stcs(reinterpret_cast<uint4*>(to), u.q);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (c + e < n) to[e] = u.e[e];
            }
        }
    }
}

lrc_status pieces_of(int64_t m, int64_t n, int cols, const char* what, int64_t* pieces, unsigned* grid) {
    *pieces = (n + cols - 1) / cols;
    return grid_of((m + kPieceRows - 1) / kPieceRows * *pieces, 1, what, grid);
}

template <typename W, typename S>
lrc_status round_as(const void* src, int64_t m, int64_t n, int64_t ldw, void* Q, void* scales, uint8_t* zeros, int group,
                    cudaStream_t s) {
    int64_t pieces;
    unsigned grid;
    lrc_status st = pieces_of(m, n, kRoundCols, "lrc_q4_round", &pieces, &grid);
    if (st != LRC_OK) return st;
    const bool whole16 = aligned16(src) && ldw * (int64_t)sizeof(W) % 16 == 0;
    auto go = [&](auto kernel) -> lrc_status {
        const cudaError_t e = launch_pdl(kernel, dim3(grid), dim3(256), 0, s, (const W*)src, m, n, ldw, whole16,
                                         (uint32_t*)Q, (S*)scales, zeros, (n + 127) / 128, pieces, lrc_packed_ld(m));
        if (e != cudaSuccess) return cuda_fail(e, "q4_round_kernel");
        return after_launch("q4_round_kernel");
    };
    auto by_group = [&](auto z, auto any) {
        constexpr bool Z = decltype(z)::value, A = decltype(any)::value;
        return group == 32   ? go(q4_round_kernel<W, S, 32, Z, A>)
               : group == 64 ? go(q4_round_kernel<W, S, 64, Z, A>)
                             : go(q4_round_kernel<W, S, 128, Z, A>);
    };
    using Yes = std::true_type;
    using No = std::false_type;
    if constexpr (sizeof(W) == 2) {
        if (!whole16) return zeros ? by_group(Yes(), Yes()) : by_group(No(), Yes());
    }
    return zeros ? by_group(Yes(), No()) : by_group(No(), No());
}

template <typename S, typename D>
lrc_status widen_as(const void* Q, const void* scales, const uint8_t* zeros, int group, int64_t m, int64_t n, void* dst,
                    int64_t ld, cudaStream_t s) {
    int64_t pieces;
    unsigned grid;
    lrc_status st = pieces_of(m, n, kPieceCols, "lrc_q4_widen", &pieces, &grid);
    if (st != LRC_OK) return st;
    auto go = [&](auto kernel) -> lrc_status {
        const cudaError_t e = launch_pdl(kernel, dim3(grid), dim3(256), 0, s, (const uint32_t*)Q, (const S*)scales, zeros,
                                         group, m, n, (n + 127) / 128, pieces, lrc_packed_ld(m), (D*)dst, ld);
        if (e != cudaSuccess) return cuda_fail(e, "q4_widen_kernel");
        return after_launch("q4_widen_kernel");
    };
    if (aligned16(dst) && ld * (int64_t)sizeof(D) % 16 == 0) return go(q4_widen_kernel<S, D, 16 / (int)sizeof(D)>);
    return go(q4_widen_kernel<S, D, 1>);
}

}  // namespace

lrc_status launch_q4_round(const void* W, lrc_fmt wfmt, int64_t m, int64_t n, int64_t ldw, void* Q, void* scales,
                           uint8_t* zeros, int group, lrc_fmt fmt, cudaStream_t s) {
    auto by_scale = [&](auto w) {
        using WT = decltype(w);
        if (fmt == LRC_F32) return round_as<WT, float>(W, m, n, ldw, Q, scales, zeros, group, s);
        if (fmt == LRC_BF16) return round_as<WT, bf16>(W, m, n, ldw, Q, scales, zeros, group, s);
        return round_as<WT, __half>(W, m, n, ldw, Q, scales, zeros, group, s);
    };
    switch (wfmt) {
        case LRC_F64: return by_scale(double());
        case LRC_F32: return by_scale(float());
        case LRC_BF16: return by_scale(bf16());
        default: return by_scale(__half());
    }
}

lrc_status launch_q4_widen(const void* Q, const void* scales, const uint8_t* zeros, int group, lrc_fmt fmt, int64_t m,
                           int64_t n, void* dst, lrc_fmt dfmt, int64_t ld, cudaStream_t s) {
    auto by_dst = [&](auto sc) {
        using ST = decltype(sc);
        if (dfmt == LRC_F64) return widen_as<ST, double>(Q, scales, zeros, group, m, n, dst, ld, s);
        if (dfmt == LRC_F32) return widen_as<ST, float>(Q, scales, zeros, group, m, n, dst, ld, s);
        if (dfmt == LRC_BF16) return widen_as<ST, bf16>(Q, scales, zeros, group, m, n, dst, ld, s);
        return widen_as<ST, __half>(Q, scales, zeros, group, m, n, dst, ld, s);
    };
    if (fmt == LRC_F32) return by_dst(float());
    if (fmt == LRC_BF16) return by_dst(bf16());
    return by_dst(__half());
}

}  // namespace lrc
