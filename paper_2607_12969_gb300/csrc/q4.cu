// q4.cu -- matrices of 4-bit codes with a scale per row and group of columns:
// rounding, widening, and the product with a few vectors (lrc_q4_round,
// lrc_q4_widen, lrc_q4_apply).
//
// What[i][c] = s (q - z).  The codes' layout is the one include/lrc.h states:
// 64-byte blocks of 128 columns, column 32 j + 8 t + e in word 4 t + j.
#include "common.cuh"
#include "elem.cuh"

namespace lrc {
namespace {

using bf16 = __nv_bfloat16;

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

// Rounding: one warp a block of 128 columns of a row, four consecutive columns
// a lane.  group / 4 neighbouring lanes share a scale.
template <typename W, typename S>
__global__ void __launch_bounds__(256)
q4_round_kernel(const W* __restrict__ src, int64_t m, int64_t n, int64_t ldw, uint32_t* __restrict__ Q,
                S* __restrict__ scales, uint8_t* __restrict__ zeros, int group, int64_t blocks, int64_t ldm) {
    const int64_t id = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
    const int lane = threadIdx.x & 31;
    if (id >= m * blocks) return;
    const int64_t row = id / blocks, block = id - row * blocks;
    const int64_t c0 = block * 128 + lane * 4;
    float w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = c0 + k < n ? src_f32(src[row * ldw + c0 + k]) : 0.f;
    float lo = 0.f, hi = 0.f;
    bool odd = false;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        lo = fminf(lo, w[k]);
        hi = fmaxf(hi, w[k]);
        odd |= !(fabsf(w[k]) <= 3.402823466e38f);
    }
    int any = odd;
    for (int o = 1; o < group / 4; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        any |= __shfl_xor_sync(0xffffffffu, any, o);
    }
    float s = zeros ? __fmul_rn(__fsub_rn(hi, lo), kFifteenth) : __fmul_rn(fmaxf(hi, -lo), kSeventh);
    S stored = el::from_f32<S>(fminf(s, largest<S>()));
    s = el::to_f32(stored);
    const bool none = s < 1.17549435e-38f;
    const float inv = none ? 0.f : __frcp_rn(s);
    if (none) stored = el::from_f32<S>(0.f);
    float z = zeros ? fminf(fmaxf(rintf(__fmul_rn(-lo, inv)), 0.f), 15.f) : 8.f;
    if (any) {
        stored = el::from_f32<S>(__int_as_float(0x7fffffff));
        z = 8.f;
    }
    uint32_t word = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float q = any ? 8.f : fminf(fmaxf(rintf(__fmul_rn(w[k], inv)) + z, 0.f), 15.f);
        word |= (uint32_t)(int)q << nibble_shift((lane & 1) * 4 + k);
    }
    word |= __shfl_xor_sync(0xffffffffu, word, 1);
    const int chunk = lane >> 1;                         // 8 columns: 4 j + t
    if (!(lane & 1)) Q[(row * blocks + block) * 16 + (chunk & 3) * 4 + (chunk >> 2)] = word;
    if (lane % (group / 4) == 0 && c0 < n) {
        const int64_t g = c0 / group;
        scales[g * ldm + row] = stored;
        if (zeros) zeros[g * ldm + row] = (uint8_t)(int)z;
    }
}

template <typename D> __device__ __forceinline__ D wide(float s, int q) { return el::from_f32<D>(__fmul_rn(s, (float)q)); }
template <> __device__ __forceinline__ double wide<double>(float s, int q) { return (double)s * (double)q; }

// Widening: one thread an entry.
template <typename S, typename D>
__global__ void __launch_bounds__(256)
q4_widen_kernel(const uint32_t* __restrict__ Q, const S* __restrict__ scales, const uint8_t* __restrict__ zeros,
                int group, int64_t m, int64_t n, int64_t blocks, int64_t ldm, D* __restrict__ dst, int64_t ld) {
    const int64_t id = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (id >= m * n) return;
    const int64_t row = id / n, c = id - row * n;
    const int chunk = (int)(c & 127) >> 3;
    const uint32_t word = Q[(row * blocks + (c >> 7)) * 16 + (chunk & 3) * 4 + (chunk >> 2)];
    const int64_t g = (c / group) * ldm + row;
    const int q = (int)((word >> nibble_shift((int)c & 7)) & 15u) - (zeros ? (int)zeros[g] : 8);
    dst[row * ld + c] = wide<D>(el::to_f32(scales[g]), q);
}

// Product: one warp a row of the matrix and four vectors, one word (8 columns)
// a lane at a time.
constexpr int kVectors = 4;
template <typename X, typename Y>
__global__ void __launch_bounds__(256)
q4_apply_kernel(const uint32_t* __restrict__ Q, const X* __restrict__ scales, const uint8_t* __restrict__ zeros,
                const X* __restrict__ x, const Y* A, Y* y, int64_t m, int64_t n, int64_t b, int group, int64_t blocks,
                int64_t ldm, int64_t ldn) {
    const int64_t row = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
    const int lane = threadIdx.x & 31;
    if (row >= m) return;
    const int64_t b0 = (int64_t)blockIdx.y * kVectors;
    float acc[kVectors] = {};
    for (int64_t w = lane; w < blocks * 16; w += 32) {
        const int slot = (int)w & 15;
        const int64_t c0 = (w >> 4) * 128 + ((slot & 3) * 4 + (slot >> 2)) * 8;
        if (c0 >= n) continue;
        const uint32_t word = Q[row * blocks * 16 + w];
        const int64_t g = (c0 / group) * ldm + row;
        const float s = el::to_f32(scales[g]);
        const int z = zeros ? zeros[g] : 8;
        float part[kVectors] = {};
        for (int e = 0; e < 8 && c0 + e < n; ++e) {
            const float q = (float)((int)((word >> nibble_shift(e)) & 15u) - z);
#pragma unroll
            for (int v = 0; v < kVectors; ++v)
                if (b0 + v < b) part[v] = fmaf(q, el::to_f32(x[(b0 + v) * ldn + c0 + e]), part[v]);
        }
#pragma unroll
        for (int v = 0; v < kVectors; ++v) acc[v] = fmaf(s, part[v], acc[v]);
    }
#pragma unroll
    for (int v = 0; v < kVectors; ++v) {
        const float r = el::warp_sum(acc[v]);
        if (lane == 0 && b0 + v < b) {
            const int64_t at = (b0 + v) * m + row;
            y[at] = el::from_f32<Y>(A ? r + el::to_f32(A[at]) : r);
        }
    }
}

lrc_status grid_of(int64_t threads, int per, const char* what, unsigned* out) {
    const int64_t g = (threads + per - 1) / per;
    if (g > 0x7fffffff) {
        set_error("%s: too large for one launch", what);
        return LRC_ERR_UNSUPPORTED;
    }
    *out = (unsigned)g;
    return LRC_OK;
}

template <typename W, typename S>
lrc_status round_as(const void* src, int64_t m, int64_t n, int64_t ldw, void* Q, void* scales, uint8_t* zeros, int group,
                    cudaStream_t s) {
    const int64_t blocks = (n + 127) / 128;
    unsigned grid;
    lrc_status st = grid_of(m * blocks * 32, 256, "lrc_q4_round", &grid);
    if (st != LRC_OK) return st;
    q4_round_kernel<W, S><<<grid, 256, 0, s>>>((const W*)src, m, n, ldw, (uint32_t*)Q, (S*)scales, zeros, group, blocks,
                                               lrc_packed_ld(m));
    return after_launch("q4_round_kernel");
}

template <typename S, typename D>
lrc_status widen_as(const void* Q, const void* scales, const uint8_t* zeros, int group, int64_t m, int64_t n, void* dst,
                    int64_t ld, cudaStream_t s) {
    unsigned grid;
    lrc_status st = grid_of(m * n, 256, "lrc_q4_widen", &grid);
    if (st != LRC_OK) return st;
    q4_widen_kernel<S, D><<<grid, 256, 0, s>>>((const uint32_t*)Q, (const S*)scales, zeros, group, m, n, (n + 127) / 128,
                                               lrc_packed_ld(m), (D*)dst, ld);
    return after_launch("q4_widen_kernel");
}

template <typename X, typename Y>
lrc_status apply_as(const void* Q, const void* scales, const uint8_t* zeros, const void* x, const void* A, void* y,
                    int64_t m, int64_t n, int64_t b, int group, cudaStream_t s) {
    unsigned grid;
    lrc_status st = grid_of(m * 32, 256, "lrc_q4_apply", &grid);
    if (st != LRC_OK) return st;
    for (int64_t b0 = 0; b0 < b; b0 += 65535 * kVectors) {
        const int64_t nb = b - b0 < 65535 * kVectors ? b - b0 : 65535 * kVectors;
        const int64_t ldn = lrc_packed_ld(n);
        q4_apply_kernel<X, Y><<<dim3(grid, (unsigned)((nb + kVectors - 1) / kVectors)), 256, 0, s>>>(
            (const uint32_t*)Q, (const X*)scales, zeros, (const X*)x + b0 * ldn, A ? (const Y*)A + b0 * m : nullptr,
            (Y*)y + b0 * m, m, n, nb, group, (n + 127) / 128, lrc_packed_ld(m), ldn);
        if ((st = after_launch("q4_apply_kernel")) != LRC_OK) return st;
    }
    return LRC_OK;
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

lrc_status launch_q4_apply(const void* Q, const void* scales, const uint8_t* zeros, const void* X, const void* A, void* Y,
                           int64_t m, int64_t n, int64_t b, int group, lrc_fmt fmt, cudaStream_t s) {
    if (fmt == LRC_F32) return apply_as<float, float>(Q, scales, zeros, X, A, Y, m, n, b, group, s);
    if (fmt == LRC_BF16) return apply_as<bf16, bf16>(Q, scales, zeros, X, A, Y, m, n, b, group, s);
    if (fmt == LRC_F16) return apply_as<__half, float>(Q, scales, zeros, X, A, Y, m, n, b, group, s);
    return apply_as<__half, __half>(Q, scales, zeros, X, A, Y, m, n, b, group, s);
}

}  // namespace lrc
