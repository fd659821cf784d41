// q4.cu -- matrices of 4-bit codes with a scale per row and group of columns:
// rounding, widening, and the product with a few vectors (lrc_q4_round,
// lrc_q4_widen, lrc_q4_apply).
//
// What[i][c] = s (q - z).  The codes' layout is the one include/lrc.h states:
// 64-byte blocks of 128 columns, column 32 j + 8 t + e in word 4 t + j.
#include "common.cuh"
#include "elem.cuh"
#include "tc.cuh"

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

// ---- product ---------------------------------------------------------------
//
// Y^T = s (q - z) X^T on the matrix instructions m16n8k16: the integers q - z
// are exact in binary16 and bfloat16 (1024 + q, or 128 + q, is the code's bits
// under a constant; subtracting 1024 + z is exact), the matrix is the A operand
// (16 rows), the vectors are the 8 columns of B.  A warp takes blocks of 128
// columns: thread (g, t) of the warp (lane 4 g + t) loads 16 bytes of the rows g
// and g + 8 of a tile, the words 4 t + j, and word j holds its columns of step j,
// 32 columns or two instructions; the order of columns within an instruction is
// free as long as B has the same, so the thread's x are 16 consecutive bytes.
// A group's sum is scaled in binary32 and added to the running one.
//
// The warps of a block share 16 MT rows and take every WARPS-th block of
// columns; their sums are added in shared memory in the order of the warps.

struct Half2 {
    using type = __half;
    // The eight q - z of a word, in order.  1024 + q for the codes in the low four
    // bits of a byte; 1024 + 16 q for the others, brought to q - z by one exact
    // multiply-add instead of a shift (shifts and masks share a pipe of half the
    // multiply-adds' rate, which is what the kernel would wait for).
    static __device__ __forceinline__ void unpack(uint32_t w, uint32_t z, uint32_t (&r)[4]) {
        const uint32_t one = 0x64006400u + z * 0x10001u;       // 1024 + z
        const uint32_t sixteenth = 0x2c002c00u;                // 1 / 16
        const uint32_t less = 0xd400d400u + z * 0x00100010u;   // -(64 + z)
        const uint32_t w8 = w >> 8;
        const uint32_t lo0 = (w & 0x000f000fu) | 0x64006400u, hi0 = (w & 0x00f000f0u) | 0x64006400u;
        const uint32_t lo1 = (w8 & 0x000f000fu) | 0x64006400u, hi1 = (w8 & 0x00f000f0u) | 0x64006400u;
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r[0]) : "r"(lo0), "r"(one));
        asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r[1]) : "r"(hi0), "r"(sixteenth), "r"(less));
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r[2]) : "r"(lo1), "r"(one));
        asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r[3]) : "r"(hi1), "r"(sixteenth), "r"(less));
    }
    static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                               uint32_t b0, uint32_t b1) {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
};
struct Bf2 {
    using type = bf16;
    // 128 + q has no room for a code above the low four bits: a shift for each.
    static __device__ __forceinline__ void unpack(uint32_t w, uint32_t z, uint32_t (&r)[4]) {
        const uint32_t less = 0x43004300u + z * 0x10001u;      // 128 + z
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t a = ((w >> (4 * u)) & 0x000f000fu) | 0x43004300u;
            asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r[u]) : "r"(a), "r"(less));
        }
    }
    static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                               uint32_t b0, uint32_t b1) {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
};

struct ApplyArgs {
    const uint4* Q;          // m rows of 4 blocks uint4
    const void* scales;
    const uint8_t* zeros;
    const void* x;           // cols rows of 16-bit elements, pitch ldx
    const void* A;
    void* y;
    int64_t m, n, blocks, groups, ldm, ldx;
    int cols;                // rows of x: vectors, or three parts of each
    bool wide;               // A and y are binary32
};

// 16 bytes of codes, read once.
__device__ __forceinline__ uint4 load_codes(const uint4* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

struct Whole { static constexpr bool value = false; };
struct Ragged { static constexpr bool value = true; };

template <typename S, int MT>
struct Stage {
    uint4 w[MT][2];
    S s[MT][2];
    uint8_t z[MT][2];
};

// OP: the instructions' element type; S: the scales' type; PARTS: columns of B
// that make one vector (3: a binary32 vector as hi + mid + lo in bfloat16).
template <typename OP, typename S, int PARTS, int GROUP, bool ZEROS, int NT, int MT, int WARPS>
__global__ void __launch_bounds__(WARPS * 32)
q4_apply_kernel(const ApplyArgs a) {
    constexpr int kRows = 16 * MT, kCols = 8 * NT, kGroups = 128 / GROUP;      // groups of a block
    __shared__ float sums[WARPS][kCols][kRows + 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int64_t row0 = (int64_t)blockIdx.x * kRows;
    const int col0 = blockIdx.y * kCols;

    // Rows and columns beyond the last are read again and not written.
    const uint4* q[MT][2];
    const S* sp[MT][2];
    const uint8_t* zp[MT][2];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            int64_t r = row0 + 16 * i + 8 * h + g;
            if (r >= a.m) r = a.m - 1;
            q[i][h] = a.Q + (r * a.blocks + warp) * 4 + t;
            // thread t of a quad holds the scale (and zero code) of step t of a block
            const int64_t at = (int64_t)(warp * kGroups + t * kGroups / 4) * a.ldm + r;
            sp[i][h] = static_cast<const S*>(a.scales) + at;
            zp[i][h] = ZEROS ? a.zeros + at : nullptr;
        }
    const uint16_t* x[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int c = min(col0 + 8 * j + g, a.cols - 1);
        x[j] = static_cast<const uint16_t*>(a.x) + (int64_t)c * a.ldx + warp * 128 + 8 * t;
    }
    tc::pdl_wait();
    tc::pdl_trigger();

    float acc[MT][NT][4] = {};
    Stage<S, MT> st[2];
    // Loads block `block` and moves the pointers on.  Steps of a ragged last block
    // whose group does not exist take another scale: their x are zeros.
    auto load = [&](Stage<S, MT>& f, int64_t block) {
        const bool there = GROUP == 128 || block * kGroups + t * kGroups / 4 < a.groups;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f.w[i][h] = load_codes(q[i][h]);
                f.s[i][h] = there ? __ldg(sp[i][h]) : el::from_f32<S>(0.f);
                if (ZEROS) f.z[i][h] = there ? __ldg(zp[i][h]) : 0;
                q[i][h] += WARPS * 4;
                sp[i][h] += (int64_t)WARPS * kGroups * a.ldm;
                if (ZEROS) zp[i][h] += (int64_t)WARPS * kGroups * a.ldm;
            }
    };
    // left: columns of the block from the thread's first one on
    auto compute = [&](const Stage<S, MT>& f, auto ragged, int left) {
        float part[MT][NT][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint4 xv[NT];
#pragma unroll
            for (int k = 0; k < NT; ++k) {
                const uint16_t* p = x[k] + 32 * j;
                if (!decltype(ragged)::value || 32 * j + 8 <= left) {
                    xv[k] = __ldg(reinterpret_cast<const uint4*>(p));
                } else {
                    uint32_t e[4] = {};
#pragma unroll
                    for (int u = 0; u < 8; ++u)
                        if (32 * j + u < left) e[u >> 1] |= (uint32_t)p[u] << (16 * (u & 1));
                    xv[k] = make_uint4(e[0], e[1], e[2], e[3]);
                }
            }
            constexpr int kSteps = GROUP / 32;           // steps of a group
            const int from = (lane & ~3) | j;
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                uint32_t r[2][4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t w = j == 0 ? f.w[i][h].x : j == 1 ? f.w[i][h].y : j == 2 ? f.w[i][h].z : f.w[i][h].w;
                    uint32_t z = 8;
                    if (ZEROS) z = GROUP == 128 ? f.z[i][h] : __shfl_sync(0xffffffffu, f.z[i][h], from);
                    OP::unpack(w, z, r[h]);
                }
#pragma unroll
                for (int k = 0; k < NT; ++k) {
                    if (j % kSteps == 0) part[i][k][0] = part[i][k][1] = part[i][k][2] = part[i][k][3] = 0.f;
                    OP::mma(part[i][k], r[0][0], r[1][0], r[0][1], r[1][1], xv[k].x, xv[k].y);
                    OP::mma(part[i][k], r[0][2], r[1][2], r[0][3], r[1][3], xv[k].z, xv[k].w);
                }
                if ((j + 1) % kSteps == 0) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float s = el::to_f32(f.s[i][h]);
                        if (GROUP != 128) s = __shfl_sync(0xffffffffu, s, from);
#pragma unroll
                        for (int k = 0; k < NT; ++k) {
                            acc[i][k][2 * h] = fmaf(s, part[i][k][2 * h], acc[i][k][2 * h]);
                            acc[i][k][2 * h + 1] = fmaf(s, part[i][k][2 * h + 1], acc[i][k][2 * h + 1]);
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int k = 0; k < NT; ++k) x[k] += WARPS * 128;
    };
    // x is padded with zeros where it is made of parts
    const int64_t whole = PARTS > 1 ? a.blocks : a.n / 128;
    int64_t block = warp;
    if (block < a.blocks) load(st[0], block);
    while (block + WARPS < whole) {
        load(st[1], block + WARPS);
        compute(st[0], Whole(), 0);
        if (block + 2 * WARPS < a.blocks) load(st[0], block + 2 * WARPS);
        compute(st[1], Whole(), 0);
        block += 2 * WARPS;
    }
    // at most two blocks are left, the last of them perhaps ragged
    if (block < a.blocks) {
        const bool more = block + WARPS < a.blocks;
        if (more) load(st[1], block + WARPS);
        if (block < whole) compute(st[0], Whole(), 0);
        else compute(st[0], Ragged(), (int)(a.n - block * 128) - 8 * t);
        if (more) compute(st[1], Ragged(), (int)(a.n - (block + WARPS) * 128) - 8 * t);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int k = 0; k < NT; ++k)
#pragma unroll
            for (int u = 0; u < 4; ++u)
                sums[warp][8 * k + 2 * t + (u & 1)][16 * i + 8 * (u >> 1) + g] = acc[i][k][u];
    __syncthreads();
    const int used = min(a.cols - col0, kCols);
    for (int e = threadIdx.x; e < used / PARTS * kRows; e += WARPS * 32) {
        const int v = e / kRows, r = e % kRows;
        if (row0 + r >= a.m) continue;
        float sum = 0.f;
#pragma unroll
        for (int p = PARTS - 1; p >= 0; --p)          // the smallest part first
#pragma unroll
            for (int w = 0; w < WARPS; ++w) sum += sums[w][v * PARTS + p][r];
        const int64_t at = (int64_t)(col0 / PARTS + v) * a.m + row0 + r;
        if (PARTS > 1 || a.wide) {
            if (a.A) sum += static_cast<const float*>(a.A)[at];
            static_cast<float*>(a.y)[at] = sum;
        } else {
            using T = typename OP::type;
            if (a.A) sum += el::to_f32(static_cast<const T*>(a.A)[at]);
            static_cast<T*>(a.y)[at] = el::from_f32<T>(sum);
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

// binary32 vectors as three bfloat16 parts, x = hi + mid + lo exactly (each cut
// off, not rounded, so that none overflows): rows 3 v, 3 v + 1, 3 v + 2 of
// `blocks` whole blocks of columns, zeros from n on.  An infinity or NaN is in
// the first part alone.
__global__ void __launch_bounds__(256)
q4_parts_kernel(const float* __restrict__ x, int64_t n, int64_t ldn, int64_t ldp, uint16_t* __restrict__ parts) {
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    tc::pdl_wait();
    tc::pdl_trigger();
    if (c >= ldp) return;
    const float v = c < n ? x[(int64_t)blockIdx.y * ldn + c] : 0.f;
    const uint32_t hi = __float_as_uint(v) & 0xffff0000u;
    const bool odd = !(fabsf(v) <= 3.402823466e38f);
    const float rest = odd ? 0.f : v - __uint_as_float(hi);
    const uint32_t mid = __float_as_uint(rest) & 0xffff0000u;
    const float last = rest - __uint_as_float(mid);
    uint16_t* p = parts + (int64_t)blockIdx.y * 3 * ldp + c;
    p[0] = odd && v != v ? 0x7fffu : (uint16_t)(hi >> 16);
    p[ldp] = (uint16_t)(mid >> 16);
    p[2 * ldp] = (uint16_t)(__float_as_uint(last) >> 16);
}

template <typename OP, typename S, int PARTS, int NT, int MT, int WARPS>
lrc_status apply_launch(const ApplyArgs& a, int group, cudaStream_t s) {
    unsigned grid;
    lrc_status st = grid_of(a.m, 16 * MT, "lrc_q4_apply", &grid);
    if (st != LRC_OK) return st;
    constexpr int kCols = 8 * NT;
    static_assert(kCols % PARTS == 0, "whole vectors a tile");
    auto go = [&](auto kernel) {
        const cudaError_t e = launch_pdl(kernel, dim3(grid, (unsigned)((a.cols + kCols - 1) / kCols)), dim3(WARPS * 32), 0, s,
                                         a);
        if (e != cudaSuccess) return cuda_fail(e, "q4_apply_kernel");
        return after_launch("q4_apply_kernel");
    };
    if (a.zeros) {
        if (group == 32) return go(q4_apply_kernel<OP, S, PARTS, 32, true, NT, MT, WARPS>);
        if (group == 64) return go(q4_apply_kernel<OP, S, PARTS, 64, true, NT, MT, WARPS>);
        return go(q4_apply_kernel<OP, S, PARTS, 128, true, NT, MT, WARPS>);
    }
    if (group == 32) return go(q4_apply_kernel<OP, S, PARTS, 32, false, NT, MT, WARPS>);
    if (group == 64) return go(q4_apply_kernel<OP, S, PARTS, 64, false, NT, MT, WARPS>);
    return go(q4_apply_kernel<OP, S, PARTS, 128, false, NT, MT, WARPS>);
}

template <typename OP, typename S, int PARTS>
lrc_status apply_tiles(const ApplyArgs& a, int group, cudaStream_t s) {
    if constexpr (PARTS == 1) {
        if (a.cols <= 8) return apply_launch<OP, S, 1, 1, 1, 8>(a, group, s);
        if (a.cols <= 16) return apply_launch<OP, S, 1, 2, 1, 8>(a, group, s);
        if (a.cols <= 32) return apply_launch<OP, S, 1, 4, 1, 8>(a, group, s);
        return apply_launch<OP, S, 1, 8, 1, 8>(a, group, s);
    } else {
        return apply_launch<OP, S, 3, 3, 1, 8>(a, group, s);
    }
}

template <typename OP, typename S, typename Y, int PARTS>
lrc_status apply_as(const void* Q, const void* scales, const uint8_t* zeros, const void* x, const void* A, void* y,
                    int64_t m, int64_t n, int64_t b, int group, cudaStream_t s) {
    ApplyArgs a{};
    a.Q = (const uint4*)Q;
    a.scales = scales;
    a.zeros = zeros;
    a.m = m;
    a.n = n;
    a.blocks = (n + 127) / 128;
    a.ldm = lrc_packed_ld(m);
    a.groups = (n + group - 1) / group;
    a.wide = sizeof(Y) == 4;
    const int64_t ldn = lrc_packed_ld(n);
    // at most this many vectors a launch
    constexpr int64_t kMost = 16384;
    for (int64_t b0 = 0; b0 < b; b0 += kMost) {
        const int64_t nb = b - b0 < kMost ? b - b0 : kMost;
        a.A = A ? (const Y*)A + b0 * m : nullptr;
        a.y = (Y*)y + b0 * m;
        a.cols = (int)nb * PARTS;
        if (PARTS == 1) {
            a.x = (const uint16_t*)x + b0 * ldn;
            a.ldx = ldn;
        } else {
            a.ldx = a.blocks * 128;
            void* ws = nullptr;
            lrc_status st = stream_workspace(s, (size_t)nb * 3 * a.ldx * 2, &ws);
            if (st != LRC_OK) return st;
            a.x = ws;
            unsigned grid;
            if ((st = grid_of(a.ldx, 256, "lrc_q4_apply", &grid)) != LRC_OK) return st;
            const cudaError_t e = launch_pdl(q4_parts_kernel, dim3(grid, (unsigned)nb), dim3(256), 0, s,
                                             (const float*)x + b0 * ldn, n, ldn, a.ldx, (uint16_t*)ws);
            if (e != cudaSuccess) return cuda_fail(e, "q4_parts_kernel");
            if ((st = after_launch("q4_parts_kernel")) != LRC_OK) return st;
        }
        const lrc_status st = apply_tiles<OP, S, PARTS>(a, group, s);
        if (st != LRC_OK) return st;
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
    if (fmt == LRC_F32) return apply_as<Bf2, float, float, 3>(Q, scales, zeros, X, A, Y, m, n, b, group, s);
    if (fmt == LRC_BF16) return apply_as<Bf2, bf16, bf16, 1>(Q, scales, zeros, X, A, Y, m, n, b, group, s);
    if (fmt == LRC_F16) return apply_as<Half2, __half, float, 1>(Q, scales, zeros, X, A, Y, m, n, b, group, s);
    return apply_as<Half2, __half, __half, 1>(Q, scales, zeros, X, A, Y, m, n, b, group, s);
}

}  // namespace lrc
