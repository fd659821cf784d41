// q4.cuh -- what the two products of a 4-bit matrix share (q4.cu: few vectors,
// q4_wide.cu: more): unpacking a word of codes, and a call's arguments.
#pragma once

#include "cluster.cuh"
#include "common.cuh"
#include "elem.cuh"
#include "tc.cuh"

namespace lrc {
namespace q4 {

using bf16 = __nv_bfloat16;

// (a & mask) | bits as one instruction.
template <uint32_t MASK, uint32_t BITS>
__device__ __forceinline__ uint32_t pick(uint32_t a) {
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(d) : "r"(a), "n"(MASK), "n"(BITS));
    return d;
}

struct Half2 {
    using type = __half;
    static constexpr bool kBf16 = false;
    // The eight q - z of a word, in order.  1024 + q for the codes in the low four
    // bits of a byte; 1024 + 16 q for the others, brought to q - z by one exact
    // multiply-add instead of a shift (shifts and masks share a pipe of half the
    // multiply-adds' rate, which is what the kernel would wait for).
    static __device__ __forceinline__ void unpack(uint32_t w, uint32_t z, uint32_t (&r)[4]) {
        const uint32_t one = 0x64006400u + z * 0x10001u;       // 1024 + z
        const uint32_t sixteenth = 0x2c002c00u;                // 1 / 16
        const uint32_t less = 0xd400d400u + z * 0x00100010u;   // -(64 + z)
        const uint32_t w8 = w >> 8;
        const uint32_t lo0 = pick<0x000f000fu, 0x64006400u>(w), hi0 = pick<0x00f000f0u, 0x64006400u>(w);
        const uint32_t lo1 = pick<0x000f000fu, 0x64006400u>(w8), hi1 = pick<0x00f000f0u, 0x64006400u>(w8);
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
    // The same with nothing to add to.
    static __device__ __forceinline__ void mma_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                     uint32_t b0, uint32_t b1) {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
    }
};
struct Bf2 {
    using type = bf16;
    static constexpr bool kBf16 = true;
    // 128 + q has no room for a code above the low four bits: a shift for each.
    // (The upper halves of products with 2^28, 2^24, 2^20 in the place of shifts,
    // on the multipliers' pipe, are slower: 47 us against 43 for 16384 x 16384.)
    static __device__ __forceinline__ void unpack(uint32_t w, uint32_t z, uint32_t (&r)[4]) {
        const uint32_t less = 0x43004300u + z * 0x10001u;      // 128 + z
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t a = pick<0x000f000fu, 0x43004300u>(w >> (4 * u));
            asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r[u]) : "r"(a), "r"(less));
        }
    }
    static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                               uint32_t b0, uint32_t b1) {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
    // The same with nothing to add to.
    static __device__ __forceinline__ void mma_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                     uint32_t b0, uint32_t b1) {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
    }
};

struct ApplyArgs {
    const uint4* Q;          // m rows of 4 blocks uint4
    const void* scales;
    const uint8_t* zeros;
    const void* x;           // cols rows of 16-bit elements, pitch ldx
    const void* A;
    void* y;
    int64_t m, blocks, groups, ldm, ldx, xcols;
    int cols, xrows;         // rows of x (vectors, or three parts of each), and of its boxes
    int R, split, depth;     // groups of 16 rows of a tile; blocks of a cluster; stages of the ring
    bool wide;               // A and y are binary32
};

// Columns of B that a tile of `cols` uses: whole vectors.
constexpr int used_cols(int cols, int PARTS) { return cols / PARTS * PARTS; }

constexpr CUtensorMapDataType map_type(float) { return CU_TENSOR_MAP_DATA_TYPE_FLOAT32; }
constexpr CUtensorMapDataType map_type(__half) { return CU_TENSOR_MAP_DATA_TYPE_FLOAT16; }
constexpr CUtensorMapDataType map_type(bf16) { return CU_TENSOR_MAP_DATA_TYPE_BFLOAT16; }

constexpr int kSmemOfSm = 227 * 1024;

// Each part of a binary32 vector after the first is 2^8 times what is left of it.
constexpr float kPartUp = 256.f;

inline lrc_status grid_of(int64_t threads, int per, const char* what, unsigned* out) {
    const int64_t g = (threads + per - 1) / per;
    if (g > 0x7fffffff) {
        set_error("%s: too large for one launch", what);
        return LRC_ERR_UNSUPPORTED;
    }
    *out = (unsigned)g;
    return LRC_OK;
}

// The end of a tile: sums of SETS sets (set s, column c, row r of the tile at sums[s *
// set + c * pitch + r], pitch a multiple of four) and of the blocks of the cluster,
// added in a fixed order, four rows a thread, the parts' powers of two taken off; then
// A and the rounding.  All loads of
// other blocks are on their way before the first is added: one after the other, their
// latency was up to half of a small product's time.
template <typename OP, int PARTS, int SETS>
__device__ __forceinline__ void finish_tile(const ApplyArgs& a, const float* sums, int set, int pitch, int rows,
                                            int64_t row0, int col0, int vectors, int rank, int threads) {
    const int quads = rows / 4;
    for (int e = rank * threads + (int)threadIdx.x; e < vectors * quads; e += a.split * threads) {
        const int v = e / quads, r = e % quads * 4;
        if (row0 + r >= a.m) continue;
        float sum[4] = {};
#pragma unroll
        for (int p = PARTS - 1; p >= 0; --p) {                    // the smallest part first
            if (p < PARTS - 1) {
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] *= 1.f / kPartUp;
            }
#pragma unroll
            for (int s = 0; s < SETS; ++s) {
                const float* at = sums + s * set + (v * PARTS + p) * pitch + r;
                float4 w[8];
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    if (q < a.split) w[q] = a.split > 1 ? cl::load4(at, q) : *reinterpret_cast<const float4*>(at);
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    if (q < a.split) sum[0] += w[q].x, sum[1] += w[q].y, sum[2] += w[q].z, sum[3] += w[q].w;
            }
        }
        const int64_t o = (int64_t)(col0 / PARTS + v) * a.m + row0 + r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (row0 + r + i >= a.m) break;
            float y = sum[i];
            if (PARTS > 1 || a.wide) {
                if (a.A) y += static_cast<const float*>(a.A)[o + i];
                static_cast<float*>(a.y)[o + i] = y;
            } else {
                using T = typename OP::type;
                if (a.A) y += el::to_f32(static_cast<const T*>(a.A)[o + i]);
                static_cast<T*>(a.y)[o + i] = el::from_f32<T>(y);
            }
        }
    }
}

// The product of more vectors (q4_wide.cu); parts: columns that make one vector.
template <typename OP, typename S, int PARTS>
lrc_status launch_wide(ApplyArgs a, int group, cudaStream_t s);

}  // namespace q4
}  // namespace lrc
