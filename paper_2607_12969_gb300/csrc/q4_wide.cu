// q4_wide.cu -- the product of a 4-bit matrix with more than a few vectors, on the
// fifth-generation tensor cores (tcgen05, accumulators and the matrix in tensor
// memory).
//
// A tile is 128 rows of the matrix and NC columns of vectors.  One warp brings
// blocks of 128 columns by TMA; three groups of four warps take every third block
// each: a thread unpacks its row's 128 codes to the integers q - z, exact in 16
// bits, and writes them to tensor memory as the A operand, one thread issues the
// products with the block's x (B, in shared memory as TMA wrote it), and every
// thread adds its row's sums of each group times the scale in binary32.  So the
// codes are unpacked once for all columns, and neither they nor the sums pass
// through shared memory.  The three groups' sums, and those of the blocks of a
// cluster, which share the columns of the matrix, are added at the end in a fixed
// order.
//
// What bounds it: the unpacking (as in q4.cu), the adding of NC sums a row and
// group, and the chain of a block (unpack, write, multiply, read), of which the
// three groups have one each in flight.
#include "q4.cuh"

#include <math.h>

#include <atomic>

namespace lrc {
namespace {

using namespace q4;

__device__ unsigned int g_err_q4_wide;

constexpr int kTeams = 3, kTeamThreads = 128, kThreads = kTeams * kTeamThreads + 32;
constexpr uint32_t kTmem = 512, kACols = 64;      // columns of tensor memory; of a team's A (128 x 128 of 16 bits)
constexpr int kMostStages = 16;

// D[tmem] (+)= A[tmem] B[smem]^T, 128 x N x 16; one thread issues.
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d), "r"(a), "l"(b_desc), "r"(idesc),
        "r"(accumulate) : "memory");
}
// 16 consecutive 32-bit columns of the warp's 32 lanes.
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}

// Shared memory of a stage, one block of 128 columns: 128 rows of 64 bytes of codes
// (64-byte swizzle), two boxes of 64 columns of x (NC rows of 128 bytes, 128-byte
// swizzle), scales and zero codes of the groups, 128 a group.
template <typename S, int GROUP, bool ZEROS, int NC>
struct WideStage {
    static constexpr int kGroups = 128 / GROUP, kX = 8192, kXBox = NC * 128, kScales = kX + 2 * kXBox;
    static constexpr int kScaleBytes = kGroups * 128 * (int)sizeof(S), kZeros = kScales + kScaleBytes;
    static constexpr int kZeroBytes = ZEROS ? kGroups * 128 : 0;
    static constexpr int kPitch = (kZeros + kZeroBytes + 1023) / 1024 * 1024;
    static constexpr int kSums = kTeams * NC * 129 * 4;
    static constexpr int kRoom = (kSmemOfSm - 3072) / kPitch;
    static constexpr int kDepth = kRoom < kMostStages ? kRoom : kMostStages;
    static_assert(kSums <= kDepth * kPitch, "the sums lie in the ring");
};

template <typename OP, typename S, int PARTS, int GROUP, bool ZEROS, int NC>
__global__ void __launch_bounds__(kThreads, 1)
q4_wide_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap xmap,
               const __grid_constant__ CUtensorMap smap, const __grid_constant__ CUtensorMap zmap,
               const __grid_constant__ ApplyArgs a, const uint32_t idesc) {
    using St = WideStage<S, GROUP, ZEROS, NC>;
    constexpr int kDepth = St::kDepth, kGroups = St::kGroups;
    // sums of so many groups fit into a team's share of tensor memory at once
    constexpr int kAtOnce = kGroups == 1 ? 1 : NC > 32 ? 1 : 2;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t full[kDepth], empty[kDepth], done[kTeams];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, team = warp >> 2;
    const int rank = blockIdx.x % a.split;
    const int64_t row0 = (int64_t)(blockIdx.x / a.split) * 128;
    const int col0 = blockIdx.y * used_cols(NC, PARTS);
    const int mine = (int)((a.blocks - rank + a.split - 1) / a.split);       // blocks of columns
    uint8_t* ring = raw + ((1024u - (tc::smem_u32(raw) & 1023u)) & 1023u);
    volatile int* abort = &abort_flag;
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int d = 0; d < kDepth; ++d) {
            tc::mbar_init(&full[d], 1);
            tc::mbar_init(&empty[d], 1);
        }
        for (int t = 0; t < kTeams; ++t) tc::mbar_init(&done[t], 1);
        tc::fence_barrier_init();
    }
    if (warp == 4 * kTeams) tc::tmem_alloc(&tmem_slot, kTmem);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = tmem_slot;
    tc::pdl_wait();
    tc::pdl_trigger();

    float acc[NC] = {};
    if (team == kTeams) {
        if (lane == 0) {
            const uint32_t bytes = 8192 + a.xrows * 256 + St::kScaleBytes + St::kZeroBytes;
            int k = 0, slot = 0;
            uint32_t phase = 1;
            for (; k < mine; ++k) {
                if (k >= kDepth && !tc::mbar_wait(&empty[slot], phase, abort, &g_err_q4_wide, 1u)) break;
                uint64_t* bar = &full[slot];
                uint8_t* to = ring + slot * St::kPitch;
                const int unit = rank + k * a.split;
                tc::mbar_arrive_expect_tx(bar, bytes);
                tc::tma_load_2d(to, &qmap, unit * 64, (int32_t)row0, bar);
                tc::tma_load_2d(to + St::kX, &xmap, unit * 128, col0, bar);
                tc::tma_load_2d(to + St::kX + St::kXBox, &xmap, unit * 128 + 64, col0, bar);
                tc::tma_load_2d(to + St::kScales, &smap, (int32_t)row0, unit * kGroups, bar);
                if (ZEROS) tc::tma_load_2d(to + St::kZeros, &zmap, (int32_t)row0, unit * kGroups, bar);
                if (++slot == kDepth) {
                    slot = 0;
                    phase ^= 1;
                }
            }
            // no copy is in flight when the block goes on
            volatile int no_abort = 0;
            for (int u = k > kDepth ? k - kDepth : 0; u < k; ++u)
                tc::mbar_wait(&full[u % kDepth], u / kDepth & 1, &no_abort, &g_err_q4_wide, 1u);
        }
        __syncwarp();
    } else {
        const int r = threadIdx.x & 127;                         // row of the tile, lane of tensor memory
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;       // the warp's first lane, in bits 16 and up
        const uint32_t ta = tmem + team * kACols, td = tmem + kTeams * kACols + team * (kAtOnce * NC);
        const bool issuer = r == 0;
        const int swz = r >> 1 & 3;
        uint32_t round = 0;
        // After a wait that gave up the blocks go on without waits: the team's threads meet
        // at its barriers for every block.
        for (int k = team; k < mine; k += kTeams) {
            const int slot = k % kDepth;
            uint8_t* from = ring + slot * St::kPitch;
            tc::mbar_wait(&full[slot], k / kDepth & 1, abort, &g_err_q4_wide, 1u);
            __syncwarp();
            uint4 w[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) w[t] = *reinterpret_cast<const uint4*>(from + r * 64 + ((t ^ swz) << 4));
            float s[kGroups];
#pragma unroll
            for (int g = 0; g < kGroups; ++g) s[g] = el::to_f32(reinterpret_cast<const S*>(from + St::kScales)[g * 128 + r]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {                        // columns 32 j ... 32 j + 31
                const uint32_t z = ZEROS ? from[St::kZeros + j * 32 / GROUP * 128 + r] : 8u;
                uint32_t v[16];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    uint32_t u[4];
                    OP::unpack(j == 0 ? w[t].x : j == 1 ? w[t].y : j == 2 ? w[t].z : w[t].w, z, u);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[4 * t + i] = u[i];
                }
                tmem_st16(ta + lanes + 16 * j, v);
            }
            tc::tmem_st_wait();
#pragma unroll
            for (int g0 = 0; g0 < kGroups; g0 += kAtOnce) {
                tc::tc_fence_before();
                tc::named_bar_sync(1 + team, kTeamThreads);
                if (issuer) {
                    tc::tc_fence_after();
                    const uint64_t x[2] = {tc::desc_sw128(tc::smem_u32(from + St::kX)),
                                           tc::desc_sw128(tc::smem_u32(from + St::kX + St::kXBox))};
#pragma unroll
                    for (int g = g0; g < g0 + kAtOnce; ++g)
#pragma unroll
                        for (int i = 0; i < GROUP / 16; ++i) {
                            const int kk = g * (GROUP / 16) + i;  // step of 16 columns
                            mma_ts(td + (g - g0) * NC, ta + 8 * kk, x[kk >> 2] + 2 * (kk & 3), idesc, i != 0);
                        }
                    tc::mma_commit(&done[team]);
                    if (g0 + kAtOnce >= kGroups) tc::mma_commit(&empty[slot]);
                }
                tc::mbar_wait(&done[team], round & 1, abort, &g_err_q4_wide, 2u);
                ++round;
                __syncwarp();
                tc::tc_fence_after();
#pragma unroll
                for (int g = g0; g < g0 + kAtOnce; ++g)
#pragma unroll
                    for (int c = 0; c < NC; c += 32) {
                        uint32_t v[32];
                        tc::tmem_ld32(td + lanes + (g - g0) * NC + c, v);
                        tc::tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 32; ++i) acc[c + i] = fmaf(s[g], __uint_as_float(v[i]), acc[c + i]);
                    }
            }
        }
        if (*abort && issuer && round) {
            // the products in flight end before the block does
            volatile int no_abort = 0;
            tc::mbar_wait(&done[team], (round - 1) & 1, &no_abort, &g_err_q4_wide, 2u, 100000000ull);
        }
    }
    tc::tc_fence_before();
    __syncthreads();                                             // the ring is free
    tc::tc_fence_after();
    if (warp == 4 * kTeams) tc::tmem_dealloc(tmem, kTmem);
    // sums[team][column][row]
    float(*sums)[NC][129] = reinterpret_cast<float(*)[NC][129]>(ring);
    if (team < kTeams) {
#pragma unroll
        for (int c = 0; c < NC; ++c) sums[team][c][threadIdx.x & 127] = acc[c];
    }
    if (a.split > 1) cl::sync();
    else __syncthreads();
    const int used = min(a.cols - col0, used_cols(NC, PARTS)) / PARTS;       // vectors of this tile
    for (int e = rank * kThreads + threadIdx.x; e < used * 128; e += a.split * kThreads) {
        const int v = e >> 7, r = e & 127;
        if (row0 + r >= a.m) continue;
        float sum = 0.f;
#pragma unroll
        for (int p = PARTS - 1; p >= 0; --p) {                   // the smallest part first
#pragma unroll
            for (int t = 0; t < kTeams; ++t) {
                const float* at = &sums[t][v * PARTS + p][r];
                if (a.split > 1)
                    for (int q = 0; q < a.split; ++q) sum += cl::load(at, q);
                else
                    sum += *at;
            }
        }
        const int64_t o = (int64_t)(col0 / PARTS + v) * a.m + row0 + r;
        if (PARTS > 1 || a.wide) {
            if (a.A) sum += static_cast<const float*>(a.A)[o];
            static_cast<float*>(a.y)[o] = sum;
        } else {
            using T = typename OP::type;
            if (a.A) sum += el::to_f32(static_cast<const T*>(a.A)[o]);
            static_cast<T*>(a.y)[o] = el::from_f32<T>(sum);
        }
    }
    if (a.split > 1) cl::sync();                                 // the sums stay until they are read
}

template <typename OP, typename S, int PARTS, int GROUP, bool ZEROS, int NC>
lrc_status wide_as(ApplyArgs a, cudaStream_t s) {
    using St = WideStage<S, GROUP, ZEROS, NC>;
    constexpr int kUsed = used_cols(NC, PARTS);
    a.xrows = a.cols < kUsed ? a.cols : kUsed;
    const int chunks = (a.cols + kUsed - 1) / kUsed;
    const int64_t tiles = (a.m + 127) / 128;
    // Blocks of a cluster: the number that fills the multiprocessors' waves best, a
    // wave's start and end taken as 14 blocks of columns.
    double best = 1e300;
    const int sms = sm_count();
    for (int split = 1; split <= 8 && split <= a.blocks; split += split < 4 ? 1 : 2) {
        const double cost = ceil((double)tiles * chunks * split / sms) * ((double)((a.blocks + split - 1) / split) + 14.);
        if (cost < best) {
            best = cost;
            a.split = split;
        }
    }
    CUtensorMap qm, xm, sm, zm{};
    lrc_status st = encode_map_2d_sw64(&qm, CU_TENSOR_MAP_DATA_TYPE_UINT8, a.Q, a.blocks * 64, a.m, a.blocks * 64, 64, 128,
                                       "Q");
    if (st != LRC_OK) return st;
    st = encode_map_2d(&xm, map_type(typename OP::type()), a.x, a.xcols, a.cols, a.ldx * 2, 64, (uint32_t)a.xrows, true,
                       "X");
    if (st != LRC_OK) return st;
    st = encode_map_2d(&sm, map_type(S()), a.scales, a.m, a.groups, a.ldm * (int64_t)sizeof(S), 128, St::kGroups, false,
                       "scales");
    if (st != LRC_OK) return st;
    if (ZEROS) {
        st = encode_map_2d(&zm, CU_TENSOR_MAP_DATA_TYPE_UINT8, a.zeros, a.m, a.groups, a.ldm, 128, St::kGroups, false,
                           "zeros");
        if (st != LRC_OK) return st;
    }
    auto kernel = q4_wide_kernel<OP, S, PARTS, GROUP, ZEROS, NC>;
    constexpr int kSmem = St::kDepth * St::kPitch + 1024;
    // the attribute is the device's: set once on each
    static std::atomic<uint64_t> set_on{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && (dev >= 64 || !(set_on.load() >> dev & 1))) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (e == cudaSuccess && dev < 64) set_on |= (uint64_t)1 << dev;
    }
    if (e != cudaSuccess) return cuda_fail(e, "q4_wide_kernel");
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(tiles * a.split), (unsigned)chunks);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)a.split;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.split > 1 ? 2 : 1;
    const uint32_t idesc = tc::idesc_f16_f32(128, NC) | (OP::kBf16 ? tc::kIdescBF16 : 0u);
    e = cudaLaunchKernelEx(&cfg, kernel, qm, xm, sm, zm, a, idesc);
    if (e != cudaSuccess) return cuda_fail(e, "q4_wide_kernel");
    return after_launch("q4_wide_kernel");
}

template <typename OP, typename S, int PARTS, int NC>
lrc_status wide_groups(const ApplyArgs& a, int group, cudaStream_t s) {
    if (a.zeros) {
        if (group == 32) return wide_as<OP, S, PARTS, 32, true, NC>(a, s);
        if (group == 64) return wide_as<OP, S, PARTS, 64, true, NC>(a, s);
        return wide_as<OP, S, PARTS, 128, true, NC>(a, s);
    }
    if (group == 32) return wide_as<OP, S, PARTS, 32, false, NC>(a, s);
    if (group == 64) return wide_as<OP, S, PARTS, 64, false, NC>(a, s);
    return wide_as<OP, S, PARTS, 128, false, NC>(a, s);
}

}  // namespace

namespace q4 {

template <typename OP, typename S, int PARTS>
lrc_status launch_wide(ApplyArgs a, int group, cudaStream_t s) {
    return a.cols <= used_cols(32, PARTS) ? wide_groups<OP, S, PARTS, 32>(a, group, s)
                                          : wide_groups<OP, S, PARTS, 64>(a, group, s);
}
template lrc_status launch_wide<Half2, __half, 1>(ApplyArgs, int, cudaStream_t);
template lrc_status launch_wide<Bf2, bf16, 1>(ApplyArgs, int, cudaStream_t);
template lrc_status launch_wide<Bf2, float, 3>(ApplyArgs, int, cudaStream_t);

}  // namespace q4

uint32_t take_q4_wide_error() {
    unsigned int v = 0;
    if (cudaMemcpyFromSymbol(&v, g_err_q4_wide, sizeof v) != cudaSuccess) return 0xffffffffu;
    if (v) {
        const unsigned int z = 0;
        cudaMemcpyToSymbol(g_err_q4_wide, &z, sizeof z);
    }
    return v;
}

}  // namespace lrc
