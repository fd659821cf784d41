// q4_wide.cu -- the product of a 4-bit matrix with more than a few vectors, on the
// fifth-generation tensor cores (tcgen05, accumulators and the matrix in tensor
// memory).
//
// A tile is 256 rows of the matrix and 64 columns of vectors, 128 columns of the
// matrix (a block) at a time, brought by TMA.  Two pairs of teams of four warps take
// every second block each, a team of a pair half of the rows: a thread unpacks its
// row's 128 codes to the integers q - z, exact in 16 bits, and writes them to tensor
// memory as the A operand, one thread issues the products with the block's x (B, in
// shared memory as TMA wrote it), and every thread adds its row's sums of each group
// times the scale in binary32.  So the codes are unpacked once for all columns, and
// neither they nor the sums pass through shared memory.  The pairs' sums, and those
// of the blocks of a cluster, which share the columns of the matrix, are added at
// the end in a fixed order.
//
// What bounds it: for 16384 x 8192 and 64 binary16 vectors (33 us) the chain of a
// block (unpack, write, multiply, read, add), of which a multiprocessor has four in
// flight -- all of tensor memory is in use -- and the polling of those who wait;
// leaving out any one step of it gains 1 to 7 us.  With 128 rows a tile (34 us) the
// vectors pass the multiprocessors' L2 ports twice as often: 128 vectors 65 us
// against 56.  Four kinds of warps that hand blocks on took 57 us.  Smaller groups are
// multiplied, read and scaled one after the other: 38 us with groups of 64, 52 of 32,
// whose four scales a thread also spill (28 to 56 bytes).  More than 64 vectors take
// the codes again for every 64: 128 56 us, 2048 740.
#include "q4.cuh"

#include <math.h>

#include <atomic>

namespace lrc {
namespace {

using namespace q4;

__device__ unsigned int g_err_q4_wide;

constexpr int kPairs = 2, kTeams = 2 * kPairs, kTeamThreads = 128, kThreads = kTeams * kTeamThreads;
constexpr int kRows = 256;
constexpr int kCols = 64;                         // columns of vectors of a tile
constexpr uint32_t kTmem = 512, kACols = 64;      // columns of tensor memory; of a team's A (128 x 128 of 16 bits)
constexpr int kMostStages = 4;                    // of a pair

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

// Shared memory of a stage, one block of 128 columns: kRows rows of 64 bytes of codes
// (64-byte swizzle), two boxes of 64 columns of x (kCols rows of 128 bytes, 128-byte
// swizzle), scales and zero codes of the groups, kRows a group.
template <typename S, int GROUP, bool ZEROS>
struct WideStage {
    static constexpr int kGroups = 128 / GROUP, kX = kRows * 64, kXBox = kCols * 128, kScales = kX + 2 * kXBox;
    static constexpr int kScaleBytes = kGroups * kRows * (int)sizeof(S), kZeros = kScales + kScaleBytes;
    static constexpr int kZeroBytes = ZEROS ? kGroups * kRows : 0;
    static constexpr int kPitch = (kZeros + kZeroBytes + 1023) / 1024 * 1024;
    static constexpr int kSums = kPairs * kCols * (kRows + 4) * 4;
    static constexpr int kRoom = (kSmemOfSm - 3072) / kPitch / kPairs;
    static constexpr int kDepth = kRoom < kMostStages ? kRoom : kMostStages;        // stages of a pair
    static_assert(kDepth >= 2 && kSums <= kPairs * kDepth * kPitch, "the sums lie in the ring");
};

template <typename OP, typename S, int PARTS, int GROUP, bool ZEROS>
__global__ void __launch_bounds__(kThreads, 1)
q4_wide_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap xmap,
               const __grid_constant__ CUtensorMap smap, const __grid_constant__ CUtensorMap zmap,
               const __grid_constant__ ApplyArgs a, const uint32_t idesc) {
    using St = WideStage<S, GROUP, ZEROS>;
    constexpr int kDepth = St::kDepth, kGroups = St::kGroups;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t full[kPairs][kDepth], empty[kPairs][kDepth], done[kTeams];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    const int warp = threadIdx.x >> 5, team = warp >> 2, pair = team >> 1, half = team & 1;
    const int rank = blockIdx.x % a.split;
    const int64_t row0 = (int64_t)(blockIdx.x / a.split) * kRows;
    const int col0 = blockIdx.y * used_cols(kCols, PARTS);
    const int mine = (int)((a.blocks - rank + a.split - 1) / a.split);       // blocks of columns
    uint8_t* base = raw + ((1024u - (tc::smem_u32(raw) & 1023u)) & 1023u);
    volatile int* abort = &abort_flag;
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int p = 0; p < kPairs; ++p)
            for (int d = 0; d < kDepth; ++d) {
                tc::mbar_init(&full[p][d], 1);
                tc::mbar_init(&empty[p][d], 2);
            }
        for (int t = 0; t < kTeams; ++t) tc::mbar_init(&done[t], 1);
        tc::fence_barrier_init();
    }
    if (warp == 0) tc::tmem_alloc(&tmem_slot, kTmem);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = tmem_slot;
    tc::pdl_wait();
    tc::pdl_trigger();

    float acc[kCols] = {};
    uint8_t* ring = base + pair * kDepth * St::kPitch;
    // the pair's n-th block, block 2 n + pair of the tile's, into its stage
    auto issue = [&](int n) {
        uint64_t* bar = &full[pair][n % kDepth];
        uint8_t* to = ring + n % kDepth * St::kPitch;
        const int unit = rank + (n * kPairs + pair) * a.split;
        tc::mbar_arrive_expect_tx(bar, kRows * 64 + a.xrows * 256 + St::kScaleBytes + St::kZeroBytes);
        tc::tma_load_2d(to, &qmap, unit * 64, (int32_t)row0, bar);
        tc::tma_load_2d(to + St::kX, &xmap, unit * 128, col0, bar);
        tc::tma_load_2d(to + St::kX + St::kXBox, &xmap, unit * 128 + 64, col0, bar);
        tc::tma_load_2d(to + St::kScales, &smap, (int32_t)row0, unit * kGroups, bar);
        if (ZEROS) tc::tma_load_2d(to + St::kZeros, &zmap, (int32_t)row0, unit * kGroups, bar);
    };
    {
        const int r = threadIdx.x & 127, row = half * 128 + r;   // lane of tensor memory, row of the tile
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;       // the warp's first lane, in bits 16 and up
        const uint32_t ta = tmem + team * kACols, td = tmem + kTeams * kACols + team * kCols;
        const bool issuer = r == 0;
        const int swz = r >> 1 & 3;
        uint32_t round = 0;
        const int blocks = (mine - pair + kPairs - 1) / kPairs;
        int issued = 0;
        const bool fetcher = half == 0 && r == 96;               // of a warp that waits at the team's barrier
        if (fetcher)
            for (; issued < kDepth && issued < blocks; ++issued) issue(issued);
        // After a wait that gave up the blocks go on without waits: the team's threads meet
        // at its barriers for every block.
        for (int k = 0; k < blocks; ++k) {
            uint8_t* from = ring + k % kDepth * St::kPitch;
            if ((warp & 3) == 0) tc::mbar_wait(&full[pair][k % kDepth], k / kDepth & 1, abort, &g_err_q4_wide, 1u);
            tc::named_bar_sync(1 + team, kTeamThreads);
            uint4 w[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) w[t] = *reinterpret_cast<const uint4*>(from + row * 64 + ((t ^ swz) << 4));
            float s[kGroups];
#pragma unroll
            for (int g = 0; g < kGroups; ++g) s[g] = el::to_f32(reinterpret_cast<const S*>(from + St::kScales)[g * kRows + row]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {                        // columns 32 j ... 32 j + 31
                const uint32_t z = ZEROS ? from[St::kZeros + j * 32 / GROUP * kRows + row] : 8u;
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
            for (int g = 0; g < kGroups; ++g) {
                tc::tc_fence_before();
                tc::named_bar_sync(1 + team, kTeamThreads);
                if (issuer) {
                    tc::tc_fence_after();
                    const uint64_t x[2] = {tc::desc_sw128(tc::smem_u32(from + St::kX)),
                                           tc::desc_sw128(tc::smem_u32(from + St::kX + St::kXBox))};
#pragma unroll
                    for (int i = 0; i < GROUP / 16; ++i) {
                        const int kk = g * (GROUP / 16) + i;      // step of 16 columns
                        mma_ts(td, ta + 8 * kk, x[kk >> 2] + 2 * (kk & 3), idesc, i != 0);
                    }
                    tc::mma_commit(&done[team]);
                    if (g + 1 == kGroups) tc::mma_commit(&empty[pair][k % kDepth]);
                }
                if ((warp & 3) == 0) tc::mbar_wait(&done[team], round & 1, abort, &g_err_q4_wide, 2u);
                // The stage of the block before is free where both teams' products are done
                // (their codes are in tensor memory).
                if (fetcher && g == 0 && k > 0 && issued < blocks && !*abort) {
                    tc::mbar_wait(&empty[pair][(k - 1) % kDepth], (k - 1) / kDepth & 1, abort, &g_err_q4_wide, 4u);
                    if (!*abort) issue(issued++);
                }
                __syncwarp();
                tc::named_bar_sync(1 + team, kTeamThreads);
                ++round;
                __syncwarp();
                tc::tc_fence_after();
#pragma unroll
                for (int c = 0; c < kCols; c += 32) {
                    uint32_t v[32];
                    tc::tmem_ld32(td + lanes + c, v);
                    tc::tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 32; ++i) acc[c + i] = fmaf(s[g], __uint_as_float(v[i]), acc[c + i]);
                }
            }
        }
        if (*abort && (issuer || fetcher)) {
            // the products and copies in flight end before the block does
            volatile int no_abort = 0;
            if (issuer && round) tc::mbar_wait(&done[team], (round - 1) & 1, &no_abort, &g_err_q4_wide, 2u, 100000000ull);
            for (int u = issued > kDepth ? issued - kDepth : 0; u < issued; ++u)
                tc::mbar_wait(&full[pair][u % kDepth], u / kDepth & 1, &no_abort, &g_err_q4_wide, 1u, 100000000ull);
        }
    }
    tc::tc_fence_before();
    __syncthreads();                                             // the ring is free
    tc::tc_fence_after();
    __syncwarp();
    if (warp == 0) tc::tmem_dealloc(tmem, kTmem);
    // sums[pair][column][row]
    float(*sums)[kCols][kRows + 4] = reinterpret_cast<float(*)[kCols][kRows + 4]>(base);
#pragma unroll
    for (int c = 0; c < kCols; ++c) sums[pair][c][threadIdx.x & (kRows - 1)] = acc[c];
    if (a.split > 1) cl::sync();
    else __syncthreads();
    const int used = min(a.cols - col0, used_cols(kCols, PARTS)) / PARTS;       // vectors of this tile
    finish_tile<OP, PARTS, kPairs>(a, &sums[0][0][0], kCols * (kRows + 4), kRows + 4, kRows, row0, col0, used, rank, kThreads);
    if (a.split > 1) cl::sync();                                 // the sums stay until they are read
}

template <typename OP, typename S, int PARTS, int GROUP, bool ZEROS>
lrc_status wide_as(ApplyArgs a, cudaStream_t s) {
    using St = WideStage<S, GROUP, ZEROS>;
    constexpr int kUsed = used_cols(kCols, PARTS);
    a.xrows = a.cols < kUsed ? a.cols : kUsed;
    const int chunks = (a.cols + kUsed - 1) / kUsed;
    const int64_t tiles = (a.m + kRows - 1) / kRows;
    // Blocks of a cluster: the number that fills the multiprocessors' waves best, a
    // wave's start and end taken as 14 blocks of columns.  (Clusters of eight blocks
    // that fill a multiprocessor each do not all find room at once: 4096 x 4096 with 64
    // vectors took 23 us with them.)
    double best = 1e300;
    const int sms = sm_count();
    for (int split = 1; split <= 4 && split <= a.blocks; ++split) {
        const double cost = ceil((double)tiles * chunks * split / sms) * ((double)((a.blocks + split - 1) / split) + 14.);
        if (cost < best) {
            best = cost;
            a.split = split;
        }
    }
    CUtensorMap qm, xm, sm, zm{};
    lrc_status st = encode_map_2d_sw64(&qm, CU_TENSOR_MAP_DATA_TYPE_UINT8, a.Q, a.blocks * 64, a.m, a.blocks * 64, 64, kRows,
                                       "Q");
    if (st != LRC_OK) return st;
    st = encode_map_2d(&xm, map_type(typename OP::type()), a.x, a.xcols, a.cols, a.ldx * 2, 64, (uint32_t)a.xrows, true,
                       "X");
    if (st != LRC_OK) return st;
    st = encode_map_2d(&sm, map_type(S()), a.scales, a.m, a.groups, a.ldm * (int64_t)sizeof(S), kRows, St::kGroups, false,
                       "scales");
    if (st != LRC_OK) return st;
    if (ZEROS) {
        st = encode_map_2d(&zm, CU_TENSOR_MAP_DATA_TYPE_UINT8, a.zeros, a.m, a.groups, a.ldm, kRows, St::kGroups, false,
                           "zeros");
        if (st != LRC_OK) return st;
    }
    auto kernel = q4_wide_kernel<OP, S, PARTS, GROUP, ZEROS>;
    constexpr int kSmem = kPairs * St::kDepth * St::kPitch + 1024;
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
    const uint32_t idesc = tc::idesc_f16_f32(128, kCols) | (OP::kBf16 ? tc::kIdescBF16 : 0u);
    e = cudaLaunchKernelEx(&cfg, kernel, qm, xm, sm, zm, a, idesc);
    if (e != cudaSuccess) return cuda_fail(e, "q4_wide_kernel");
    return after_launch("q4_wide_kernel");
}

}  // namespace

namespace q4 {

template <typename OP, typename S, int PARTS>
lrc_status launch_wide(ApplyArgs a, int group, cudaStream_t s) {
    if (a.zeros) {
        if (group == 32) return wide_as<OP, S, PARTS, 32, true>(a, s);
        if (group == 64) return wide_as<OP, S, PARTS, 64, true>(a, s);
        return wide_as<OP, S, PARTS, 128, true>(a, s);
    }
    if (group == 32) return wide_as<OP, S, PARTS, 32, false>(a, s);
    if (group == 64) return wide_as<OP, S, PARTS, 64, false>(a, s);
    return wide_as<OP, S, PARTS, 128, false>(a, s);
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
