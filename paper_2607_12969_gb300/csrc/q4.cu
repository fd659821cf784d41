// q4.cu -- the product of a matrix of 4-bit codes with vectors (lrc_q4_apply): the
// kernel for up to 32 columns of them, and the choice.
//
// What[i][c] = s (q - z).  The codes' layout is the one include/lrc.h states:
// 64-byte blocks of 128 columns, column 32 j + 8 t + e in word 4 t + j.
#include <math.h>

#include <atomic>

#include "q4.cuh"

namespace lrc {
namespace {

using namespace q4;

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
// A block has R groups of 16 rows and two warps for each, which take alternate
// pairs of blocks of columns.  One more warp brings codes, x, scales and zero
// codes of 512 columns at a time by TMA into a ring of stages that all warps
// read, so that x passes the L2 port once a block and not once a warp.  The
// blocks of a cluster share the columns of a tile; their sums are added in the
// order of their ranks through distributed shared memory.
//
// What bounds it: 16384 x 16384 and one bfloat16 vector take 28 us, 4.9 TB/s of 6.8,
// with no unit full: the unpacking, 11 (binary16 9) instructions for eight codes, 7 (5)
// of them on the pipe of half rate, is 55 % of that pipe's time, HBM 57 %; what is
// missing is overlap of the two, with one block a multiprocessor.  With more vectors
// every warp reads the block's x for its own 16 rows: 16384 x 8192 and 32 binary16
// vectors 30 us, 12287 x 16381 and 7 binary32 ones (21 columns) 40.  A ring for each warp 39 us; loads to registers, whose x of L1
// come in order behind the codes of memory, slower still; one run of stages for each
// resident block, joined by counters, 34.

__device__ unsigned int g_err_q4;

// Shared memory of a stage of 512 columns for 16 R rows: two boxes of 128 bytes of
// codes a row, eight boxes of 64 columns of x (kCols rows of 128 bytes), all with
// the 128-byte swizzle; scales and zero codes of the groups, 16 R values a group.
template <typename S, int GROUP, bool ZEROS, int NT>
struct StageOf {
    static constexpr int kCols = 8 * NT, kGroups = 512 / GROUP, kXBox = kCols * 128;
    int codes, scales, zeros, scale_bytes, pitch;
    __host__ __device__ explicit StageOf(int R)
        : codes(R * 2048), scales(2 * codes + 8 * kXBox), zeros(0), scale_bytes(kGroups * 16 * R * (int)sizeof(S)), pitch(0) {
        zeros = scales + (scale_bytes + 127) / 128 * 128;                          // TMA boxes start at 128 bytes
        pitch = (zeros + (ZEROS ? kGroups * 16 * R : 0) + 1023) / 1024 * 1024;
    }
    __host__ __device__ int bytes(int R, int xrows) const {                        // what the copies bring
        return 2 * codes + xrows * 1024 + scale_bytes + (ZEROS ? kGroups * 16 * R : 0);
    }
};

// Groups of 16 rows of a tile at most: 15 warps of a block have 128 registers a
// thread, 17 would have 96.
constexpr int kMostRows = 7;
constexpr int kMostDepth = 8;      // stages of a ring

// OP: the instructions' element type; S: the scales' type; PARTS: columns of B
// that make one vector (3: a binary32 vector's parts in bfloat16).
template <typename OP, typename S, int PARTS, int GROUP, bool ZEROS, int NT>
__global__ void __launch_bounds__(64 * kMostRows + 32, 1)
q4_apply_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap xmap,
                const __grid_constant__ CUtensorMap smap, const __grid_constant__ CUtensorMap zmap,
                const __grid_constant__ ApplyArgs a) {
    using St = StageOf<S, GROUP, ZEROS, NT>;
    const St lay(a.R);
    constexpr int kCols = St::kCols;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t full[kMostDepth], empty[kMostDepth];
    __shared__ int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = 2 * a.R, threads = 64 * a.R + 32;
    const int rows = 16 * a.R, rank = blockIdx.x % a.split;
    const int64_t row0 = (int64_t)(blockIdx.x / a.split) * rows;
    const int stages = (int)((a.blocks + 3) / 4);
    const int mine = (stages - rank + a.split - 1) / a.split;         // stages of this block
    uint8_t* ring = raw + ((1024u - (tc::smem_u32(raw) & 1023u)) & 1023u);
    volatile int* abort = &abort_flag;
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int d = 0; d < a.depth; ++d) {
            tc::mbar_init(&full[d], 1);
            tc::mbar_init(&empty[d], warps);
        }
        tc::fence_barrier_init();
    }
    __syncthreads();
    tc::pdl_wait();
    tc::pdl_trigger();

    if (warp == warps) {
        if (lane == 0) {
            const uint32_t bytes = lay.bytes(a.R, a.xrows);
            int k = 0, slot = 0;
            uint32_t phase = 1;
            for (; k < mine; ++k) {
                if (k >= a.depth && !tc::mbar_wait(&empty[slot], phase, abort, &g_err_q4, 1u)) break;
                uint64_t* bar = &full[slot];
                uint8_t* to = ring + slot * lay.pitch;
                const int unit = rank + k * a.split;
                tc::mbar_arrive_expect_tx(bar, bytes);
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    tc::tma_load_2d(to + q * lay.codes, &qmap, unit * 256 + q * 128, (int32_t)row0, bar);
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    tc::tma_load_2d(to + 2 * lay.codes + q * St::kXBox, &xmap, unit * 512 + q * 64, 0, bar);
                tc::tma_load_2d(to + lay.scales, &smap, (int32_t)row0, unit * St::kGroups, bar);
                if (ZEROS) tc::tma_load_2d(to + lay.zeros, &zmap, (int32_t)row0, unit * St::kGroups, bar);
                if (++slot == a.depth) {
                    slot = 0;
                    phase ^= 1;
                }
            }
            // no copy is in flight when the block goes on
            volatile int no_abort = 0;
            for (int u = k > a.depth ? k - a.depth : 0; u < k; ++u)
                tc::mbar_wait(&full[u % a.depth], u / a.depth & 1, &no_abort, &g_err_q4, 1u);
        }
        __syncwarp();
    }
    float acc[NT][4] = {};
    const int g = lane >> 2, t = lane & 3, half = warp & 1;
    // Row of eight (and column of eight) that the lanes of g take: neighbouring g
    // in opposite halves of a swizzled row, so that 16-byte loads meet no bank
    // conflict.
    const int rho = g >> 1 | (g & 1) << 2;
    const int row = 16 * (warp >> 1) + rho;           // and row + 8
    if (warp < warps) {
        const int swz[2] = {(t ^ rho) << 4, ((4 | t) ^ rho) << 4};
        // Columns beyond the last read the last again (a broadcast) where one tile
        // of eight holds them all; else whatever is there: their sums are not used.
        const int xrow = NT == 1 ? min(rho, a.xrows - 1) : rho;
        const int xat[2] = {xrow * 128 + ((t ^ xrow) << 4), xrow * 128 + (((4 | t) ^ xrow) << 4)};
        const uint8_t* codes = ring + half * lay.codes + row * 128;
        const uint8_t* xs = ring + 2 * lay.codes + half * 4 * St::kXBox;
        const uint8_t* scales = ring + lay.scales + (half * St::kGroups / 2 * rows + row) * (int)sizeof(S);
        const uint8_t* zeros = ring + lay.zeros + half * St::kGroups / 2 * rows + row;
        int slot = 0, off = 0;
        uint32_t phase = 0;
        for (int k = 0; k < mine; ++k) {
            if (!tc::mbar_wait(&full[slot], phase, abort, &g_err_q4, 1u)) break;
            // two blocks of 128 columns (those beyond the last have x, codes and
            // scales of zero)
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                uint4 w[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) w[h] = *reinterpret_cast<const uint4*>(codes + off + h * 1024 + swz[blk]);
                float part[NT][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint4 xv[NT];
#pragma unroll
                    for (int c = 0; c < NT; ++c)
                        xv[c] = *reinterpret_cast<const uint4*>(xs + off + (2 * blk + (j >> 1)) * St::kXBox + c * 1024 +
                                                                xat[j & 1]);
                    constexpr int kSteps = GROUP / 32;           // steps of a group
                    const int group = (4 * blk + j) / kSteps;
                    uint32_t r[2][4];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t word = j == 0 ? w[h].x : j == 1 ? w[h].y : j == 2 ? w[h].z : w[h].w;
                        OP::unpack(word, ZEROS ? zeros[off + group * rows + 8 * h] : 8u, r[h]);
                    }
#pragma unroll
                    for (int c = 0; c < NT; ++c) {
                        if (j % kSteps == 0) OP::mma_first(part[c], r[0][0], r[1][0], r[0][1], r[1][1], xv[c].x, xv[c].y);
                        else OP::mma(part[c], r[0][0], r[1][0], r[0][1], r[1][1], xv[c].x, xv[c].y);
                        OP::mma(part[c], r[0][2], r[1][2], r[0][3], r[1][3], xv[c].z, xv[c].w);
                    }
                    if ((j + 1) % kSteps == 0) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float s = el::to_f32(
                                *reinterpret_cast<const S*>(scales + off + (group * rows + 8 * h) * (int)sizeof(S)));
#pragma unroll
                            for (int c = 0; c < NT; ++c) {
                                acc[c][2 * h] = fmaf(s, part[c][2 * h], acc[c][2 * h]);
                                acc[c][2 * h + 1] = fmaf(s, part[c][2 * h + 1], acc[c][2 * h + 1]);
                            }
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&empty[slot]);
            off += lay.pitch;
            if (++slot == a.depth) {
                slot = off = 0;
                phase ^= 1;
            }
        }
    }
    __syncthreads();                                              // the ring is free
    // sums[half][column][row]
    float* sums = reinterpret_cast<float*>(ring);
    const int pitch = rows + 4;
    if (warp < warps) {
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int u = 0; u < 4; ++u)      // column 2 t + u of eight, t or t + 4 of the vectors
                sums[(half * kCols + 8 * c + t + 4 * (u & 1)) * pitch + row + 8 * (u >> 1)] = acc[c][u];
    }
    if (a.split > 1) cl::sync();
    else __syncthreads();
    finish_tile<OP, PARTS, 2>(a, sums, kCols * pitch, pitch, rows, row0, 0, a.cols / PARTS, rank, threads);
    if (a.split > 1) cl::sync();                              // the sums stay until they are read
}

// binary32 vectors as three bfloat16 parts, x = hi + 2^-8 mid + 2^-16 lo (each cut
// off, not rounded, so that none overflows): rows 3 v, 3 v + 1, 3 v + 2 of `blocks`
// whole blocks of columns, zeros from n on.  The powers of two bring each part to hi's
// size: what is left of x has 8 bits fewer each time and every binary32 number is a
// multiple of 2^-149, so the parts are multiples of 2^-133, bfloat16's smallest number,
// and hold all of x however small it is.  (Not brought up, the last bits of entries
// below 2^-110 were lost, 1e-4 of one of 2^-120.)  finish_tile takes the powers off the
// sums.  An infinity or NaN is in the first part alone.
__global__ void __launch_bounds__(256)
q4_parts_kernel(const float* __restrict__ x, int64_t n, int64_t ldn, int64_t ldp, uint16_t* __restrict__ parts) {
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    tc::pdl_wait();
    tc::pdl_trigger();
    if (c >= ldp) return;
    const float v = c < n ? x[(int64_t)blockIdx.y * ldn + c] : 0.f;
    const uint32_t hi = __float_as_uint(v) & 0xffff0000u;
    const bool odd = !(fabsf(v) <= 3.402823466e38f);
    const float rest = odd ? 0.f : (v - __uint_as_float(hi)) * kPartUp;
    const uint32_t mid = __float_as_uint(rest) & 0xffff0000u;
    const float last = (rest - __uint_as_float(mid)) * kPartUp;
    uint16_t* p = parts + (int64_t)blockIdx.y * 3 * ldp + c;
    p[0] = odd && v != v ? 0x7fffu : (uint16_t)(hi >> 16);
    p[ldp] = (uint16_t)(mid >> 16);
    p[2 * ldp] = (uint16_t)(__float_as_uint(last) >> 16);
}

// Groups of rows of a tile and blocks of a cluster: what takes the shortest by a
// model of a multiprocessor's time, in units of what it takes for 16 rows and a
// stage (0.11 us).  A block needs five such a stage at least however few its rows
// are (the latency of its warps' chain), and sixteen to start and to end.  It takes the
// multiprocessors as one pool, although a cluster needs room in one part of them, and
// counts two blocks of four groups of rows on each, although instances of more than 112
// registers (three tiles of columns in part, four) have room for one there: 2254 x 3764
// and 29 binary16 vectors take 16.6 us, with one counted 7.7, but 4446 x 13988 and 7
// binary32 ones 25 and 32.
inline void choose_tile(ApplyArgs* a) {
    const int stages = (int)((a->blocks + 3) / 4), sms = sm_count();
    double best = 1e300;
    for (int R = kMostRows; R >= 1; --R) {
        const int64_t tiles = ((a->m + 15) / 16 + R - 1) / R;
        const int slots = (R > 4 ? 1 : 2) * sms;
        for (int split = 1; split <= 8 && split <= stages; split += split < 4 ? 1 : 2) {
            const double blocks = (double)tiles * split;
            const double waves = ceil(blocks / slots), beside = blocks < slots ? ceil(blocks / sms) : slots / sms;
            const double cost = waves * (fmax(beside * R, 5.) * ((stages + split - 1) / split) + 16.);
            if (cost < best) {
                best = cost;
                a->R = R;
                a->split = split;
            }
        }
    }
}

template <typename OP, typename S, int PARTS, int GROUP, bool ZEROS, int NT>
lrc_status apply_launch(ApplyArgs a, cudaStream_t s) {
    using St = StageOf<S, GROUP, ZEROS, NT>;
    a.xrows = a.cols;
    choose_tile(&a);
    const uint32_t rows = 16 * a.R;
    const St lay(a.R);
    const int room = kSmemOfSm / (a.R > 4 ? 1 : 2) - 3072;
    a.depth = room / lay.pitch < kMostDepth ? room / lay.pitch : kMostDepth;
    CUtensorMap qm, xm, sm, zm{};
    lrc_status st = encode_map_2d(&qm, CU_TENSOR_MAP_DATA_TYPE_UINT8, a.Q, a.blocks * 64, a.m, a.blocks * 64, 128, rows,
                                  true, "Q");
    if (st != LRC_OK) return st;
    st = encode_map_2d(&xm, map_type(typename OP::type()), a.x, a.xcols, a.cols, a.ldx * 2, 64, (uint32_t)a.xrows, true,
                       "X");
    if (st != LRC_OK) return st;
    st = encode_map_2d(&sm, map_type(S()), a.scales, a.m, a.groups, a.ldm * (int64_t)sizeof(S), rows, St::kGroups, false,
                       "scales");
    if (st != LRC_OK) return st;
    if (ZEROS) {
        st = encode_map_2d(&zm, CU_TENSOR_MAP_DATA_TYPE_UINT8, a.zeros, a.m, a.groups, a.ldm, rows, St::kGroups, false,
                           "zeros");
        if (st != LRC_OK) return st;
    }
    unsigned grid;
    if ((st = grid_of((a.m + rows - 1) / rows * a.split, 1, "lrc_q4_apply", &grid)) != LRC_OK) return st;
    auto kernel = q4_apply_kernel<OP, S, PARTS, GROUP, ZEROS, NT>;
    const int smem = a.depth * lay.pitch + 1024;
    // the attribute is the device's: set once on each
    static std::atomic<uint64_t> set_on{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && (dev >= 64 || !(set_on.load() >> dev & 1))) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemOfSm - 1024);
        if (e == cudaSuccess && dev < 64) set_on |= (uint64_t)1 << dev;
    }
    if (e != cudaSuccess) return cuda_fail(e, "q4_apply_kernel");
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(64 * a.R + 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)a.split;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.split > 1 ? 2 : 1;
    e = cudaLaunchKernelEx(&cfg, kernel, qm, xm, sm, zm, a);
    if (e != cudaSuccess) return cuda_fail(e, "q4_apply_kernel");
    return after_launch("q4_apply_kernel");
}

template <typename OP, typename S, int PARTS, int NT>
lrc_status apply_groups(const ApplyArgs& a, int group, cudaStream_t s) {
    if (a.zeros) {
        if (group == 32) return apply_launch<OP, S, PARTS, 32, true, NT>(a, s);
        if (group == 64) return apply_launch<OP, S, PARTS, 64, true, NT>(a, s);
        return apply_launch<OP, S, PARTS, 128, true, NT>(a, s);
    }
    if (group == 32) return apply_launch<OP, S, PARTS, 32, false, NT>(a, s);
    if (group == 64) return apply_launch<OP, S, PARTS, 64, false, NT>(a, s);
    return apply_launch<OP, S, PARTS, 128, false, NT>(a, s);
}

// As many tiles of eight columns as the vectors need.
template <typename OP, typename S, int PARTS>
lrc_status apply_tiles(const ApplyArgs& a, int group, cudaStream_t s) {
    if (a.cols <= 8) return apply_groups<OP, S, PARTS, 1>(a, group, s);
    if (a.cols <= 16) return apply_groups<OP, S, PARTS, 2>(a, group, s);
    if (a.cols <= 24) return apply_groups<OP, S, PARTS, 3>(a, group, s);
    return apply_groups<OP, S, PARTS, 4>(a, group, s);
}

// Columns up to which the product is mma.sync's.  Either way one pass over the codes;
// this one's warps hand nothing on, so it starts sooner: 1000 x 4000 and 30 bfloat16
// vectors 7.0 us here, 11.4 on tcgen05; 12287 x 16381 and 10 binary32 vectors (30
// columns) 49 and 91; 16384 x 8192 and 32 binary16 vectors 30.1 and 30.4, 4096 x 4096
// 14.9 and 11.4.  Above, this one would pass over the codes again: 48 vectors 52 us
// here, 32 there.
constexpr int kFew = 32;

template <typename OP, typename S, typename Y, int PARTS>
lrc_status apply_as(const void* Q, const void* scales, const uint8_t* zeros, const void* x, const void* A, void* y,
                    int64_t m, int64_t n, int64_t b, int group, cudaStream_t s) {
    ApplyArgs a{};
    a.Q = (const uint4*)Q;
    a.scales = scales;
    a.zeros = zeros;
    a.m = m;
    a.blocks = (n + 127) / 128;
    a.ldm = lrc_packed_ld(m);
    a.groups = (n + group - 1) / group;
    a.wide = sizeof(Y) == 4;
    const int64_t ldn = lrc_packed_ld(n);
    // vectors a launch: 16384, of binary32 ones as many as have parts of 256 MB
    int64_t most = 16384;
    if (PARTS > 1 && most > (int64_t)(256 << 20) / (a.blocks * 768)) most = (int64_t)(256 << 20) / (a.blocks * 768);
    if (most < 1) most = 1;
    for (int64_t b0 = 0; b0 < b; b0 += most) {
        const int64_t nb = b - b0 < most ? b - b0 : most;
        a.A = A ? (const Y*)A + b0 * m : nullptr;
        a.y = (Y*)y + b0 * m;
        a.cols = (int)nb * PARTS;
        if (PARTS == 1) {
            a.x = (const uint16_t*)x + b0 * ldn;
            a.ldx = ldn;
            a.xcols = n;
        } else {
            a.ldx = a.xcols = a.blocks * 128;
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
        const lrc_status st = a.cols > kFew ? q4::launch_wide<OP, S, PARTS>(a, group, s) : apply_tiles<OP, S, PARTS>(a, group, s);
        if (st != LRC_OK) return st;
    }
    return LRC_OK;
}

}  // namespace

lrc_status launch_q4_apply(const void* Q, const void* scales, const uint8_t* zeros, const void* X, const void* A, void* Y,
                           int64_t m, int64_t n, int64_t b, int group, lrc_fmt fmt, cudaStream_t s) {
    if (fmt == LRC_F32) return apply_as<Bf2, float, float, 3>(Q, scales, zeros, X, A, Y, m, n, b, group, s);
    if (fmt == LRC_BF16) return apply_as<Bf2, bf16, bf16, 1>(Q, scales, zeros, X, A, Y, m, n, b, group, s);
    if (fmt == LRC_F16) return apply_as<Half2, __half, float, 1>(Q, scales, zeros, X, A, Y, m, n, b, group, s);
    return apply_as<Half2, __half, __half, 1>(Q, scales, zeros, X, A, Y, m, n, b, group, s);
}

uint32_t take_q4_error() {
    unsigned int v = 0;
    if (cudaMemcpyFromSymbol(&v, g_err_q4, sizeof v) != cudaSuccess) return 0xffffffffu;
    if (v) {
        const unsigned int z = 0;
        cudaMemcpyToSymbol(g_err_q4, &z, sizeof z);
    }
    return v;
}

}  // namespace lrc
