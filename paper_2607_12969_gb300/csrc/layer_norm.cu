// layer_norm.cu -- layer norm of rows and its gradient (lrc_layer_norm,
// lrc_layer_norm_grad), binary32 arithmetic.
//
//   y = (x - mu) r gamma + beta
//   dx = r (d - mean(d) - xh mean(d xh)),  d = dy gamma,  xh = (x - mu) r
//   dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy
//
// Up to 32768 columns (the gradient 65536) a row is read once and held on chip
// between its sums and its result, in registers, where rows are many first in shared
// memory; longer rows are read three times.  HBM is the floor; what keeps each kernel
// from it stands at the kernel.
#include <type_traits>

#include "cluster.cuh"
#include "common.cuh"
#include "elem.cuh"
#include "tc.cuh"

namespace lrc {
namespace {

using bf16 = __nv_bfloat16;

__device__ unsigned int g_err_norm;

// ---- elements of a row -------------------------------------------------------

// Eight elements from an address on a 16-byte boundary (32 for binary32: two loads).
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void load8(const __half* p, float (&v)[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        v[2 * i] = f.x, v[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ void load8(const bf16* p, float (&v)[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(__half* p, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(tc::pack_half2(v[0], v[1]), tc::pack_half2(v[2], v[3]),
                                              tc::pack_half2(v[4], v[5]), tc::pack_half2(v[6], v[7]));
}
__device__ __forceinline__ void store8(bf16* p, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(tc::pack_bf162(v[0], v[1]), tc::pack_bf162(v[2], v[3]),
                                              tc::pack_bf162(v[4], v[5]), tc::pack_bf162(v[6], v[7]));
}

using el::f2;
using el::pair;
using el::split;
using el::add2;
using el::mul2;
using el::fma2;
__device__ __forceinline__ float both_of(f2 a) {
    float x, y;
    split(a, x, y);
    return x + y;
}

// Eight values of a thread: columns c ... c + 7 where VEC, else c, c + step, ...
// (a warp's elements side by side: rows that start anywhere); `none` beyond cols.
template <bool VEC, typename T>
__device__ __forceinline__ void load_row(const T* row, int c, int step, int cols, float none, float (&v)[8]) {
    if (VEC && c + 8 <= cols) {
        load8(row + c, v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = VEC ? c + e : c + e * step;
            v[e] = i < cols ? el::to_f32(row[i]) : none;
        }
    }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store_row(T* row, int c, int step, int cols, const float (&v)[8]) {
    if (VEC && c + 8 <= cols) {
        store8(row + c, v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = VEC ? c + e : c + e * step;
            if (i < cols) row[i] = el::from_f32<T>(v[e]);
        }
    }
}
// The same of gamma or beta, whose type is known at run time.
template <bool VEC>
__device__ __forceinline__ void load_param(const void* p, int kind, int c, int step, int cols, float none,
                                           float (&v)[8]) {
    if (!p) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = none;
    } else if (kind == 0) {
        load_row<VEC>(static_cast<const float*>(p), c, step, cols, none, v);
    } else if (kind == 1) {
        load_row<VEC>(static_cast<const __half*>(p), c, step, cols, none, v);
    } else {
        load_row<VEC>(static_cast<const bf16*>(p), c, step, cols, none, v);
    }
}

// Sum over the block's threads (a whole number of warps), in every thread; sh: a
// float a warp, used again only after another barrier.
__device__ __forceinline__ float block_sum(float x, float* sh) {
    x = el::warp_sum(x);
    if (blockDim.x == 32) return x;
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
    __syncthreads();
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    return el::warp_sum(lane < warps ? sh[lane] : 0.f);
}

// ---- forward -----------------------------------------------------------------

struct NormArgs {
    const void* x;
    const void* gamma;
    const void* beta;
    void* y;
    float* mean;
    float* rstd;
    int64_t rows, cols, ldx, ldy;
    float eps;
    int pk;                  // type of gamma and beta
};

// A thread's eight elements as they came: 16-bit ones stay packed between the
// row's sums and its result (fewer registers, more rows on a multiprocessor).
template <typename T>
struct Held {
    uint32_t w[4];
    __device__ void set(const float (&v)[8]);
};
template <> __device__ __forceinline__ void Held<__half>::set(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = tc::pack_half2(v[2 * i], v[2 * i + 1]);
}
template <> __device__ __forceinline__ void Held<bf16>::set(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = tc::pack_bf162(v[2 * i], v[2 * i + 1]);
}
template <>
struct Held<float> {
    float v[8];
    __device__ __forceinline__ void set(const float (&u)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = u[e];
    }
};
__device__ __forceinline__ void get(const Held<float>& h, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = h.v[e];
}
template <typename T> __device__ __forceinline__ void get(const Held<T>& h, float (&v)[8]) {
    load8(reinterpret_cast<const T*>(h.w), v);
}

// One row for each blockDim.x threads (blockDim.y rows a block, more than one where
// a warp takes a row), VPT groups of eight elements a thread.  One barrier: with
// m_i the mean and q_i the sum of squares about it of the n_i elements of a part,
// the whole has q = sum_i (q_i + n_i (m_i - m)^2), first over the lanes of a warp,
// then over the warps.  A few hundred rows wait for the call (64 x 8192 of binary16 7
// us).  Six blocks of 256 threads and 16-bit rows on a multiprocessor: rows that start
// anywhere spill 48 to 80 bytes a thread for it, 400 x 4097 9.9 us against 11.1 with
// four blocks, but 8191 x 511 13.7 and 13.1, 500 x 7001 19.5 and 13.4.
template <typename X, typename Y, bool VEC, int VPT, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS > 256 ? 1 : sizeof(X) == 2 ? 6 : 4) norm_kernel(const NormArgs a) {
    __shared__ float sh[2][32];
    const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    tc::pdl_wait();
    tc::pdl_trigger();
    if (row >= a.rows) return;               // whole warps: blockDim.x = 32 where blockDim.y > 1
    const X* x = static_cast<const X*>(a.x) + row * a.ldx;
    const int T = blockDim.x, cols = (int)a.cols, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto column = [&](int k) { return VEC ? (k * T + (int)threadIdx.x) * 8 : k * T * 8 + (int)threadIdx.x; };
    const int step = VEC ? 1 : T;
    Held<X> held[VPT];
    float s = 0.f, count = 0.f;
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        float v[8];
        load_row<VEC>(x, column(k), T, cols, 0.f, v);
        held[k].set(v);
    }
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        float v[8];
        get(held[k], v);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += v[e];
        const int left = (cols - column(k) + step - 1) / step;
        count += (float)(left < 0 ? 0 : left > 8 ? 8 : left);
    }
    const float n = el::warp_sum(count);
    s = el::warp_sum(s);
    const float m = n > 0.f ? s / n : 0.f;   // of the warp's elements
    float q = 0.f;
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        float v[8];
        get(held[k], v);
        const int c = column(k);
        if (c + 7 * step < cols) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] -= m;
                q = fmaf(v[e], v[e], q);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = c + e * step < cols ? v[e] - m : 0.f;
                q = fmaf(v[e], v[e], q);
            }
        }
    }
    q = el::warp_sum(q);
    float mu = m;
    if (T > 32) {
        // (a warp's number of elements is known to the others by its place)
        if (lane == 0) sh[0][warp] = s, sh[1][warp] = q;
        __syncthreads();
        const int warps = T >> 5;
        const float sw = lane < warps ? sh[0][lane] : 0.f, qw = lane < warps ? sh[1][lane] : 0.f;
        float nw = 0.f;
        if (lane < warps) {
            if (VEC) {
                for (int k = 0; k < VPT; ++k) nw += (float)min(max(cols - (k * T + lane * 32) * 8, 0), 256);
            } else {
                for (int k = 0; k < VPT * 8; ++k) nw += (float)min(max(cols - k * T - lane * 32, 0), 32);
            }
        }
        mu = el::warp_sum(sw) / (float)a.cols;
        const float d = nw > 0.f ? sw / nw - mu : 0.f;
        q = el::warp_sum(fmaf(nw * d, d, qw));
    }
    const float r = 1.f / sqrtf(q / (float)a.cols + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[row] = mu;
        if (a.rstd) a.rstd[row] = r;
    }
    Y* y = static_cast<Y*>(a.y) + row * a.ldy;
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int c = column(k);
        float v[8], w[8];
        get(held[k], v);
        load_param<VEC>(a.gamma, a.pk, c, T, cols, 1.f, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (v[e] - mu) * r * w[e];
        load_param<VEC>(a.beta, a.pk, c, T, cols, 0.f, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += w[e];
        store_row<VEC>(y, c, T, cols, v);
    }
}

// Where the rows of a tensor start within 16 bytes: their copies keep it, so that
// whole 16 bytes of a row go by one bulk copy and its first and last elements by
// plain loads.  Nothing beside the row is read.
template <typename T>
struct Span {
    uint32_t head, body, mis;                // elements before and within the bulk copy; bytes past a boundary
    __device__ Span(const T* row, int64_t cols) {
        constexpr uint32_t kPer = 16 / sizeof(T);
        mis = (uint32_t)(reinterpret_cast<uintptr_t>(row) & 15u);
        head = min((uint32_t)cols, ((16u - mis) & 15u) / (uint32_t)sizeof(T));
        body = ((uint32_t)cols - head) / kPer * kPer;
    }
};

constexpr int kMostRing = 8;                 // rows of a ring
constexpr int kRing = 225 * 1024;            // bytes of the rings of a multiprocessor
constexpr int kStreamThreads = 1024;         // of a block, at most
constexpr int kMostTeams = 15;               // of a block: a named barrier each

// s / n with `inv` next to 1 / n (0 for no elements): the product, and its remainder's.
__device__ __forceinline__ float quotient(float s, float n, float inv) {
    const float near = s * inv;
    return isinf(near) ? near : fmaf(fmaf(-near, n, s), inv, near);
}

// x^(-1/2): the approximation after one Newton step.
__device__ __forceinline__ float reciprocal_root(float x) {
    const float r = rsqrtf(x), s = fmaf(0.5f * r, fmaf(-x * r, r, 1.f), r);
    return x > 0.f && x < __int_as_float(0x7f800000) ? s : r;        // not for 0 and infinity
}

// Many rows: a block's teams of blockDim.x threads (blockDim.y of them) take every
// (number of teams)-th row each, in a ring in shared memory that bulk copies fill
// rows ahead; gamma and beta are there too, in binary32, for all teams.  A row is in
// registers between its sums and its result, and its place is free at its one
// barrier; the sums as in norm_kernel.  VEC: every row starts on a 16-byte boundary,
// eight columns side by side a thread; else a warp's columns are side by side, and
// the result passes through shared memory, from where its whole 16 bytes go by one
// bulk copy.  EDGES: x has elements outside the bulk copies, which the team's first
// warp loads when it asks for the copies and puts beside them a row later.
// What bounds it (8192 x 8192 of bfloat16, 55 us, 4.9 TB/s of 6.8): a quarter of the
// warp's instructions wait for shared memory, whose pipe is 60 % busy, two thirds of
// that with gamma and beta; 2.5 instructions a cycle.  Blocks that keep them apart
// in every block (two a multiprocessor) have room for fewer rows: 62 us.
template <typename X, typename Y, bool VEC, bool EDGES, int G>
__global__ void __launch_bounds__(kStreamThreads, 1)
norm_stream_kernel(const __grid_constant__ NormArgs a, const int depth) {
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ float sums[2][2][32];         // [parity][sum][warp]
    __shared__ uint64_t all_full[kMostTeams][kMostRing];
    __shared__ int abort_flag;
    const int T = blockDim.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, cols = (int)a.cols;
    const X* x = static_cast<const X*>(a.x);
    const int team = threadIdx.y, first = blockIdx.x * blockDim.y + team, teams = gridDim.x * blockDim.y;
    const int mine = first < a.rows ? (int)((a.rows - first + teams - 1) / teams) : 0;
    uint64_t* full = all_full[team];
    const uint32_t pitch = ((uint32_t)(cols * sizeof(X)) + 31) & ~15u;
    const uint32_t stage_pitch = VEC ? 0 : ((uint32_t)(cols * sizeof(Y)) + 31) & ~15u;
    volatile int* abort = &abort_flag;
    if (threadIdx.x == 0) {
        if (team == 0) abort_flag = 0;
        for (int d = 0; d < depth; ++d) tc::mbar_init(&full[d], EDGES ? 2 : 1);
        tc::fence_barrier_init();
    }
    __syncthreads();
    tc::pdl_wait();
    tc::pdl_trigger();

    float* gamma = reinterpret_cast<float*>(smem);
    float* beta = gamma + T * 8 * G;
    uint8_t* stage = reinterpret_cast<uint8_t*>(beta + T * 8 * G) + team * (depth * pitch + stage_pitch);
    uint8_t* ring = stage + stage_pitch;
    int edge_at = -1;                        // where this lane's element goes, -1 for none
    X edge = el::from_f32<X>(0.f);
    auto issue = [&](int k, int slot) {      // warp 0 (without edges, its first thread)
        const X* xr = x + (first + (int64_t)k * teams) * a.ldx;
        uint8_t* to = ring + slot * pitch;
        if (!EDGES) {
            tc::mbar_arrive_expect_tx(&full[slot], cols * (uint32_t)sizeof(X));
            tc::bulk_load(to, xr, cols * (uint32_t)sizeof(X), &full[slot]);
            return;
        }
        const Span<X> sx(xr, cols);
        if (lane == 0) {
            const uint32_t bytes = sx.body * sizeof(X);
            tc::mbar_arrive_expect_tx(&full[slot], bytes);
            if (bytes) tc::bulk_load(to + sx.mis + sx.head * sizeof(X), xr + sx.head, bytes, &full[slot]);
        }
        // lanes 0 ... 7 have the elements before the bulk copy, 8 ... 15 those after it
        const bool after = lane & 8;
        const uint32_t i = (lane & 7) + (after ? sx.head + sx.body : 0);
        edge_at = -1;
        if (lane < 16 && i < (after ? (uint32_t)cols : sx.head)) {
            edge_at = (int)(slot * pitch + sx.mis + i * sizeof(X));
            edge = xr[i];
        }
    };
    auto put_edges = [&](int slot) {         // warp 0: of the row last asked for
        if (edge_at >= 0) *reinterpret_cast<X*>(ring + edge_at) = edge;
        tc::fence_proxy_async_smem();        // a later copy may write there
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&full[slot]);
    };
    int issued = 0;
    if (EDGES ? warp == 0 : threadIdx.x == 0)
        for (; issued < depth && issued < mine; ++issued) {
            if (EDGES && issued) put_edges(issued - 1);
            issue(issued, issued);
        }
    // (VEC: the first four columns of every thread side by side, then the others; else
    // gamma and beta of a column side by side)
    for (int c = team * T + threadIdx.x; c < cols; c += T * blockDim.y) {
        const int at = VEC ? ((c / (8 * T) * 2 + (c >> 2 & 1)) * T + (c >> 3) % T) * 4 + (c & 3) : 2 * c;
        gamma[at] = a.gamma ? el::load_as(a.gamma, a.pk, c) : 1.f;
        (VEC ? beta : gamma + 1)[at] = a.beta ? el::load_as(a.beta, a.pk, c) : 0.f;
    }
    if (EDGES && warp == 0 && issued) put_edges(issued - 1);
    __syncthreads();

    const int step = VEC ? 1 : T;
    auto column = [&](int k) { return VEC ? (k * T + (int)threadIdx.x) * 8 : k * T * 8 + (int)threadIdx.x; };
    // numbers of elements of this warp and of warp `lane`
    auto elements = [&](int w) {
        int n = 0;
        if (VEC) {
            for (int k = 0; k < G; ++k) n += min(max(cols - (k * T + w * 32) * 8, 0), 256);
        } else {
            for (int k = 0; k < G * 8; ++k) n += min(max(cols - k * T - w * 32, 0), 32);
        }
        return (float)n;
    };
    const int warps = T >> 5, warp0 = team * warps;
    const float n = elements(warp), inv = n > 0.f ? 1.f / n : 0.f;
    const float inv_cols = 1.f / (float)a.cols;
    const float n_l = lane < warps ? elements(lane) : 0.f, inv_l = n_l > 0.f ? 1.f / n_l : 0.f;
    int slot = 0, p = 0, waiting = -1;       // waiting: place whose edges are not there yet
    uint32_t phase = 0;
    for (int k = 0; k < mine; ++k) {
        const int64_t row = first + (int64_t)k * teams;
        // after a wait that gave up the rows go on without copies or waits
        tc::mbar_wait(&full[slot], phase, abort, &g_err_norm, 1u);
        const X* at = reinterpret_cast<const X*>(ring + slot * pitch + (VEC ? 0 : (reinterpret_cast<uintptr_t>(x + row * a.ldx) & 15u)));
        f2 v[G][4], s2 = 0, q2 = 0;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float w[8];
            if (!VEC && column(g) + 7 * T < cols) {
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = el::to_f32(at[column(g) + e * T]);
            } else {
                load_row<VEC>(at, column(g), T, cols, 0.f, w);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[g][e] = pair(w[2 * e], w[2 * e + 1]);
                s2 = add2(s2, v[g][e]);
            }
        }
        const float s = el::warp_sum(both_of(s2)), m = quotient(s, n, inv);
        const f2 m2 = pair(-m, -m);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int c = column(g);
            if (c + 7 * step < cols) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f2 d = add2(v[g][e], m2);
                    q2 = fma2(d, d, q2);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float d0, d1;
                    split(add2(v[g][e], m2), d0, d1);
                    const f2 d = pair(c + 2 * e * step < cols ? d0 : 0.f, c + (2 * e + 1) * step < cols ? d1 : 0.f);
                    q2 = fma2(d, d, q2);
                }
            }
        }
        const float q = el::warp_sum(both_of(q2));
        if (lane == 0) sums[p][0][warp0 + warp] = s, sums[p][1][warp0 + warp] = q;
        if (!VEC && threadIdx.x == 0) tc::bulk_wait_read<0>();       // the last result has left `stage`
        tc::named_bar_sync(1 + team, T);     // every warp has the row in registers
        if (EDGES ? warp == 0 : threadIdx.x == 0) {
            if (EDGES && waiting >= 0) put_edges(waiting);
            waiting = -1;
            if (issued < mine && !*abort) {
                issue(issued, slot);
                ++issued;
                waiting = slot;
            }
        }
        if (++slot == depth) {
            slot = 0;
            phase ^= 1;
        }
        const float sw = lane < warps ? sums[p][0][warp0 + lane] : 0.f, qw = lane < warps ? sums[p][1][warp0 + lane] : 0.f;
        p ^= 1;
        float mu = sw;
#pragma unroll
        for (int o = 16; o; o >>= 1) mu += __shfl_xor_sync(0xffffffffu, mu, o);
        mu = quotient(mu, (float)a.cols, inv_cols);
        const float d = n_l > 0.f ? quotient(sw, n_l, inv_l) - mu : 0.f;
        float var = fmaf(n_l * d, d, qw);
#pragma unroll
        for (int o = 16; o; o >>= 1) var += __shfl_xor_sync(0xffffffffu, var, o);
        const float r = reciprocal_root(fmaf(var, inv_cols, a.eps));
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mu;
            if (a.rstd) a.rstd[row] = r;
        }
        Y* y = static_cast<Y*>(a.y) + row * a.ldy;
        const f2 mu2 = pair(-mu, -mu), r2 = pair(r, r);
        const Span<Y> sy(y, cols);
        Y* out = reinterpret_cast<Y*>(stage + sy.mis);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int c = column(g);
            float w[8], b[8], u[8];
            if (VEC) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int i = (g * 2 + h) * T + (int)threadIdx.x;
                    const float4 wv = reinterpret_cast<const float4*>(gamma)[i], bv = reinterpret_cast<const float4*>(beta)[i];
                    w[4 * h] = wv.x, w[4 * h + 1] = wv.y, w[4 * h + 2] = wv.z, w[4 * h + 3] = wv.w;
                    b[4 * h] = bv.x, b[4 * h + 1] = bv.y, b[4 * h + 2] = bv.z, b[4 * h + 3] = bv.w;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 wb = reinterpret_cast<const float2*>(gamma)[c + e * T];
                    w[e] = wb.x, b[e] = wb.y;
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                split(fma2(mul2(add2(v[g][e], mu2), r2), pair(w[2 * e], w[2 * e + 1]), pair(b[2 * e], b[2 * e + 1])), u[2 * e], u[2 * e + 1]);
            if (VEC) store_row<true>(y, c, T, cols, u);
            else if (c + 7 * T < cols) store_row<false>(out, c, T, 0x7fffffff, u);
            else store_row<false>(out, c, T, cols, u);
        }
        if (!VEC) {
            tc::fence_proxy_async_smem();
            tc::named_bar_sync(1 + team, T);
            if (threadIdx.x == 0 && sy.body) {
                tc::bulk_store(y + sy.head, out + sy.head, sy.body * (uint32_t)sizeof(Y));
                tc::bulk_commit();
            }
            if (threadIdx.x >= T - 16) {     // the elements before (at most seven) and after that copy
                const uint32_t e = threadIdx.x & 15, i = e < 8 ? e : sy.head + sy.body + e - 8;
                if (i < (e < 8 ? sy.head : (uint32_t)cols)) y[i] = out[i];
            }
        }
    }
    if (!VEC && threadIdx.x == 0) tc::bulk_wait<0>();
    if (warp == 0 && *abort) {
        // the copies in flight end before the block does
        if (EDGES && waiting >= 0) put_edges(waiting);
        volatile int no_abort = 0;
        if (lane == 0)
            for (int u = issued > depth ? issued - depth : 0; u < issued; ++u)
                tc::mbar_wait(&full[u % depth], u / depth & 1, &no_abort, &g_err_norm, 1u, 100000000ull);
    }
}

// Rows too long for the registers of a block: read three times (from L2 after the
// first): 2048 x 40000 of bfloat16 160 us.
template <typename X, typename Y>
__global__ void __launch_bounds__(1024) norm_long_kernel(const NormArgs a) {
    __shared__ float sh[2][32];
    tc::pdl_wait();
    tc::pdl_trigger();
    const X* x = static_cast<const X*>(a.x) + blockIdx.x * a.ldx;
    Y* y = static_cast<Y*>(a.y) + blockIdx.x * a.ldy;
    float s = 0.f;
    for (int64_t c = threadIdx.x; c < a.cols; c += 1024) s += el::to_f32(x[c]);
    const float n = (float)a.cols, mu = block_sum(s, sh[0]) / n;
    s = 0.f;
    for (int64_t c = threadIdx.x; c < a.cols; c += 1024) {
        const float d = el::to_f32(x[c]) - mu;
        s = fmaf(d, d, s);
    }
    const float r = 1.f / sqrtf(block_sum(s, sh[1]) / n + a.eps);
    for (int64_t c = threadIdx.x; c < a.cols; c += 1024) {
        const float g = a.gamma ? el::load_as(a.gamma, a.pk, c) : 1.f, b = a.beta ? el::load_as(a.beta, a.pk, c) : 0.f;
        y[c] = el::from_f32<Y>(fmaf((el::to_f32(x[c]) - mu) * r, g, b));
    }
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[blockIdx.x] = mu;
        if (a.rstd) a.rstd[blockIdx.x] = r;
    }
}

// ---- gradient ----------------------------------------------------------------

struct GradArgs {
    const void* dy;
    const void* x;
    const void* gamma;
    const float* mean;
    const float* rstd;
    void* dx;                // nullptr: not wanted
    float* part;             // sums over a block's rows of dy xh and of dy, 2 x cols a block; nullptr: not wanted
    int64_t rows, cols, lddy, ldx, lddx;
    int64_t slice;           // columns of a block of a cluster
    int depth;               // rows of the ring
    int pk;
};

constexpr int kGradThreads = 512;            // of a block, at most

// A cluster takes every (number of clusters)-th row, each of its blocks a slice of
// the columns, eight a thread: the threads keep the sums over the rows of their
// columns.  Rows come into a ring in shared memory, a row's place free once every
// warp has met at the row's barrier; a row is in registers (as xh and d) while its
// two sums are added over the block and the cluster.  gamma is in shared memory,
// and one thread asks for the copies.
// What bounds it (8192 x 8192 of bfloat16, 80 us, 5.0 TB/s of 6.8): the chain of a
// row's sums, with one row of 16 warps at a time (1.75 instructions a cycle, no pipe
// above 20 %); 1024 threads with eight columns each take 121 us, 256 with 32 91
// (sixteen in single arithmetic: 120).  More than 8192 columns add the cluster's
// exchange to every row's chain: 4096 x 16384 150 us.  Rows that start
// anywhere pass element by element: 8191 x 4097 131 us against 49 for 8192 x 4096
// (results by way of shared memory, as in norm_stream_kernel: 125, but 28 against 25
// for 4099 x 1138 of binary32).
// VEC: every row starts on a 16-byte boundary and a thread takes eight columns
// side by side; else a warp's columns are side by side.  EDGES: rows have elements
// outside the bulk copies, which warp 0 loads when it asks for the copies and puts
// beside them a row later.
template <typename X, typename Y, bool VEC, bool EDGES, int EG>
__global__ void __launch_bounds__(kGradThreads, 1) norm_grad_kernel(const __grid_constant__ GradArgs a) {
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ float sums[2][2][16];         // [parity][sum][warp]
    __shared__ float totals[2][8][2];        // [parity][block of the cluster][sum]
    __shared__ uint64_t full[kMostRing], got[2];
    __shared__ int abort_flag;
    const int T = blockDim.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t ranks = cl::size(), rank = cl::rank();
    const int clusters = gridDim.x / ranks, first = blockIdx.x / ranks;
    const int64_t c0 = rank * a.slice;
    const int cols = (int)min(a.slice, a.cols - c0);                       // this block's columns
    const X* x = static_cast<const X*>(a.x) + c0;
    const Y* dy = static_cast<const Y*>(a.dy) + c0;
    const int mine = first < a.rows ? (int)((a.rows - first + clusters - 1) / clusters) : 0;
    const uint32_t ypart = (uint32_t)(a.slice * sizeof(X) + 16), pitch = ypart + (uint32_t)(a.slice * sizeof(Y) + 16);
    volatile int* abort = &abort_flag;
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int d = 0; d < a.depth; ++d) tc::mbar_init(&full[d], EDGES ? 2 : 1);
        for (int p = 0; p < 2; ++p) tc::mbar_init(&got[p], ranks * 2);
        tc::fence_barrier_init();
    }
    if (ranks > 1) cl::sync();           // every block's barriers are there
    else __syncthreads();
    tc::pdl_wait();
    tc::pdl_trigger();

    float* gamma = reinterpret_cast<float*>(ring + a.depth * pitch);
    const void* gp = a.gamma ? static_cast<const uint8_t*>(a.gamma) + c0 * (a.pk ? 2 : 4) : nullptr;
    // Lanes 0 ... 15 have the elements of x before (at most seven) and after the bulk
    // copy, the others those of dy: where they go, -1 for none, and their values.
    int edge_at = -1;
    X xe = el::from_f32<X>(0.f);
    Y ye = el::from_f32<Y>(0.f);
    auto issue = [&](int k, int slot) {      // warp 0 (without edges, its first thread)
        const int64_t row = first + (int64_t)k * clusters;
        const X* xr = x + row * a.ldx;
        const Y* yr = dy + row * a.lddy;
        uint8_t* to = ring + slot * pitch;
        if (!EDGES) {
            tc::mbar_arrive_expect_tx(&full[slot], cols * (uint32_t)(sizeof(X) + sizeof(Y)));
            tc::bulk_load(to, xr, cols * (uint32_t)sizeof(X), &full[slot]);
            tc::bulk_load(to + ypart, yr, cols * (uint32_t)sizeof(Y), &full[slot]);
            return;
        }
        const Span<X> sx(xr, cols);
        const Span<Y> sy(yr, cols);
        if (lane == 0) {
            const uint32_t xb = sx.body * sizeof(X), yb = sy.body * sizeof(Y);
            tc::mbar_arrive_expect_tx(&full[slot], xb + yb);
            if (xb) tc::bulk_load(to + sx.mis + sx.head * sizeof(X), xr + sx.head, xb, &full[slot]);
            if (yb) tc::bulk_load(to + ypart + sy.mis + sy.head * sizeof(Y), yr + sy.head, yb, &full[slot]);
        }
        const bool of_y = lane >= 16, after = lane & 8;
        const uint32_t head = of_y ? sy.head : sx.head, body = of_y ? sy.body : sx.body;
        const uint32_t i = (lane & 7) + (after ? head + body : 0);
        edge_at = -1;
        if (i < (after ? (uint32_t)cols : head)) {
            edge_at = (int)(slot * pitch + (of_y ? ypart + sy.mis + i * sizeof(Y) : sx.mis + i * sizeof(X)));
            if (of_y) ye = yr[i];
            else xe = xr[i];
        }
    };
    auto put_edges = [&](int slot) {         // warp 0: of the row last asked for
        if (edge_at >= 0) {
            if (lane >= 16) *reinterpret_cast<Y*>(ring + edge_at) = ye;
            else *reinterpret_cast<X*>(ring + edge_at) = xe;
        }
        tc::fence_proxy_async_smem();        // a later copy may write there
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&full[slot]);
    };
    int issued = 0;
    if (EDGES ? warp == 0 : threadIdx.x == 0)
        for (; issued < a.depth && issued < mine; ++issued) {
            if (EDGES && issued) put_edges(issued - 1);
            issue(issued, issued);
        }
    for (int c = threadIdx.x; c < cols; c += T) gamma[c] = gp ? el::load_as(gp, a.pk, c) : 1.f;
    if (EDGES && warp == 0 && issued) put_edges(issued - 1);
    __syncthreads();

    auto column = [&](int k) { return VEC ? (k * T + (int)threadIdx.x) * 8 : k * T * 8 + (int)threadIdx.x; };
    // eight elements of a row in the ring (or of gamma), 0 beyond the columns
    auto take = [&](const auto* at, int c, f2(&v)[4]) {
        float w[8];
        if (VEC && c + 8 <= cols) {
            load8(at + c, w);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int i = VEC ? c + e : c + e * T;
                w[e] = i < cols ? el::to_f32(at[i]) : 0.f;
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = pair(w[2 * e], w[2 * e + 1]);
    };
    f2 sg[EG][4], sb[EG][4];
#pragma unroll
    for (int g = 0; g < EG; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) sg[g][e] = sb[g][e] = 0;
    const float inv = 1.f / (float)a.cols;
    X* dx = a.dx ? static_cast<X*>(a.dx) + c0 + first * a.lddx : nullptr;
    float mu_next = mine ? __ldg(a.mean + first) : 0.f, r_next = mine ? __ldg(a.rstd + first) : 0.f;
    int slot = 0, p = 0, waiting = -1;       // waiting: place whose edges are not there yet
    uint32_t phase = 0, turn = 0;
    for (int k = 0; k < mine; ++k) {
        const float mu = mu_next, r = r_next;
        if (k + 1 < mine) {
            const int row = first + (k + 1) * clusters;
            mu_next = __ldg(a.mean + row), r_next = __ldg(a.rstd + row);
        }
        // After a wait that gave up the rows go on without copies or waits: the
        // cluster's blocks meet for every row.
        tc::mbar_wait(&full[slot], phase, abort, &g_err_norm, 1u);
        const uint8_t* at = ring + slot * pitch;
        uint32_t xmis = 0, ymis = 0;
        if (!VEC) {
            const int64_t row = first + (int64_t)k * clusters;
            xmis = (uint32_t)reinterpret_cast<uintptr_t>(x + row * a.ldx) & 15u;
            ymis = (uint32_t)reinterpret_cast<uintptr_t>(dy + row * a.lddy) & 15u;
        }
        f2 xh[EG][4], d[EG][4], s2 = 0, t2 = 0;
        const f2 mu2 = pair(-mu, -mu), r2 = pair(r, r);
#pragma unroll
        for (int g = 0; g < EG; ++g) {
            f2 w[4];
            take(reinterpret_cast<const X*>(at + xmis), column(g), xh[g]);
            take(reinterpret_cast<const Y*>(at + ypart + ymis), column(g), d[g]);
            take(gamma, column(g), w);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                xh[g][e] = mul2(add2(xh[g][e], mu2), r2);
                sb[g][e] = add2(sb[g][e], d[g][e]);
                sg[g][e] = fma2(d[g][e], xh[g][e], sg[g][e]);
                d[g][e] = mul2(d[g][e], w[e]);
                s2 = add2(s2, d[g][e]);
                t2 = fma2(d[g][e], xh[g][e], t2);
            }
        }
        float s = both_of(s2), t = both_of(t2);
        // both sums at once: the lower half warp adds s, the upper one t
        float both = (lane < 16 ? s : t) + __shfl_xor_sync(0xffffffffu, lane < 16 ? t : s, 16);
#pragma unroll
        for (int o = 8; o; o >>= 1) both += __shfl_xor_sync(0xffffffffu, both, o);
        if ((lane & 15) == 0) sums[p][lane >> 4][warp] = both;
        __syncthreads();                     // every warp has the row in registers
        if (EDGES ? warp == 0 : threadIdx.x == 0) {
            if (EDGES && waiting >= 0) put_edges(waiting);
            waiting = -1;
            if (issued < mine && !*abort) {
                issue(issued, slot);
                ++issued;
                waiting = slot;
            }
        }
        const int warps = T >> 5, l = lane & 15;
        both = l < warps ? sums[p][lane >> 4][l] : 0.f;
#pragma unroll
        for (int o = 8; o; o >>= 1) both += __shfl_xor_sync(0xffffffffu, both, o);
        if (ranks > 1) {
            // Each block gives its totals to every block of the cluster.  (A block that
            // gives those of row k + 2 has all of row k + 1, which the others gave after
            // they had read those of row k.)
            if (warp == 0 && l == 0)
                for (uint32_t w = 0; w < ranks; ++w) {
                    cl::store(&totals[p][rank][lane >> 4], w, both);
                    cl::arrive(&got[p], w);
                }
            cl::wait(&got[p], turn, abort, &g_err_norm, 2u);
            both = 0.f;
            for (uint32_t w = 0; w < ranks; ++w) both += totals[p][w][lane >> 4];
            turn ^= p;
        }
        p ^= 1;
        if (++slot == a.depth) {
            slot = 0;
            phase ^= 1;
        }
        both *= inv * r;
        s = __shfl_sync(0xffffffffu, both, 0);
        t = __shfl_sync(0xffffffffu, both, 16);
        if (dx) {
            const f2 s3 = pair(-s, -s), t3 = pair(-t, -t);
#pragma unroll
            for (int g = 0; g < EG; ++g) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) split(fma2(xh[g][e], t3, fma2(r2, d[g][e], s3)), v[2 * e], v[2 * e + 1]);
                store_row<VEC>(dx, column(g), T, cols, v);
            }
            dx += clusters * a.lddx;
        }
    }
    if (warp == 0 && *abort) {
        // the copies in flight end before the block does
        if (EDGES && waiting >= 0) put_edges(waiting);
        volatile int no_abort = 0;
        if (lane == 0)
            for (int u = issued > a.depth ? issued - a.depth : 0; u < issued; ++u)
                tc::mbar_wait(&full[u % a.depth], u / a.depth & 1, &no_abort, &g_err_norm, 1u, 100000000ull);
    }
    if (a.part) {
        float* part = a.part + (int64_t)first * 2 * a.cols + c0;
#pragma unroll
        for (int g = 0; g < EG; ++g) {
            float vg[8], vb[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                split(sg[g][e], vg[2 * e], vg[2 * e + 1]);
                split(sb[g][e], vb[2 * e], vb[2 * e + 1]);
            }
            if (VEC && a.cols % 4 == 0) {
                store_row<true>(part, column(g), 1, cols, vg);
                store_row<true>(part + a.cols, column(g), 1, cols, vb);
            } else {
                store_row<false>(part, column(g), VEC ? 1 : T, cols, vg);
                store_row<false>(part + a.cols, column(g), VEC ? 1 : T, cols, vb);
            }
        }
    }
    if (ranks > 1) cl::sync();           // no block ends before the others have given it theirs
}

// Rows too long for that: dx a row a block, the columns' sums apart (1000 x 70000 of
// bfloat16 548 us).
template <typename X, typename Y>
__global__ void __launch_bounds__(1024) norm_grad_long_kernel(const GradArgs a) {
    __shared__ float sh[2][32];
    tc::pdl_wait();
    tc::pdl_trigger();
    const Y* dy = static_cast<const Y*>(a.dy) + blockIdx.x * a.lddy;
    const X* x = static_cast<const X*>(a.x) + blockIdx.x * a.ldx;
    X* dx = static_cast<X*>(a.dx) + blockIdx.x * a.lddx;
    const float mu = a.mean[blockIdx.x], r = a.rstd[blockIdx.x], n = (float)a.cols;
    float s = 0.f, t = 0.f;
    for (int64_t c = threadIdx.x; c < a.cols; c += 1024) {
        const float d = el::to_f32(dy[c]) * (a.gamma ? el::load_as(a.gamma, a.pk, c) : 1.f);
        s += d;
        t = fmaf(d, (el::to_f32(x[c]) - mu) * r, t);
    }
    s = block_sum(s, sh[0]) / n;
    t = block_sum(t, sh[1]) / n;
    for (int64_t c = threadIdx.x; c < a.cols; c += 1024) {
        const float d = el::to_f32(dy[c]) * (a.gamma ? el::load_as(a.gamma, a.pk, c) : 1.f);
        dx[c] = el::from_f32<X>(r * (d - s - (el::to_f32(x[c]) - mu) * r * t));
    }
}

template <typename X, typename Y>
__global__ void __launch_bounds__(256) norm_columns_kernel(const GradArgs a) {
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    tc::pdl_wait();
    tc::pdl_trigger();
    if (c >= a.cols) return;
    float g = 0.f, b = 0.f;
    for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
        const float d = el::to_f32(static_cast<const Y*>(a.dy)[r * a.lddy + c]);
        g = fmaf(d, (el::to_f32(static_cast<const X*>(a.x)[r * a.ldx + c]) - a.mean[r]) * a.rstd[r], g);
        b += d;
    }
    a.part[(int64_t)blockIdx.y * 2 * a.cols + c] = g;
    a.part[((int64_t)blockIdx.y * 2 + 1) * a.cols + c] = b;
}

// The partial sums of the columns added in a fixed order: 32 columns a block, its
// eight warps every eighth part each, eight of those joined before they are added, so
// that a part passes a 64th of their number of additions and seven more (one after the
// other, 57 of 456 parts a warp made most of the error of dgamma and dbeta).
// blockIdx.y: dgamma or dbeta.
__device__ __forceinline__ float joined(const float (&v)[8]) {
    return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
}
__global__ void __launch_bounds__(256)
norm_columns_sum_kernel(const float* part, int parts, int64_t cols, float* dgamma, float* dbeta) {
    __shared__ float sh[8][32];
    float* out = blockIdx.y ? dbeta : dgamma;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    tc::pdl_wait();
    tc::pdl_trigger();
    if (!out) return;
    float s = 0.f, v[8];
    if (c < cols) {
        const int64_t next = 16 * cols;                       // to the warp's next part
        const float* p = part + (2 * warp + blockIdx.y) * cols + c;
        int left = (parts - warp + 7) / 8;
        for (; left >= 8; left -= 8, p += 8 * next) {
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = p[u * next];
            s += joined(v);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = u < left ? p[u * next] : 0.f;
        s += joined(v);
    }
    sh[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < cols) {
#pragma unroll
        for (int w = 0; w < 8; ++w) v[w] = sh[w][lane];
        out[c] = joined(v);
    }
}

int kind_of(lrc_fmt f) { return f == LRC_F32 ? 0 : f == LRC_BF16 ? 2 : 1; }

// Rows of elements of `es` bytes all start on a 16-byte boundary.
bool rows_aligned(const void* p, int64_t ld, int64_t es, int64_t rows) {
    return !p || (aligned16(p) && (rows < 2 || ld * es % 16 == 0));
}

lrc_status too_long(const char* what) {
    set_error("%s: cols too large", what);
    return LRC_ERR_UNSUPPORTED;
}

template <typename X, typename Y>
lrc_status norm_as(const NormArgs& a, cudaStream_t s) {
    const bool vec = rows_aligned(a.x, a.ldx, sizeof(X), a.rows) && rows_aligned(a.y, a.ldy, sizeof(Y), a.rows) &&
                     rows_aligned(a.gamma, 0, 1, 1) && rows_aligned(a.beta, 0, 1, 1);
    const int64_t groups = (a.cols + 7) / 8;
    auto go = [&](auto kernel, int vpt) -> lrc_status {
        const unsigned T = (unsigned)((groups + 32 * vpt - 1) / (32 * vpt) * 32);
        const unsigned per = T == 32 ? 4 : 1;
        const cudaError_t e = launch_pdl(kernel, dim3((unsigned)((a.rows + per - 1) / per)), dim3(T, per), 0, s, a);
        if (e != cudaSuccess) return cuda_fail(e, "norm_kernel");
        return after_launch("norm_kernel");
    };
    // Many rows: 256 threads a row or fewer, so that a multiprocessor has several rows
    // at different points of their chain; few rows: eight values a thread.
    const bool many = a.rows >= 2 * (int64_t)sm_count();
    // Rows enough to pay for bringing gamma and beta to every multiprocessor, long
    // enough for a few warps: norm_stream_kernel against norm_kernel, bfloat16, us.
    //   8192 x 8192: 55, 75.  4096: 31, 40.  2048: 21, 24.  1024: 19, 13.
    //   8191 x 4097: 46, 107.  1025: 22, 29.  513: 15, 18.
    //   2600 x 8192: 26, 30.  1300: 20.4, 20.2.  700: 12.0, 9.9.
    //   700 x 4097: 10, 20.  1025: 7.8, 6.9.
    if (a.rows >= (vec ? 16 : 4) * (int64_t)sm_count() && groups <= 2048 && groups > (vec ? 128 : 64)) {
        const int pitch = ((int)(a.cols * (int64_t)sizeof(X)) + 31) & ~15;
        const int stage = vec ? 0 : ((int)(a.cols * (int64_t)sizeof(Y)) + 31) & ~15;
        // 32 columns a thread (a warp's sums and its row's ends are half of its
        // instructions) where the teams that fit, two rows in the ring each, fill a
        // block; else 16: 8192 x 8192 of binary32 (two teams of 256 threads, or of 512)
        // is 7 % slower with 32, of bfloat16 9 % faster; 8191 x 1025 24 us and 22.
        int G = 4, teams = 0, depth = 0, params = 0;
        unsigned T = 0;
        for (; G >= 2; G /= 2) {
            T = (unsigned)((groups + 32 * G - 1) / (32 * G) * 32);
            params = (int)T * 8 * G * 8;
            teams = T < 64 ? kMostTeams : (int)(1024 / T) < kMostTeams ? (int)(1024 / T) : kMostTeams;
            const int room = kRing - params;
            while (teams && room / teams < stage + 2 * pitch) --teams;
            depth = teams ? (room / teams - stage) / pitch : 0;
            if (groups > 256 && teams * T >= 768) break;
        }
        if (G < 2) G = 2;
        if (depth > kMostRing) depth = kMostRing;
        if (teams) {
            auto pick = [&](auto g) {
                constexpr int kG = decltype(g)::value;
                return !vec ? norm_stream_kernel<X, Y, false, true, kG>
                            : a.cols % 8 ? norm_stream_kernel<X, Y, true, true, kG> : norm_stream_kernel<X, Y, true, false, kG>;
            };
            auto kernel = G == 2 ? pick(std::integral_constant<int, 2>()) : pick(std::integral_constant<int, 4>());
            cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRing);
            if (e != cudaSuccess) return cuda_fail(e, "norm_stream_kernel");
            e = launch_pdl(kernel, dim3((unsigned)sm_count()), dim3(T, (unsigned)teams), (size_t)(teams * (depth * pitch + stage) + params), s, a, depth);
            if (e != cudaSuccess) return cuda_fail(e, "norm_stream_kernel");
            return after_launch("norm_stream_kernel");
        }
    }
    if (many && groups <= 1024) {
        if (groups <= 256) return vec ? go(norm_kernel<X, Y, true, 1, 256>, 1) : go(norm_kernel<X, Y, false, 1, 256>, 1);
        if (groups <= 512) return vec ? go(norm_kernel<X, Y, true, 2, 256>, 2) : go(norm_kernel<X, Y, false, 2, 256>, 2);
        return vec ? go(norm_kernel<X, Y, true, 4, 256>, 4) : go(norm_kernel<X, Y, false, 4, 256>, 4);
    }
    if (groups <= 1024) return vec ? go(norm_kernel<X, Y, true, 1, 1024>, 1) : go(norm_kernel<X, Y, false, 1, 1024>, 1);
    if (groups <= 2048) return vec ? go(norm_kernel<X, Y, true, 2, 1024>, 2) : go(norm_kernel<X, Y, false, 2, 1024>, 2);
    if (groups <= 4096) return vec ? go(norm_kernel<X, Y, true, 4, 1024>, 4) : go(norm_kernel<X, Y, false, 4, 1024>, 4);
    const cudaError_t e = launch_pdl(norm_long_kernel<X, Y>, dim3((unsigned)a.rows), dim3(1024), 0, s, a);
    if (e != cudaSuccess) return cuda_fail(e, "norm_long_kernel");
    return after_launch("norm_long_kernel");
}

// Columns of a block at most, blocks of a cluster at most, bytes of its ring.
constexpr int64_t kSlice = 8192;

template <typename X, typename Y>
lrc_status norm_grad_as(GradArgs a, float* dgamma, float* dbeta, cudaStream_t s) {
    const bool sums = dgamma || dbeta;
    int ranks = (int)((a.cols + kSlice - 1) / kSlice < 16 ? (a.cols + kSlice - 1) / kSlice : 16);
    const bool fits = ranks <= 8 && a.rows > 0;
    const int64_t sms = sm_count();
    int64_t parts = 0;
    int resident = 1;
    bool vec = false;
    unsigned threads = 0;
    int pitch = 0, eg = 1;
    if (fits) {
        a.slice = ((a.cols + ranks - 1) / ranks + 7) / 8 * 8;
        vec = rows_aligned(a.x, a.ldx, sizeof(X), a.rows) && rows_aligned(a.dy, a.lddy, sizeof(Y), a.rows) &&
              rows_aligned(a.dx, a.lddx, sizeof(X), a.rows) && rows_aligned(a.gamma, 0, 1, 1);
        eg = a.slice > 2048 ? 2 : 1;
        threads = (unsigned)((a.slice / 8 + 32 * eg - 1) / (32 * eg) * 32);
        // Blocks of a multiprocessor: two rows of 4096 side by side (49 us for 8192 of
        // them against 59 with one, 65 with four of half the columns a thread); shorter
        // rows up to 512 threads, six at most: each block has partial sums to write.
        resident = threads > 256 ? 1 : eg == 2 ? 2 : (int)(512 / threads > 6 ? 6 : 512 / threads);
        pitch = (int)(a.slice * (int64_t)(sizeof(X) + sizeof(Y)) + 32);
        a.depth = (kRing / resident - (resident > 1 ? 2048 : 0) - (int)a.slice * 4) / pitch;
        if (a.depth > kMostRing) a.depth = kMostRing;
        parts = sms * resident / ranks;
        if (parts > a.rows) parts = a.rows;
    } else if (a.rows > 0) {
        parts = a.rows < 128 ? a.rows : 128;
    }
    lrc_status st;
    if (sums) {
        if ((a.cols + 31) / 32 > 0x7fffffff) return too_long("lrc_layer_norm_grad");
        void* ws = nullptr;
        if ((st = stream_workspace(s, (size_t)(parts ? parts : 1) * 2 * a.cols * 4, &ws)) != LRC_OK) return st;
        a.part = static_cast<float*>(ws);
    }
    cudaError_t e;
    if (fits && (sums || a.dx)) {
        // (slices but the last are whole groups of eight columns)
        auto pick = [&](auto g) {
            constexpr int G = decltype(g)::value;
            return !vec ? norm_grad_kernel<X, Y, false, true, G>
                        : a.cols % 8 ? norm_grad_kernel<X, Y, true, true, G> : norm_grad_kernel<X, Y, true, false, G>;
        };
        auto kernel = eg == 1 ? pick(std::integral_constant<int, 1>()) : pick(std::integral_constant<int, 2>());
        const int smem = a.depth * pitch + (int)a.slice * 4;
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRing);
        if (e != cudaSuccess) return cuda_fail(e, "norm_grad_kernel");
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)(parts * ranks));
        cfg.blockDim = dim3(threads);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = s;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)ranks;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = ranks > 1 ? 2 : 1;
        if ((e = cudaLaunchKernelEx(&cfg, kernel, a)) != cudaSuccess) return cuda_fail(e, "norm_grad_kernel");
        if ((st = after_launch("norm_grad_kernel")) != LRC_OK) return st;
    } else if (!fits && a.rows > 0) {
        if (sums) {
            e = launch_pdl(norm_columns_kernel<X, Y>, dim3((unsigned)((a.cols + 255) / 256), (unsigned)parts), dim3(256), 0, s, a);
            if (e != cudaSuccess) return cuda_fail(e, "norm_columns_kernel");
            if ((st = after_launch("norm_columns_kernel")) != LRC_OK) return st;
        }
        if (a.dx) {
            e = launch_pdl(norm_grad_long_kernel<X, Y>, dim3((unsigned)a.rows), dim3(1024), 0, s, a);
            if (e != cudaSuccess) return cuda_fail(e, "norm_grad_long_kernel");
            if ((st = after_launch("norm_grad_long_kernel")) != LRC_OK) return st;
        }
    }
    if (!sums) return LRC_OK;
    e = launch_pdl(norm_columns_sum_kernel, dim3((unsigned)((a.cols + 31) / 32), 2), dim3(256), 0, s, (const float*)a.part,
                   (int)parts, a.cols, dgamma, dbeta);
    if (e != cudaSuccess) return cuda_fail(e, "norm_columns_sum_kernel");
    return after_launch("norm_columns_sum_kernel");
}

}  // namespace

lrc_status launch_layer_norm(const void* X, const void* gamma, const void* beta, void* Y, float* mean, float* rstd,
                             int64_t rows, int64_t cols, int64_t ldx, int64_t ldy, float eps, lrc_fmt fmt, lrc_fmt pfmt,
                             cudaStream_t s) {
    const NormArgs a{X, gamma, beta, Y, mean, rstd, rows, cols, ldx, ldy, eps, kind_of(pfmt)};
    if (fmt == LRC_F32) return norm_as<float, float>(a, s);
    if (fmt == LRC_BF16) return norm_as<bf16, bf16>(a, s);
    if (fmt == LRC_F16) return norm_as<__half, float>(a, s);
    return norm_as<__half, __half>(a, s);
}

lrc_status launch_layer_norm_grad(const void* dY, const void* X, const void* gamma, const float* mean, const float* rstd,
                                  void* dX, float* dgamma, float* dbeta, int64_t rows, int64_t cols, int64_t lddy,
                                  int64_t ldx, int64_t lddx, lrc_fmt fmt, lrc_fmt pfmt, cudaStream_t s) {
    GradArgs a{};
    a.dy = dY;
    a.x = X;
    a.gamma = gamma;
    a.mean = mean;
    a.rstd = rstd;
    a.dx = dX;
    a.rows = rows;
    a.cols = cols;
    a.lddy = lddy;
    a.ldx = ldx;
    a.lddx = lddx;
    a.pk = kind_of(pfmt);
    if (fmt == LRC_F32) return norm_grad_as<float, float>(a, dgamma, dbeta, s);
    if (fmt == LRC_BF16) return norm_grad_as<bf16, bf16>(a, dgamma, dbeta, s);
    if (fmt == LRC_F16) return norm_grad_as<__half, float>(a, dgamma, dbeta, s);
    return norm_grad_as<__half, __half>(a, dgamma, dbeta, s);
}

uint32_t take_norm_error() {
    unsigned int v = 0;
    if (cudaMemcpyFromSymbol(&v, g_err_norm, sizeof v) != cudaSuccess) return 0xffffffffu;
    if (v) {
        const unsigned int z = 0;
        cudaMemcpyToSymbol(g_err_norm, &z, sizeof z);
    }
    return v;
}

}  // namespace lrc
