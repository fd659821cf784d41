// distill.cu -- distillation from a teacher's top logits (lrc_distill,
// lrc_distill_grad), binary32 arithmetic.
//
// With the row's largest logit m, s = sum_j exp((z_j - m) / tau) and the teacher's p:
//   lse = m / tau + log s,
//   loss = tau^2 w sum_k p_k (log p_k - ((z_{i_k} - m) / tau - log s)),
//   dz_j = tau w g (exp((z_j - m) / tau) / s - sum over k with i_k = j of p_k).
// The difference comes first, in two-lane instructions (1024 x 32768 binary32 forward
// 31.3 us; 30.2 with z k - m k, one multiply-add): a rounded m k would change every
// term, by 4e-5 of it for logits near 1000, and m k leaves binary32 for a row of the
// lowest number.
//
// Long rows are bound by HBM (a row read once, its gradient written once): 4096 rows
// of 65536 bfloat16 199 us, 5.4 TB/s; the gradient alone for 1021 rows of 50001
// binary16 35 us, 5.9 TB/s.  Shorter ones, and the forward pass, by the end of each row
// (the block's maximum and sum, the logarithm, the loss, the teacher's places), when
// most of the block waits: 2048 x 32768 bfloat16 forward 38 us (floor 20), 4096 x 8192
// binary16 37 with the gradient (20).  Rows that do not fit into the ring are read
// twice, from the L2 as far as the rows at work fit there: 512 x 262144 bfloat16 133
// us, 256 of binary32 132 (floors 79).  A few rows wait for a chain of loads and the
// call: 16 of 32768 binary32 8 us.
//
// Persistent blocks, one row at a time (or a cluster a row where rows are few, each
// block a slice).  One warp brings the row in chunks by bulk copies into a ring in
// shared memory, a few prepare the next rows' teacher entries (a row each: a chain of
// two loads from memory and a softmax, longer than many a row's copies), the others
// form the running maximum and sum chunk by chunk as they come and, where the row
// fits into the ring, the gradient from the same copy; else the chunks come again.  The ring holds the next row's first chunks by then.  At the places of
// the teacher's entries the gradient is written once more at the end of the row.
#include <math.h>

#include "cluster.cuh"
#include "common.cuh"
#include "elem.cuh"
#include "tc.cuh"

namespace lrc {
namespace {

using bf16 = __nv_bfloat16;

__device__ unsigned int g_err_distill;

constexpr int kMaxTop = 1024;
constexpr int kMostChunks = 32;
constexpr float kLog2e = 1.4426950408889634f;

struct Args {
    const void* Z;
    const void* T;
    const int64_t* idx;
    const float* w;
    const float* lse_in;
    const float* g;
    float* loss;
    float* lse_out;
    void* dZ;
    int64_t rows, V, ldz, ldt, lddz, slice;
    int K, table;            // teacher entries; places of the table that finds repeated ones
    int chunks;              // of the ring
    bool keep;               // the slice stays in the ring until its gradient is written
    float tau;
    int tkind;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// The larger one; a NaN where there is one.
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// 16 bytes of elements (kVec of them) as binary32 and back.
template <typename T> constexpr int kVec = 16 / (int)sizeof(T);
__device__ __forceinline__ void widen(const uint4& a, float (&v)[4], float) {
    v[0] = __uint_as_float(a.x), v[1] = __uint_as_float(a.y), v[2] = __uint_as_float(a.z), v[3] = __uint_as_float(a.w);
}
__device__ __forceinline__ void widen(const uint4& a, float (&v)[8], __half) {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        v[2 * i] = f.x, v[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ void widen(const uint4& a, float (&v)[8], bf16) {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
}
__device__ __forceinline__ uint4 narrow(const float (&v)[4], float) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
__device__ __forceinline__ uint4 narrow(const float (&v)[8], __half) {
    return make_uint4(tc::pack_half2(v[0], v[1]), tc::pack_half2(v[2], v[3]), tc::pack_half2(v[4], v[5]),
                      tc::pack_half2(v[6], v[7]));
}
__device__ __forceinline__ uint4 narrow(const float (&v)[8], bf16) {
    return make_uint4(tc::pack_bf162(v[0], v[1]), tc::pack_bf162(v[2], v[3]), tc::pack_bf162(v[4], v[5]),
                      tc::pack_bf162(v[6], v[7]));
}

// What is taken off the logits of a row whose largest one is m: nothing where there
// is none.
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }

// Running maximum and sum of exp2((z - m) k): m = -infinity has s = 0; a NaN or
// +infinity makes s NaN.
struct Running {
    float m = -INFINITY, s = 0.f, base = 0.f;
    __device__ __forceinline__ void raise(float to, float k) {
        const float mm = max_nan(m, to);
        if (mm != m) {                               // (a NaN too)
            s *= ex2((m - mm) * k);
            m = base = mm;
        }
    }
    __device__ __forceinline__ void join(float om, float os, float k) {
        const float mm = max_nan(m, om);
        s = (m == mm ? s : s * ex2((m - mm) * k)) + (om == mm ? os : os * ex2((om - mm) * k));
        m = mm;
    }
};

// What the teacher's warp leaves for a row.
struct Teacher {
    float c;                 // tau w g, 0 where the row has no gradient
    float lw;                // tau w, 0 where the row has no loss (tau^2 alone may leave binary32)
    int repeated;            // some place is named more than once
};

// Warps that prepare teacher entries: one for each row that is prepared ahead.
constexpr int teachers(int THREADS) { return THREADS > 256 ? 4 : 2; }
constexpr int all_threads(int THREADS) { return THREADS + 32 + 32 * teachers(THREADS); }

// Shared memory: ring | a teacher's warp each: at, log p, z of the K entries, table.
template <typename T, int THREADS>
__global__ void __launch_bounds__(all_threads(THREADS), 512 / THREADS) distill_kernel(const __grid_constant__ Args a) {
    constexpr int kChunk = THREADS * 32;                      // bytes: two vectors a thread
    constexpr int kWarps = THREADS / 32, N = kVec<T>, kAhead = teachers(THREADS);
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ uint64_t full[kMostChunks], empty[kMostChunks], tfull[kAhead], tempty[kAhead], got;
    __shared__ float part_m[2][kWarps], part_s[2][kWarps];    // [row parity][warp]
    __shared__ float all_m[8], all_s[8];                      // [block of the cluster]
    __shared__ Teacher teacher[kAhead];
    __shared__ int abort_flag;
    int* at = reinterpret_cast<int*>(ring + a.chunks * kChunk);          // [kAhead][K]
    float* lpk = reinterpret_cast<float*>(at + kAhead * a.K);
    float* zk = lpk + kAhead * a.K;
    int* tables = reinterpret_cast<int*>(zk + kAhead * a.K);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t ranks = cl::size(), rank = cl::rank();
    const int clusters = gridDim.x / ranks, first = blockIdx.x / ranks;
    const int64_t c0 = rank * a.slice;
    const int len = (int)min(a.slice, a.V - c0);              // elements of this block's slice
    const int mine = first < a.rows ? (int)((a.rows - first + clusters - 1) / clusters) : 0;
    const T* Z = static_cast<const T*>(a.Z) + c0;
    T* dZ = a.dZ ? static_cast<T*>(a.dZ) + c0 : nullptr;
    const bool sums = a.lse_in == nullptr;
    const float it = 1.f / a.tau, k2 = kLog2e * it;
    const float it_rest = fmaf(-it, a.tau, 1.f) * it;         // 1 / tau = it + it_rest
    const el::f2 kk = el::pair(k2, k2);
    volatile int* abort = &abort_flag;
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int d = 0; d < a.chunks; ++d) {
            tc::mbar_init(&full[d], 1);
            tc::mbar_init(&empty[d], kWarps);
        }
        for (int p = 0; p < kAhead; ++p) {
            tc::mbar_init(&tfull[p], 1);
            tc::mbar_init(&tempty[p], kWarps);
        }
        tc::mbar_init(&got, ranks);
        tc::fence_barrier_init();
    }
    if (ranks > 1) cl::sync();                            // every block's barriers are there
    else __syncthreads();
    tc::pdl_wait();
    tc::pdl_trigger();
    // A row's slice: `head` elements up to a 16-byte boundary, nvec vectors, the rest.
    auto head_of = [&](const T* z) {
        return min((uint32_t)len, (16u - (uint32_t)(reinterpret_cast<uintptr_t>(z) & 15u)) % 16u / (uint32_t)sizeof(T));
    };

    if (warp == kWarps) {
        // ---- the copies
        if (lane == 0) {
            int slot = 0;
            uint32_t phase = 1, used = 0;
            bool go = true;
            for (int r = 0; r < mine && go; ++r) {
                const T* z = Z + (first + (int64_t)r * clusters) * a.ldz;
                const uint32_t head = head_of(z), bytes = (len - head) / N * 16;
                const uint8_t* src = reinterpret_cast<const uint8_t*>(z + head);
                const int times = sums && dZ && !a.keep ? 2 : 1;
                for (int pass = 0; pass < times && go; ++pass)
                    for (uint32_t o = 0; o < bytes; o += kChunk) {
                        if (used >= (uint32_t)a.chunks &&
                            !tc::mbar_wait(&empty[slot], phase, abort, &g_err_distill, 1u)) {
                            go = false;
                            break;
                        }
                        const uint32_t n = min(bytes - o, (uint32_t)kChunk);
                        tc::mbar_arrive_expect_tx(&full[slot], n);
                        tc::bulk_load(ring + slot * kChunk, src + o, n, &full[slot]);
                        ++used;
                        if (++slot == a.chunks) {
                            slot = 0;
                            phase ^= 1;
                        }
                    }
            }
            // no copy is in flight when the block ends
            volatile int no_abort = 0;
            for (uint32_t u = used > (uint32_t)a.chunks ? used - a.chunks : 0; u < used; ++u)
                tc::mbar_wait(&full[u % a.chunks], u / a.chunks & 1, &no_abort, &g_err_distill, 1u);
        }
        __syncwarp();
    } else if (warp > kWarps) {
        // ---- the teacher's entries, rows ahead
        const float none = -INFINITY;
        const int p = warp - kWarps - 1;
        int* table = tables + p * a.table;
        uint32_t phase = 1;
        for (int r = p; r < mine; r += kAhead) {
            if (r >= kAhead) tc::mbar_wait(&tempty[p], phase, abort, &g_err_distill, 1u);
            phase ^= 1;
            __syncwarp();
            const int64_t row = first + (int64_t)r * clusters;
            const T* z = static_cast<const T*>(a.Z) + row * a.ldz;
            int* my_at = at + p * a.K;
            float *my_lp = lpk + p * a.K, *my_z = zk + p * a.K;
            float top = none;
#pragma unroll 4
            for (int k = lane; k < a.K; k += 32) {
                const int64_t i = __ldg(a.idx + row * a.ldt + k);
                const bool there = i >= 0 && i < a.V;
                const float t = there ? el::load_as(a.T, a.tkind, row * a.ldt + k) : none;
                const bool in = t != none;                    // (a NaN is)
                my_at[k] = in ? (int)i : -1;
                my_z[k] = in ? el::to_f32(z[i]) : 0.f;
                my_lp[k] = t;
                top = max_nan(top, t);
            }
            const float w = a.w ? __ldg(a.w + row) : 1.f, g = a.g ? __ldg(a.g + row) : 1.f;
            for (int e = lane; e < a.table; e += 32) table[e] = -1;
#pragma unroll
            for (int o = 16; o; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
            float s = 0.f;
            for (int k = lane; k < a.K; k += 32) s += expf((my_lp[k] - top) * it);
            s = el::warp_sum(s);
            const float ls = logf(s);
            int repeated = 0;
            __syncwarp();
            for (int k = lane; k < a.K; k += 32) {
                const int i = my_at[k];
                my_lp[k] = i < 0 ? none : fmaf(my_lp[k] - top, it, -ls);
                if (i >= 0) {
                    uint32_t h = (uint32_t)i * 2654435761u >> 16;
                    while (true) {                            // (the table has twice as many places)
                        h &= a.table - 1;
                        const int was = atomicCAS(&table[h], -1, i);
                        if (was == i) repeated = 1;
                        if (was == i || was == -1) break;
                        ++h;
                    }
                }
            }
            repeated = __any_sync(0xffffffffu, repeated);
            if (lane == 0) {
                const bool on = top != none && w != 0.f;
                teacher[p].c = on && g != 0.f ? a.tau * w * g : 0.f;
                teacher[p].lw = on ? a.tau * w : 0.f;
                teacher[p].repeated = repeated;
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&tfull[p]);
        }
    } else {
        // ---- sums and gradient
        int slot = 0;
        uint32_t phase = 0;
        // Elements outside the vectors: lanes 0 ... 7 of the first warp have those before,
        // 8 ... 15 those after; loaded a row ahead.
        int edge = -1;
        float edge_z = 0.f, edge_next = 0.f;
        auto edge_of = [&](int r, float* v) {
            if (warp != 0 || r >= mine || lane >= 16) return -1;
            const T* z = Z + (first + (int64_t)r * clusters) * a.ldz;
            const uint32_t head = head_of(z), body = (len - head) / N * N;
            const uint32_t i = lane < 8 ? lane : lane - 8 + head + body;
            if (i >= (lane < 8 ? head : (uint32_t)len)) return -1;
            *v = el::to_f32(z[i]);
            return (int)i;
        };
        int edge_at_next = edge_of(0, &edge_next);
        // Each block gives its maximum and sum of the cluster's one row to every block of
        // it.  (No block writes a gradient before all have their teacher's places' logits,
        // which may lie where it is written.)
        auto exchange = [&](float m, float s) {
            if (threadIdx.x < ranks) {
                cl::store(&all_m[rank], threadIdx.x, m);
                cl::store(&all_s[rank], threadIdx.x, s);
                cl::arrive(&got, threadIdx.x);
            }
            cl::wait(&got, 0, abort, &g_err_distill, 2u);
        };
        int ahead = -1;                      // the row's teacher entries
        uint32_t tphase = 1;
        for (int r = 0; r < mine; ++r) {
            const int p = r & 1;
            if (++ahead == kAhead) ahead = 0;
            if (ahead == 0) tphase ^= 1;
            const int64_t row = first + (int64_t)r * clusters;
            const T* z = Z + row * a.ldz;
            const uint32_t head = head_of(z);
            const int nvec = (len - head) / N;
            edge = edge_at_next;
            edge_z = edge_next;
            edge_at_next = edge_of(r + 1, &edge_next);
            const int slot0 = slot;
            // q_j = exp2((z_j - base) k2) over, with over = 1 / s, or, for a given lse that
            // base is next to tau times of, the exponential of what that leaves
            float base, over, log_s = 0.f;
            if (sums) {
                Running run;
                for (int o = 0; o < nvec; o += 2 * THREADS) {
                    tc::mbar_wait(&full[slot], phase, abort, &g_err_distill, 1u);
                    const uint4* v = reinterpret_cast<const uint4*>(ring + slot * kChunk);
                    float x[2][N];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        if (o + u * THREADS + (int)threadIdx.x < nvec) {
                            widen(v[u * THREADS + threadIdx.x], x[u], T());
                        } else {
#pragma unroll
                            for (int e = 0; e < N; ++e) x[u][e] = -INFINITY;
                        }
                    }
                    if (!(dZ && a.keep)) {
                        __syncwarp();
                        if (lane == 0) tc::mbar_arrive(&empty[slot]);
                    }
                    if (++slot == a.chunks) {
                        slot = 0;
                        phase ^= 1;
                    }
                    float top = x[0][0];
#pragma unroll
                    for (int e = 1; e < 2 * N; ++e) top = max_nan(top, x[e / N][e % N]);
                    run.raise(top, k2);
                    float s[4] = {};
                    const el::f2 less = el::pair(-run.base, -run.base);
#pragma unroll
                    for (int e = 0; e < 2 * N; e += 2) {
                        float y0, y1;
                        el::split(el::mul2(el::add2(el::pair(x[e / N][e % N], x[e / N][e % N + 1]), less), kk), y0, y1);
                        s[e & 3] += ex2(y0);
                        s[(e & 3) + 1] += ex2(y1);
                    }
                    run.s += (s[0] + s[1]) + (s[2] + s[3]);
                }
                if (edge >= 0) {
                    run.raise(edge_z, k2);
                    run.s += ex2((edge_z - run.base) * k2);
                }
                float m = run.m;
#pragma unroll
                for (int o = 16; o; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
                float s = el::warp_sum(run.m == m ? run.s : run.s * ex2((run.m - m) * k2));
                if (lane == 0) part_m[p][warp] = m, part_s[p][warp] = s;
                tc::named_bar_sync(1, THREADS);
                Running all;
#pragma unroll
                for (int i = 0; i < kWarps; ++i) all.m = max_nan(all.m, part_m[p][i]);
#pragma unroll
                for (int i = 0; i < kWarps; ++i) {
                    const float pm = part_m[p][i];
                    all.s += pm == all.m ? part_s[p][i] : part_s[p][i] * ex2((pm - all.m) * k2);
                }
                if (ranks > 1) {
                    tc::mbar_wait(&tfull[ahead], tphase, abort, &g_err_distill, 1u);
                    exchange(all.m, all.s);
                    Running both;
                    for (uint32_t i = 0; i < ranks; ++i) both.join(all_m[i], all_s[i], k2);
                    all = both;
                }
                base = base_of(all.m);
                over = __fdividef(1.f, all.s);
                log_s = logf(all.s);
                if (a.lse_out && rank == 0 && threadIdx.x == 0) a.lse_out[row] = fmaf(all.m, it, fmaf(base, it_rest, log_s));
            } else {
                if (ranks > 1) {
                    tc::mbar_wait(&tfull[ahead], tphase, abort, &g_err_distill, 1u);
                    exchange(0.f, 0.f);
                }
                const float L = __ldg(a.lse_in + row);
                base = fmaxf(fminf(L * a.tau, 3.402823466e38f), -3.402823466e38f);
                over = expf(-fmaf(L, a.tau, -base) * it);
            }
            tc::mbar_wait(&tfull[ahead], tphase, abort, &g_err_distill, 1u);
            const float c = teacher[ahead].c, cq = c * over;
            const el::f2 less = el::pair(-base, -base), cq2 = el::pair(cq, cq);
            const int* my_at = at + ahead * a.K;
            const float *my_lp = lpk + ahead * a.K, *my_z = zk + ahead * a.K;
            if (a.loss && rank == 0 && warp == 0) {
                float kl = 0.f;
                for (int k = lane; k < a.K; k += 32) {
                    const float pk = expf(my_lp[k]);
                    if (pk != 0.f) kl = fmaf(pk, my_lp[k] - fmaf(my_z[k] - base, it, -log_s), kl);
                }
                kl = el::warp_sum(kl);
                const float lw = teacher[ahead].lw;
                if (lane == 0) a.loss[row] = lw != 0.f ? lw * (a.tau * kl) : 0.f;
            }
            if (dZ) {
                T* d = dZ + row * a.lddz;
                const bool same = ((reinterpret_cast<uintptr_t>(d) ^ reinterpret_cast<uintptr_t>(z)) & 15u) == 0;
                const bool again = sums && a.keep;            // the chunks of the sum, still there
                int at_slot = again ? slot0 : slot;
                for (int o = 0; o < nvec; o += 2 * THREADS) {
                    if (!again) tc::mbar_wait(&full[at_slot], phase, abort, &g_err_distill, 1u);
                    uint4* v = reinterpret_cast<uint4*>(ring + at_slot * kChunk);
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int i = o + u * THREADS + threadIdx.x;
                        if (i < nvec) {
                            float x[N];
                            uint4 out = make_uint4(0, 0, 0, 0);
                            if (c != 0.f) {
                                widen(v[u * THREADS + threadIdx.x], x, T());
#pragma unroll
                                for (int e = 0; e < N; e += 2) {
                                    el::split(el::mul2(el::add2(el::pair(x[e], x[e + 1]), less), kk), x[e], x[e + 1]);
                                    el::split(el::mul2(el::pair(ex2(x[e]), ex2(x[e + 1])), cq2), x[e], x[e + 1]);
                                }
                                out = narrow(x, T());
                            }
                            if (same) *reinterpret_cast<uint4*>(d + head + (int64_t)i * N) = out;
                            else v[u * THREADS + threadIdx.x] = out;
                        }
                    }
                    if (!same) {
                        // a warp's vectors side by side, element by element (1021 x 50001
                        // binary16 and its gradient 66 us, where both start alike 54)
                        __syncwarp();
                        const T* from = reinterpret_cast<const T*>(v);
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const int v0 = u * THREADS + warp * 32;
                            const int n = min(nvec - (o + v0), 32) * N;
#pragma unroll 4
                            for (int e = lane; e < n; e += 32) d[head + (int64_t)(o + v0) * N + e] = from[v0 * N + e];
                        }
                        tc::fence_proxy_async_smem();         // the place's next copy comes after these writes
                    }
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(&empty[at_slot]);
                    if (++at_slot == a.chunks) {
                        at_slot = 0;
                        if (!again) phase ^= 1;
                    }
                }
                if (!again) slot = at_slot;
                if (edge >= 0) d[edge] = el::from_f32<T>(c != 0.f ? cq * ex2((edge_z - base) * k2) : 0.f);
                tc::named_bar_sync(1, THREADS);
                if (c != 0.f) {
                    for (int k = threadIdx.x; k < a.K; k += THREADS) {
                        const int64_t i = (int64_t)my_at[k] - c0;
                        if (my_at[k] < 0 || i < 0 || i >= len) continue;
                        float sum = expf(my_lp[k]);
                        if (teacher[ahead].repeated) {
                            sum = 0.f;
                            for (int o = 0; o < a.K; ++o)
                                if (my_at[o] == my_at[k]) sum += expf(my_lp[o]);
                        }
                        d[i] = el::from_f32<T>(fmaf(cq, ex2((my_z[k] - base) * k2), -c * sum));
                    }
                }
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&tempty[ahead]);
        }
    }
    if (ranks > 1) cl::sync();           // no block ends before the others have given it theirs
}

constexpr int kSmem = 216 * 1024;            // of a multiprocessor, for rings and teacher entries

template <typename T, int THREADS>
lrc_status distill_launch(Args a, int ranks, int resident, cudaStream_t s) {
    constexpr int kChunk = THREADS * 32;
    const int extra = teachers(THREADS) * 4 * (3 * a.K + a.table);
    int room = kSmem / resident - extra - (resident > 1 ? 2048 : 0);
    a.chunks = room / kChunk < kMostChunks ? room / kChunk : kMostChunks;
    const int64_t need = (a.slice * (int64_t)sizeof(T) + kChunk - 1) / kChunk;
    a.keep = need <= a.chunks;
    const int smem = a.chunks * kChunk + extra;
    auto kernel = distill_kernel<T, THREADS>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return cuda_fail(e, "distill_kernel");
    int64_t clusters = (int64_t)sm_count() * resident / ranks;
    if (clusters > a.rows) clusters = a.rows;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(clusters * ranks));
    cfg.blockDim = dim3(all_threads(THREADS));
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
    e = cudaLaunchKernelEx(&cfg, kernel, a);
    if (e != cudaSuccess) return cuda_fail(e, "distill_kernel");
    return after_launch("distill_kernel");
}

template <typename T>
lrc_status distill_as(Args a, cudaStream_t s) {
    // Few rows: a cluster of up to eight blocks each (a block for every multiprocessor at
    // most, so that each cluster has one row), of 4096 elements at least.
    // (Clusters for rows that no block can keep are slower than reading them twice, the
    // second time from L2: 215 us against 133 for 512 rows of 262144 bfloat16.)
    int ranks = 1;
    while (ranks < 8 && a.rows * ranks * 2 <= sm_count() && a.V >= ranks * 2 * 4096) ranks *= 2;
    a.slice = ((a.V + ranks - 1) / ranks + 7) / 8 * 8;
    // Rows of up to 16 KB: four small blocks on a multiprocessor, whose rows' chains
    // overlap (4096 rows of 8192 binary16: 37 us, with two 44 us); up to 98 KB: two
    // where the sum is formed (2048 rows of 32768 bfloat16: 58 us, with one 69 us), one
    // for the gradient alone (1021 x 50001 binary16: 36 us, with two 40 us).
    const int64_t bytes = a.slice * (int64_t)sizeof(T);
    if (bytes > (a.lse_in ? 48 : 98) * 1024) return distill_launch<T, 512>(a, ranks, 1, s);
    if (bytes > 16 * 1024) return distill_launch<T, 256>(a, ranks, 2, s);
    return distill_launch<T, 128>(a, ranks, 4, s);
}

}  // namespace

lrc_status launch_distill(const void* Z, const void* T, const int64_t* idx, const float* w, const float* lse_in,
                          const float* g, float* loss, float* lse_out, void* dZ, int64_t rows, int64_t V, int64_t K,
                          int64_t ldz, int64_t ldt, int64_t lddz, float tau, lrc_fmt fmt, lrc_fmt tfmt, cudaStream_t s) {
    Args a{};
    a.Z = Z;
    a.T = T;
    a.idx = idx;
    a.w = w;
    a.lse_in = lse_in;
    a.g = g;
    a.loss = loss;
    a.lse_out = lse_out;
    a.dZ = dZ;
    a.rows = rows;
    a.V = V;
    a.ldz = ldz;
    a.ldt = ldt;
    a.lddz = lddz;
    a.K = (int)K;
    a.table = 64;
    while (a.table < 2 * K) a.table *= 2;
    a.tau = tau;
    a.tkind = tfmt == LRC_F32 ? 0 : tfmt == LRC_BF16 ? 2 : 1;
    if (fmt == LRC_F32) return distill_as<float>(a, s);
    if (fmt == LRC_BF16) return distill_as<bf16>(a, s);
    return distill_as<__half>(a, s);
}

int distill_max_top() { return kMaxTop; }

uint32_t take_distill_error() {
    unsigned int v = 0;
    if (cudaMemcpyFromSymbol(&v, g_err_distill, sizeof v) != cudaSuccess) return 0xffffffffu;
    if (v) {
        const unsigned int z = 0;
        cudaMemcpyToSymbol(g_err_distill, &z, sizeof z);
    }
    return v;
}

}  // namespace lrc
