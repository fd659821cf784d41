// distill.cu -- distillation from a teacher's top logits (lrc_distill,
// lrc_distill_grad), binary32 arithmetic.
//
// With z' = z / tau, the row's log-sum-exp L and the teacher's p:
//   loss = tau^2 w sum_k p_k (log p_k - (z'_{i_k} - L)),
//   dz_j = tau w g (exp(z'_j - L) - sum over k with i_k = j of p_k).
#include "common.cuh"
#include "elem.cuh"

namespace lrc {
namespace {

using bf16 = __nv_bfloat16;

constexpr int kThreads = 256;
constexpr int kMaxTop = 1024;

__device__ __forceinline__ float block_all(float x, float* sh, bool maximum) {
    x = maximum ? el::warp_max(x) : el::warp_sum(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
    __syncthreads();
    x = sh[0];
    for (int i = 1; i < (int)blockDim.x / 32; ++i) x = maximum ? fmaxf(x, sh[i]) : x + sh[i];
    return x;
}

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
    int64_t V, K, ldz, ldt, lddz;
    float tau;
    int tkind;
};

// One block a row.
template <typename T>
__global__ void __launch_bounds__(kThreads) distill_kernel(Args a) {
    __shared__ float sh[kThreads / 32];
    __shared__ float p[kMaxTop];
    __shared__ int64_t at[kMaxTop];
    const int64_t row = blockIdx.x;
    const T* z = static_cast<const T*>(a.Z) + row * a.ldz;
    const float it = 1.f / a.tau;
    // the row's log-sum-exp
    float L;
    if (a.lse_in) {
        L = a.lse_in[row];
    } else {
        float top = -INFINITY;
        bool odd = false;
        for (int64_t j = threadIdx.x; j < a.V; j += kThreads) {
            const float v = el::to_f32(z[j]);
            odd |= v != v;
            top = fmaxf(top, v);
        }
        top = block_all(top, sh, true);
        const float m = top == -INFINITY ? 0.f : top;
        float s = 0.f;
        for (int64_t j = threadIdx.x; j < a.V; j += kThreads) s += expf((el::to_f32(z[j]) - m) * it);
        s = block_all(odd ? NAN : s, sh, false);
        L = m * it + logf(s);
        if (a.lse_out && threadIdx.x == 0) a.lse_out[row] = L;
    }
    // the teacher's probabilities
    float tt = -INFINITY;
    for (int64_t k = threadIdx.x; k < a.K; k += kThreads) {
        const int64_t i = a.idx[row * a.ldt + k];
        const bool there = i >= 0 && i < a.V;
        at[k] = there ? i : -1;
        p[k] = there ? el::load_as(a.T, a.tkind, row * a.ldt + k) * it : -INFINITY;
        tt = fmaxf(tt, p[k] != p[k] ? INFINITY : p[k]);
    }
    tt = block_all(tt, sh, true);
    const float w = a.w ? a.w[row] : 1.f;
    const float up = a.g ? a.g[row] : 1.f;
    const bool on = tt > -INFINITY && w != 0.f;
    float s = 0.f;
    for (int64_t k = threadIdx.x; k < a.K; k += kThreads) s += expf(p[k] - tt);
    s = block_all(s, sh, false);
    const float lt = tt + logf(s);
    float kl = 0.f;
    for (int64_t k = threadIdx.x; k < a.K; k += kThreads) {
        const float lp = p[k] - lt, q = expf(lp);
        if (q != 0.f) kl += q * (lp - (el::to_f32(z[at[k] < 0 ? 0 : at[k]]) * it - L));
        p[k] = q;
    }
    kl = block_all(kl, sh, false);
    if (a.loss && threadIdx.x == 0) a.loss[row] = on ? a.tau * a.tau * w * kl : 0.f;
    if (!a.dZ) return;
    T* d = static_cast<T*>(a.dZ) + row * a.lddz;
    const float c = on && up != 0.f ? a.tau * w * up : 0.f;
    // the places of the teacher's entries are kept apart: d may be z
    constexpr int kEach = kMaxTop / kThreads;
    float mine[kEach];
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const int64_t k = threadIdx.x + u * kThreads;
        mine[u] = 0.f;
        if (c != 0.f && k < a.K && at[k] >= 0) {
            float sum = 0.f;
            for (int64_t o = 0; o < a.K; ++o)
                if (at[o] == at[k]) sum += p[o];
            mine[u] = c * (expf(el::to_f32(z[at[k]]) * it - L) - sum);
        }
    }
    __syncthreads();
    for (int64_t j = threadIdx.x; j < a.V; j += kThreads)
        d[j] = el::from_f32<T>(c != 0.f ? c * expf(el::to_f32(z[j]) * it - L) : 0.f);
    __syncthreads();
    if (c != 0.f) {
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            const int64_t k = threadIdx.x + u * kThreads;
            if (k < a.K && at[k] >= 0) d[at[k]] = el::from_f32<T>(mine[u]);
        }
    }
}

}  // namespace

lrc_status launch_distill(const void* Z, const void* T, const int64_t* idx, const float* w, const float* lse_in,
                          const float* g, float* loss, float* lse_out, void* dZ, int64_t rows, int64_t V, int64_t K,
                          int64_t ldz, int64_t ldt, int64_t lddz, float tau, lrc_fmt fmt, lrc_fmt tfmt, cudaStream_t s) {
    Args a{Z, T, idx, w, lse_in, g, loss, lse_out, dZ, V, K, ldz, ldt, lddz, tau,
           tfmt == LRC_F32 ? 0 : tfmt == LRC_BF16 ? 2 : 1};
    if (fmt == LRC_F32) distill_kernel<float><<<(unsigned)rows, kThreads, 0, s>>>(a);
    else if (fmt == LRC_BF16) distill_kernel<bf16><<<(unsigned)rows, kThreads, 0, s>>>(a);
    else distill_kernel<__half><<<(unsigned)rows, kThreads, 0, s>>>(a);
    return after_launch("distill_kernel");
}

int distill_max_top() { return kMaxTop; }

}  // namespace lrc
