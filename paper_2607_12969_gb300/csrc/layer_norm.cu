// layer_norm.cu -- layer norm of rows and its gradient (lrc_layer_norm,
// lrc_layer_norm_grad), binary32 arithmetic.
#include "common.cuh"
#include "elem.cuh"

namespace lrc {
namespace {

using bf16 = __nv_bfloat16;

constexpr int kThreads = 256;

// Sum over the block, in every thread.
__device__ __forceinline__ float block_sum(float x, float* sh) {
    x = el::warp_sum(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
    __syncthreads();
    x = 0.f;
    for (int i = 0; i < (int)blockDim.x / 32; ++i) x += sh[i];
    return x;
}

template <typename X, typename Y>
__global__ void __launch_bounds__(kThreads)
norm_kernel(const X* x, const void* gamma, const void* beta, int pk, Y* y, float* mean, float* rstd, int64_t cols,
            int64_t ldx, int64_t ldy, float eps) {
    __shared__ float sh[kThreads / 32];
    const X* xr = x + (int64_t)blockIdx.x * ldx;
    Y* yr = y + (int64_t)blockIdx.x * ldy;
    float s = 0.f;
    for (int64_t c = threadIdx.x; c < cols; c += kThreads) s += el::to_f32(xr[c]);
    const float mu = block_sum(s, sh) / (float)cols;
    s = 0.f;
    for (int64_t c = threadIdx.x; c < cols; c += kThreads) {
        const float d = el::to_f32(xr[c]) - mu;
        s = fmaf(d, d, s);
    }
    const float r = 1.f / sqrtf(block_sum(s, sh) / (float)cols + eps);
    for (int64_t c = threadIdx.x; c < cols; c += kThreads) {
        const float g = gamma ? el::load_as(gamma, pk, c) : 1.f, b = beta ? el::load_as(beta, pk, c) : 0.f;
        yr[c] = el::from_f32<Y>(fmaf((el::to_f32(xr[c]) - mu) * r, g, b));
    }
    if (threadIdx.x == 0) {
        if (mean) mean[blockIdx.x] = mu;
        if (rstd) rstd[blockIdx.x] = r;
    }
}

// Partial column sums over the rows blockIdx.y, blockIdx.y + gridDim.y, ...:
// part[2 y][c] of dy xh, part[2 y + 1][c] of dy.
template <typename X, typename Y>
__global__ void __launch_bounds__(kThreads)
norm_columns_kernel(const Y* dy, const X* x, const float* mean, const float* rstd, int64_t rows, int64_t cols,
                    int64_t lddy, int64_t ldx, float* part) {
    const int64_t c = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (c >= cols) return;
    float g = 0.f, b = 0.f;
    for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
        const float d = el::to_f32(dy[r * lddy + c]);
        g = fmaf(d, (el::to_f32(x[r * ldx + c]) - mean[r]) * rstd[r], g);
        b += d;
    }
    part[(int64_t)blockIdx.y * 2 * cols + c] = g;
    part[((int64_t)blockIdx.y * 2 + 1) * cols + c] = b;
}

__global__ void __launch_bounds__(kThreads)
norm_columns_sum_kernel(const float* part, int parts, int64_t cols, float* dgamma, float* dbeta) {
    const int64_t c = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (c >= cols) return;
    float g = 0.f, b = 0.f;
    for (int p = 0; p < parts; ++p) {
        g += part[(int64_t)p * 2 * cols + c];
        b += part[((int64_t)p * 2 + 1) * cols + c];
    }
    if (dgamma) dgamma[c] = g;
    if (dbeta) dbeta[c] = b;
}

template <typename X, typename Y>
__global__ void __launch_bounds__(kThreads)
norm_grad_kernel(const Y* dy, const X* x, const void* gamma, int pk, const float* mean, const float* rstd, X* dx,
                 int64_t cols, int64_t lddy, int64_t ldx, int64_t lddx) {
    __shared__ float sh[kThreads / 32];
    const Y* dr = dy + (int64_t)blockIdx.x * lddy;
    const X* xr = x + (int64_t)blockIdx.x * ldx;
    X* o = dx + (int64_t)blockIdx.x * lddx;
    const float mu = mean[blockIdx.x], r = rstd[blockIdx.x];
    float s = 0.f, t = 0.f;
    for (int64_t c = threadIdx.x; c < cols; c += kThreads) {
        const float d = el::to_f32(dr[c]) * (gamma ? el::load_as(gamma, pk, c) : 1.f);
        s += d;
        t = fmaf(d, (el::to_f32(xr[c]) - mu) * r, t);
    }
    s = block_sum(s, sh) / (float)cols;
    t = block_sum(t, sh) / (float)cols;
    for (int64_t c = threadIdx.x; c < cols; c += kThreads) {
        const float d = el::to_f32(dr[c]) * (gamma ? el::load_as(gamma, pk, c) : 1.f);
        o[c] = el::from_f32<X>(r * (d - s - (el::to_f32(xr[c]) - mu) * r * t));
    }
}

int kind_of(lrc_fmt f) { return f == LRC_F32 ? 0 : f == LRC_BF16 ? 2 : 1; }

template <typename X, typename Y>
lrc_status norm_as(const void* x, const void* gamma, const void* beta, void* y, float* mean, float* rstd, int64_t rows,
                   int64_t cols, int64_t ldx, int64_t ldy, float eps, int pk, cudaStream_t s) {
    norm_kernel<X, Y><<<(unsigned)rows, kThreads, 0, s>>>((const X*)x, gamma, beta, pk, (Y*)y, mean, rstd, cols, ldx, ldy,
                                                          eps);
    return after_launch("norm_kernel");
}

template <typename X, typename Y>
lrc_status norm_grad_as(const void* dy, const void* x, const void* gamma, const float* mean, const float* rstd, void* dx,
                        float* dgamma, float* dbeta, int64_t rows, int64_t cols, int64_t lddy, int64_t ldx, int64_t lddx,
                        int pk, cudaStream_t s) {
    const int64_t slabs = (cols + kThreads - 1) / kThreads;
    if (slabs > 0x7fffffff) {
        set_error("lrc_layer_norm_grad: cols too large");
        return LRC_ERR_UNSUPPORTED;
    }
    lrc_status st;
    if (dgamma || dbeta) {
        const int parts = rows < 128 ? (int)rows : 128;
        void* ws = nullptr;
        if ((st = stream_workspace(s, (size_t)(parts ? parts : 1) * 2 * cols * 4, &ws)) != LRC_OK) return st;
        if (parts) {
            norm_columns_kernel<X, Y><<<dim3((unsigned)slabs, parts), kThreads, 0, s>>>(
                (const Y*)dy, (const X*)x, mean, rstd, rows, cols, lddy, ldx, (float*)ws);
            if ((st = after_launch("norm_columns_kernel")) != LRC_OK) return st;
        }
        norm_columns_sum_kernel<<<(unsigned)slabs, kThreads, 0, s>>>((const float*)ws, parts, cols, dgamma, dbeta);
        if ((st = after_launch("norm_columns_sum_kernel")) != LRC_OK) return st;
    }
    if (dx && rows) {
        norm_grad_kernel<X, Y><<<(unsigned)rows, kThreads, 0, s>>>((const Y*)dy, (const X*)x, gamma, pk, mean, rstd,
                                                                   (X*)dx, cols, lddy, ldx, lddx);
        return after_launch("norm_grad_kernel");
    }
    return LRC_OK;
}

}  // namespace

lrc_status launch_layer_norm(const void* X, const void* gamma, const void* beta, void* Y, float* mean, float* rstd,
                             int64_t rows, int64_t cols, int64_t ldx, int64_t ldy, float eps, lrc_fmt fmt, lrc_fmt pfmt,
                             cudaStream_t s) {
    const int pk = kind_of(pfmt);
    if (fmt == LRC_F32) return norm_as<float, float>(X, gamma, beta, Y, mean, rstd, rows, cols, ldx, ldy, eps, pk, s);
    if (fmt == LRC_BF16) return norm_as<bf16, bf16>(X, gamma, beta, Y, mean, rstd, rows, cols, ldx, ldy, eps, pk, s);
    if (fmt == LRC_F16) return norm_as<__half, float>(X, gamma, beta, Y, mean, rstd, rows, cols, ldx, ldy, eps, pk, s);
    return norm_as<__half, __half>(X, gamma, beta, Y, mean, rstd, rows, cols, ldx, ldy, eps, pk, s);
}

lrc_status launch_layer_norm_grad(const void* dY, const void* X, const void* gamma, const float* mean, const float* rstd,
                                  void* dX, float* dgamma, float* dbeta, int64_t rows, int64_t cols, int64_t lddy,
                                  int64_t ldx, int64_t lddx, lrc_fmt fmt, lrc_fmt pfmt, cudaStream_t s) {
    const int pk = kind_of(pfmt);
    auto go = [&](auto x, auto y) {
        return norm_grad_as<decltype(x), decltype(y)>(dY, X, gamma, mean, rstd, dX, dgamma, dbeta, rows, cols, lddy, ldx,
                                                      lddx, pk, s);
    };
    if (fmt == LRC_F32) return go(float(), float());
    if (fmt == LRC_BF16) return go(bf16(), bf16());
    if (fmt == LRC_F16) return go(__half(), float());
    return go(__half(), __half());
}

}  // namespace lrc
