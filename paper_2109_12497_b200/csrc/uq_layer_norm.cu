// Layer norm over the rows of a matrix, forward (optionally with the result quantized to microscaled 4-bit values on the way
// out) and backward (with the reduction of the weight's and the bias's gradient over all rows).
//
//   mean = sum x / n    var = sum (x - mean)^2 / n    rstd = 1 / sqrt(var + eps)    y = (x - mean) rstd gamma + beta
//   xh = (x - mean) rstd    t = dy gamma    dx = rstd (t - sum t / n - xh sum (t xh) / n)
//   dgamma = sum over rows of dy xh         dbeta = sum over rows of dy
//
// Everything is held in binary32; a result is rounded once, to the type of its array.
#include "uq_mx.cuh"

namespace uq {
namespace {

constexpr int kLnThreads = 256;
constexpr int kLnGrid = 296;                    // partial sums of the weight's gradient: two CTAs per SM

// The sum over a CTA, the same in every thread, in an order that depends only on the launch's shape.
__device__ __forceinline__ float cta_sum(float v, float *scratch)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    __syncthreads();
    if (lane == 0) scratch[warp] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kLnThreads / 32; ++w) s += scratch[w];
    return s;
}

template <int DT>
__global__ void __launch_bounds__(kLnThreads) layer_norm_kernel(const void *__restrict__ x, int64_t rows, int64_t cols, int64_t ld,
                                                                const float *__restrict__ gamma, const float *__restrict__ beta, float eps,
                                                                void *__restrict__ y, int64_t y_ld, float *mean_out, float *rstd_out,
                                                                uq_mx q, uint32_t *status)
{
    __shared__ float scratch[kLnThreads / 32];
    grid_dependency_prologue();
    const bool wide = ((uintptr_t)x & 15) == 0 && (ld * Elem<DT>::BYTES & 15) == 0;
    const bool wide_y = ((uintptr_t)y & 15) == 0 && (y_ld * Elem<DT>::BYTES & 15) == 0;
    const int64_t chunks = (cols + 7) >> 3;
    const int64_t all = q.codes != nullptr ? mx_ktiles(cols) * 16 : (chunks + 31) / 32 * 32;
    const float n = (float)cols;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        float s = 0.0f;
        for (int64_t c = threadIdx.x; c < chunks; c += kLnThreads) {
            float v[8];
            load8<DT>(x, row * ld + c * 8, (int)min((int64_t)8, cols - c * 8), wide, v);
#pragma unroll
            for (int t = 0; t < 8; ++t) s += v[t];
        }
        const float mean = cta_sum(s, scratch) / n;
        s = 0.0f;
        for (int64_t c = threadIdx.x; c < chunks; c += kLnThreads) {
            float v[8];
            const int have = (int)min((int64_t)8, cols - c * 8);
            load8<DT>(x, row * ld + c * 8, have, wide, v);
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const float d = t < have ? v[t] - mean : 0.0f;
                s = __fmaf_rn(d, d, s);
            }
        }
        const float rstd = 1.0f / sqrtf(cta_sum(s, scratch) / n + eps);
        if (threadIdx.x == 0) {
            if (mean_out != nullptr) mean_out[row] = mean;
            if (rstd_out != nullptr) rstd_out[row] = rstd;
        }
        for (int64_t c0 = threadIdx.x & ~31; c0 < all; c0 += kLnThreads) {
            const int64_t c = c0 + (threadIdx.x & 31);
            const int have = (int)max((int64_t)0, min((int64_t)8, cols - c * 8));
            float v[8];
            load8<DT>(x, row * ld + c * 8, have, wide, v);
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                if (t < have) {
                    v[t] = (v[t] - mean) * rstd;
                    if (gamma != nullptr) v[t] *= __ldg(gamma + c * 8 + t);
                    if (beta != nullptr) v[t] += __ldg(beta + c * 8 + t);
                }
            }
            if (y != nullptr) store8<DT>(y, row * y_ld + c * 8, have, wide_y, v);
            if (q.codes != nullptr) {
                if constexpr (DT == UQ_BF16) {
#pragma unroll
                    for (int t = 0; t < 8; ++t) v[t] = __uint_as_float(bf16_bits(v[t]) << 16);
                }
                uint32_t m = max_abs_bits(v);
                m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
                m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
                const uint32_t byte = mx_scale_byte(m);
                uint32_t codes = 0;
                if (byte != 255u) {
                    const float inv = mx_inverse(byte);
#pragma unroll
                    for (int t = 0; t < 8; ++t) v[t] *= inv;
                    codes = e2m1x8_nearest(v);
                } else if (status != nullptr) {
                    atomicOr(status, UQ_STATUS_NONFINITE);
                }
                if (c < mx_blocks(cols) * 4) *(uint32_t *)(q.codes + row * q.code_stride + c * 4) = codes;
                if ((c & 3) == 0 && c < all) q.scales[mx_scale_at(row, c >> 2, mx_ktiles(cols))] = (uint8_t)byte;
            }
        }
    }
}

// A CTA takes every gridDim.x-th row; its sums for dgamma and dbeta are a row pair of `partial`, a thread's columns its own.
template <int DT>
__global__ void __launch_bounds__(kLnThreads) layer_norm_backward_kernel(const void *__restrict__ dy, int64_t dy_ld,
                                                                         const void *__restrict__ x, int64_t x_ld, int64_t rows, int64_t cols,
                                                                         const float *__restrict__ gamma, const float *__restrict__ mean_in,
                                                                         const float *__restrict__ rstd_in, void *__restrict__ dx,
                                                                         int64_t dx_ld, float *__restrict__ partial)
{
    __shared__ float scratch[kLnThreads / 32];
    grid_dependency_prologue();
    const bool wide_dy = ((uintptr_t)dy & 15) == 0 && (dy_ld * Elem<DT>::BYTES & 15) == 0;
    const bool wide_x = ((uintptr_t)x & 15) == 0 && (x_ld * Elem<DT>::BYTES & 15) == 0;
    const bool wide_dx = ((uintptr_t)dx & 15) == 0 && (dx_ld * Elem<DT>::BYTES & 15) == 0;
    const int64_t chunks = (cols + 7) >> 3;
    const float n = (float)cols;
    float *pg = partial + (int64_t)blockIdx.x * 2 * cols, *pb = pg + cols;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const float mean = __ldg(mean_in + row), rstd = __ldg(rstd_in + row);
        float s1 = 0.0f, s2 = 0.0f;
        for (int64_t c = threadIdx.x; c < chunks; c += kLnThreads) {
            const int have = (int)min((int64_t)8, cols - c * 8);
            float d[8], v[8];
            load8<DT>(dy, row * dy_ld + c * 8, have, wide_dy, d);
            load8<DT>(x, row * x_ld + c * 8, have, wide_x, v);
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                if (t < have) {
                    const float xh = (v[t] - mean) * rstd, g = gamma != nullptr ? d[t] * __ldg(gamma + c * 8 + t) : d[t];
                    s1 += g;
                    s2 = __fmaf_rn(g, xh, s2);
                }
            }
        }
        const float m1 = cta_sum(s1, scratch) / n, m2 = cta_sum(s2, scratch) / n;
        const bool first = row == blockIdx.x;
        for (int64_t c = threadIdx.x; c < chunks; c += kLnThreads) {
            const int have = (int)min((int64_t)8, cols - c * 8);
            float d[8], v[8];
            load8<DT>(dy, row * dy_ld + c * 8, have, wide_dy, d);
            load8<DT>(x, row * x_ld + c * 8, have, wide_x, v);
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                if (t < have) {
                    const int64_t i = c * 8 + t;
                    const float xh = (v[t] - mean) * rstd, g = gamma != nullptr ? d[t] * __ldg(gamma + i) : d[t];
                    pg[i] = first ? d[t] * xh : __fmaf_rn(d[t], xh, pg[i]);
                    pb[i] = first ? d[t] : pb[i] + d[t];
                    v[t] = rstd * (g - m1 - xh * m2);
                }
            }
            if (dx != nullptr) store8<DT>(dx, row * dx_ld + c * 8, have, wide_dx, v);
        }
    }
}

// The partial sums of all CTAs, in their order.
template <int GT>
__global__ void __launch_bounds__(kLnThreads) weight_gradient_kernel(const float *__restrict__ partial, int parts, int64_t cols, void *dgamma,
                                                                     void *dbeta)
{
    grid_dependency_prologue();
    const int64_t c = (int64_t)blockIdx.x * kLnThreads + threadIdx.x;
    if (c >= cols) return;
    float g = 0.0f, b = 0.0f;
    for (int p = 0; p < parts; ++p) {
        g += partial[(int64_t)p * 2 * cols + c];
        b += partial[(int64_t)p * 2 * cols + cols + c];
    }
    if (dgamma != nullptr) store1<GT>(dgamma, c, g);
    if (dbeta != nullptr) store1<GT>(dbeta, c, b);
}

int backward_parts(int64_t rows) { return (int)min(rows, (int64_t)kLnGrid); }

}  // namespace

size_t layer_norm_workspace_bytes(int64_t rows, int64_t cols) { return (size_t)backward_parts(rows) * 2 * cols * sizeof(float); }

cudaError_t launch_layer_norm(const void *x, int64_t rows, int64_t cols, int64_t ld, int dtype, const float *gamma, const float *beta,
                              float eps, void *y, int64_t y_ld, float *mean, float *rstd, const uq_mx &q, uint32_t *status,
                              cudaStream_t st)
{
    const dim3 grid((unsigned)min(rows, (int64_t)148 * 8));
    if (dtype == UQ_BF16)
        launch_k(layer_norm_kernel<UQ_BF16>, grid, dim3(kLnThreads), st, x, rows, cols, ld, gamma, beta, eps, y, y_ld, mean, rstd, q, status);
    else
        launch_k(layer_norm_kernel<UQ_F32>, grid, dim3(kLnThreads), st, x, rows, cols, ld, gamma, beta, eps, y, y_ld, mean, rstd, q, status);
    return cudaGetLastError();
}

cudaError_t launch_layer_norm_backward(const void *dy, int64_t dy_ld, const void *x, int64_t x_ld, int64_t rows, int64_t cols, int dtype,
                                       const float *gamma, const float *mean, const float *rstd, void *dx, int64_t dx_ld, void *dgamma,
                                       void *dbeta, int grad_dtype, void *workspace, cudaStream_t st)
{
    const int parts = backward_parts(rows);
    float *partial = (float *)workspace;
    if (rows > 0) {
        if (dtype == UQ_BF16)
            launch_k(layer_norm_backward_kernel<UQ_BF16>, dim3(parts), dim3(kLnThreads), st, dy, dy_ld, x, x_ld, rows, cols, gamma, mean, rstd,
                     dx, dx_ld, partial);
        else
            launch_k(layer_norm_backward_kernel<UQ_F32>, dim3(parts), dim3(kLnThreads), st, dy, dy_ld, x, x_ld, rows, cols, gamma, mean, rstd,
                     dx, dx_ld, partial);
        if (cudaError_t e = cudaGetLastError()) return e;
    }
    if (dgamma == nullptr && dbeta == nullptr) return cudaSuccess;
    const dim3 grid((unsigned)((cols + kLnThreads - 1) / kLnThreads));
    if (grad_dtype == UQ_BF16) launch_k(weight_gradient_kernel<UQ_BF16>, grid, dim3(kLnThreads), st, (const float *)partial, parts, cols, dgamma, dbeta);
    else launch_k(weight_gradient_kernel<UQ_F32>, grid, dim3(kLnThreads), st, (const float *)partial, parts, cols, dgamma, dbeta);
    return cudaGetLastError();
}

}  // namespace uq
