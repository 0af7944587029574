// out[i][j] = sum over k of a[i][k] b[j][k] (+ add[i][j]) of two microscaled 4-bit matrices.
#include "uq_mx.cuh"

namespace uq {
namespace {

constexpr int kPThreads = 256;

// A tile of 64 x 64 per CTA; one block of 32 columns of both operands at a time as binary32 in shared memory, 4 x 4 sums a thread.
template <int DT>
__global__ void __launch_bounds__(kPThreads) product_kernel(uq_mx a, uq_mx b, const void *add, int64_t add_ld, void *out, int64_t ld)
{
    __shared__ float as[32][68], bs[32][68];
    grid_dependency_prologue();
    const int64_t across = (b.rows + 63) / 64, i0 = blockIdx.x / across * 64, j0 = blockIdx.x % across * 64, nb = mx_blocks(a.cols), kt = mx_ktiles(a.cols);
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    float sum[4][4] = {};
    for (int64_t blk = 0; blk < nb; ++blk) {
        const int r = tid >> 2, part = tid & 3;
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const uq_mx &m = side ? b : a;
            const int64_t row = (side ? j0 : i0) + r;
            uint32_t codes = 0;
            float scale = 0.0f;
            if (row < m.rows) {
                codes = __ldg((const uint32_t *)(m.codes + row * m.code_stride + blk * 16 + part * 4));
                scale = mx_scale_value(__ldg(m.scales + mx_scale_at(row, blk, kt)));
            }
#pragma unroll
            for (int t = 0; t < 8; ++t) (side ? bs : as)[part * 8 + t][r] = mx_code_value(codes >> (4 * t)) * scale;
        }
        __syncthreads();
#pragma unroll 8
        for (int k = 0; k < 32; ++k) {
            float u[4], w[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) { u[t] = as[k][ty * 4 + t]; w[t] = bs[k][tx * 4 + t]; }
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int t = 0; t < 4; ++t) sum[p][t] = __fmaf_rn(u[p], w[t], sum[p][t]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int64_t i = i0 + ty * 4 + p, j = j0 + tx * 4 + t;
            if (i < a.rows && j < b.rows) {
                float v = sum[p][t];
                if (add != nullptr) {
                    if constexpr (DT == UQ_BF16) v += __uint_as_float((uint32_t)((const unsigned short *)add)[i * add_ld + j] << 16);
                    else v += ((const float *)add)[i * add_ld + j];
                }
                store1<DT>(out, i * ld + j, v);
            }
        }
}

}  // namespace

cudaError_t launch_mx_product(const uq_mx &a, const uq_mx &b, const void *add, int64_t add_ld, void *out, int64_t ld, int dtype,
                              uint32_t *status, cudaStream_t st)
{
    (void)status;
    const dim3 grid((unsigned)((b.rows + 63) / 64 * ((a.rows + 63) / 64)));
    if (dtype == UQ_BF16) launch_k(product_kernel<UQ_BF16>, grid, dim3(kPThreads), st, a, b, add, add_ld, out, ld);
    else launch_k(product_kernel<UQ_F32>, grid, dim3(kPThreads), st, a, b, add, add_ld, out, ld);
    return cudaGetLastError();
}

}  // namespace uq
