// Microscaled 4-bit quantization of a matrix with blocks along its rows, along its columns (the transposed matrix), or both
// from one read, and the values that codes stand for.
//
// A CTA owns a tile of 128 x 128 values: that is one scale tile of either orientation (512 contiguous bytes), and 64
// contiguous bytes of every row of codes.  Rows: 16 lanes hold a row's 128 values, eight each; four lanes are a block, whose
// largest magnitude two shuffles find.  Columns: the tile (and the draws, made once per eight values of a row and used in both
// orientations) is kept in shared memory and read back two columns per lane.
#include "uq_mx.cuh"

namespace uq {
namespace {

constexpr int kQThreads = 256;

template <int DT> struct TileWord;                        // two neighbouring columns of a row in shared memory
template <> struct TileWord<UQ_BF16> { using T = uint32_t; };
template <> struct TileWord<UQ_F32> { using T = uint2; };

__device__ __forceinline__ float lo_of(uint32_t w) { return bf16lo(w); }
__device__ __forceinline__ float hi_of(uint32_t w) { return bf16hi(w); }
__device__ __forceinline__ float lo_of(uint2 w) { return __uint_as_float(w.x); }
__device__ __forceinline__ float hi_of(uint2 w) { return __uint_as_float(w.y); }

// Word (two columns) `c2` of row `r` of a tile in shared memory; eight words between groups of 32 rows keep the lanes of a
// column pass (8 column pairs x 4 blocks) on different banks.
__device__ __forceinline__ int tile_at(int r, int c2) { return r * 64 + (r >> 5) * 8 + c2; }
constexpr int kTileWords = 128 * 64 + 4 * 8;

template <int DT, bool SR>
__global__ void __launch_bounds__(kQThreads) quantize_tile_kernel(const void *__restrict__ x, int64_t rows, int64_t cols, int64_t ld,
                                                                  PhiloxKey key, uq_mx q, uq_mx qt, uint32_t *status)
{
    using Word = typename TileWord<DT>::T;
    extern __shared__ __align__(16) unsigned char smem[];
    Word *tile = (Word *)smem;
    uint32_t *draws = (uint32_t *)(smem + sizeof(Word) * kTileWords);
    grid_dependency_prologue();
    const int64_t ktq = mx_ktiles(cols), ktt = mx_ktiles(rows);
    const int64_t r0 = blockIdx.x / ktq * kMxTile, c0 = blockIdx.x % ktq * kMxTile;
    const int tid = threadIdx.x, lane = tid & 31;
    const bool wide = ((uintptr_t)x & 15) == 0 && (ld * Elem<DT>::BYTES & 15) == 0;
    const bool along_rows = q.codes != nullptr, along_cols = qt.codes != nullptr;
    bool bad = false;

    const int chunk = tid & 15;                           // eight columns
    const int64_t c = c0 + chunk * 8;
    const int have = (int)min((int64_t)8, max((int64_t)0, cols - c));
#pragma unroll 2
    for (int r = tid >> 4; r < kMxTile; r += kQThreads / 16) {
        const int64_t row = r0 + r;
        const bool in = row < rows;
        float v[8];
        load8<DT>(x, row * ld + c, in ? have : 0, wide, v);
        uint4 h = make_uint4(0, 0, 0, 0);
        if constexpr (SR) h = philox4x32_10(key, (uint32_t)(c >> 3), (uint32_t)row, 0u, kMxTag);
        if (along_cols) {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                Word w;
                if constexpr (DT == UQ_BF16) w = (__float_as_uint(v[2 * t]) >> 16) | (__float_as_uint(v[2 * t + 1]) & 0xFFFF0000u);
                else w = make_uint2(__float_as_uint(v[2 * t]), __float_as_uint(v[2 * t + 1]));
                tile[tile_at(r, chunk * 4 + t)] = w;
            }
            if constexpr (SR) {
                uint32_t *d = draws + tile_at(r, chunk * 4);
                d[0] = h.x; d[1] = h.y; d[2] = h.z; d[3] = h.w;
            }
        }
        if (along_rows) {
            uint32_t m = max_abs_bits(v);
            m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
            m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
            const uint32_t byte = mx_scale_byte(m);
            uint32_t codes = 0;
            if (byte != 255u) {
                const float inv = mx_inverse(byte);
#pragma unroll
                for (int t = 0; t < 8; ++t) v[t] *= inv;
                if constexpr (SR) codes = e2m1x8_stochastic(v, h);
                else codes = e2m1x8_nearest(v);
            } else {
                bad = true;
            }
            if (in && c < mx_blocks(cols) * 32) *(uint32_t *)(q.codes + row * q.code_stride + (c >> 1)) = codes;
            if ((lane & 3) == 0) q.scales[mx_scale_at(row, c >> 5, ktq)] = (uint8_t)(in ? byte : 0u);
        }
    }
    if (along_cols) {
        __syncthreads();
        const int block = (tid >> 3) & 3, pair = (tid >> 5) * 8 + (tid & 7);
        uint32_t m0 = 0, m1 = 0;
#pragma unroll 8
        for (int t = 0; t < 32; ++t) {
            const Word w = tile[tile_at(block * 32 + t, pair)];
            m0 = max(m0, abs_bits(lo_of(w)));
            m1 = max(m1, abs_bits(hi_of(w)));
        }
        const uint32_t b0 = mx_scale_byte(m0), b1 = mx_scale_byte(m1);
        const float inv0 = b0 == 255u ? 0.0f : mx_inverse(b0), inv1 = b1 == 255u ? 0.0f : mx_inverse(b1);
        bad = bad || b0 == 255u || b1 == 255u;
        uint32_t out0[4], out1[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float v0[8], v1[8];
            uint32_t h[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const int at = tile_at(block * 32 + g * 8 + t, pair);
                const Word w = tile[at];
                v0[t] = lo_of(w) * inv0;
                v1[t] = hi_of(w) * inv1;
                if constexpr (SR) h[t] = draws[at];
            }
            if constexpr (SR) {
                uint4 e, o;
                e.x = __byte_perm(h[0], h[1], 0x5410); o.x = __byte_perm(h[0], h[1], 0x7632);
                e.y = __byte_perm(h[2], h[3], 0x5410); o.y = __byte_perm(h[2], h[3], 0x7632);
                e.z = __byte_perm(h[4], h[5], 0x5410); o.z = __byte_perm(h[4], h[5], 0x7632);
                e.w = __byte_perm(h[6], h[7], 0x5410); o.w = __byte_perm(h[6], h[7], 0x7632);
                out0[g] = e2m1x8_stochastic(v0, e);
                out1[g] = e2m1x8_stochastic(v1, o);
            } else {
                out0[g] = e2m1x8_nearest(v0);
                out1[g] = e2m1x8_nearest(v1);
            }
            if (b0 == 255u) out0[g] = 0;
            if (b1 == 255u) out1[g] = 0;
        }
        const int64_t col = c0 + pair * 2, blk = (r0 >> 5) + block;
        const bool inb = blk < mx_blocks(rows);
        if (col < cols && inb) *(uint4 *)(qt.codes + col * qt.code_stride + blk * 16) = make_uint4(out0[0], out0[1], out0[2], out0[3]);
        if (col + 1 < cols && inb) *(uint4 *)(qt.codes + (col + 1) * qt.code_stride + blk * 16) = make_uint4(out1[0], out1[1], out1[2], out1[3]);
        qt.scales[mx_scale_at(col, blk, ktt)] = (uint8_t)(inb ? b0 : 0u);
        qt.scales[mx_scale_at(col + 1, blk, ktt)] = (uint8_t)(inb ? b1 : 0u);
    }
    if (status != nullptr && bad) atomicOr(status, UQ_STATUS_NONFINITE);
}

// Eight values per thread.
template <int DT>
__global__ void __launch_bounds__(kQThreads) dequantize_kernel(uq_mx q, void *__restrict__ out, int64_t ld)
{
    grid_dependency_prologue();
    const int64_t chunks = (q.cols + 7) >> 3, kt = mx_ktiles(q.cols);
    const bool wide = ((uintptr_t)out & 15) == 0 && (ld * Elem<DT>::BYTES & 15) == 0;
    const int64_t n = q.rows * chunks, step = (int64_t)gridDim.x * kQThreads;
    for (int64_t i = (int64_t)blockIdx.x * kQThreads + threadIdx.x; i < n; i += step) {
        const int64_t row = i / chunks, c = (i - row * chunks) * 8;
        const uint32_t codes = __ldg((const uint32_t *)(q.codes + row * q.code_stride + (c >> 1)));
        const float scale = mx_scale_value(__ldg(q.scales + mx_scale_at(row, c >> 5, kt)));
        float v[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) v[t] = mx_code_value(codes >> (4 * t)) * scale;
        store8<DT>(out, row * ld + c, (int)min((int64_t)8, q.cols - c), wide, v);
    }
}

template <int DT, bool SR>
void launch_tile(const void *x, int64_t rows, int64_t cols, int64_t ld, const PhiloxKey &key, const uq_mx &q, const uq_mx &qt,
                 uint32_t *status, cudaStream_t st)
{
    const size_t smem = qt.codes == nullptr ? 0 : (size_t)kTileWords * ((DT == UQ_BF16 ? 4 : 8) + (SR ? 4 : 0));
    auto kernel = quantize_tile_kernel<DT, SR>;
    if (smem > 48 * 1024) cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    launch_k_smem(kernel, dim3((unsigned)(mx_ktiles(cols) * mx_ktiles(rows))), dim3(kQThreads), smem, st, x, rows, cols, ld, key, q, qt,
                  status);
}

}  // namespace

cudaError_t launch_mx_quantize(const void *x, int64_t rows, int64_t cols, int64_t ld, int dtype, uint64_t seed, int rng_bits,
                               const uq_mx &q, const uq_mx &qt, uint32_t *status, cudaStream_t st)
{
    const PhiloxKey key = philox_key(seed);
    if (dtype == UQ_BF16) {
        if (rng_bits) launch_tile<UQ_BF16, true>(x, rows, cols, ld, key, q, qt, status, st);
        else launch_tile<UQ_BF16, false>(x, rows, cols, ld, key, q, qt, status, st);
    } else {
        if (rng_bits) launch_tile<UQ_F32, true>(x, rows, cols, ld, key, q, qt, status, st);
        else launch_tile<UQ_F32, false>(x, rows, cols, ld, key, q, qt, status, st);
    }
    return cudaGetLastError();
}

cudaError_t launch_mx_dequantize(const uq_mx &q, void *out, int64_t ld, int dtype, cudaStream_t st)
{
    const int64_t n = q.rows * ((q.cols + 7) >> 3);
    const unsigned grid = (unsigned)min((n + kQThreads - 1) / kQThreads, (int64_t)148 * 64);
    if (dtype == UQ_BF16) launch_k(dequantize_kernel<UQ_BF16>, dim3(grid), dim3(kQThreads), st, q, out, ld);
    else launch_k(dequantize_kernel<UQ_F32>, dim3(grid), dim3(kQThreads), st, q, out, ld);
    return cudaGetLastError();
}

}  // namespace uq
