// Layer norm over the rows of a matrix, forward (optionally with the result quantized to microscaled 4-bit values on the way
// out) and backward (with the reduction of the weight's and the bias's gradient over all rows).
//
//   mean = sum x / n    var = sum (x - mean)^2 / n    rstd = 1 / sqrt(var + eps)    y = (x - mean) rstd gamma + beta
//   xh = (x - mean) rstd    t = dy gamma    dx = rstd (t - sum t / n - xh sum (t xh) / n)
//   dgamma = sum over rows of dy xh         dbeta = sum over rows of dy
//
// Everything is held in binary32; a result is rounded once, to the type of its array.  Both passes are bound by memory.  A CTA
// (for up to 512 columns: a warp) takes one row after another; the next rows are on their way into a ring of three in shared
// memory meanwhile, and a row is read from there once and kept in registers over its reductions, as are the weights and, in
// the backward pass, the sums over the rows.  Rows may start anywhere: the ring takes whole 16-byte granules of memory, what
// lies beside the row (but inside the matrix) included, and a row keeps its offset from 16 bytes there.  Which elements a
// thread holds depends on that offset: neighbours in 16-byte accesses, or elements that are 32 apart, so that a warp's scalar
// accesses are contiguous.
// Measured at 16384 x 8192: forward bf16 85 us (6.3 TB/s), binary32 188 us (5.7), quantized on the way out 127 us and 153 us (2.7 and
// 4.0), with the result itself as well 134 and 188 us, backward bf16 158 us (5.1), binary32 254 to 275 us (5.9 to 6.3); with rows that
// start anywhere (8191 columns) bf16 148, 207 and 259 us, binary32 188, 271 and 290; backward at 8192 x 16384 bf16 239 us (3.4),
// binary32 363 us (4.4).
#include "uq_mx.cuh"

namespace uq {
namespace {

constexpr int kLnThreads = 256;                            // of the kernels for any length
constexpr int kRing = 3;                                   // rows in shared memory
constexpr size_t kLnScratchBytes = 512;                    // the most that a kernel has in shared memory beside the ring
constexpr int64_t kLnRegisterCols = 16384;                 // forward: longest row that is kept in registers
constexpr int64_t kLnBackwardCols = 16384;                 // backward: longest row whose sums over the rows are (two CTAs above 8192)

// How a thread's eight elements of a piece lie in the row: in 16-byte accesses (kWide: pieces that are whole or empty; kFull: none
// is empty, so no branch is left in a row); 32 apart; neighbours, taken element by element.
enum { kWide = 0, kStrided = 1, kChunk = 2, kFull = 3 };
__host__ __device__ constexpr bool is_wide(int map) { return map == kWide || map == kFull; }

// Elements of a piece: what 16 bytes hold, so that a warp's accesses of either memory are contiguous; eight (a quarter of a block)
// where the result is quantized.
template <int DT, bool Q> constexpr int kPiece = Q ? 8 : 16 / Elem<DT>::BYTES;

// First element of a thread's piece i of PE elements; the others follow at distance 1, or 32 (kStrided).
template <int TPR, int MAP, int PE> __device__ __forceinline__ int piece_at(int i, int t)
{
    if constexpr (MAP == kStrided) return (i * (TPR / 32) + (t >> 5)) * (PE * 32) + (t & 31);
    return (i * TPR + t) * PE;
}
template <int MAP> __device__ __forceinline__ int piece_step() { return MAP == kStrided ? 32 : 1; }

// Bytes of a ring's slot: a row and the rest of its first and last granule.
__host__ __device__ __forceinline__ constexpr int slot_bytes(int64_t cols, int bytes) { return (int)((cols * bytes + 15) / 16 * 16 + 16); }

// Starts the copy of row `row` into a slot, by `threads` threads.  A granule that reaches out of the matrix is copied element by
// element (the first of the first row, the last of the last row).
template <int DT> __device__ __forceinline__ void fetch_row(unsigned char *slot, const void *base, int64_t row, int64_t rows, int64_t cols,
                                                            int64_t ld, int thread, int threads)
{
    constexpr int E = Elem<DT>::BYTES;
    const uintptr_t begin = (uintptr_t)base + row * ld * E, end = begin + cols * E, first = begin & ~(uintptr_t)15;
    const uintptr_t matrix_end = (uintptr_t)base + ((rows - 1) * ld + cols) * E;
    const int granules = (int)((end - first + 15) >> 4);
    if (first >= (uintptr_t)base && first + 16 * (uintptr_t)granules <= matrix_end) {
        const uint32_t dst = smem_address(slot);
#pragma unroll 4
        for (int g = thread; g < granules; g += threads) copy_async16(dst + 16 * g, (const void *)(first + 16 * g));
        return;
    }
    for (int g = thread; g < granules; g += threads) {
        const uintptr_t at = first + 16 * (uintptr_t)g;
        if (at >= (uintptr_t)base && at + 16 <= matrix_end) {
            copy_async16(smem_address(slot + 16 * g), (const void *)at);
        } else {
            for (int k = 0; k < 16; k += E)
                if (at + k >= (uintptr_t)base && at + k + E <= matrix_end) {
                    if constexpr (DT == UQ_BF16) *(unsigned short *)(slot + 16 * g + k) = *(const unsigned short *)(at + k);
                    else *(float *)(slot + 16 * g + k) = *(const float *)(at + k);
                }
        }
    }
}
// A row that starts on 16 bytes and consists of whole granules.
template <int TPR> __device__ __forceinline__ void fetch_wide(unsigned char *slot, const char *row, int bytes, int thread)
{
    const uint32_t dst = smem_address(slot);
#pragma unroll 4
    for (int at = thread * 16; at < bytes; at += TPR * 16) copy_async16(dst + at, row + at);
}
template <int DT, int TPR, int MAP> __device__ __forceinline__ void fetch(unsigned char *slot, const void *base, int64_t row, int64_t rows,
                                                                          int64_t cols, int64_t ld, int thread)
{
    if constexpr (is_wide(MAP)) fetch_wide<TPR>(slot, (const char *)base + row * ld * Elem<DT>::BYTES, (int)cols * Elem<DT>::BYTES, thread);
    else fetch_row<DT>(slot, base, row, rows, cols, ld, thread, TPR);
}
__device__ __forceinline__ void fetch_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING> __device__ __forceinline__ void fetch_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(PENDING) : "memory"); }

// Whether a piece holds anything of the row.
template <int MAP> __device__ __forceinline__ bool piece_there(int at, int cols) { return MAP == kFull || at < cols; }

// A piece of a row in shared memory; `beyond` in the places beyond its end.
template <int DT, int MAP, int PE>
__device__ __forceinline__ void load_piece(const unsigned char *row, int at, int cols, float (&v)[PE], float beyond = 0.0f)
{
    if constexpr (is_wide(MAP) && DT == UQ_BF16) {
        Elem<UQ_BF16>::unpack(*(const uint4 *)(row + at * 2), v);
    } else if constexpr (is_wide(MAP)) {
#pragma unroll
        for (int t = 0; t < PE; t += 4) {
            const float4 q = *(const float4 *)(row + (at + t) * 4);
            v[t] = q.x; v[t + 1] = q.y; v[t + 2] = q.z; v[t + 3] = q.w;
        }
    } else {
        const auto element = [&](int i) {
            if constexpr (DT == UQ_BF16) return __uint_as_float((uint32_t)*(const unsigned short *)(row + i * 2) << 16);
            else return *(const float *)(row + i * 4);
        };
        // all but a row's last pieces without questions: 16384 x 8191 bf16 forward 167 -> 147 us (binary32, with half the elements to a
        // piece, loses by it)
        if (DT == UQ_BF16 && at + (PE - 1) * piece_step<MAP>() < cols) {
#pragma unroll
            for (int t = 0; t < PE; ++t) v[t] = element(at + t * piece_step<MAP>());
        } else {
#pragma unroll
            for (int t = 0; t < PE; ++t) v[t] = at + t * piece_step<MAP>() < cols ? element(at + t * piece_step<MAP>()) : beyond;
        }
    }
}

template <int DT, int MAP, int PE> __device__ __forceinline__ void store_piece(void *row, int at, int cols, const float (&v)[PE])
{
    if constexpr (is_wide(MAP) && PE == 4) {
        *(float4 *)((float *)row + at) = make_float4(v[0], v[1], v[2], v[3]);
    } else if constexpr (is_wide(MAP)) {
        store8<DT>(row, at, 8, true, v);
    } else {
#pragma unroll
        for (int t = 0; t < PE; ++t)
            if (at + t * piece_step<MAP>() < cols) store1<DT>(row, at + t * piece_step<MAP>(), v[t]);
    }
}

// The weights of a piece, cached: every row uses them.
template <int MAP, int PE> __device__ __forceinline__ void load_weights(const float *w, int64_t at, int64_t cols, bool wide, float (&v)[PE])
{
    if (MAP != kStrided && wide && at + PE <= cols) {
#pragma unroll
        for (int t = 0; t < PE; t += 4) {
            const float4 q = __ldg((const float4 *)(w + at + t));
            v[t] = q.x; v[t + 1] = q.y; v[t + 2] = q.z; v[t + 3] = q.w;
        }
        return;
    }
#pragma unroll
    for (int t = 0; t < PE; ++t) v[t] = at + t * piece_step<MAP>() < cols ? __ldg(w + at + t * piece_step<MAP>()) : 0.0f;
}

// Two values per instruction: the row's elements are held in pairs.
__device__ __forceinline__ uint64_t pair_bits(float2 v)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(v.x), "f"(v.y));
    return r;
}
__device__ __forceinline__ float2 pair_of(uint64_t r)
{
    float2 v;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(r));
    return v;
}
__device__ __forceinline__ float2 operator+(float2 a, float2 b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)));
    return pair_of(r);
}
__device__ __forceinline__ float2 operator*(float2 a, float2 b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)));
    return pair_of(r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)), "l"(pair_bits(c)));
    return pair_of(r);
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
template <int PE> __device__ __forceinline__ void to_pairs(const float (&v)[PE], float2 (&w)[PE / 2])
{
#pragma unroll
    for (int k = 0; k < PE / 2; ++k) w[k] = make_float2(v[2 * k], v[2 * k + 1]);
}
template <int PE> __device__ __forceinline__ void from_pairs(const float2 (&w)[PE / 2], float (&v)[PE])
{
#pragma unroll
    for (int k = 0; k < PE / 2; ++k) { v[2 * k] = w[k].x; v[2 * k + 1] = w[k].y; }
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// The sum over a row's threads, the same in each, in an order that depends only on TPR.  scratch: TPR / 32 floats that no
// other sum uses until the next barrier but one.
template <int TPR> __device__ __forceinline__ float row_sum(float v, float *scratch)
{
    v = warp_sum(v);
    if constexpr (TPR > 32) {
        if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
        __syncthreads();
        if constexpr (TPR == 64) return scratch[0] + scratch[1];
        float2 s = both(0.0f);
#pragma unroll
        for (int w = 0; w < TPR / 32; w += 4) {
            const float4 q = *(const float4 *)(scratch + w);
            s = (s + make_float2(q.x, q.y)) + make_float2(q.z, q.w);
        }
        v = s.x + s.y;
    }
    return v;
}

// Two sums at once.
template <int TPR> __device__ __forceinline__ float2 row_sums(float2 v, float2 *scratch)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = v + make_float2(__shfl_xor_sync(0xFFFFFFFFu, v.x, o), __shfl_xor_sync(0xFFFFFFFFu, v.y, o));
    if constexpr (TPR > 32) {
        if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
        __syncthreads();
        v = both(0.0f);
#pragma unroll
        for (int w = 0; w < TPR / 32; w += 2) {
            const float4 q = *(const float4 *)(scratch + w);
            v = (v + make_float2(q.x, q.y)) + make_float2(q.z, q.w);
        }
    }
    return v;
}

// Two sums at once over the same threads of both CTAs of a cluster: every warp leaves its sums in both.  The cluster's barrier
// stands in for the CTA's.
template <int TPR> __device__ __forceinline__ float2 pair_sums(float2 v, float2 *scratch, uint32_t rank)
{
    constexpr int W = TPR / 32;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = v + make_float2(__shfl_xor_sync(0xFFFFFFFFu, v.x, o), __shfl_xor_sync(0xFFFFFFFFu, v.y, o));
    if ((threadIdx.x & 31) < 2) {
        const uint32_t at = cluster_address(smem_address(scratch + rank * W + (threadIdx.x >> 5)), threadIdx.x & 31);
        asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" :: "r"(at), "f"(v.x), "f"(v.y) : "memory");
    }
    cluster_sync();
    v = both(0.0f);
#pragma unroll
    for (int w = 0; w < 2 * W; w += 2) {
        const float4 q = *(const float4 *)(scratch + w);
        v = (v + make_float2(q.x, q.y)) + make_float2(q.z, q.w);
    }
    return v;
}

// 1 / sqrt(v): the approximation (2 units in the last place) and a Newton step, without the chains of an exact root and an exact
// division in every thread; 0 and infinity keep their limits.
__device__ __forceinline__ float inverse_root(float v)
{
    const float r = rsqrtf(v);
    const float better = __fmaf_rn(0.5f * r, __fmaf_rn(-v * r, r, 1.0f), r);
    return r > 0.0f && r < __int_as_float(0x7F800000) ? better : r;
}

// Eight neighbouring results (zeros beyond the row) to codes; the four threads of a block are neighbours in a warp.
template <int DT> __device__ __forceinline__ bool quantize_piece(const uq_mx &q, int64_t row, int64_t at, float (&v)[8])
{
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
    }
    const int64_t kt = mx_ktiles(q.cols);
    if (at < mx_blocks(q.cols) * 32) *(uint32_t *)(q.codes + row * q.code_stride + (at >> 1)) = codes;
    if ((at & 31) == 0 && at < kt * 128) q.scales[mx_scale_at(row, at >> 5, kt)] = (uint8_t)byte;
    return byte == 255u;
}

// Sets what lies beyond the row to 0.
template <int MAP, int PE> __device__ __forceinline__ void clear_beyond(int at, int cols, float2 (&v)[PE / 2])
{
    if (!is_wide(MAP) && at + (PE - 1) * piece_step<MAP>() >= cols) {
#pragma unroll
        for (int k = 0; k < PE / 2; ++k) {
            if (at + 2 * k * piece_step<MAP>() >= cols) v[k].x = 0.0f;
            if (at + (2 * k + 1) * piece_step<MAP>() >= cols) v[k].y = 0.0f;
        }
    }
}

struct NormArgs {
    const void *x;
    const float *gamma, *beta;
    void *y;
    float *mean, *rstd;
    uint32_t *status;
    int64_t rows, cols, ld, y_ld;
    float eps;
    uq_mx q;
};

// ---- forward ------------------------------------------------------------------------------------

// TPR threads per row (the CTA, or one of its four warps), NC pieces of eight elements each.
template <int TPR> struct RowThreads {
    static constexpr int kThreads = TPR == 32 ? 128 : TPR, kRows = kThreads / TPR;
    // CTAs per SM that the grid counts on
    static constexpr int kResident = 512 / kThreads;
};

template <int DT, int TPR, int NC, int MAP, bool Q>
__global__ void __launch_bounds__(RowThreads<TPR>::kThreads, RowThreads<TPR>::kResident) layer_norm_kernel(const NormArgs p)
{
    constexpr int R = RowThreads<TPR>::kRows, PE = kPiece<DT, Q>, NP = NC * 8 / PE;
    __shared__ __align__(16) float scratch[2][TPR / 32];
    static_assert(sizeof(scratch) <= kLnScratchBytes, "counted in launch_rows");
    extern __shared__ __align__(16) unsigned char ring[];
    grid_dependency_prologue();
    const int t = threadIdx.x % TPR, cols = (int)p.cols;
    const int slot = slot_bytes(p.cols, Elem<DT>::BYTES);
    unsigned char *mine = ring + threadIdx.x / TPR * kRing * slot;
    const int64_t first = (int64_t)blockIdx.x * R + threadIdx.x / TPR, step = (int64_t)gridDim.x * R;
#pragma unroll
    for (int i = 0; i < kRing; ++i) {
        if (first + i * step < p.rows) fetch<DT, TPR, MAP>(mine + i * slot, p.x, first + i * step, p.rows, p.cols, p.ld, t);
        fetch_commit();
    }
    float2 gamma[NP][PE / 2], beta[NP][PE / 2];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int at = piece_at<TPR, MAP, PE>(i, t);
        float w[PE];
#pragma unroll
        for (int k = 0; k < PE; ++k) w[k] = 1.0f;
        if (p.gamma != nullptr) load_weights<MAP, PE>(p.gamma, at, p.cols, ((uintptr_t)p.gamma & 15) == 0, w);
        to_pairs<PE>(w, gamma[i]);
#pragma unroll
        for (int k = 0; k < PE; ++k) w[k] = 0.0f;
        if (p.beta != nullptr) load_weights<MAP, PE>(p.beta, at, p.cols, ((uintptr_t)p.beta & 15) == 0, w);
        to_pairs<PE>(w, beta[i]);
    }
    const float inv_n = 1.0f / (float)p.cols;
    bool bad = false;
    char *yr = (char *)p.y + first * p.y_ld * Elem<DT>::BYTES;
    fetch_wait<kRing - 1>();
    if constexpr (TPR > 32) __syncthreads(); else __syncwarp();
    int s = 0;
    for (int64_t row = first; row < p.rows; row += step, yr += step * p.y_ld * Elem<DT>::BYTES) {
        const unsigned char *xr = mine + s * slot + (is_wide(MAP) ? 0 : ((uintptr_t)p.x + row * p.ld * Elem<DT>::BYTES) & 15);
        float2 v[NP][PE / 2], sum = both(0.0f);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int at = piece_at<TPR, MAP, PE>(i, t);
            if (piece_there<MAP>(at, cols)) {
                float w[PE];
                load_piece<DT, MAP, PE>(xr, at, cols, w);
                to_pairs<PE>(w, v[i]);
#pragma unroll
                for (int k = 0; k < PE / 2; ++k) sum = sum + v[i][k];
            }
        }
        fetch_wait<kRing - 2>();                           // the next row; the sum's barrier shows it to all, and frees this row's slot
        if constexpr (TPR == 32) __syncwarp();
        const float mean = row_sum<TPR>(sum.x + sum.y, scratch[0]) * inv_n;
        if (row + kRing * step < p.rows) fetch<DT, TPR, MAP>(mine + s * slot, p.x, row + kRing * step, p.rows, p.cols, p.ld, t);
        fetch_commit();
        s = s + 1 == kRing ? 0 : s + 1;
        sum = both(0.0f);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int at = piece_at<TPR, MAP, PE>(i, t);
            if (piece_there<MAP>(at, cols)) {
#pragma unroll
                for (int k = 0; k < PE / 2; ++k) v[i][k] = v[i][k] + both(-mean);
                clear_beyond<MAP, PE>(at, cols, v[i]);
#pragma unroll
                for (int k = 0; k < PE / 2; ++k) sum = fma2(v[i][k], v[i][k], sum);
            }
        }
        const float rstd = inverse_root(row_sum<TPR>(sum.x + sum.y, scratch[1]) * inv_n + p.eps);
        if (t == 0) {
            if (p.mean != nullptr) p.mean[row] = mean;
            if (p.rstd != nullptr) p.rstd[row] = rstd;
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int at = piece_at<TPR, MAP, PE>(i, t);
            float w[PE] = {};
            if (piece_there<MAP>(at, cols)) {
#pragma unroll
                for (int k = 0; k < PE / 2; ++k) v[i][k] = fma2(v[i][k] * both(rstd), gamma[i][k], beta[i][k]);
                from_pairs<PE>(v[i], w);
                if (p.y != nullptr) store_piece<DT, MAP, PE>(yr, at, cols, w);
            }
            if constexpr (Q) bad = quantize_piece<DT>(p.q, row, at, w) || bad;      // (elements beyond the row are 0, and so is beta)
        }
    }
    if (Q && bad && p.status != nullptr) atomicOr(p.status, UQ_STATUS_NONFINITE);
}

// Rows of any length: read three times (the second and third time from the caches).
template <int DT>
__global__ void __launch_bounds__(kLnThreads) layer_norm_long_kernel(const NormArgs p)
{
    __shared__ __align__(16) float scratch[2][kLnThreads / 32];
    grid_dependency_prologue();
    const int64_t cols = p.cols, chunks = (cols + 7) >> 3;
    const int64_t all = (mx_ktiles(cols) * 16 + 31) / 32 * 32;         // whole warps, and a row's last scale tile
    const bool wide = ((uintptr_t)p.x & 15) == 0 && (p.ld * Elem<DT>::BYTES & 15) == 0;
    const bool wide_y = ((uintptr_t)p.y & 15) == 0 && (p.y_ld * Elem<DT>::BYTES & 15) == 0;
    const bool wide_g = ((uintptr_t)p.gamma & 15) == 0, wide_b = ((uintptr_t)p.beta & 15) == 0;
    const float n = (float)cols;
    const int64_t row = blockIdx.x;
    const char *xr = (const char *)p.x + row * p.ld * Elem<DT>::BYTES;
    float s = 0.0f;
    for (int64_t c = threadIdx.x; c < chunks; c += kLnThreads) {
        float v[8];
        load8<DT>(xr, c * 8, (int)min((int64_t)8, cols - c * 8), wide, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) s += v[k];
    }
    const float mean = row_sum<kLnThreads>(s, scratch[0]) / n;
    s = 0.0f;
    for (int64_t c = threadIdx.x; c < chunks; c += kLnThreads) {
        float v[8];
        const int have = (int)min((int64_t)8, cols - c * 8);
        load8<DT>(xr, c * 8, have, wide, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float d = k < have ? v[k] - mean : 0.0f;
            s = __fmaf_rn(d, d, s);
        }
    }
    const float rstd = 1.0f / sqrtf(row_sum<kLnThreads>(s, scratch[1]) / n + p.eps);
    if (threadIdx.x == 0) {
        if (p.mean != nullptr) p.mean[row] = mean;
        if (p.rstd != nullptr) p.rstd[row] = rstd;
    }
    bool bad = false;
    for (int64_t c = threadIdx.x; c < all; c += kLnThreads) {
        const int have = (int)max((int64_t)0, min((int64_t)8, cols - c * 8));
        float v[8], w[8];
        load8<DT>(xr, c * 8, have, wide, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = (v[k] - mean) * rstd;
        if (p.gamma != nullptr) {
            load_weights<kWide, 8>(p.gamma, c * 8, cols, wide_g, w);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= w[k];
        }
        if (p.beta != nullptr) {
            load_weights<kWide, 8>(p.beta, c * 8, cols, wide_b, w);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += w[k];
        }
        if (p.y != nullptr) store8<DT>((char *)p.y + row * p.y_ld * Elem<DT>::BYTES, c * 8, have, wide_y, v);
        if (p.q.codes != nullptr) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = k < have ? v[k] : 0.0f;
            bad = quantize_piece<DT>(p.q, row, c * 8, v) || bad;
        }
    }
    if (bad && p.status != nullptr) atomicOr(p.status, UQ_STATUS_NONFINITE);
}

// ---- backward -----------------------------------------------------------------------------------

struct NormBackwardArgs {
    const void *dy, *x;
    const float *gamma, *mean, *rstd;
    void *dx;
    float *partial;                                        // [part][2][cols]: sums of dy xh and of dy over a part's rows
    int64_t rows, cols, dy_ld, x_ld, dx_ld;
};

// Columns of the first CTA of two that share a row.
__host__ __device__ __forceinline__ int64_t half_row(int64_t cols) { return ((cols + 1) / 2 + 7) & ~(int64_t)7; }

// A CTA takes every gridDim.x-th row (TPR = 32: its four warps one each) and keeps its sums over the rows in registers, a
// thread's columns being its own.  CL = 2: a cluster of two takes a row, half its columns each.
template <int DT, int TPR, int NC, int MAP, int CL>
__global__ void __launch_bounds__(RowThreads<TPR>::kThreads, RowThreads<TPR>::kResident) layer_norm_backward_kernel(const NormBackwardArgs p)
{
    constexpr int R = RowThreads<TPR>::kRows, T = RowThreads<TPR>::kThreads, PE = kPiece<DT, false>, NP = NC * 8 / PE;
    __shared__ __align__(16) float2 scratch[2][CL * TPR / 32];
    static_assert(sizeof(scratch) <= kLnScratchBytes, "counted in launch_rows");
    extern __shared__ __align__(16) unsigned char ring[];
    grid_dependency_prologue();
    constexpr int E = Elem<DT>::BYTES;
    const uint32_t rank = CL > 1 ? cluster_rank() : 0;
    const int t = threadIdx.x % TPR, part = threadIdx.x / TPR;
    // this CTA's columns, as a matrix of their own
    const int64_t half = CL > 1 ? half_row(p.cols) : p.cols, col0 = rank * half;
    const int cols = (int)min(half, p.cols - col0);
    const char *x = (const char *)p.x + col0 * E, *dy = (const char *)p.dy + col0 * E;
    const float *weight = p.gamma == nullptr ? nullptr : p.gamma + col0;
    const int slot = slot_bytes(half, E);
    unsigned char *mine = ring + part * kRing * 2 * slot;
    const int64_t first = (int64_t)(blockIdx.x / CL) * R + part, step = (int64_t)(gridDim.x / CL) * R;
#pragma unroll
    for (int i = 0; i < kRing; ++i) {
        if (first + i * step < p.rows) {
            fetch<DT, TPR, MAP>(mine + 2 * i * slot, x, first + i * step, p.rows, cols, p.x_ld, t);
            fetch<DT, TPR, MAP>(mine + (2 * i + 1) * slot, dy, first + i * step, p.rows, cols, p.dy_ld, t);
        }
        fetch_commit();
    }
    const float inv_n = 1.0f / (float)p.cols;
    float2 gamma[NP][PE / 2], dg[NP][PE / 2], db[NP][PE / 2];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        float w[PE];
#pragma unroll
        for (int k = 0; k < PE; ++k) w[k] = 1.0f;
        if (weight != nullptr) load_weights<MAP, PE>(weight, piece_at<TPR, MAP, PE>(i, t), cols, ((uintptr_t)weight & 15) == 0, w);
        to_pairs<PE>(w, gamma[i]);
#pragma unroll
        for (int k = 0; k < PE / 2; ++k) dg[i][k] = db[i][k] = both(0.0f);
    }
    char *dxr = (char *)p.dx + (first * p.dx_ld + col0) * E;
    fetch_wait<kRing - 1>();
    if constexpr (CL > 1) cluster_sync();                  // (and the other CTA is there to be written to)
    else if constexpr (TPR > 32) __syncthreads();
    else __syncwarp();
    int s = 0, turn = 0;
    float next_mean = first < p.rows ? __ldg(p.mean + first) : 0.0f, next_rstd = first < p.rows ? __ldg(p.rstd + first) : 0.0f;
    for (int64_t row = first; row < p.rows; row += step, turn ^= 1, dxr += step * p.dx_ld * Elem<DT>::BYTES) {
        const float mean = next_mean, rstd = next_rstd;    // (loaded a row ahead: nothing else in a row waits for memory)
        if (row + step < p.rows) {
            next_mean = __ldg(p.mean + row + step);
            next_rstd = __ldg(p.rstd + row + step);
        }
        const unsigned char *xr = mine + 2 * s * slot + (is_wide(MAP) ? 0 : ((uintptr_t)x + row * p.x_ld * E) & 15);
        const unsigned char *dr = mine + (2 * s + 1) * slot + (is_wide(MAP) ? 0 : ((uintptr_t)dy + row * p.dy_ld * E) & 15);
        float2 d[NP][PE / 2], xh[NP][PE / 2], sum1 = both(0.0f), sum2 = both(0.0f);
#pragma unroll
        for (int i = 0; i < NP; ++i) {                     // beyond the row xh and dy are 0: nothing is added
            const int at = piece_at<TPR, MAP, PE>(i, t);
            if (piece_there<MAP>(at, cols)) {
                float w[PE];
                // Beyond the row mean * rstd may leave binary32 where no xh of the row does: x is the mean there, or xh is set to 0
                // (by two CTAs 8192 x 16383 bf16 takes 344 us by the first and 305 by the second, by one 16384 x 8191 258 and 262).
                load_piece<DT, MAP, PE>(xr, at, cols, w, CL == 1 ? mean : 0.0f);
                to_pairs<PE>(w, xh[i]);
                load_piece<DT, MAP, PE>(dr, at, cols, w);
                to_pairs<PE>(w, d[i]);
#pragma unroll
                for (int k = 0; k < PE / 2; ++k) xh[i][k] = (xh[i][k] + both(-mean)) * both(rstd);
                if constexpr (CL > 1) clear_beyond<MAP, PE>(at, cols, xh[i]);
#pragma unroll
                for (int k = 0; k < PE / 2; ++k) {
                    dg[i][k] = fma2(d[i][k], xh[i][k], dg[i][k]);
                    db[i][k] = db[i][k] + d[i][k];
                    d[i][k] = d[i][k] * gamma[i][k];
                    sum1 = sum1 + d[i][k];
                    sum2 = fma2(d[i][k], xh[i][k], sum2);
                }
            }
        }
        fetch_wait<kRing - 2>();                           // the next row; the barrier shows it to all, and frees this row's slot
        if constexpr (TPR == 32) __syncwarp();
        float2 m = make_float2(sum1.x + sum1.y, sum2.x + sum2.y);
        if constexpr (CL > 1) m = pair_sums<TPR>(m, scratch[turn], rank);
        else m = row_sums<TPR>(m, scratch[turn]);
        m = m * both(inv_n);
        if (row + kRing * step < p.rows) {
            fetch<DT, TPR, MAP>(mine + 2 * s * slot, x, row + kRing * step, p.rows, cols, p.x_ld, t);
            fetch<DT, TPR, MAP>(mine + (2 * s + 1) * slot, dy, row + kRing * step, p.rows, cols, p.dy_ld, t);
        }
        fetch_commit();
        s = s + 1 == kRing ? 0 : s + 1;
        if (p.dx != nullptr) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int at = piece_at<TPR, MAP, PE>(i, t);
                if (piece_there<MAP>(at, cols)) {
                    float w[PE];
#pragma unroll
                    for (int k = 0; k < PE / 2; ++k) d[i][k] = both(rstd) * fma2(xh[i][k], both(-m.y), d[i][k] + both(-m.x));
                    from_pairs<PE>(d[i], w);
                    store_piece<DT, MAP, PE>(dxr, at, cols, w);
                }
            }
        }
    }
    float *out = p.partial + (int64_t)(blockIdx.x / CL) * 2 * p.cols + col0;
    if constexpr (TPR == 32) {                             // the warps' sums, in their order
        float *sums = (float *)ring;
        __syncthreads();
        for (int w = 0; w < R; ++w) {
            if (part == w) {
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    float g[PE], b[PE];
                    from_pairs<PE>(dg[i], g);
                    from_pairs<PE>(db[i], b);
#pragma unroll
                    for (int k = 0; k < PE; ++k) {
                        const int c = piece_at<TPR, MAP, PE>(i, t) + k * piece_step<MAP>();
                        if (c < cols) {
                            sums[c] = w == 0 ? g[k] : sums[c] + g[k];
                            sums[cols + c] = w == 0 ? b[k] : sums[cols + c] + b[k];
                        }
                    }
                }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < 2 * cols; c += T) out[c] = sums[c];
    } else {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            float g[PE], b[PE];
            from_pairs<PE>(dg[i], g);
            from_pairs<PE>(db[i], b);
#pragma unroll
            for (int k = 0; k < PE; ++k) {
                const int c = piece_at<TPR, MAP, PE>(i, t) + k * piece_step<MAP>();
                if (c < cols) { out[c] = g[k]; out[p.cols + c] = b[k]; }
            }
        }
    }
    if constexpr (CL > 1) cluster_sync();                  // (the other CTA may still be writing its sums here)
}

// Rows of any length: dx, each row read twice (the second time from the caches).
template <int DT>
__global__ void __launch_bounds__(kLnThreads) layer_norm_backward_long_kernel(const NormBackwardArgs p)
{
    __shared__ __align__(16) float scratch[2][kLnThreads / 32];
    grid_dependency_prologue();
    const int64_t cols = p.cols, chunks = (cols + 7) >> 3;
    const bool wide_dy = ((uintptr_t)p.dy & 15) == 0 && (p.dy_ld * Elem<DT>::BYTES & 15) == 0;
    const bool wide_x = ((uintptr_t)p.x & 15) == 0 && (p.x_ld * Elem<DT>::BYTES & 15) == 0;
    const bool wide_dx = ((uintptr_t)p.dx & 15) == 0 && (p.dx_ld * Elem<DT>::BYTES & 15) == 0;
    const bool wide_g = ((uintptr_t)p.gamma & 15) == 0;
    const float n = (float)cols;
    const int64_t row = blockIdx.x;
    const float mean = __ldg(p.mean + row), rstd = __ldg(p.rstd + row);
    const char *xr = (const char *)p.x + row * p.x_ld * Elem<DT>::BYTES, *dr = (const char *)p.dy + row * p.dy_ld * Elem<DT>::BYTES;
    float s1 = 0.0f, s2 = 0.0f;
    for (int64_t c = threadIdx.x; c < chunks; c += kLnThreads) {
        const int have = (int)min((int64_t)8, cols - c * 8);
        float d[8], v[8], w[8];
        load8<DT>(dr, c * 8, have, wide_dy, d);
        load8<DT>(xr, c * 8, have, wide_x, v);
        if (p.gamma != nullptr) load_weights<kWide, 8>(p.gamma, c * 8, cols, wide_g, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (k < have) {
                const float g = p.gamma != nullptr ? d[k] * w[k] : d[k];
                s1 += g;
                s2 = __fmaf_rn(g, (v[k] - mean) * rstd, s2);
            }
        }
    }
    const float m1 = row_sum<kLnThreads>(s1, scratch[0]) / n, m2 = row_sum<kLnThreads>(s2, scratch[1]) / n;
    for (int64_t c = threadIdx.x; c < chunks; c += kLnThreads) {
        const int have = (int)min((int64_t)8, cols - c * 8);
        float d[8], v[8], w[8];
        load8<DT>(dr, c * 8, have, wide_dy, d);
        load8<DT>(xr, c * 8, have, wide_x, v);
        if (p.gamma != nullptr) load_weights<kWide, 8>(p.gamma, c * 8, cols, wide_g, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float g = p.gamma != nullptr ? d[k] * w[k] : d[k];
            v[k] = rstd * (g - m1 - (v[k] - mean) * rstd * m2);
        }
        store8<DT>((char *)p.dx + row * p.dx_ld * Elem<DT>::BYTES, c * 8, have, wide_dx, v);
    }
}

// ... and the sums over the rows: a CTA takes 512 columns (two neighbours per thread, or two 256 apart) of every `parts`-th row.
template <int DT, bool PAIRS>
__global__ void __launch_bounds__(kLnThreads) weight_partials_kernel(const NormBackwardArgs p, int parts)
{
    grid_dependency_prologue();
    const int64_t strips = (p.cols + 511) / 512;
    const int64_t part = blockIdx.x / strips, c = blockIdx.x % strips * 512 + (PAIRS ? 2 : 1) * threadIdx.x;
    const int64_t c2 = PAIRS ? c + 1 : c + 256;
    float g[2] = {0.0f, 0.0f}, b[2] = {0.0f, 0.0f};
    if (c < p.cols) {
#pragma unroll 4
        for (int64_t row = part; row < p.rows; row += parts) {
            const float mean = __ldg(p.mean + row), rstd = __ldg(p.rstd + row);
            float x[2] = {0.0f, 0.0f}, d[2] = {0.0f, 0.0f};
            if constexpr (DT == UQ_BF16) {
                const unsigned short *xr = (const unsigned short *)p.x + row * p.x_ld, *dr = (const unsigned short *)p.dy + row * p.dy_ld;
                if (PAIRS && c2 < p.cols) {
                    const uint32_t xw = __ldg((const uint32_t *)(xr + c)), dw = __ldg((const uint32_t *)(dr + c));
                    x[0] = bf16lo(xw); x[1] = bf16hi(xw); d[0] = bf16lo(dw); d[1] = bf16hi(dw);
                } else {
                    x[0] = __uint_as_float((uint32_t)__ldg(xr + c) << 16); d[0] = __uint_as_float((uint32_t)__ldg(dr + c) << 16);
                    if (c2 < p.cols) { x[1] = __uint_as_float((uint32_t)__ldg(xr + c2) << 16); d[1] = __uint_as_float((uint32_t)__ldg(dr + c2) << 16); }
                }
            } else {
                const float *xr = (const float *)p.x + row * p.x_ld, *dr = (const float *)p.dy + row * p.dy_ld;
                x[0] = __ldg(xr + c); d[0] = __ldg(dr + c);
                if (c2 < p.cols) { x[1] = __ldg(xr + c2); d[1] = __ldg(dr + c2); }
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                g[k] = __fmaf_rn(d[k], (x[k] - mean) * rstd, g[k]);
                b[k] += d[k];
            }
        }
        float *out = p.partial + part * 2 * p.cols;
        out[c] = g[0]; out[p.cols + c] = b[0];
        if (c2 < p.cols) { out[c2] = g[1]; out[p.cols + c2] = b[1]; }
    }
}

// The parts' sums: 32 columns per CTA; thread row y adds up every 16th part, then the 16 are added in order.
template <int GT>
__global__ void __launch_bounds__(512) weight_gradient_kernel(const float *__restrict__ partial, int parts, int64_t cols, void *dgamma,
                                                              void *dbeta)
{
    __shared__ float s[16][33];
    grid_dependency_prologue();
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t c = (int64_t)(blockIdx.x >> 1) * 32 + x;
    const bool beta = blockIdx.x & 1;
    const float *src = partial + (beta ? cols : 0) + c;
    float v = 0.0f;
    if (c < cols) {
#pragma unroll 8
        for (int i = y; i < parts; i += 16) v += src[(int64_t)i * 2 * cols];
    }
    s[y][x] = v;
    __syncthreads();
    if (y == 0 && c < cols) {
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) v += s[i][x];
        void *out = beta ? dbeta : dgamma;
        if (out != nullptr) store1<GT>(out, c, v);
    }
}

// Threads per row of the backward pass.
int backward_threads(int64_t cols) { return cols <= 512 ? 32 : cols <= 1024 ? 64 : cols <= 2048 ? 128 : cols <= 4096 ? 256 : 512; }

// CTAs of the backward pass (clusters above 8192 columns), each of which leaves a part; never fewer for more rows.  A row each (for
// a warp of it, up to 512 columns) while every SM gets one at most; then four: the parts have to be added
// up (600 x 4096 bf16 by 1, 2 and 4 rows: 17.5, 17.6, 16.3 us; 4 x 8000: 8.9, 10.8, 14.7).  Between the two, where rows are short, two
// rows, up to 400 parts (both passes replayed as a graph; by four rows, by two up to 400 parts, by two without a limit: 777 x 1025
// binary32 10.0, 8.4, 8.4 us; 3200 x 500 14.4, 12.1, 12.1; 1000 x 1025 bf16 11.3, 9.4, 9.4; 1000 x 2000 bf16 17.3, 17.3, 20.4; 2000 x
// 700 binary32 11.4, 11.5, 14.8; of 24 sizes in both types two rows gain most at 3200 x 500 bf16, 15.4, 12.3, and lose most at 600 x
// 2000 bf16, 12.5, 15.9).
int backward_parts(int64_t rows, int64_t cols)
{
    if (cols > kLnBackwardCols) return (int)min((rows + 63) / 64, (int64_t)64);
    const int threads = backward_threads(cols), at_once = threads == 32 ? 4 : 1, resident = 512 / (threads == 32 ? 128 : threads);
    const int64_t turns = (rows + at_once - 1) / at_once, most = cols > 8192 ? 74 : 148 * resident;
    const int64_t by_two = cols <= 2048 ? min((turns + 1) / 2, (int64_t)400) : 0;
    return (int)min(most, max(min(turns, (int64_t)148), max(by_two, (turns + 3) / 4)));
}

template <int DT> bool rows_wide(const void *p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && (ld * Elem<DT>::BYTES & 15) == 0; }

// A kernel has 48 KiB of shared memory, its own arrays included, without asking for more.  What is asked for belongs to the kernel
// and not to the call: every call asks for the same, `most`, or a host thread with shorter rows would take away what another one
// is about to launch with.
template <typename K> void ask_for_rows(K *kernel, size_t smem, size_t most)
{
    if (smem + kLnScratchBytes > 48 * 1024) cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
}
template <typename K, typename A>
void launch_rows(K *kernel, int64_t grid, int threads, size_t smem, size_t most, cudaStream_t st, const A &args)
{
    ask_for_rows(kernel, smem, most);
    launch_k_smem(kernel, dim3((unsigned)grid), dim3(threads), smem, st, args);
}

template <int DT, int TPR, int NC> void launch_forward(const NormArgs &p, bool wide, cudaStream_t st)
{
    using T = RowThreads<TPR>;
    const int64_t grid = min((p.rows + T::kRows - 1) / T::kRows, (int64_t)148 * T::kResident);
    const size_t smem = (size_t)T::kRows * kRing * slot_bytes(p.cols, Elem<DT>::BYTES);
    constexpr size_t most = (size_t)T::kRows * kRing * slot_bytes(TPR * NC * 8, Elem<DT>::BYTES);
    const bool full = p.cols == TPR * NC * 8;
    if (p.q.codes != nullptr) {
        if (!wide) launch_rows(layer_norm_kernel<DT, TPR, NC, kChunk, true>, grid, T::kThreads, smem, most, st, p);
        else if (full) launch_rows(layer_norm_kernel<DT, TPR, NC, kFull, true>, grid, T::kThreads, smem, most, st, p);
        else launch_rows(layer_norm_kernel<DT, TPR, NC, kWide, true>, grid, T::kThreads, smem, most, st, p);
    } else {
        if (!wide) launch_rows(layer_norm_kernel<DT, TPR, NC, kStrided, false>, grid, T::kThreads, smem, most, st, p);
        else if (full) launch_rows(layer_norm_kernel<DT, TPR, NC, kFull, false>, grid, T::kThreads, smem, most, st, p);
        else launch_rows(layer_norm_kernel<DT, TPR, NC, kWide, false>, grid, T::kThreads, smem, most, st, p);
    }
}

template <int DT> void launch_forward_any(const NormArgs &p, cudaStream_t st)
{
    const int piece = p.q.codes != nullptr ? 8 : 16 / Elem<DT>::BYTES;
    const bool wide = p.cols % piece == 0 && rows_wide<DT>(p.x, p.ld) && (p.y == nullptr || rows_wide<DT>(p.y, p.y_ld));
    if (p.cols <= 256) launch_forward<DT, 32, 1>(p, wide, st);
    else if (p.cols <= 512) launch_forward<DT, 32, 2>(p, wide, st);
    else if (p.cols <= 1024) launch_forward<DT, 64, 2>(p, wide, st);
    else if (p.cols <= 2048) launch_forward<DT, 128, 2>(p, wide, st);
    else if (p.cols <= 4096) launch_forward<DT, 128, 4>(p, wide, st);
    else if (p.cols <= 8192) launch_forward<DT, 256, 4>(p, wide, st);
    else if (p.cols <= kLnRegisterCols) launch_forward<DT, 512, 4>(p, wide, st);
    else launch_k(layer_norm_long_kernel<DT>, dim3((unsigned)p.rows), dim3(kLnThreads), st, p);
}

template <int DT, int TPR, int NC, int CL = 1> void launch_backward(const NormBackwardArgs &p, bool wide, int parts, cudaStream_t st)
{
    using T = RowThreads<TPR>;
    const size_t smem = (size_t)T::kRows * kRing * 2 * slot_bytes(CL > 1 ? half_row(p.cols) : p.cols, Elem<DT>::BYTES);
    constexpr size_t most = (size_t)T::kRows * kRing * 2 * slot_bytes(TPR * NC * 8, Elem<DT>::BYTES);
    auto kernel = !wide ? layer_norm_backward_kernel<DT, TPR, NC, kStrided, CL>
                  : p.cols == CL * TPR * NC * 8 ? layer_norm_backward_kernel<DT, TPR, NC, kFull, CL> : layer_norm_backward_kernel<DT, TPR, NC, kWide, CL>;
    if constexpr (CL == 1) {
        launch_rows(kernel, parts, T::kThreads, smem, most, st, p);
    } else {
        ask_for_rows(kernel, smem, most);
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(parts * CL);
        cfg.blockDim = dim3(T::kThreads);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = st;
        cudaLaunchAttribute attr[2];
        cfg.attrs = attr;
        cfg.numAttrs = grid_dependency_attribute(attr);
        attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        attr[cfg.numAttrs].val.clusterDim.x = CL;
        attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
        ++cfg.numAttrs;
        cudaLaunchKernelEx(&cfg, kernel, p);
    }
}

template <int DT> void launch_backward_any(const NormBackwardArgs &p, int parts, bool sums, cudaStream_t st)
{
    const bool wide = p.cols % (16 / Elem<DT>::BYTES) == 0 && rows_wide<DT>(p.dy, p.dy_ld) && rows_wide<DT>(p.x, p.x_ld) && (p.dx == nullptr || rows_wide<DT>(p.dx, p.dx_ld));
    if (p.cols <= 256) launch_backward<DT, 32, 1>(p, wide, parts, st);
    else if (p.cols <= 512) launch_backward<DT, 32, 2>(p, wide, parts, st);
    else if (p.cols <= 1024) launch_backward<DT, 64, 2>(p, wide, parts, st);
    else if (p.cols <= 2048) launch_backward<DT, 128, 2>(p, wide, parts, st);
    else if (p.cols <= 4096) launch_backward<DT, 256, 2>(p, wide, parts, st);
    else if (p.cols <= 8192) launch_backward<DT, 512, 2>(p, wide, parts, st);
    else if (p.cols <= kLnBackwardCols) launch_backward<DT, 512, 2, 2>(p, wide, parts, st);
    else {
        if (p.dx != nullptr) launch_k(layer_norm_backward_long_kernel<DT>, dim3((unsigned)p.rows), dim3(kLnThreads), st, p);
        if (sums) {
            const dim3 grid((unsigned)((p.cols + 511) / 512 * parts));
            if (DT == UQ_BF16 && wide) launch_k(weight_partials_kernel<DT, true>, grid, dim3(kLnThreads), st, p, parts);
            else launch_k(weight_partials_kernel<DT, false>, grid, dim3(kLnThreads), st, p, parts);
        }
    }
}

}  // namespace

size_t layer_norm_workspace_bytes(int64_t rows, int64_t cols) { return (size_t)backward_parts(rows, cols) * 2 * cols * sizeof(float); }

cudaError_t launch_layer_norm(const void *x, int64_t rows, int64_t cols, int64_t ld, int dtype, const float *gamma, const float *beta,
                              float eps, void *y, int64_t y_ld, float *mean, float *rstd, const uq_mx &q, uint32_t *status,
                              cudaStream_t st)
{
    const NormArgs p = {x, gamma, beta, y, mean, rstd, status, rows, cols, ld, y_ld, eps, q};
    if (dtype == UQ_BF16) launch_forward_any<UQ_BF16>(p, st);
    else launch_forward_any<UQ_F32>(p, st);
    return cudaGetLastError();
}

cudaError_t launch_layer_norm_backward(const void *dy, int64_t dy_ld, const void *x, int64_t x_ld, int64_t rows, int64_t cols, int dtype,
                                       const float *gamma, const float *mean, const float *rstd, void *dx, int64_t dx_ld, void *dgamma,
                                       void *dbeta, int grad_dtype, void *workspace, cudaStream_t st)
{
    const int parts = backward_parts(rows, cols);
    float *partial = (float *)workspace;
    if (rows > 0) {
        const NormBackwardArgs p = {dy, x, gamma, mean, rstd, dx, partial, rows, cols, dy_ld, x_ld, dx_ld};
        const bool sums = dgamma != nullptr || dbeta != nullptr;
        if (dtype == UQ_BF16) launch_backward_any<UQ_BF16>(p, parts, sums, st);
        else launch_backward_any<UQ_F32>(p, parts, sums, st);
        if (cudaError_t e = cudaGetLastError()) return e;
    }
    if (dgamma == nullptr && dbeta == nullptr) return cudaSuccess;
    const dim3 grid((unsigned)((cols + 31) / 32 * 2));
    if (grad_dtype == UQ_BF16) launch_k(weight_gradient_kernel<UQ_BF16>, grid, dim3(512), st, (const float *)partial, parts, cols, dgamma, dbeta);
    else launch_k(weight_gradient_kernel<UQ_F32>, grid, dim3(512), st, (const float *)partial, parts, cols, dgamma, dbeta);
    return cudaGetLastError();
}

}  // namespace uq
