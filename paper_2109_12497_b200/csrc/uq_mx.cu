// Microscaled 4-bit quantization of a matrix with blocks along its rows, along its columns (the transposed matrix), or both
// from one read, and the values that codes stand for.
//
// A CTA owns a tile of 128 x 128 values: that is one scale tile of either orientation (512 contiguous bytes), and 64
// contiguous bytes of every row of codes.  In either orientation a lane holds eight neighbours of a block and four lanes are a
// block, whose largest magnitude two shuffles find.  Columns are read back from the tile in shared memory, bf16 values and the
// draws (made once per eight values of a row, used in both orientations) by transposing matrix loads.
// To the nearest and along rows it is bound by memory (16384 x 8192 bf16 57 to 60 us, 5.7 to 6.0 TB/s, binary32 93 us, 6.5); along
// columns it takes 68 and 144 us, both ways 100 and 163 (the floors by bytes are 53 and 94 us one way, 64 and 105 both).  Where it
// draws, it is bound by arithmetic: 38 instructions per value both ways, 22 of them on the integer pipe, which is 75 % busy (bf16
// along rows, along columns, both ways 131, 134, 210 us; binary32 142, 202, 292).
#include "uq_mx.cuh"

namespace uq {
namespace {

constexpr int kQThreads = 256;

// The tile in shared memory.  16-bit elements: rows of 256 bytes whose 16-byte granules are exchanged so that the eight rows that
// one transposing load takes (two neighbours at a distance of eight rows each) lie on different banks.  Binary32: rows of 528
// bytes and 32 more after eight rows, for the same reason (a warp reads eight columns of four rows, eight rows apart).
__device__ __forceinline__ uint32_t granule_at(int row, int granule) { return row * 256 + ((granule ^ (((row >> 3) & 3) * 2 + (row & 1))) << 4); }
__device__ __forceinline__ uint32_t word_at(int row, int col) { return (row * 132 + (row >> 3) * 8 + col) * 4; }
template <int DT, int TR> constexpr int kTileBytes = DT == UQ_BF16 ? TR * 256 : (TR * 132 + TR / 8 * 8) * 4;

// Eight rows (8 q .. 8 q + 7 of the 32 from `row` on, for q = lane % 4) of column `granule` * 8 + lane / 4 of a 16-bit tile, in
// pairs: matrix i holds rows 2 i and 2 i + 1 of each group of eight.
__device__ __forceinline__ uint4 column_of_halves(uint32_t tile, int row, int granule, int lane)
{
    const int i = lane >> 3, k = lane & 7;                 // this lane names row k of matrix i
    const uint32_t at = tile + granule_at(row + 8 * (k >> 1) + 2 * i + (k & 1), granule);
    uint4 v;
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}

// The draws of eight neighbours of a row: Philox4x32-10 with counter (col / 8, row, 0, kMxTag).  Its third word is 0 and only the
// second changes from row to row, so a thread that stays in its columns makes what the first two rounds take from the first,
// third and fourth word once (DrawColumn), and 17 of the 20 wide multiplies are left.
struct DrawColumn { uint32_t c0, c1, c3; };
__device__ __forceinline__ DrawColumn draw_column(const PhiloxKey &k, uint32_t block)
{
    const uint64_t p0 = (uint64_t)kPhiloxM0 * block;       // round 0: c0 = row ^ k0, c1 = 0, c2 = hi ^ tag ^ k1, c3 = lo
    const uint64_t p1 = (uint64_t)kPhiloxM1 * ((uint32_t)(p0 >> 32) ^ kMxTag ^ k.k[1]);
    return {(uint32_t)(p1 >> 32) ^ k.k[2], (uint32_t)p1, (uint32_t)p0 ^ k.k[3]};
}
__device__ __forceinline__ uint4 draw_row(const PhiloxKey &k, const DrawColumn &d, uint32_t row)
{
    const uint64_t p = (uint64_t)kPhiloxM0 * (row ^ k.k[0]);
    uint32_t c0 = d.c0, c1 = d.c1, c2 = (uint32_t)(p >> 32) ^ d.c3, c3 = (uint32_t)p;
#pragma unroll
    for (int r = 2; r < 10; ++r) {
        const uint64_t p0 = (uint64_t)kPhiloxM0 * c0, p1 = (uint64_t)kPhiloxM1 * c2;
        c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k.k[2 * r];
        c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k.k[2 * r + 1];
        c1 = (uint32_t)p1; c3 = (uint32_t)p0;
    }
    return make_uint4(c0, c1, c2, c3);
}

// Eight neighbours of a row into the tile in shared memory.
template <int DT> __device__ __forceinline__ void keep_eight(unsigned char *tile, int r, int chunk, const Eight<DT> &x)
{
    if constexpr (DT == UQ_BF16) {
        *(uint4 *)(tile + granule_at(r, chunk)) = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
    } else {
        // four lanes their first half, the next four their second: eight lanes then cover all banks
        const bool second = chunk & 4;
        const uint4 a = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]), b = make_uint4(x.w[4], x.w[5], x.w[6], x.w[7]);
        *(uint4 *)(tile + word_at(r, chunk * 8 + (second ? 4 : 0))) = second ? b : a;
        *(uint4 *)(tile + word_at(r, chunk * 8 + (second ? 0 : 4))) = second ? a : b;
    }
}
// Eight values from `at` on, whatever its alignment; `have` of them exist.  bf16: five words that the values touch (what lies beside
// the row, but inside the matrix, included), cut where a half is over; single values at the matrix's ends and a row's end.  (Whole
// 16-byte granules, completed by the next lane's, read memory in fewer instructions but take longer: 8192 x 8191 stochastic both
// ways 143 us against 131, binary32 175 against 152.)
template <int DT> __device__ __forceinline__ void load_cut(const char *at, const char *begin, const char *end, int have, Eight<DT> &x)
{
    if constexpr (DT == UQ_BF16) {
        const char *first = (const char *)((uintptr_t)at & ~(uintptr_t)3);
        if (have == 8 && first >= begin && first + 20 <= end) {
            const uint32_t shift = ((uintptr_t)at & 2) * 8;
            uint32_t w[5];
#pragma unroll
            for (int t = 0; t < 5; ++t) w[t] = __ldg((const uint32_t *)first + t);
#pragma unroll
            for (int t = 0; t < 4; ++t) x.w[t] = __funnelshift_r(w[t], w[t + 1], shift);
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint32_t lo = 2 * t < have ? __ldg((const unsigned short *)at + 2 * t) : 0u;
                const uint32_t hi = 2 * t + 1 < have ? __ldg((const unsigned short *)at + 2 * t + 1) : 0u;
                x.w[t] = lo | hi << 16;
            }
        }
    } else {
#pragma unroll
        for (int t = 0; t < 8; ++t) x.w[t] = t < have ? __ldg((const uint32_t *)at + t) : 0u;
    }
}

// WIDE: rows start on 16 bytes and consist of whole groups of eight.  TR: rows of x per CTA, a whole tile or a quarter of one (where
// there are few tiles).
template <int DT, bool SR, bool WIDE, int TR>
__global__ void __launch_bounds__(kQThreads, SR ? 3 : DT == UQ_BF16 && WIDE ? 5 : 4) quantize_tile_kernel(const void *__restrict__ x, int64_t rows, int64_t cols, int64_t ld,
                                                                  const PhiloxKey key, const uq_mx q, const uq_mx qt, uint32_t *status)
{
    constexpr int E = Elem<DT>::BYTES, BATCH = TR == 32 ? 2 : DT == UQ_BF16 ? 8 : 4;
    extern __shared__ __align__(16) unsigned char smem[];
    constexpr bool COLS = DT == UQ_BF16 || TR == 32;       // (binary32 columns: always a quarter of a tile)
    const bool along_rows = q.codes != nullptr, along_cols = COLS && qt.codes != nullptr;
    unsigned char *scales_q = smem, *scales_t = smem + 512, *tile = smem + 1024, *draws = tile + kTileBytes<DT, TR>;
    grid_dependency_prologue();
    const int64_t ktq = mx_ktiles(cols), ktt = mx_ktiles(rows);
    const int64_t tc = blockIdx.x % ktq, r0 = blockIdx.x / ktq * TR, tr = r0 / kMxTile, c0 = tc * kMxTile;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rows_here = (int)min((int64_t)TR, rows - r0), cols_here = (int)min((int64_t)kMxTile, cols - c0);
    const char *end = (const char *)x + ((rows - 1) * ld + cols) * E;
    bool bad = false;

    const int chunk = tid & 15, first = tid >> 4;          // eight columns, of every 16th row
    const int have = max(0, min(8, cols_here - chunk * 8));
    const DrawColumn mine = draw_column(key, (uint32_t)((c0 >> 3) + chunk));
#pragma unroll 1
    for (int batch = 0; batch < TR / 16; batch += BATCH) {
        Eight<DT> v[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int r = first + (batch + k) * 16;
            if constexpr (WIDE) {
                uint4 a = make_uint4(0, 0, 0, 0), b = a;
                if (r < rows_here && chunk * 8 < cols_here) {
                    const char *at = (const char *)x + ((r0 + r) * ld + c0 + chunk * 8) * E;
                    a = ld_stream(at);
                    if constexpr (DT == UQ_F32) b = ld_stream(at + 16);
                }
                v[k].w[0] = a.x; v[k].w[1] = a.y; v[k].w[2] = a.z; v[k].w[3] = a.w;
                if constexpr (DT == UQ_F32) { v[k].w[4] = b.x; v[k].w[5] = b.y; v[k].w[6] = b.z; v[k].w[7] = b.w; }
            } else {
                load_cut<DT>((const char *)x + ((r0 + r) * ld + c0 + chunk * 8) * E, (const char *)x, end, r < rows_here ? have : 0, v[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int r = first + (batch + k) * 16;
            uint4 h = make_uint4(0, 0, 0, 0);
            if constexpr (SR) h = draw_row(key, mine, (uint32_t)(r0 + r));
            if (along_cols) {
                keep_eight<DT>(tile, r, chunk, v[k]);
                if constexpr (SR) *(uint4 *)(draws + granule_at(r, chunk)) = h;
            }
            if (along_rows) {
                uint32_t byte;
                const uint32_t codes = quantize_eight<DT, SR>(v[k], h, byte);
                bad = bad || byte == 255u;
                if (r < rows_here && chunk * 8 < ((cols_here + 31) & ~31))
                    *(uint32_t *)(q.codes + (r0 + r) * q.code_stride + ((c0 + chunk * 8) >> 1)) = codes;
                if ((lane & 3) == 0) scales_q[(r & 31) * 16 + (r >> 5) * 4 + (chunk >> 2)] = (uint8_t)byte;
            }
        }
    }
    __syncthreads();
    if (along_cols) {
        // a warp: 16 columns in two groups of eight, the four blocks of each
        const int group = lane >> 2, part = lane & 3;
#pragma unroll 1
        for (int g = warp * 2; g < warp * 2 + 2; ++g) {
            const int col = g * 8 + group;
            unsigned char *out = qt.codes + (c0 + col) * qt.code_stride + r0 / 2 + part * 4;
#pragma unroll
            for (int blk = 0; blk < TR / 32; ++blk) {
                Eight<DT> v;
                uint4 h = make_uint4(0, 0, 0, 0);
                if constexpr (DT == UQ_BF16) {
                    const uint4 w = column_of_halves(smem_address(tile), blk * 32, g, lane);
                    v.w[0] = w.x; v.w[1] = w.y; v.w[2] = w.z; v.w[3] = w.w;
                } else {
#pragma unroll
                    for (int t = 0; t < 8; ++t) v.w[t] = *(const uint32_t *)(tile + word_at(blk * 32 + part * 8 + t, col));
                }
                if constexpr (SR) h = column_of_halves(smem_address(draws), blk * 32, g, lane);
                uint32_t byte;
                const uint32_t codes = quantize_eight<DT, SR>(v, h, byte);
                bad = bad || byte == 255u;
                if (col < cols_here && blk * 32 < rows_here) *(uint32_t *)(out + blk * 16) = codes;
                if (part == 0) scales_t[(col & 31) * 16 + (col >> 5) * 4 + blk] = (uint8_t)byte;
            }
        }
        __syncthreads();
    }
    uint8_t *to_q = q.scales + (tr * ktq + tc) * 512, *to_t = qt.scales + (tc * ktt + tr) * 512;
    if constexpr (TR == kMxTile) {
        if (along_rows && warp == 0) *(uint4 *)(to_q + lane * 16) = *(const uint4 *)(scales_q + lane * 16);
        if (along_cols && warp == 1) *(uint4 *)(to_t + lane * 16) = *(const uint4 *)(scales_t + lane * 16);
    } else {                                               // four bytes of 32 rows, a byte of 128 columns
        const int quarter = (int)(r0 / 32) & 3;
        if (along_rows && warp == 0) *(uint32_t *)(to_q + lane * 16 + quarter * 4) = *(const uint32_t *)(scales_q + lane * 16);
        if (along_cols && warp >= 4) {
            const int col = tid - 128, at = (col & 31) * 16 + (col >> 5) * 4;
            to_t[at + quarter] = scales_t[at];
        }
    }
    if (status != nullptr && bad) atomicOr(status, UQ_STATUS_NONFINITE);
}

// ---- values -------------------------------------------------------------------------------------

// bf16 patterns of four magnitude codes, as their high and low bytes: a byte permute looks four codes up at once.
__device__ __forceinline__ uint32_t code_high_bytes(uint32_t codes) { return __byte_perm(0x3F3F3F00u, 0x40404040u, codes & 0x7777u); }
__device__ __forceinline__ uint32_t code_low_bytes(uint32_t codes) { return __byte_perm(0xC0800000u, 0xC0804000u, codes & 0x7777u); }

// The values of eight codes, without their scale, as bf16 pairs.
__device__ __forceinline__ void code_values(uint32_t codes, uint32_t (&w)[4])
{
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const uint32_t c = half ? codes >> 16 : codes;
        const uint32_t twice = __byte_perm(c, 0, 0x1100), low_nibbles = twice << 4;       // signs to bit 7 of four bytes
        const uint32_t signs = (low_nibbles & 0x00FF00FFu) | (twice & 0xFF00FF00u);
        const uint32_t hi = code_high_bytes(c) | (signs & 0x80808080u), lo = code_low_bytes(c);
        w[2 * half] = __byte_perm(lo, hi, 0x5140);
        w[2 * half + 1] = __byte_perm(lo, hi, 0x7362);
    }
}

// 2^e as a bf16 pair; products with it are exact (subnormal results too).
__device__ __forceinline__ uint32_t scale_pair(uint32_t byte)
{
    const uint32_t v = byte == 255u ? 0x7FFFu : byte == 0u ? 0x0040u : byte << 7;
    return v | v << 16;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// A warp takes units of 256 columns of four rows: eight neighbours a lane (binary32: four, and four 128 columns on), or, where
// rows of out do not start on 16 bytes, a row, eight values a lane that are 32 apart: a store is contiguous.
constexpr int kDequantRows = 4;
template <int DT, bool WIDE>
__global__ void __launch_bounds__(kQThreads) dequantize_kernel(const uq_mx q, void *__restrict__ out, int64_t ld)
{
    grid_dependency_prologue();
    constexpr int R = WIDE ? kDequantRows : 1;
    const int64_t pieces = (q.cols + 255) >> 8, kt = mx_ktiles(q.cols), step = (int64_t)gridDim.x * (kQThreads / 32);
    const int64_t row_step = step / pieces, piece_step = step - row_step * pieces;      // (one division, not one for every unit)
    const int lane = threadIdx.x & 31;
    const int64_t start = (int64_t)blockIdx.x * (kQThreads / 32) + (threadIdx.x >> 5);
    int64_t group = start / pieces, piece = start - group * pieces;
    while (group * R < q.rows) {
        const int64_t row = group * R;
        const int there = (int)min((int64_t)R, q.rows - row);
        if constexpr (WIDE) {
            constexpr int N = DT == UQ_BF16 ? 8 : 4;
#pragma unroll
            for (int k = 0; k < 8 / N; ++k) {
                const int64_t c = piece * 256 + k * 128 + lane * N;
                if (c >= q.cols) break;
                const unsigned char *codes = q.codes + row * q.code_stride + (c >> 1);
                const uint8_t *scales = q.scales + mx_scale_at(row, c >> 5, kt);        // the rows' are 16 bytes apart
                char *at = (char *)out + (row * ld + c) * Elem<DT>::BYTES;
                const int have = (int)min((int64_t)N, q.cols - c);
                uint32_t code[R], byte[R];
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (r < there) {
                        if constexpr (N == 8) code[r] = __ldg((const uint32_t *)(codes + r * q.code_stride));
                        else code[r] = __ldg((const unsigned short *)(codes + r * q.code_stride));
                        byte[r] = __ldg(scales + 16 * r);
                    }
#pragma unroll
                for (int r = 0; r < R; ++r, at += ld * Elem<DT>::BYTES) {
                    if (r >= there) break;
                    uint32_t w[4];
                    code_values(code[r], w);
                    if (DT == UQ_BF16 && have == N) {
                        const uint32_t scale = scale_pair(byte[r]);
                        *(uint4 *)at = make_uint4(mul_bf16x2(w[0], scale), mul_bf16x2(w[1], scale), mul_bf16x2(w[2], scale), mul_bf16x2(w[3], scale));
                    } else {
                        const float scale = mx_scale_value(byte[r]);
                        float v[8];
#pragma unroll
                        for (int t = 0; t < N / 2; ++t) mul_pair(bf16lo(w[t]), bf16hi(w[t]), scale, scale, v[2 * t], v[2 * t + 1]);
                        if (DT == UQ_F32 && have == N) *(float4 *)at = make_float4(v[0], v[1], v[2], v[3]);
                        else {
#pragma unroll
                            for (int t = 0; t < N; ++t)
                                if (t < have) store1<DT>(at, t, v[t]);
                        }
                    }
                }
            }
        } else {
            // lane l fetches codes 8 l .. 8 l + 7 of the piece and (of the first eight lanes) the scale of block l
            const int64_t first = piece * 256, left = q.cols - first - lane;
            uint32_t codes = 0, byte = 0;
            if (first + lane * 8 < q.cols) codes = __ldg((const uint32_t *)(q.codes + row * q.code_stride + (first >> 1)) + lane);
            if (lane < 8 && first + lane * 32 < q.cols) byte = __ldg(q.scales + mx_scale_at(row, piece * 8 + lane, kt));
            const float mine = mx_scale_value(byte);
            char *at = (char *)out + (row * ld + first + lane) * Elem<DT>::BYTES;
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const uint32_t code = __shfl_sync(0xFFFFFFFFu, codes, 4 * t + (lane >> 3)) >> (4 * (lane & 7));
                const float scale = __shfl_sync(0xFFFFFFFFu, mine, t);
                if (32 * t < left) store1<DT>(at, 32 * t, mx_code_value(code) * scale);
            }
        }
        group += row_step;
        piece += piece_step;
        if (piece >= pieces) { piece -= pieces; ++group; }
    }
}

// A CTA takes a quarter of a tile where there are few tiles (bf16, both ways, stochastic: 1023 x 2037 11.7 -> 7.0 us, 2048 x 2048
// 12.8 -> 9.5, 2048 x 4096 17.3 -> 17.6, 4096 x 4096 28.5 -> 33.6), and wherever binary32 columns go through shared memory, whose
// whole tile leaves an SM few CTAs (4096 x 4096 41.9 -> 37.9 us, 16384 x 8192 340 -> 294; rows alone 146 -> 183).
constexpr int64_t kQuarterTiles = 300;

template <int DT, bool SR>
void launch_tile(const void *x, int64_t rows, int64_t cols, int64_t ld, const PhiloxKey &key, const uq_mx &q, const uq_mx &qt,
                 uint32_t *status, cudaStream_t st)
{
    const bool wide = ((uintptr_t)x & 15) == 0 && (ld * Elem<DT>::BYTES & 15) == 0 && (cols & 7) == 0;
    const int64_t tiles = mx_ktiles(cols) * mx_ktiles(rows);
    const bool small = tiles <= kQuarterTiles || (DT == UQ_F32 && qt.codes != nullptr);
    const size_t tile = small ? kTileBytes<DT, 32> + (SR ? kTileBytes<UQ_BF16, 32> : 0) : kTileBytes<UQ_BF16, 128> * (SR ? 2 : 1);
    const size_t smem = 1024 + (qt.codes != nullptr ? tile : 0);
    auto kernel = small ? (wide ? quantize_tile_kernel<DT, SR, true, 32> : quantize_tile_kernel<DT, SR, false, 32>)
                        : (wide ? quantize_tile_kernel<DT, SR, true, 128> : quantize_tile_kernel<DT, SR, false, 128>);
    if (smem > 48 * 1024) cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    launch_k_smem(kernel, dim3((unsigned)(small ? 4 * tiles : tiles)), dim3(kQThreads), smem, st, x, rows, cols, ld, key, q, qt, status);
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
    const bool wide = ((uintptr_t)out & 15) == 0 && (ld * (dtype == UQ_BF16 ? 2 : 4) & 15) == 0;
    const int64_t warps = (wide ? (q.rows + kDequantRows - 1) / kDequantRows : q.rows) * ((q.cols + 255) >> 8);
    const unsigned grid = (unsigned)min((warps * 32 + kQThreads - 1) / kQThreads, (int64_t)148 * 64);
    if (dtype == UQ_BF16) launch_k(wide ? dequantize_kernel<UQ_BF16, true> : dequantize_kernel<UQ_BF16, false>, dim3(grid), dim3(kQThreads), st, q, out, ld);
    else launch_k(wide ? dequantize_kernel<UQ_F32, true> : dequantize_kernel<UQ_F32, false>, dim3(grid), dim3(kQThreads), st, q, out, ld);
    return cudaGetLastError();
}

}  // namespace uq
