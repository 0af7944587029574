// out[i][j] = sum over k of a[i][k] b[j][k] (+ add[i][j]) of two microscaled 4-bit matrices, on the tensor cores.
//
// The multiply takes 64 columns of both operands and their scales (one power of two per 32) and adds up in binary32 in tensor
// memory.  b's rows (the weights; out's columns) are the instruction's 128 rows, i.e. tensor memory's lanes, and a's rows (the
// tokens) its columns: few tokens then cost few columns, and a warp's 32 lanes are 32 neighbouring elements of a row of out, so
// stores need no staging whatever out's alignment and stride.
#include "uq_tensor.cuh"
#include "uq_mx.cuh"

namespace uq {
namespace {

struct ProductArgs {
    int64_t m, n, k;                                       // rows of a, rows of b, columns of both
    int64_t ktiles;                                        // scale tiles along a row
    const uint8_t *scales_a, *scales_b;
    const void *add;
    void *out;
    int64_t add_ld, ld;
    uint32_t *status;
    int32_t split;                                         // CTAs (of one cluster) that share a tile's columns
};

constexpr int kRows = 128;                                 // of b per tile
constexpr int kStageK = 256;                               // columns per stage: 128 bytes of a row
constexpr int kPThreads = 192;                             // warp 0 copies, warp 1 multiplies, warps 2 to 5 store

template <int DT> __device__ __forceinline__ void store_result(const ProductArgs &p, int64_t i, int64_t j, float v)
{
    if (p.add != nullptr) {
        if constexpr (DT == UQ_BF16) v += __uint_as_float((uint32_t)((const unsigned short *)p.add)[i * p.add_ld + j] << 16);
        else v += ((const float *)p.add)[i * p.add_ld + j];
    }
    store1<DT>(p.out, i * p.ld + j, v);
}

template <int NT> struct ProductShape {
    static constexpr int kStageBytes = kRows * 128 + NT * 128 + 2048;
    static constexpr int kStages = NT == 128 ? 3 : 6;
    static constexpr int kScaleColumns = 16;               // per stage: 2 x 4 of each operand
    static constexpr int kColumns = NT + kStages * kScaleColumns <= 128 ? 128 : 256;
    static constexpr int kSmem = kStages * kStageBytes + 1024 + 256;
};

// A tile of 128 rows of b and NT of a.  With split > 1 the CTAs of a cluster take a share of the columns each, put their sums
// into shared memory, and each adds up a share of the tile in the CTAs' order.
template <int NT, int DT>
__global__ void __launch_bounds__(kPThreads) product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                            const ProductArgs p)
{
    using S = ProductShape<NT>;
    constexpr int ST = S::kStages;
    extern __shared__ unsigned char raw[];
    unsigned char *base = (unsigned char *)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    const uint32_t data = smem_address(base);
    uint64_t *bars = (uint64_t *)(base + ST * S::kStageBytes);            // full, empty, done
    const uint32_t full = smem_address(bars), empty = full + 8 * ST, done = full + 16 * ST;
    uint32_t *tmem_slot = (uint32_t *)(bars + 2 * ST + 1);
    volatile int *gave_up = (volatile int *)(tmem_slot + 1);
    volatile int *issued = gave_up + 1;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = p.split > 1 ? cluster_rank() : 0;
    const int64_t tiles_n = (p.n + kRows - 1) / kRows;
    const int64_t tile = blockIdx.x / p.split, n0 = tile % tiles_n * kRows, m0 = tile / tiles_n * NT;
    const int64_t stages = (p.k + kStageK - 1) / kStageK;
    const int s0 = (int)(stages * rank / p.split), s1 = (int)(stages * (rank + 1) / p.split);

    grid_dependency_trigger();
    if (tid == 0) {
        for (int s = 0; s < 2 * ST + 1; ++s) barrier_init(full + 8 * s, 1);
        *gave_up = 0;
        *issued = 0;
        barrier_init_visible();
    }
    grid_dependency_wait();                                // tensor memory too is taken only after the kernel in front has given its back
    if (warp == 1) tmem_alloc(smem_address(tmem_slot), S::kColumns);
    tensor_fence_before();
    __syncthreads();
    tensor_fence_after();
    const uint32_t tmem = *(volatile uint32_t *)tmem_slot;

    if (warp == 0 && lane == 0) {
        for (int i = s0; i < s1; ++i) {
            const int s = (i - s0) % ST, round = (i - s0) / ST;
            if (round > 0 && !barrier_wait(empty + 8 * s, (round - 1) & 1, gave_up)) break;
            const uint32_t at = data + s * S::kStageBytes, bar = full + 8 * s;
            const uint32_t scale_bytes = p.ktiles - 2 * (int64_t)i >= 2 ? 1024 : 512;
            barrier_expect(bar, kRows * 128 + NT * 128 + 2 * scale_bytes);
            copy_tile(at, &map_b, i * 128, (int)n0, bar);
            copy_tile(at + kRows * 128, &map_a, i * 128, (int)m0, bar);
            copy_bulk(at + kRows * 128 + NT * 128, p.scales_b + ((n0 >> 7) * p.ktiles + 2 * (int64_t)i) * 512, scale_bytes, bar);
            copy_bulk(at + kRows * 128 + NT * 128 + 1024, p.scales_a + ((m0 >> 7) * p.ktiles + 2 * (int64_t)i) * 512, scale_bytes, bar);
            *issued = i - s0 + 1;
        }
    } else if (warp == 1 && lane == 0) {
        for (int i = s0; i < s1; ++i) {
            const int s = (i - s0) % ST, round = (i - s0) / ST;
            if (!barrier_wait(full + 8 * s, round & 1, gave_up)) break;
            tensor_fence_after();
            const uint32_t at = data + s * S::kStageBytes, scales = at + kRows * 128 + NT * 128;
            const uint32_t sb = tmem + NT + s * S::kScaleColumns, sa = sb + 8;
            const uint64_t db = operand_descriptor(at), da = operand_descriptor(at + kRows * 128);
            const int64_t left = p.k - (int64_t)i * kStageK;
#pragma unroll
            for (int h = 0; h < 2; ++h) {                  // a scale tile: 128 columns
                if (left > 128 * h) {
                    tmem_copy_scales(sb + 4 * h, scales_descriptor(scales + 512 * h));
                    tmem_copy_scales(sa + 4 * h, scales_descriptor(scales + 1024 + 512 * h));
#pragma unroll
                    for (int q = 0; q < 2; ++q)
                        if (left > 128 * h + 64 * q)
                            mma_mxf4(tmem, db + (2 * h + q) * 2, da + (2 * h + q) * 2, mxf4_instruction(kRows, NT, q), sb + 4 * h, sa + 4 * h,
                                     i > s0 || h > 0 || q > 0);
                }
            }
            tensor_commit(empty + 8 * s);
        }
        tensor_commit(done);
        int again = 0;                                     // (a wait of its own: tensor memory is given back only when nothing writes it)
        if (!barrier_wait(done, 0, &again)) *gave_up = 1;
    }
    __syncwarp();

    if (warp >= 2) {
        barrier_wait(done, 0, gave_up);
        tensor_fence_after();
        const int quarter = warp & 3;
        const int64_t j = n0 + quarter * 32 + lane;
        const uint32_t acc = tmem + ((uint32_t)(quarter * 32) << 16);
#pragma unroll 1
        for (int c = 0; c < NT; c += 16) {
            float v[16];
            tmem_load16(acc + c, v);
            tmem_load_wait();
            if (p.split > 1) {
                float *sums = (float *)base;               // every stage has been read: [column][lane]
#pragma unroll
                for (int t = 0; t < 16; ++t) sums[(c + t) * kRows + quarter * 32 + lane] = v[t];
            } else if (j < p.n) {
                const int have = (int)min((int64_t)16, p.m - m0 - c);
#pragma unroll
                for (int t = 0; t < 16; ++t)
                    if (t < have) store_result<DT>(p, m0 + c + t, j, v[t]);
            }
        }
        tensor_fence_before();
    }
    __syncthreads();
    if (*gave_up != 0 && tid == 0) {
        // copies that are still on their way must land before the CTA's memory is another's
        if (p.status != nullptr) atomicOr(p.status, UQ_STATUS_TIMEOUT);
        const int n = *issued;
        for (int i = n > ST ? n - ST : 0; i < n; ++i) {
            int again = 0;
            barrier_wait(full + 8 * (i % ST), (i / ST) & 1, &again);
        }
    }
    __syncwarp();
    if (warp == 1) {
        tensor_fence_after();
        tmem_free(tmem, S::kColumns);
    }
    if (p.split > 1) {
        cluster_sync();
        const int share = NT / p.split;
        for (int e = tid; e < share * kRows; e += kPThreads) {
            const int c = (int)rank * share + e / kRows, l = e % kRows;
            float v = 0.0f;
            for (int r = 0; r < p.split; ++r) v += cluster_load(cluster_address(data + (c * kRows + l) * 4, r));
            if (m0 + c < p.m && n0 + l < p.n) store_result<DT>(p, m0 + c, n0 + l, v);
        }
        cluster_sync();                                    // the others may still be reading here
    }
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                 CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled()
{
    static const EncodeTiled fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            f = nullptr;
        return (EncodeTiled)f;
    }();
    return fn;
}

// Tiles of 128 bytes x `rows` rows of a matrix's codes; what lies outside the matrix reads as zeros.
bool codes_map(CUtensorMap *map, const uq_mx &q, int rows)
{
    const EncodeTiled encode = encode_tiled();
    const cuuint64_t size[2] = {(cuuint64_t)mx_blocks(q.cols) * 16, (cuuint64_t)q.rows}, stride[1] = {(cuuint64_t)q.code_stride};
    const cuuint32_t box[2] = {128, (cuuint32_t)rows}, step[2] = {1, 1};
    return encode != nullptr &&
           encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, q.codes, size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int NT, int DT> cudaError_t launch_tiles(const uq_mx &a, const uq_mx &b, ProductArgs p, cudaStream_t st)
{
    using S = ProductShape<NT>;
    auto kernel = product_kernel<NT, DT>;
    CUtensorMap map_a, map_b;
    if (!codes_map(&map_a, a, NT) || !codes_map(&map_b, b, kRows)) return cudaErrorInvalidValue;
    cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    const int64_t tiles = (p.n + kRows - 1) / kRows * ((p.m + NT - 1) / NT), stages = (p.k + kStageK - 1) / kStageK;
    // more CTAs per tile while that still leaves an SM each, and two stages
    p.split = 1;
    while (p.split < 8 && tiles * p.split * 2 <= 148 && stages >= p.split * 4) p.split *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * p.split));
    cfg.blockDim = dim3(kPThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    cfg.attrs = attr;
    cfg.numAttrs = grid_dependency_attribute(attr);
    if (p.split > 1) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        attr[cfg.numAttrs].val.clusterDim.x = p.split;
        attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
        ++cfg.numAttrs;
    }
    cudaLaunchKernelEx(&cfg, kernel, map_a, map_b, (const ProductArgs)p);
    return cudaGetLastError();
}

template <int DT> cudaError_t launch_product(const uq_mx &a, const uq_mx &b, const ProductArgs &p, cudaStream_t st)
{
    if (p.m <= 16) return launch_tiles<16, DT>(a, b, p, st);
    if (p.m <= 32) return launch_tiles<32, DT>(a, b, p, st);
    if (p.m <= 64) return launch_tiles<64, DT>(a, b, p, st);
    return launch_tiles<128, DT>(a, b, p, st);
}

}  // namespace

cudaError_t launch_mx_product(const uq_mx &a, const uq_mx &b, const void *add, int64_t add_ld, void *out, int64_t ld, int dtype,
                              uint32_t *status, cudaStream_t st)
{
    const ProductArgs p = {a.rows, b.rows, a.cols, mx_ktiles(a.cols), a.scales, b.scales, add, out, add_ld, ld, status, 1};
    return dtype == UQ_BF16 ? launch_product<UQ_BF16>(a, b, p, st) : launch_product<UQ_F32>(a, b, p, st);
}

}  // namespace uq
