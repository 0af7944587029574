// out[i][j] = sum over k of a[i][k] b[j][k] (+ add[i][j]) of two microscaled 4-bit matrices, on the tensor cores.
//
// The multiply takes 64 columns of both operands and their scales (one power of two per 32) and adds up in binary32 in tensor
// memory.  b's rows (the weights; out's columns) are the instruction's 128 rows, i.e. tensor memory's lanes, and a's rows (the
// tokens) its columns: few tokens then cost few columns, and a warp's 32 lanes are 32 neighbouring elements of a row of out, so
// stores need no staging whatever out's alignment and stride.
//
// Few tokens are bound by reading the weights.  From HBM, where a model's layers lie between one token and the next (a ring of
// matrices of 400 MB, as a graph): 1 x 8192 x 4096 (17.8 MB) 6.4 us, 2.8 TB/s, 16 x 16384 x 8192 14.0 us, 5.1 TB/s, 37 x 10000 x 5010 9.8
// us, 2.8 TB/s; the same matrix again and again, out of the L2 cache: 5.2, 8.9 and 8.2 us.  Large products are bound by the tensor
// core and the board's power (8192^3: 184 us after a pause, 6.0 PFLOP/s; 207 to 214 us back to back).
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
    int32_t split;                                         // CTAs (of one cluster) that share a tile's columns: 1, 2, 4 or 8
};

constexpr int kRows = 128;                                 // of b per tile
constexpr int kStageK = 256;                               // columns per stage: 128 bytes of a row
// Warp 0 copies, warp 1 multiplies, the others store: PARTS warps for each quarter of the lanes, taking turns of 16 columns.
constexpr int kPairParts = 4;
constexpr int threads_of(int parts) { return 64 + 128 * parts; }

template <int DT> __device__ __forceinline__ float load1(const void *base, int64_t at)
{
    if constexpr (DT == UQ_BF16) return __uint_as_float((uint32_t)((const unsigned short *)base)[at] << 16);
    else return ((const float *)base)[at];
}

template <int DT> __device__ __forceinline__ void store_result(const ProductArgs &p, int64_t i, int64_t j, float v)
{
    if (p.add != nullptr) v += load1<DT>(p.add, i * p.add_ld + j);
    store1<DT>(p.out, i * p.ld + j, v);
}

// 16 rows of out (or of what is added) from row i on, in this lane's column of the 32 from j0 on; `have` of them exist.  A row's
// address is the same for a warp; a lane adds its offset, which stays.
template <int DT> __device__ __forceinline__ void load_column(const void *base, int64_t ld, int64_t i, int64_t j0, int lane, int have, float (&v)[16])
{
    const char *row = (const char *)base + (i * ld + j0) * Elem<DT>::BYTES;
    const uint32_t off = lane * Elem<DT>::BYTES;
    if (have >= 16) {
#pragma unroll
        for (int t = 0; t < 16; ++t, row += ld * Elem<DT>::BYTES) v[t] = load1<DT>(row + off, 0);
    } else {
#pragma unroll
        for (int t = 0; t < 16; ++t, row += ld * Elem<DT>::BYTES) v[t] = t < have ? load1<DT>(row + off, 0) : 0.0f;
    }
}
template <int DT> __device__ __forceinline__ void store_column(void *base, int64_t ld, int64_t i, int64_t j0, int lane, int have, const float (&v)[16])
{
    char *row = (char *)base + (i * ld + j0) * Elem<DT>::BYTES;
    const uint32_t off = lane * Elem<DT>::BYTES;
    if (have >= 16) {
#pragma unroll
        for (int t = 0; t < 16; ++t, row += ld * Elem<DT>::BYTES) store1<DT>(row + off, 0, v[t]);
    } else {
#pragma unroll
        for (int t = 0; t < 16; ++t, row += ld * Elem<DT>::BYTES)
            if (t < have) store1<DT>(row + off, 0, v[t]);
    }
}

// The multiplies of one stage: four of 64 columns (fewer in the row's last stage), with the copies of their scales to tensor
// memory in front.  One thread issues everything that the tensor core does, so its instructions count: descriptors are their
// low words plus constants, and nothing is decided in a whole stage.  `codes`, `scales`: low descriptor words of b's rows (a's
// are A_AT bytes behind) and of b's scales (a's are 1024 bytes behind); `columns`: where the scales go.
template <int CTAS, int NT, int A_AT> __device__ __forceinline__ void multiply_stage(uint32_t sums, uint32_t codes, uint32_t scales,
                                                                                     uint32_t columns, int steps, bool onto)
{
    constexpr int M = CTAS * kRows, W = (NT + 127) / 128, HALF = 4 + 4 * W;
    const auto operand = [](uint32_t lo) { return (uint64_t)lo | operand_descriptor(0) & 0xFFFFFFFF00000000ull; };
    const auto scale = [](uint32_t lo) { return (uint64_t)lo | scales_descriptor(0) & 0xFFFFFFFF00000000ull; };
#pragma unroll
    for (int h = 0; h < 2; ++h) {                          // a scale tile: 128 columns
        if (h == 1 && steps <= 2) continue;
        const uint32_t sb = columns + h * HALF, sa = sb + 4;
        tmem_copy_scales<CTAS>(sb, scale(scales + h * (512 >> 4)));
#pragma unroll
        for (int w = 0; w < W; ++w) tmem_copy_scales<CTAS>(sa + 4 * w, scale(scales + ((1024 + w * 1024 + h * 512) >> 4)));
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            if (q == 1 && steps == 2 * h + 1) continue;
            const uint32_t at = codes + (2 * h + q) * (32 >> 4);
            mma_mxf4<CTAS>(sums, operand(at), operand(at + (A_AT >> 4)), mxf4_instruction(M, NT, q), sb, sa, onto || h > 0 || q > 0);
        }
    }
}

template <int NT> struct ProductShape {
    static constexpr int kStageBytes = kRows * 128 + NT * 128 + 2048;
    static constexpr int kStages = NT == 128 ? 3 : NT == 16 ? 5 : 4;      // two CTAs fit an SM
    static constexpr int kParts = NT >= 64 ? 2 : 1, kThreads = threads_of(kParts);
    static constexpr int kScaleColumns = 16;               // per stage: 2 x 4 of each operand
    static constexpr int kColumns = NT + kStages * kScaleColumns <= 128 ? 128 : 256;
    static constexpr int kSmem = kStages * kStageBytes + 1024 + 256;
};

// Adds up columns c0 .. c1 - 1 of a tile's sums from the R CTAs of a cluster, in their order: four neighbouring rows of b per thread
// and piece, the loads of U pieces from all CTAs in flight together.
template <int DT, int U, int R, int THREADS>
__device__ __forceinline__ void join_sums(const ProductArgs &p, uint32_t data, int c0, int c1, int64_t m0, int64_t n0)
{
    const int pieces = (c1 - c0) * (kRows / 4);
    for (int e = threadIdx.x; e < pieces; e += U * THREADS) {
        float4 w[U][R];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (e + u * THREADS < pieces) {
                    const int i = e + u * THREADS;
                    w[u][r] = cluster_load4(cluster_address(data + ((c0 + i / (kRows / 4)) * kRows + i % (kRows / 4) * 4) * 4, r));
                }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = e + u * THREADS, c = c0 + i / (kRows / 4), l = i % (kRows / 4) * 4;
            if (i >= pieces) break;
            float4 v = w[u][0];
#pragma unroll
            for (int r = 1; r < R; ++r) { v.x += w[u][r].x; v.y += w[u][r].y; v.z += w[u][r].z; v.w += w[u][r].w; }
            const int64_t left = p.n - n0 - l;
            if (left > 0) store_result<DT>(p, m0 + c, n0 + l, v.x);
            if (left > 1) store_result<DT>(p, m0 + c, n0 + l + 1, v.y);
            if (left > 2) store_result<DT>(p, m0 + c, n0 + l + 2, v.z);
            if (left > 3) store_result<DT>(p, m0 + c, n0 + l + 3, v.w);
        }
    }
}

// A tile of 128 rows of b and NT of a.  With split > 1 the CTAs of a cluster take a share of the columns each, put their sums
// into shared memory, and each adds up a share of the tile in the CTAs' order.
template <int NT, int DT>
__global__ void __launch_bounds__(ProductShape<NT>::kThreads) product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
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

    const int tid = threadIdx.x, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), lane = tid & 31;
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
    if (warp == 1) tmem_alloc<1>(smem_address(tmem_slot), S::kColumns);
    tensor_fence_before();
    __syncthreads();
    tensor_fence_after();
    const uint32_t tmem = *(volatile uint32_t *)tmem_slot;

    if (warp == 0) {
        const bool one = elect_lane();
        const uint8_t *scales_b = p.scales_b + (n0 >> 7) * p.ktiles * 512, *scales_a = p.scales_a + (m0 >> 7) * p.ktiles * 512;
        for (int i = s0, s = 0, parity = 1; i < s1; ++i) {
            if (i - s0 >= ST && !barrier_wait_warp(empty + 8 * s, parity, gave_up)) break;
            const uint32_t at = data + s * S::kStageBytes, bar = full + 8 * s;
            const uint32_t scale_bytes = p.ktiles - 2 * (int64_t)i >= 2 ? 1024 : 512;
            if (one) {
                barrier_expect(bar, kRows * 128 + NT * 128 + 2 * scale_bytes);
                copy_tile(at, &map_b, i * 128, (int)n0, bar);
                copy_tile(at + kRows * 128, &map_a, i * 128, (int)m0, bar);
                copy_bulk(at + kRows * 128 + NT * 128, scales_b + (int64_t)i * 1024, scale_bytes, bar);
                copy_bulk(at + kRows * 128 + NT * 128 + 1024, scales_a + (int64_t)i * 1024, scale_bytes, bar);
                *issued = i - s0 + 1;
            }
            __syncwarp();
            if (++s == ST) { s = 0; parity ^= 1; }
        }
    } else if (warp == 1) {
        const bool one = elect_lane();                     // the same for all: a commit waits for what its own thread has issued
        const uint32_t codes = (uint32_t)operand_descriptor(data), scales = (uint32_t)scales_descriptor(data + kRows * 128 + NT * 128);
        for (int i = s0, s = 0, parity = 0; i < s1; ++i) {
            if (!barrier_wait_warp(full + 8 * s, parity, gave_up)) break;
            tensor_fence_after();
            const int steps = (int)min((int64_t)4, (p.k - (int64_t)i * kStageK + 63) >> 6);
            if (one) {
                multiply_stage<1, NT, kRows * 128>(tmem, codes + s * (S::kStageBytes >> 4), scales + s * (S::kStageBytes >> 4),
                                                   tmem + NT + s * S::kScaleColumns, steps, i > s0);
                tensor_commit<1>(empty + 8 * s);
            }
            __syncwarp();
            if (++s == ST) { s = 0; parity ^= 1; }
        }
        if (one) tensor_commit<1>(done);
        __syncwarp();
        int again = 0;                                     // (a wait of its own: tensor memory is given back only when nothing writes it)
        if (!barrier_wait_warp(done, 0, &again)) *gave_up = 1;
    }
    __syncwarp();

    if (warp >= 2) {
        barrier_wait_warp(done, 0, gave_up);
        tensor_fence_after();
        const int quarter = warp & 3;
        const int64_t j0 = n0 + quarter * 32;
        const uint32_t acc = tmem + ((uint32_t)(quarter * 32) << 16);
#pragma unroll 1
        for (int c = ((warp - 2) >> 2) * 16; c < NT; c += 16 * S::kParts) {
            float v[16];
            __syncwarp();
            tmem_load16(acc + c, v);
            tmem_load_wait();
            if (p.split > 1) {
                float *sums = (float *)base;               // every stage has been read: [column][lane]
#pragma unroll
                for (int t = 0; t < 16; ++t) sums[(c + t) * kRows + quarter * 32 + lane] = v[t];
            } else if (j0 + lane < p.n && m0 + c < p.m) {
                const int have = (int)min((int64_t)16, p.m - m0 - c);
                if (p.add != nullptr) {                    // all of it first: it may be out itself, so no load moves in front of a store
                    float w[16];
                    load_column<DT>(p.add, p.add_ld, m0 + c, j0, lane, have, w);
#pragma unroll
                    for (int t = 0; t < 16; ++t) v[t] += w[t];
                }
                store_column<DT>(p.out, p.ld, m0 + c, j0, lane, have, v);
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
        tmem_free<1>(tmem, S::kColumns);
    }
    if (p.split > 1) {
        cluster_sync();
        const int c0 = NT * (int)rank / p.split, c1 = min(NT * ((int)rank + 1) / p.split, (int)min((int64_t)NT, p.m - m0));
        if (p.split == 2) join_sums<DT, 4, 2, S::kThreads>(p, data, c0, c1, m0, n0);
        else if (p.split == 4) join_sums<DT, 2, 4, S::kThreads>(p, data, c0, c1, m0, n0);
        else join_sums<DT, 1, 8, S::kThreads>(p, data, c0, c1, m0, n0);
        cluster_sync();                                    // the others may still be reading here
    }
}

// ---- large products: pairs of CTAs ----------------------------------------------------------------
//
// A pair of CTAs multiplies 256 rows of b (128 in either CTA's tensor memory) by NT of a: each fetches its 128 rows of b, half of
// a's rows, and the scales of both; the even CTA issues the multiplies for both.  Per multiply-add that is half the shared memory
// traffic and half the reads of a single CTA's tile of 128 x 128.  The pairs stay and take one tile after another; a tile's sums
// are stored while the next tile is multiplied.  Tensor memory holds the sums of two tiles that overlap in the columns that the
// scales leave too few: those are stored first, and the next tile starts when they are.

template <int NT> struct PairShape {
    static constexpr int kStageBytes = kRows * 128 + NT / 2 * 128 + 1024 + (NT + 127) / 128 * 1024;
    static constexpr int kStages = 6;
    static constexpr int kScaleSlots = 3;                  // a slot's scales are overwritten when its multiplies are done
    static constexpr int kSlotColumns = 2 * (4 + (NT + 127) / 128 * 4);
    static constexpr int kScales = 512 - kScaleSlots * kSlotColumns;      // first column of the scales
    static constexpr int kSecond = kScales - NT < NT ? (kScales - NT) / 16 * 16 : NT;   // first column of the second tile's sums
    static constexpr int kShared = NT - kSecond;           // columns that are stored first
    static_assert(kShared >= 16 * kPairParts && kSecond + NT <= kScales, "each storing warp has a part of the shared columns");
    static constexpr int kSmem = kStages * kStageBytes + 1024 + 256;
};

// The tile at a place in the order of the work: groups of eight rows of tiles, so that what runs at one time shares its operands
// in the L2 cache.
__device__ __forceinline__ void tile_place(int64_t t, int64_t tiles_m, int64_t tiles_n, int64_t *tm, int64_t *tn)
{
    const int64_t group = t / (8 * tiles_n), first = group * 8, height = min((int64_t)8, tiles_m - first), in = t - group * 8 * tiles_n;
    *tm = first + in % height;
    *tn = in / height;
}

template <int NT, int DT>
__global__ void __launch_bounds__(threads_of(kPairParts)) __cluster_dims__(2, 1, 1)
product_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                    const __grid_constant__ CUtensorMap map_sa, const __grid_constant__ CUtensorMap map_sb, const ProductArgs p)
{
    using S = PairShape<NT>;
    constexpr int ST = S::kStages;
    extern __shared__ unsigned char raw[];
    unsigned char *base = (unsigned char *)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    const uint32_t data = smem_address(base);
    uint64_t *bars = (uint64_t *)(base + ST * S::kStageBytes);
    const uint32_t full = smem_address(bars), empty = full + 8 * ST, sums_ready = full + 16 * ST, sums_free = sums_ready + 8, drained = sums_ready + 16;
    uint32_t *tmem_slot = (uint32_t *)(bars + 2 * ST + 3);
    volatile int *gave_up = (volatile int *)(tmem_slot + 1);
    volatile int *issued = gave_up + 1;

    const int tid = threadIdx.x, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), lane = tid & 31;
    const uint32_t rank = cluster_rank();
    const int64_t tiles_n = (p.n + 255) / 256, tiles_m = (p.m + NT - 1) / NT, tiles = tiles_m * tiles_n;
    const int64_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int stages = (int)((p.k + kStageK - 1) / kStageK);

    grid_dependency_trigger();
    if (tid == 0) {
        for (int s = 0; s < 2 * ST + 1; ++s) barrier_init(full + 8 * s, 1);
        barrier_init(sums_free, 8 * kPairParts);           // the storing warps of both CTAs
        barrier_init(drained, 1);
        *gave_up = 0;
        *issued = 0;
        barrier_init_visible();
    }
    grid_dependency_wait();
    if (warp == 1) tmem_alloc<2>(smem_address(tmem_slot), 512);
    tensor_fence_before();
    __syncthreads();
    cluster_sync();                                        // both CTAs' barriers are there
    tensor_fence_after();
    const uint32_t tmem = *(volatile uint32_t *)tmem_slot;

    if (warp == 0) {
        const bool one = elect_lane();
        const uint32_t leader_full = cluster_address(full, 0);
        int use = 0, s = 0, parity = 1;                    // stages filled so far; the next one, and the parity of its release
        bool going = true;
        for (int64_t t = pair; going && t < tiles; t += pairs) {
            int64_t tm, tn;
            tile_place(t, tiles_m, tiles_n, &tm, &tn);
            const int row_b = (int)(tn * 256 + rank * 128), row_a = (int)(tm * NT + rank * (NT / 2)), strip_a = (int)(tm * NT >> 7);
            for (int i = 0; i < stages; ++i) {
                going = use < ST || barrier_wait_warp(empty + 8 * s, parity, gave_up);
                if (!going) break;
                const uint32_t at = data + s * S::kStageBytes, bar = leader_full + 8 * s;
                ++use;
                if (one) {
                    if (rank == 0) barrier_expect(full + 8 * s, 2 * S::kStageBytes);
                    copy_tile_pair(at, &map_b, i * 128, row_b, bar);
                    copy_tile_pair(at + kRows * 128, &map_a, i * 128, row_a, bar);
                    copy_tile_pair(at + kRows * 128 + NT / 2 * 128, &map_sb, i * 256, row_b >> 7, bar);
                    copy_tile_pair(at + kRows * 128 + NT / 2 * 128 + 1024, &map_sa, i * 256, strip_a, bar);
                    *issued = use;
                }
                __syncwarp();
                if (++s == ST) { s = 0; parity ^= 1; }
            }
        }
    } else if (warp == 1 && rank == 0) {
        const bool one = elect_lane();                     // the same for all: a commit waits for what its own thread has issued
        const uint32_t codes = (uint32_t)operand_descriptor(data), scales = (uint32_t)scales_descriptor(data + kRows * 128 + NT / 2 * 128);
        const int last_steps = (int)((p.k - (int64_t)(stages - 1) * kStageK + 63) >> 6);
        int s = 0, parity = 0, slot = 0, turn = 0;
        int old = -S::kScaleSlots, old_parity = 0;         // the stage whose scales are overwritten (below 0: none yet)
        bool going = true;
        for (int64_t t = pair; going && t < tiles; t += pairs, ++turn) {
            if (turn > 0 && !barrier_wait_warp(sums_free, (turn - 1) & 1, gave_up)) break;
            tensor_fence_after();
            const uint32_t sums = tmem + (turn & 1) * S::kSecond;
            for (int i = 0; i < stages; ++i) {
                going = (old < 0 || barrier_wait_warp(empty + 8 * old, old_parity, gave_up)) && barrier_wait_warp(full + 8 * s, parity, gave_up);
                if (!going) break;
                tensor_fence_after();
                if (one) {
                    multiply_stage<2, NT, kRows * 128>(sums, codes + s * (S::kStageBytes >> 4), scales + s * (S::kStageBytes >> 4),
                                                       tmem + S::kScales + slot * S::kSlotColumns, i + 1 < stages ? 4 : last_steps, i > 0);
                    tensor_commit<2>(empty + 8 * s);
                }
                __syncwarp();
                if (++s == ST) { s = 0; parity ^= 1; }
                if (++slot == S::kScaleSlots) slot = 0;
                if (++old == ST) { old = 0; old_parity ^= 1; }
            }
            if (going && one) tensor_commit<2>(sums_ready);
            __syncwarp();
        }
        if (*gave_up != 0) {                               // tensor memory is given back only when nothing writes it
            int again = 0;
            if (one) tensor_commit<2>(drained);
            __syncwarp();
            barrier_wait_warp(drained, 0, &again);
        }
    } else if (warp >= 2) {
        // What is added to a piece is loaded a piece ahead, the first piece's before the sums are there.
        const int quarter = warp & 3, part = (warp - 2) >> 2;
        const uint32_t free_bar = cluster_address(sums_free, 0);
        int turn = 0;
        for (int64_t t = pair; t < tiles; t += pairs, ++turn) {
            int64_t tm, tn;
            tile_place(t, tiles_m, tiles_n, &tm, &tn);
            const int64_t j0 = tn * 256 + rank * 128 + quarter * 32, m0 = tm * NT;
            const uint32_t sums = tmem + (turn & 1) * S::kSecond + ((uint32_t)(quarter * 32) << 16);
            // the first of two overlapping tiles shares its last columns, the second its first
            const int first = turn & 1 ? 0 : NT - S::kShared;
            const auto column = [&](int done) { return first + done < NT ? first + done : first + done - NT; };
            const auto rows_there = [&](int c) { return (int)max((int64_t)0, min((int64_t)16, p.m - m0 - c)); };
            const bool mine = j0 + lane < p.n;
            float w[16];
            if (p.add != nullptr && mine) load_column<DT>(p.add, p.add_ld, m0 + column(part * 16), j0, lane, rows_there(column(part * 16)), w);
            if (!barrier_wait_warp(sums_ready, turn & 1, gave_up)) break;
            tensor_fence_after();
#pragma unroll 1
            for (int done = part * 16; done < NT; done += 16 * kPairParts) {
                const int c = column(done), have = rows_there(c);
                float v[16];
                __syncwarp();
                tmem_load16(sums + c, v);
                tmem_load_wait();
                if (done < S::kShared && done + 16 * kPairParts >= S::kShared) {
                    tensor_fence_before();
                    __syncwarp();
                    if (lane == 0) cluster_arrive(free_bar);
                }
                if (p.add != nullptr) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) v[k] += w[k];
                    const int after = done + 16 * kPairParts, next = column(after < NT ? after : done);
                    if (after < NT && mine) load_column<DT>(p.add, p.add_ld, m0 + next, j0, lane, rows_there(next), w);
                }
                if (have > 0 && mine) store_column<DT>(p.out, p.ld, m0 + c, j0, lane, have, v);
            }
        }
    }
    __syncwarp();
    __syncthreads();
    if (*gave_up != 0 && tid == 0) {
        if (p.status != nullptr) atomicOr(p.status, UQ_STATUS_TIMEOUT);
        // copies of both CTAs that are still on their way must land before their memory is another's
        const int n = *issued;
        for (int i = n > ST ? n - ST : 0; rank == 0 && i < n; ++i) {
            int again = 0;
            barrier_wait(full + 8 * (i % ST), (i / ST) & 1, &again);
        }
    }
    __syncwarp();
    tensor_fence_before();
    cluster_sync();                                        // the pair's other CTA is done with this one's memory
    if (warp == 1) {
        tensor_fence_after();
        tmem_free<2>(tmem, 512);
    }
}

// An allocation of tensor memory waits until there is enough, and CTAs of a cluster that wait for one another's SM could wait for
// good.  None has to wait: shared memory lets two CTAs of product_kernel onto an SM, whose columns (512 there are) fit beside each
// other, or one of a pair, which takes all columns, with no other.
constexpr int kSmShared = 228 * 1024, kCtaShared = 1024;   // bytes of an SM, and what each CTA takes of them beside its own
template <int... NT> constexpr int least_smem()
{
    int least = kSmShared;
    ((least = ProductShape<NT>::kSmem + kCtaShared < least ? ProductShape<NT>::kSmem + kCtaShared : least), ...);
    return least;
}
template <int... NT> constexpr bool half_the_columns() { return ((ProductShape<NT>::kColumns <= 256) && ...); }
static_assert(3 * least_smem<16, 32, 64, 128>() > kSmShared && half_the_columns<16, 32, 64, 128>(), "two CTAs per SM at most, half of the columns each");
static_assert(PairShape<256>::kSmem + kCtaShared + least_smem<16, 32, 64, 128>() > kSmShared, "a pair's CTA has its SM to itself");

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

// Two scale tiles (1024 bytes) of `strips` strips of 128 rows.
bool scales_map(CUtensorMap *map, const uq_mx &q, int strips)
{
    const EncodeTiled encode = encode_tiled();
    const cuuint64_t size[2] = {(cuuint64_t)mx_ktiles(q.cols) * 128, (cuuint64_t)mx_ktiles(q.rows)}, stride[1] = {size[0] * 4};
    const cuuint32_t box[2] = {256, (cuuint32_t)strips}, step[2] = {1, 1};
    return encode != nullptr &&
           encode(map, CU_TENSOR_MAP_DATA_TYPE_INT32, 2, q.scales, size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int NT, int DT> cudaError_t launch_pairs(const uq_mx &a, const uq_mx &b, const ProductArgs &p, cudaStream_t st)
{
    using S = PairShape<NT>;
    auto kernel = product_pair_kernel<NT, DT>;
    CUtensorMap map_a, map_b, map_sa, map_sb;
    if (!codes_map(&map_a, a, NT / 2) || !codes_map(&map_b, b, kRows) || !scales_map(&map_sa, a, (NT + 127) / 128) || !scales_map(&map_sb, b, 1))
        return cudaErrorInvalidValue;
    cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    const int64_t tiles = (p.n + 255) / 256 * ((p.m + NT - 1) / NT);
    launch_k_smem(kernel, dim3((unsigned)(min(tiles, (int64_t)74) * 2)), dim3(threads_of(kPairParts)), S::kSmem, st, map_a, map_b, map_sa, map_sb, p);
    return cudaGetLastError();
}

// CTAs that share a tile's columns, from measured costs in microseconds: a stage takes 0.2 + 0.0014 NT of one CTA on an SM (two on
// an SM share it), joining the sums 1.3 + 0.014 NT, and 0.015 NT more where clusters share SMs.  4 x 4096 x 4096: 5.5 alone, 4.4 by
// four; 182 x 836 x 7433: 14.7 and, by eight, 7.7; 128 x 8192 x 8192: 16.2 and, by two, 13.8; 512 x 4096 x 4096, which has an SM for
// each tile as it is: 7.3 and, by two, 11.1.
int best_split(int nt, int64_t tiles, int64_t stages)
{
    int best = 1;
    double least = 1e30;
    for (int s = 1; s <= 8 && s <= stages && (s == 1 || tiles * s <= 296); s *= 2) {
        const double load = tiles * s > 148 ? (double)(tiles * s) / 148.0 : 1.0;
        const double join = s > 1 ? 1.3 + 0.014 * nt + (tiles * s > 148 ? 0.015 * nt : 0.0) : 0.0;
        const double t = load * (double)((stages + s - 1) / s) * (0.2 + 0.0014 * nt) + join;
        if (t < least) { least = t; best = s; }
    }
    return best;
}

template <int NT, int DT> cudaError_t launch_tiles(const uq_mx &a, const uq_mx &b, ProductArgs p, cudaStream_t st)
{
    using S = ProductShape<NT>;
    auto kernel = product_kernel<NT, DT>;
    CUtensorMap map_a, map_b;
    if (!codes_map(&map_a, a, NT) || !codes_map(&map_b, b, kRows)) return cudaErrorInvalidValue;
    cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    const int64_t tiles = (p.n + kRows - 1) / kRows * ((p.m + NT - 1) / NT), stages = (p.k + kStageK - 1) / kStageK;
    p.split = best_split(NT, tiles, stages);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * p.split));
    cfg.blockDim = dim3(S::kThreads);
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
    // Pairs where there are more tiles of 128 x 128 than SMs (us, pairs against tiles: 700 x 5000 x 3000 9.3 and 11.1, 2000^3 8.9 and
    // 10.6, 1024 x 4096 x 4096 10.7 and 10.9, 2048 x 2304 x 1024 7.0 and 6.1; with an SM for each tile 512 x 4096 x 4096 10.0 and 7.4).
    if ((p.n + 127) / 128 * ((p.m + 127) / 128) > 148) return launch_pairs<256, DT>(a, b, p, st);
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
