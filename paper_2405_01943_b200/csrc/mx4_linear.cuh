// What the kernels of dass_linear_mx4 share: the arguments, the tensor maps, the walk of the persistent kernels over groups
// of rows.  Internal header.
#pragma once

#include "linear_common.cuh"
#include "mx4_common.cuh"
#include "tc_common.cuh"

namespace dass {

struct Mx4Matrix { const uint8_t *codes, *scales; };       // null codes: absent

struct Mx4Args {
    LinearArgs a;              // X null where x holds the rows; W, W_up and their strides unused; bf16
    Mx4Matrix x, w, up;        // rows [T x K]; weights [groups x N x K]
};

// Codes and scales of group g's matrix.
__host__ __device__ __forceinline__ Mx4Matrix mx4_group(const Mx4Matrix &m, int64_t g, int64_t N, int64_t K)
{
    return {m.codes + g * N * mx4_pitch(K), m.scales + g * ((N + MX4_TILE_ROWS - 1) / MX4_TILE_ROWS) * mx4_k_tiles(K) * MX4_TILE_BYTES};
}

// Warps of a block of mx4_few.cu.  16 hide the decoding's latency where each of them has two turns of k at least (up to 8 rows,
// 1 x 4096 x 4096: 6.8 against 7.2 us, 1 x 14336 x 4096 15.2 against 18.2; but 1 x 2048 x 2048 gated 8.3 against 6.4).
inline int mx4_few_warps(int64_t K, int eights, int split) { return eights == 1 && mx4_k_tiles(K) >= 32 * split ? 16 : 8; }

// ------------------------------------------------------------------ waits of the warp that issues the products
// A wait that finds its barrier complete still takes 130 cycles, as long as a short slab's products.  So the issuing warp
// asks for the next stage's barrier before it issues this one's products, and looks at the answer after them.
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Arrives on a barrier of the pair's leader for what is in TMEM: its order is the tcgen05 fence's before it, and there is no
// memory to be made visible (a release at cluster scope also waits for the warp's stores to Y: 1000 cycles).
__device__ __forceinline__ void mbar_arrive_tmem(uint32_t cluster_addr)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// A ring's place: stage and the parity of its barriers' phase.
struct Mx4Ring {
    uint32_t stage = 0, phase = 0;
    __device__ __forceinline__ void step(uint32_t stages) { if (++stage == stages) { stage = 0; phase ^= 1u; } }
};

// ------------------------------------------------------------------ descriptors of the block-scaled products
// Descriptor of 32 rows of 16 bytes, one after the other, for tcgen05.cp: 8-row groups 128 bytes apart, no swizzle.
__device__ __forceinline__ uint64_t smem_desc_scales(uint32_t addr)
{
    return (uint64_t)((addr & 0x3ffffu) >> 4) | ((uint64_t)(128 >> 4) << 32) | (1ull << 46);
}
// Instruction descriptor of kind::mxf4: A = B = e2m1, both K-major, scales ue8m0, D = f32; sf: which half of a scale word.
__host__ __device__ constexpr uint32_t idesc_mxf4(int m, int n, int sf)
{
    return ((uint32_t)sf << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(m >> 7) << 27) | ((uint32_t)sf << 29);
}

// ------------------------------------------------------------------ the persistent kernels' walk
// Every group's rows are cut into tiles by themselves, of `rows` rows from the multiple of `align` at or below the group's first
// one.  The host does not know the offsets, so every CTA builds the prefix sums of the groups' tile counts once (in `table`:
// first tiles, then first rows, then ends) and finds its items in them.  Inside a group the items run over MX4_BAND row
// tiles before they step to the next columns, so that the CTAs at work at one time share a patch of tiles through L2.
constexpr int MX4_BAND = 8;
constexpr uint32_t MX4_TABLE_BYTES = (3 * LIN_MAX_GROUPS + 4) * 4;

struct Mx4Item { int g; int tile, row, row_lo, row_hi, col; };   // the row tile, counted over all groups, its first row, the group's rows, the first column

__device__ __forceinline__ void mx4_count_tiles(int *table, const int32_t *offsets, int groups, int64_t T, int align, int rows, int threads)
{
    for (int g = threadIdx.x; g < groups; g += threads) {
        int64_t lo, hi;
        lin_group_rows(offsets, g, T, lo, hi);
        table[g + 1] = hi > lo ? (int)((hi - (lo & ~(int64_t)(align - 1)) + rows - 1) / rows) : 0;
        table[LIN_MAX_GROUPS + 4 + g] = (int)lo;
        table[2 * LIN_MAX_GROUPS + 4 + g] = (int)hi;
    }
}
// Inclusive prefix sums over the groups, by one warp.
__device__ __forceinline__ void mx4_sum_tiles(int *table, int groups)
{
    const int lane = threadIdx.x & 31;
    int carry = 0;
    for (int g0 = 0; g0 < groups; g0 += 32) {
        int v = g0 + lane < groups ? table[g0 + lane + 1] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(FULL_MASK, v, o);
            v += lane >= o ? up : 0;
        }
        v += carry;
        if (g0 + lane < groups) table[g0 + lane + 1] = v;
        carry = __shfl_sync(FULL_MASK, v, 31);
    }
    if (lane == 0) table[0] = 0;
}
// The idx-th item of the walk; false past the last one.
__device__ __forceinline__ bool mx4_item(const int *table, int groups, int align, int rows, int col_tiles, int cols_per_tile, int64_t idx, Mx4Item &it)
{
    const int *lo = table + LIN_MAX_GROUPS + 4, *hi = lo + LIN_MAX_GROUPS;
    if (idx >= (int64_t)table[groups] * col_tiles) return false;
    int a = 0, b = groups;                                           // table[a] * col_tiles <= idx < table[b] * col_tiles
    while (b - a > 1) {
        const int m = (a + b) >> 1;
        if ((int64_t)table[m] * col_tiles <= idx) a = m; else b = m;
    }
    const int tiles = table[a + 1] - table[a];
    const int64_t rem = idx - (int64_t)table[a] * col_tiles;
    const int band = (int)(rem / ((int64_t)MX4_BAND * col_tiles));
    const int r2 = (int)(rem - (int64_t)band * MX4_BAND * col_tiles);
    const int left = tiles - band * MX4_BAND;
    const int nb = left < MX4_BAND ? left : MX4_BAND;
    const int ct = r2 / nb;
    it.g = a;
    it.row_lo = lo[a];
    it.row_hi = hi[a];
    const int nth = band * MX4_BAND + (r2 - ct * nb);
    it.tile = table[a] + nth;
    it.row = (lo[a] & ~(align - 1)) + nth * rows;
    it.col = ct * cols_per_tile;
    return true;
}

// ------------------------------------------------------------------ blocks of Y whose columns are lanes
// Where a TMEM lane is a column of Y a thread holds one column, and a store from there would move 2 bytes.  A warp's block of
// rows x 32 columns therefore passes through shared memory (64 bytes a row), where the residual waits before it.
// Rows lo .. hi - 1 exist, and `left` columns (32 or more: all).  Called by a whole warp; ends with a warp barrier.
__device__ __forceinline__ void mx4_block_in(uint16_t *block, const uint16_t *from, int64_t ld, bool vec, int lo, int hi, int left)
{
    const int lane = threadIdx.x & 31;
    if (vec && left >= 32) {
#pragma unroll 4
        for (int r = lo + (lane >> 2); r < hi; r += 8)
            *reinterpret_cast<uint4 *>(block + r * 32 + (lane & 3) * 8) = DASS_LD(reinterpret_cast<const uint4 *>(from + r * ld + (lane & 3) * 8));
    } else {
#pragma unroll 4
        for (int r = lo; r < hi; ++r)
            if (lane < left) block[r * 32 + lane] = DASS_LD(from + r * ld + lane);
    }
    __syncwarp();
}
__device__ __forceinline__ void mx4_block_out(const uint16_t *block, uint16_t *to, int64_t ld, bool vec, int lo, int hi, int left)
{
    const int lane = threadIdx.x & 31;
    __syncwarp();
    if (vec && left >= 32) {
#pragma unroll 4
        for (int r = lo + (lane >> 2); r < hi; r += 8)
            DASS_ST(reinterpret_cast<uint4 *>(to + r * ld + (lane & 3) * 8), *reinterpret_cast<const uint4 *>(block + r * 32 + (lane & 3) * 8));
    } else {
#pragma unroll 4
        for (int r = lo; r < hi; ++r)
            if (lane < left) DASS_ST(to + r * ld + lane, block[r * 32 + lane]);
    }
    __syncwarp();
}
// V results of this lane's column, rows r0 .. r0 + V - 1 of the block: plus what the block holds there, if it does, rounded.
template <int V>
__device__ __forceinline__ void mx4_block_set(uint16_t *block, int r0, const float (&y)[V], bool add)
{
    uint16_t *at = block + r0 * 32 + (threadIdx.x & 31);
#pragma unroll
    for (int i = 0; i < V; i += 2) {
        float a = y[i], b = y[i + 1];
        if (add) {
            a += __uint_as_float((uint32_t)at[i * 32] << 16);
            b += __uint_as_float((uint32_t)at[i * 32 + 32] << 16);
        }
        const uint32_t w = pack_bf16x2(a, b);
        at[i * 32] = (uint16_t)w;
        at[i * 32 + 32] = (uint16_t)(w >> 16);
    }
}

// ------------------------------------------------------------------ tensor maps
// `mats` matrices of codes [rows x pitch bytes], one after the other: boxes of 128 bytes x box_rows with the 128-byte swizzle;
// rows past a matrix's end read as zero.
inline bool mx4_codes_map(CUtensorMap *map, const void *codes, int64_t mats, int64_t rows, int64_t K, int box_rows)
{
    const EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const int64_t pitch = mx4_pitch(K);
    const cuuint64_t dims[3] = {(cuuint64_t)pitch, (cuuint64_t)rows, (cuuint64_t)mats};
    const cuuint64_t strides[2] = {(cuuint64_t)pitch, (cuuint64_t)(rows * pitch)};
    const cuuint32_t box[3] = {128, (cuuint32_t)box_rows, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void *>(codes), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Scale tiles [tiles along the rows x tiles along k x 512 bytes]: boxes of two k tiles.
inline bool mx4_scales_map(CUtensorMap *map, const void *scales, int64_t row_tiles, int64_t K)
{
    const EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const int64_t k_tiles = mx4_k_tiles(K);
    const cuuint64_t dims[3] = {MX4_TILE_BYTES / 4, (cuuint64_t)k_tiles, (cuuint64_t)row_tiles};
    const cuuint64_t strides[2] = {MX4_TILE_BYTES, (cuuint64_t)k_tiles * MX4_TILE_BYTES};
    const cuuint32_t box[3] = {MX4_TILE_BYTES / 4, 2, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<void *>(scales), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace dass
