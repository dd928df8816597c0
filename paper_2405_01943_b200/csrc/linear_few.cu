// dass_linear for bf16 and few rows (a decode step): every weight is read once and meets at most 32 rows of X, so the
// time is that of streaming the weights.
//
// A block of 8 warps owns 16 columns of Y, that is 16 weight rows; the warps take k in turns of 64, so that the block
// reads 1 KB runs of each of its rows, straight into the registers of mma.m16n8k16: A = 16 weight rows, B = 8 rows of X
// at a time.  A dot product may take its k in any order as long as both sides agree, so a lane loads 8 consecutive k (16
// bytes) of its row and uses them as the fragment's scattered k.  The tensor instruction only has to keep ahead of the
// memory here; no shared-memory round trip, TMEM or tensor map stands between a load and its use, and blocks are small
// enough that the last wave is short.  A cluster of SPLIT blocks shares the columns and splits k further where there are
// few columns; sums over the warps and the cluster's blocks are taken in a fixed order.
//
// Bound by the launch and the latency of a few loads: 512 x 1024 3.5 us, 2048 x 2048 5.8 us for up to 8 rows (linear_mid.cu:
// 5.9 and 7.7); 14336 x 4096 gated 44 us, 5.2 TB/s (linear_mid.cu 40).
#include "linear_common.cuh"
#include "linear_tc.cuh"
#include "tc_pair.cuh"

namespace dass {

constexpr int LW_WARPS = 8;
constexpr int LW_THREADS = LW_WARPS * 32;
constexpr int LW_COLS = 16;          // columns of Y (weight rows) of a block
constexpr int LW_STEP = 64;          // k of a warp's turn

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 8 elements of a row from k on; elements at and past K read as zero (and are not touched).
template <bool STREAM>
__device__ __forceinline__ uint4 lw_load8(const uint16_t *row, int64_t k, int64_t K)
{
    if (k + 8 <= K) {
        const uint4 *p = reinterpret_cast<const uint4 *>(row + k);
        return STREAM ? DASS_LD_CS(p) : DASS_LD_G(p);
    }
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (k + i < K) w[i >> 1] |= (uint32_t)DASS_LD(row + k + i) << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// NT: rows of X in eights.  Grid: SPLIT x column tiles x row tiles, clusters of SPLIT along x.
template <int NT, bool GLU>
__global__ void __launch_bounds__(LW_THREADS)
linear_few_kernel(const LinearArgs a, int col_tiles, int split)
{
    constexpr int M = GLU ? 2 : 1;
    constexpr int SUMS = M * LW_COLS * NT * 8;
    __shared__ float part[LW_WARPS][SUMS];
    __shared__ float sum[SUMS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, q = lane & 3;
    const int64_t block = blockIdx.x / split;
    const int rank = blockIdx.x - (int)block * split;
    lin_zero_outside<true>(a.offsets, a.groups, a.T, a.N, a.Y, a.ldy, false, (int64_t)blockIdx.x * LW_THREADS + threadIdx.x,
                           (int64_t)gridDim.x * LW_THREADS);
    const LinTile tile = lin_find_tile(a.offsets, a.groups, a.T, NT * 8, block / col_tiles);
    if (tile.g < 0) return;                                  // the whole cluster
    const int64_t n0 = (block % col_tiles) * LW_COLS;

    const uint16_t *w[M][2], *x[NT];
#pragma unroll
    for (int h = 0; h < 2; ++h) {                            // rows past the last column are read as the last: never stored
        const int64_t n = n0 + g + 8 * h < a.N ? n0 + g + 8 * h : a.N - 1;
        const int64_t at = (int64_t)tile.g * a.group_stride + n * a.ldw;
        w[0][h] = static_cast<const uint16_t *>(a.W) + at;
        if constexpr (GLU) w[1][h] = static_cast<const uint16_t *>(a.W_up) + at;
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int64_t t = tile.lo + i * 8 + g < tile.hi ? tile.lo + i * 8 + g : tile.lo;
        x[i] = static_cast<const uint16_t *>(a.X) + t * a.ldx;
    }
    float acc[M][NT][4];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[m][i][c] = 0.f;

#pragma unroll 2
    for (int64_t k0 = (int64_t)(rank * LW_WARPS + warp) * LW_STEP; k0 < a.K; k0 += (int64_t)split * LW_WARPS * LW_STEP) {
        uint4 wv[M][2][2], xv[NT][2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int64_t k = k0 + s * 32 + q * 8;
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) wv[m][h][s] = lw_load8<true>(w[m][h], k, a.K);
#pragma unroll
            for (int i = 0; i < NT; ++i) xv[i][s] = lw_load8<false>(x[i], k, a.K);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int m = 0; m < M; ++m) {
                    mma_16816(acc[m][i], wv[m][0][s].x, wv[m][1][s].x, wv[m][0][s].y, wv[m][1][s].y, xv[i][s].x, xv[i][s].y);
                    mma_16816(acc[m][i], wv[m][0][s].z, wv[m][1][s].z, wv[m][0][s].w, wv[m][1][s].w, xv[i][s].z, xv[i][s].w);
                }
    }
    // sum over the warps, then over the cluster's blocks
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                part[warp][(m * NT * 8 + i * 8 + 2 * q + (c & 1)) * LW_COLS + g + 8 * (c >> 1)] = acc[m][i][c];
    __syncthreads();
    for (int o = threadIdx.x; o < SUMS; o += LW_THREADS) {
        float s = part[0][o];
#pragma unroll
        for (int v = 1; v < LW_WARPS; ++v) s += part[v][o];
        sum[o] = s;
    }
    __syncwarp();                                            // the cluster barrier wants whole warps
    if (split > 1) cluster_sync_all(); else __syncthreads();
    const int rows = (int)(tile.hi - tile.lo);
    const uint32_t sum_addr = smem_u32(sum);
    for (int o = threadIdx.x + rank * LW_THREADS; o < rows * LW_COLS; o += split * LW_THREADS) {
        const int64_t t = tile.lo + o / LW_COLS, n = n0 + o % LW_COLS;
        if (n >= a.N) continue;
        float p[M];
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int at = m * NT * 8 * LW_COLS + o;
            if (split > 1) {
                p[m] = 0.f;
                for (int r = 0; r < split; ++r) p[m] += ld_cluster(map_to_cta(sum_addr + at * 4, r));
            } else {
                p[m] = sum[at];
            }
        }
        float b[1] = {0.f};
        if (a.bias) { row_load<true, 1>(a.bias, (int64_t)tile.g * a.N + n, b); p[0] += b[0]; }
        float y[1] = {p[0]};
        lt_act_all(y, a.act);
        if constexpr (GLU) {
            if (a.bias_up) { row_load<true, 1>(a.bias_up, (int64_t)tile.g * a.N + n, b); p[1] += b[0]; }
            y[0] *= p[1];
        }
        if (a.residual) { row_load<true, 1>(a.residual, t * a.ldr + n, b); y[0] += b[0]; }
        row_store<true, 1>(a.Y, t * a.ldy + n, y);
    }
    __syncwarp();
    if (split > 1) cluster_sync_all();                       // the others may still read this block's sums
}

template <int NT, bool GLU>
static cudaError_t lw_launch(const LinearArgs &a, int64_t row_tiles, int split)
{
    const int col_tiles = (int)((a.N + LW_COLS - 1) / LW_COLS);
    if (row_tiles * col_tiles * split > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(row_tiles * col_tiles * split));
    cfg.blockDim = dim3(LW_THREADS);
    cfg.stream = a.st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, linear_few_kernel<NT, GLU>, a, col_tiles, split);
}

// nt: rows of X in eights (1, 2 or 4); split: blocks that share the contraction (1, 2, 4 or 8)
dass_status linear_few_launch(const LinearArgs &a, int nt, int split)
{
    const int64_t row_tiles = a.offsets ? a.T / (8 * nt) + lin_active_groups(a) : (a.T + 8 * nt - 1) / (8 * nt);
    cudaError_t e;
    if (a.W_up) e = nt == 1 ? lw_launch<1, true>(a, row_tiles, split) : nt == 2 ? lw_launch<2, true>(a, row_tiles, split) : lw_launch<4, true>(a, row_tiles, split);
    else e = nt == 1 ? lw_launch<1, false>(a, row_tiles, split) : nt == 2 ? lw_launch<2, false>(a, row_tiles, split) : lw_launch<4, false>(a, row_tiles, split);
    return e == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

}  // namespace dass
