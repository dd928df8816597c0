// dass_linear for bf16 and some tens of rows (per group): too many for linear_few.cu's registers, too few to fill the
// 256-row tiles of linear_tc.cu, and still bound by reading the weights once.
//
// The operands change sides: M = 128 weight rows (columns of Y), N = NT rows of X, so a tensor instruction is as long as
// there are rows.  One block per 128 columns and NT rows; TMA fills a ring of weight (and up-weight) and X tiles, one
// lane issues the MMAs, and two or more blocks share an SM so that one's first loads and epilogue run under another's
// stream.  A cluster of SPLIT blocks divides k where there are few columns.  The accumulators (a TMEM lane is a column of
// Y) go through shared memory, where they turn into runs of 8 columns of one row and where the cluster's blocks add up
// their parts, in order, each for its share of the rows.
//
// Bound by the weights' bytes where there are enough blocks: 32 rows over 8 experts of 4096 x 14336 run at 6.4 TB/s of
// weights in the GLU form (290 us) and 6.6 back (140 us); linear_tc.cu takes 326 and 164, linear_few.cu 316 and 152.  A
// product of few columns is bound by the start and the k-blocks of one block (0.2 us each): 4096 x 4096, 64 rows, 14 us.
//
// Every wait is bounded, as in linear_tc.cu.
#include "linear_common.cuh"
#include "linear_tc.cuh"
#include "tc_common.cuh"
#include "tc_pair.cuh"

namespace dass {

constexpr int LM_COLS = 128;        // columns of Y (weight rows) per block: MMA M
constexpr int LM_BK = 64;
constexpr int LM_THREADS = 320;     // TMA, MMA and 8 epilogue warps, two to a quarter of the TMEM lanes
constexpr int LM_PITCH = LM_COLS + 4;
constexpr uint32_t LM_W_BYTES = LM_COLS * LM_BK * 2;

template <int NT, bool GLU> struct LmShape {
    static constexpr uint32_t STAGE = LM_W_BYTES * (GLU ? 2 : 1) + NT * LM_BK * 2;
    static constexpr uint32_t SUMS = (GLU ? 2 : 1) * NT * LM_PITCH * 4;              // partial sums, over the drained ring
    static constexpr uint32_t EXTRA = 1024 /* alignment slack */ + 256 /* barriers */;
    static constexpr int DEEP = (int)((226u * 1024u - EXTRA) / STAGE) < 12 ? (int)((226u * 1024u - EXTRA) / STAGE) : 12;   // one block to an SM
    // two blocks to an SM, where a ring of three stages is left to each
    static constexpr int SHARED = (int)((113u * 1024u - EXTRA) / STAGE) >= 3 ? (int)((113u * 1024u - EXTRA) / STAGE) : DEEP;
    static_assert(SUMS <= SHARED * STAGE, "the partial sums take the ring's place");
    static constexpr uint32_t TMEM = (GLU ? 2 : 1) * NT < 32 ? 32 : (GLU ? 2 : 1) * NT;
};

struct LmParams {
    LinearArgs a;
    int col_tiles, row_tiles, k_blocks, split, stages;
    int vec;                // Y, R and the biases allow 16-byte accesses
    int *timeouts;
};

// 8 values of a bf16 row: columns n .. n + 7 (STEP 1), or n, n + 16 .. n + 112 (STEP 16); columns past N are zero.
template <int STEP>
__device__ __forceinline__ void lm_load8(const void *row, int64_t at, int n, int N, float (&v)[8])
{
    if (STEP == 1 && n + 8 <= N) { row_load<true, 8>(row, at + n, v); return; }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float x[1] = {0.f};
        if (n + i * STEP < N) row_load<true, 1>(row, at + n + i * STEP, x);
        v[i] = x[0];
    }
}

// Rows r0 .. r1 - 1 of the block's tile: the cluster's partial sums added up, the epilogue, the store.  A thread has 8
// columns of a row: consecutive ones where Y, R and the biases allow 16-byte accesses, else every 16th, so that half a
// warp moves 32 contiguous bytes.
template <int NT, bool GLU, int STEP>
__device__ __forceinline__ void lm_finish(const LmParams &p, const LinTile &tile, int col, int r0, int r1, const float *sums)
{
    constexpr int M = GLU ? 2 : 1;
    const LinearArgs &a = p.a;
    const uint32_t sums_addr = smem_u32(sums);
    const int N = (int)a.N;
    for (int o = r0 * 16 + threadIdx.x; o < r1 * 16; o += LM_THREADS) {
        const int r = o >> 4, c = STEP == 1 ? (o & 15) * 8 : o & 15, n = col + c;
        if (n >= N) continue;
        const int64_t t = tile.lo + r;
        float acc[M][8];
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int at = (m * NT + r) * LM_PITCH + c;
            if (p.split > 1) {
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[m][i] = 0.f;
                for (int s = 0; s < p.split; ++s) {
                    const uint32_t from = map_to_cta(sums_addr + at * 4, s);
                    if constexpr (STEP == 1) {
                        const float4 u = ld_cluster4(from), v = ld_cluster4(from + 16);
                        acc[m][0] += u.x; acc[m][1] += u.y; acc[m][2] += u.z; acc[m][3] += u.w;
                        acc[m][4] += v.x; acc[m][5] += v.y; acc[m][6] += v.z; acc[m][7] += v.w;
                    } else {
                        float v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = ld_cluster(from + i * STEP * 4);
#pragma unroll
                        for (int i = 0; i < 8; ++i) acc[m][i] += v[i];
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[m][i] = sums[at + i * STEP];
            }
        }
        float y[8], b[8];
        if (a.bias) {
            lm_load8<STEP>(a.bias, (int64_t)tile.g * N, n, N, b);
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[0][i] += b[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = acc[0][i];
        lt_act_all(y, a.act);
        if constexpr (GLU) {
            if (a.bias_up) {
                lm_load8<STEP>(a.bias_up, (int64_t)tile.g * N, n, N, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[1][i] += b[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] *= acc[M - 1][i];
        }
        if (a.residual) {
            lm_load8<STEP>(a.residual, t * a.ldr, n, N, b);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] += b[i];
        }
        if (STEP == 1 && n + 8 <= N) {
            row_store<true, 8>(a.Y, t * a.ldy + n, y);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float one[1] = {y[i]};
                if (n + i * STEP < N) row_store<true, 1>(a.Y, t * a.ldy + n + i * STEP, one);
            }
        }
    }
}

template <int NT, bool GLU>
__global__ void __launch_bounds__(LM_THREADS)
linear_mid_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                  const __grid_constant__ CUtensorMap map_up, const __grid_constant__ LmParams p)
{
    using S = LmShape<NT, GLU>;
    constexpr int M = GLU ? 2 : 1;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t *aligned = smem_raw + (base - raw);
    uint64_t *bars = reinterpret_cast<uint64_t *>(aligned + p.stages * S::STAGE);
    const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + 8 * p.stages, bar_acc = bar_empty + 8 * p.stages;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 2 * p.stages + 1);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    float *sums = reinterpret_cast<float *>(aligned);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const LinearArgs &a = p.a;
    const int64_t block = blockIdx.x / p.split;
    const int rank = blockIdx.x - (int)block * p.split;
    lin_zero_outside<true>(a.offsets, a.groups, a.T, a.N, a.Y, a.ldy, p.vec != 0, (int64_t)blockIdx.x * LM_THREADS + threadIdx.x,
                           (int64_t)gridDim.x * LM_THREADS);
    // the row tiles of one set of columns are neighbours: they read the same weights
    const LinTile tile = lin_find_tile(a.offsets, a.groups, a.T, NT, block % p.row_tiles);
    if (tile.g < 0) return;                                       // the whole cluster
    const int col = (int)(block / p.row_tiles) * LM_COLS;
    const int kb0 = (int)((int64_t)p.k_blocks * rank / p.split), kb1 = (int)((int64_t)p.k_blocks * (rank + 1) / p.split);

    if (threadIdx.x == 64) {                                      // the descriptors' first fetch runs beside the set-up
        tma_prefetch_map(&map_w);
        if constexpr (GLU) tma_prefetch_map(&map_up);
        tma_prefetch_map(&map_x);
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
        mbar_init(bar_acc, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(tmem_slot), S::TMEM);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    // Both issuing warps run their loops whole and elect a lane for the instructions: inside a one-lane branch the
    // operands are not uniform, and four MMAs alone take 225 cycles to issue.
    if (warp == 0) {
        uint32_t stage = 0, phase = 0;
        bool ok = true;
        const uint64_t pol_w = l2_policy_evict_first(), pol_x = l2_policy_evict_last();
        for (int kb = kb0; kb < kb1; ++kb) {
            if (!warp_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag)) { ok = false; break; }
            const uint32_t sbase = base + stage * S::STAGE, full = bar_full + 8 * stage;
            if (elect_one()) {
                mbar_arrive_expect_tx(full, S::STAGE);
                tma_load_3d_hint(sbase, &map_w, full, kb * LM_BK, col, tile.g, pol_w);
                if constexpr (GLU) tma_load_3d_hint(sbase + LM_W_BYTES, &map_up, full, kb * LM_BK, col, tile.g, pol_w);
                tma_load_2d_hint(sbase + M * LM_W_BYTES, &map_x, full, kb * LM_BK, (int)tile.lo, pol_x);
            }
            __syncwarp();
            if ((int)++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
        if (!ok && lane == 0) { *abort_flag = 1; atomicAdd(p.timeouts, 1); }
    } else if (warp == 1) {
        constexpr uint32_t idesc = idesc_bf16_f32(LM_COLS, NT);
        uint32_t stage = 0, phase = 0;
        bool ok = true;
        for (int kb = kb0; kb < kb1; ++kb) {
            if (!warp_wait(bar_full + 8 * stage, phase, abort_flag)) { ok = false; break; }
            tc_fence_after();
            const uint32_t sbase = base + stage * S::STAGE;
            if (elect_one()) {
                const uint64_t db = smem_desc_sw128(sbase + M * LM_W_BYTES);
#pragma unroll
                for (int m = 0; m < M; ++m) {
                    const uint64_t da = smem_desc_sw128(sbase + m * LM_W_BYTES);
#pragma unroll
                    for (int k = 0; k < LM_BK / 16; ++k)
                        umma_bf16(tmem_base + m * NT, da + 2 * k, db + 2 * k, idesc, (kb > kb0 || k > 0) ? 1u : 0u);
                }
                umma_commit(bar_empty + 8 * stage);
                if (kb + 1 == kb1) umma_commit(bar_acc);
            }
            __syncwarp();
            if ((int)++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
        if (!ok && lane == 0) { *abort_flag = 1; atomicAdd(p.timeouts, 1); }
    } else {
        // accumulators to shared memory: lane = column of Y, accumulator column = row of X
        const int quad = warp & 3;
        if (warp_wait(bar_acc, 0, abort_flag)) {
            tc_fence_after();
            const uint32_t addr = tmem_base + ((uint32_t)(quad * 32) << 16);
#pragma unroll 1
            for (int c = ((warp - 2) >> 2) * 16; c < M * NT; c += 32) {
                uint32_t v[16];
                tmem_ld_16(addr + c, v);
                tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < 16; ++j) sums[(c + j) * LM_PITCH + quad * 32 + lane] = __uint_as_float(v[j]);
            }
        } else if (lane == 0) {
            *abort_flag = 1;
            atomicAdd(p.timeouts, 1);
        }
    }
    tc_fence_before();
    __syncwarp();                                                 // the cluster barrier wants whole warps
    if (p.split > 1) cluster_sync_all(); else __syncthreads();
    if (*abort_flag) {
        for (int i = 0; i < 20; ++i) __nanosleep(1000000);       // failure path: let what was issued land
    } else {
        const int rows = (int)(tile.hi - tile.lo);
        const int r0 = NT * rank / p.split, r1 = NT * (rank + 1) / p.split < rows ? NT * (rank + 1) / p.split : rows;
        if (p.vec) lm_finish<NT, GLU, 1>(p, tile, col, r0, r1, sums);
        else lm_finish<NT, GLU, 16>(p, tile, col, r0, r1, sums);
    }
    __syncwarp();
    if (p.split > 1) cluster_sync_all(); else __syncthreads();   // sums may still be read by the cluster's other blocks
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, S::TMEM);
    }
}

// ------------------------------------------------------------------ host side
int device_sm_count();                                                                                       // dass_abi.cu
int *linear_timeouts();                                                                                      // linear.cu
bool tc_make_map(CUtensorMap *map, const void *ptr, int64_t rows, int64_t cols, int64_t ld, int box_rows);   // calib_tc.cu
bool tc_make_map_3d(CUtensorMap *map, const void *ptr, int64_t mats, int64_t rows, int64_t cols, int64_t ld, int64_t mat_stride, int box_rows);   // linear_tc.cu

template <int NT, bool GLU>
static dass_status lm_launch(const LinearArgs &a, int split)
{
    using S = LmShape<NT, GLU>;
    static DeviceMask configured{0ull};               // per device
    if (ensure_dynamic_smem(linear_mid_kernel<NT, GLU>, (int)(S::DEEP * S::STAGE + S::EXTRA), configured) != cudaSuccess) return DASS_ERR_CUDA;
    CUtensorMap mx, mw, mu;
    if (!tc_make_map(&mx, a.X, a.T, a.K, a.ldx, NT) || !tc_make_map_3d(&mw, a.W, a.groups, a.N, a.K, a.ldw, a.group_stride, LM_COLS) ||
        !tc_make_map_3d(&mu, GLU ? a.W_up : a.W, a.groups, a.N, a.K, a.ldw, a.group_stride, LM_COLS))
        return DASS_ERR_CUDA;
    LmParams p;
    p.a = a;
    p.col_tiles = (int)((a.N + LM_COLS - 1) / LM_COLS);
    p.k_blocks = (int)((a.K + LM_BK - 1) / LM_BK);
    const int64_t groups = lin_active_groups(a);
    p.row_tiles = (int)(a.offsets ? a.T / NT + groups : (a.T + NT - 1) / NT);
    const int64_t blocks = (int64_t)p.col_tiles * (a.offsets ? groups : p.row_tiles);      // that will have work
    p.split = split < p.k_blocks ? split : 1;
    p.stages = blocks * p.split * 10 <= 8 * device_sm_count() ? S::DEEP : S::SHARED;        // clusters do not fill every SM
    p.vec = lin_wide_ok(a);
    p.timeouts = linear_timeouts();
    if (!p.timeouts) return DASS_ERR_CUDA;
    const int64_t grid = (int64_t)p.col_tiles * p.row_tiles * p.split;
    if (grid > 0x7fffffffll) return DASS_ERR_UNSUPPORTED;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(LM_THREADS);
    cfg.dynamicSmemBytes = p.stages * S::STAGE + S::EXTRA;
    cfg.stream = a.st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, linear_mid_kernel<NT, GLU>, mx, mw, mu, p) == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

// nt: rows per tile (16, 32, 64 or 128); split: blocks that share the contraction (1, 2, 4 or 8)
dass_status linear_mid_launch(const LinearArgs &a, int nt, int split)
{
    if (a.W_up) return nt == 16 ? lm_launch<16, true>(a, split) : nt == 32 ? lm_launch<32, true>(a, split) : nt == 64 ? lm_launch<64, true>(a, split) : lm_launch<128, true>(a, split);
    return nt == 16 ? lm_launch<16, false>(a, split) : nt == 32 ? lm_launch<32, false>(a, split) : nt == 64 ? lm_launch<64, false>(a, split) : lm_launch<128, false>(a, split);
}

}  // namespace dass
