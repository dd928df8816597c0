// dass_linear for bf16 and many rows on the sm_100a tensor cores: Y = act(X W^T + b) [* (X W_up^T + b_up)] + R, dense or
// per expert.
//
// A persistent kernel run by CTA pairs (a cluster of 2) that drive tcgen05.mma.cta_group::2 of shape 256 x 256 x 16:
//   * M = 256 rows of X, 128 to each CTA; N = 256 accumulator columns: 256 columns of Y, or, in the GLU form, 128 of the
//     gate product (the leader CTA loads W) beside the same 128 of the up product (its peer loads W_up);
//   * two accumulators of 256 TMEM columns: the epilogue of one tile runs under the products of the next.
//   warp 0      TMA into a 6-stage, 128B-swizzled ring;  warp 1  TMEM, MMAs (leader);  warps 2..5  epilogue
// Groups: every expert's rows are cut into tiles of 256 by themselves.  A tile may begin at any row (the row coordinate
// of a TMA box is free) and reads on into the next expert's rows; those results are not stored.  The host does not know
// the offsets, so every CTA builds the prefix sums of the experts' tile counts once and finds its items in them.  Inside
// an expert the items run over 8 row tiles before they step to the next columns: the pairs at work at one time then
// share a patch of about 8 x 9 tiles through L2.
//
// Every wait is bounded: when one runs out the CTA raises an abort flag, records DASS_ERR_TIMEOUT for
// dass_linear_status, lets its roles drain and frees its TMEM before it returns.
#include "linear_common.cuh"
#include "linear_tc.cuh"
#include "tc_common.cuh"
#include "tc_pair.cuh"

namespace dass {

constexpr int LT_BM = 128;          // rows per CTA
constexpr int LT_BN = 256;          // accumulator columns
constexpr int LT_BK = 64;           // k per stage: one 128-byte swizzle row
constexpr int LT_STAGES = 6;
constexpr int LT_THREADS = 192;
constexpr int LT_BAND = 8;          // row tiles that are walked before the next columns
constexpr uint32_t LT_TILE_BYTES = 128 * LT_BK * 2;
constexpr uint32_t LT_STAGE_BYTES = 2 * LT_TILE_BYTES;
constexpr uint32_t LT_TABLE_BYTES = (LIN_MAX_GROUPS + 1) * 4;
constexpr uint32_t LT_SMEM_BYTES = LT_STAGES * LT_STAGE_BYTES + 1024 /* alignment slack */ + 256 /* barriers */ + LT_TABLE_BYTES;

struct LtParams {
    const int32_t *offsets;
    const uint16_t *bias, *bias_up, *residual;
    uint16_t *Y;
    int64_t ldr, ldy, T;
    int N, groups, col_tiles, k_blocks, cols_per_tile;
    int y_vec, r_vec;               // whole 16-byte accesses
    int *status;
};

struct LtItem { int g; int row, row_end, col; };

// The idx-th item of the grid's walk; false past the last one.
__device__ __forceinline__ bool lt_item(const LtParams &p, const int *first_tile, int64_t idx, LtItem &it)
{
    if (idx >= (int64_t)first_tile[p.groups] * p.col_tiles) return false;
    int a = 0, b = p.groups;                                         // first_tile[a] * col_tiles <= idx < first_tile[b] * col_tiles
    while (b - a > 1) {
        const int m = (a + b) >> 1;
        if ((int64_t)first_tile[m] * p.col_tiles <= idx) a = m; else b = m;
    }
    const int tiles = first_tile[a + 1] - first_tile[a];
    const int64_t rem = idx - (int64_t)first_tile[a] * p.col_tiles;
    const int band = (int)(rem / ((int64_t)LT_BAND * p.col_tiles));
    const int r2 = (int)(rem - (int64_t)band * LT_BAND * p.col_tiles);
    const int left = tiles - band * LT_BAND;
    const int nb = left < LT_BAND ? left : LT_BAND;
    const int ct = r2 / nb;
    int64_t lo, hi;
    lin_group_rows(p.offsets, a, p.T, lo, hi);
    it.g = a;
    it.row = (int)lo + (band * LT_BAND + (r2 - ct * nb)) * 2 * LT_BM;
    it.row_end = (int)hi;
    it.col = ct * p.cols_per_tile;
    return true;
}

// A column's bias for the lanes of a warp: lane l holds column n0 + l.
__device__ __forceinline__ float lt_bias(const uint16_t *bias, int64_t at, int n, int N)
{
    return bias && n < N ? __uint_as_float((uint32_t)DASS_LD(bias + at + n) << 16) : 0.f;
}

template <bool GLU, int ACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(LT_THREADS, 1)
linear_tc_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                 const __grid_constant__ CUtensorMap map_up, const LtParams p)
{
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;                 // swizzled tiles need 1024-byte alignment
    uint8_t *aligned = smem_raw + (base - raw);
    uint64_t *bars = reinterpret_cast<uint64_t *>(aligned + LT_STAGES * LT_STAGE_BYTES);
    const uint32_t bar_full = smem_u32(bars);                     // [stages], used in the leader
    const uint32_t bar_empty = bar_full + 8 * LT_STAGES;          // [stages], per CTA
    const uint32_t bar_acc_full = bar_empty + 8 * LT_STAGES;      // [2], per CTA
    const uint32_t bar_acc_empty = bar_acc_full + 16;             // [2], leader: 8 epilogue warps arrive
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 2 * LT_STAGES + 4);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    int *first_tile = reinterpret_cast<int *>(reinterpret_cast<uint8_t *>(bars) + 256);

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();                      // 0 = leader
    const int64_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < LT_STAGES; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(bar_acc_full + 8 * s, 1); mbar_init(bar_acc_empty + 8 * s, 8); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    for (int g = threadIdx.x; g < p.groups; g += LT_THREADS) {
        int64_t lo, hi;
        lin_group_rows(p.offsets, g, p.T, lo, hi);
        first_tile[g + 1] = (int)((hi - lo + 2 * LT_BM - 1) / (2 * LT_BM));
    }
    if (warp == 1) {
        tmem_alloc_pair(smem_u32(tmem_slot), 512);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) {                                              // inclusive prefix sums over the groups
        int carry = 0;
        for (int g0 = 0; g0 < p.groups; g0 += 32) {
            int v = g0 + lane < p.groups ? first_tile[g0 + lane + 1] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int up = __shfl_up_sync(FULL_MASK, v, o);
                v += lane >= o ? up : 0;
            }
            v += carry;
            if (g0 + lane < p.groups) first_tile[g0 + lane + 1] = v;
            carry = __shfl_sync(FULL_MASK, v, 31);
        }
        if (lane == 0) first_tile[0] = 0;
    }
    __syncthreads();
    cluster_sync_all();            // both CTAs' barriers are initialised and both TMEM allocations exist
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer (one per CTA)
        if (lane == 0) {
            uint32_t stage = 0, phase = 0;
            bool ok = true;
            const uint32_t leader_full = map_to_cta(bar_full, 0);
            const uint64_t pol = l2_policy_evict_last();
            const CUtensorMap *map_b = GLU && rank ? &map_up : &map_w;
            LtItem it;
            for (int64_t idx = pair; ok && lt_item(p, first_tile, idx, it); idx += pairs) {
                const int a_row = it.row + (int)rank * LT_BM;
                const int b_row = it.col + (GLU ? 0 : (int)rank * 128);
                for (int kb = 0; kb < p.k_blocks; ++kb) {
                    if (!mbar_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag)) { ok = false; break; }
                    const uint32_t sbase = base + stage * LT_STAGE_BYTES;
                    const uint32_t fb = leader_full + 8 * stage;
                    if (rank == 0) mbar_arrive_expect_tx(bar_full + 8 * stage, 2 * LT_STAGE_BYTES);   // both CTAs' bytes
                    tma_load_2d_pair(sbase, &map_x, fb, kb * LT_BK, a_row, pol);
                    tma_load_3d_pair(sbase + LT_TILE_BYTES, map_b, fb, kb * LT_BK, b_row, it.g, pol);
                    if (++stage == LT_STAGES) { stage = 0; phase ^= 1u; }
                }
            }
            if (!ok) { *abort_flag = 1; atomicExch(p.status, (int)DASS_ERR_TIMEOUT); }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer (leader CTA only)
        if (lane == 0 && rank == 0) {
            constexpr uint32_t idesc = idesc_bf16_f32(2 * LT_BM, LT_BN);
            uint32_t stage = 0, phase = 0, tile = 0;
            bool ok = true;
            const int64_t items = (int64_t)first_tile[p.groups] * p.col_tiles;
            for (int64_t idx = pair; ok && idx < items; idx += pairs, ++tile) {
                const uint32_t as = tile & 1u;
                if (!mbar_wait(bar_acc_empty + 8 * as, ((tile >> 1) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
                tc_fence_after();
                const uint32_t acc_addr = tmem_base + as * LT_BN;
                for (int kb = 0; kb < p.k_blocks; ++kb) {
                    if (!mbar_wait(bar_full + 8 * stage, phase, abort_flag)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t sbase = base + stage * LT_STAGE_BYTES;
                    const uint64_t da = smem_desc_sw128(sbase);
                    const uint64_t db = smem_desc_sw128(sbase + LT_TILE_BYTES);
#pragma unroll
                    for (int k = 0; k < LT_BK / 16; ++k)
                        umma_bf16_pair(acc_addr, da + 2 * k, db + 2 * k, idesc, (kb > 0 || k > 0) ? 1u : 0u);   // 32 bytes per k step
                    umma_commit_pair(bar_empty + 8 * stage, (uint16_t)3);   // slot free in both CTAs
                    if (++stage == LT_STAGES) { stage = 0; phase ^= 1u; }
                }
                if (ok) umma_commit_pair(bar_acc_full + 8 * as, (uint16_t)3);   // accumulator ready in both CTAs
            }
            if (!ok) { *abort_flag = 1; atomicExch(p.status, (int)DASS_ERR_TIMEOUT); }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ epilogue (4 warps, this CTA's 128 rows)
        lin_zero_outside<true>(p.offsets, p.groups, p.T, p.N, p.Y, p.ldy, p.y_vec != 0, (int64_t)blockIdx.x * 128 + threadIdx.x - 64, (int64_t)gridDim.x * 128);
        const int quad = warp & 3;                               // TMEM lanes 32*quad .. 32*quad+31
        const uint32_t lane_addr = tmem_base + ((uint32_t)(quad * 32) << 16);
        const uint32_t leader_acc_empty = map_to_cta(bar_acc_empty, 0);
        uint32_t tile = 0;
        bool ok = true;
        LtItem it;
        for (int64_t idx = pair; ok && lt_item(p, first_tile, idx, it); idx += pairs, ++tile) {
            const uint32_t as = tile & 1u;
            if (!mbar_wait(bar_acc_full + 8 * as, (tile >> 1) & 1u, abort_flag)) { ok = false; break; }
            tc_fence_after();
            const int64_t t = (int64_t)it.row + rank * LT_BM + quad * 32 + lane;   // this thread's row
            const bool mine = t < it.row_end;
            uint16_t *row = p.Y + (mine ? t : 0) * p.ldy;
            const uint16_t *res = p.residual ? p.residual + (mine ? t : 0) * p.ldr : nullptr;
            const int64_t b_at = (int64_t)it.g * p.N;
            const uint32_t acc_addr = lane_addr + as * LT_BN;
#pragma unroll 1
            for (int c = 0; c < (GLU ? LT_BN / 2 : LT_BN); c += 32) {
                const int n0 = it.col + c;
                if (n0 >= p.N) break;
                uint32_t a[32], u[GLU ? 32 : 1], w[16];
                tmem_ld_32(acc_addr + c, a);
                if constexpr (GLU) tmem_ld_32(acc_addr + LT_BN / 2 + c, u);
                const bool whole = n0 + 32 <= p.N;
                if (mine && res) {
                    if (p.r_vec && whole) {
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            const uint4 x = DASS_LD(reinterpret_cast<const uint4 *>(res + n0) + v);
                            w[4 * v] = x.x; w[4 * v + 1] = x.y; w[4 * v + 2] = x.z; w[4 * v + 3] = x.w;
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const uint32_t lo = n0 + 2 * j < p.N ? DASS_LD(res + n0 + 2 * j) : 0;
                            const uint32_t hi = n0 + 2 * j + 1 < p.N ? DASS_LD(res + n0 + 2 * j + 1) : 0;
                            w[j] = lo | (hi << 16);
                        }
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) w[j] = 0u;
                }
                const float bn = lt_bias(p.bias, b_at, n0 + lane, p.N);
                const float bu = GLU ? lt_bias(p.bias_up, b_at, n0 + lane, p.N) : 0.f;
                tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    float y[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float x = __uint_as_float(a[2 * j + h]);
                        if (p.bias) x += __shfl_sync(FULL_MASK, bn, 2 * j + h);
                        x = lt_act<ACT>(x);
                        if constexpr (GLU) {
                            float v = __uint_as_float(u[2 * j + h]);
                            if (p.bias_up) v += __shfl_sync(FULL_MASK, bu, 2 * j + h);
                            x *= v;
                        }
                        y[h] = x + __uint_as_float(h ? (w[j] & 0xffff0000u) : (w[j] << 16));
                    }
                    w[j] = pack_bf16x2(y[0], y[1]);
                }
                if (!mine) continue;
                if (p.y_vec && whole) {
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        DASS_ST(reinterpret_cast<uint4 *>(row + n0) + v, make_uint4(w[4 * v], w[4 * v + 1], w[4 * v + 2], w[4 * v + 3]));
                } else {
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (n0 + j < p.N) DASS_ST(row + n0 + j, (uint16_t)((j & 1) ? (w[j >> 1] >> 16) : (w[j >> 1] & 0xffffu)));
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {                                     // release the accumulator to the leader's MMA warp
                if (rank == 0) mbar_arrive(bar_acc_empty + 8 * as);
                else mbar_arrive_cluster(leader_acc_empty + 8 * as);
            }
        }
        if (!ok && lane == 0) { *abort_flag = 1; atomicExch(p.status, (int)DASS_ERR_TIMEOUT); }
    }

    // ---------------------------------------------------------------- teardown
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        // failure path only: give copies and MMAs that were already issued time to land before the
        // shared memory and the TMEM columns are handed back
        for (int i = 0; i < 20; ++i) __nanosleep(1000000);
        __syncthreads();
    }
    cluster_sync_all();            // the peer no longer signals into this CTA's shared memory or uses the pair's TMEM
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem_base, 512);
    }
}

// ------------------------------------------------------------------ host side
template <bool GLU, int ACT>
static cudaError_t lt_launch(const CUtensorMap &mx, const CUtensorMap &mw, const CUtensorMap &mu, const LtParams &p, int grid, cudaStream_t st)
{
    static DeviceMask configured{0ull};               // per device
    const cudaError_t ce = ensure_dynamic_smem(linear_tc_kernel<GLU, ACT>, (int)LT_SMEM_BYTES, configured);
    if (ce != cudaSuccess) return ce;
    linear_tc_kernel<GLU, ACT><<<grid, LT_THREADS, LT_SMEM_BYTES, st>>>(mx, mw, mu, p);
    return cudaGetLastError();
}
template <bool GLU>
static cudaError_t lt_pick(int act, const CUtensorMap &mx, const CUtensorMap &mw, const CUtensorMap &mu, const LtParams &p, int grid, cudaStream_t st)
{
    switch (act) {
    case DASS_ACT_SILU: return lt_launch<GLU, DASS_ACT_SILU>(mx, mw, mu, p, grid, st);
    case DASS_ACT_GELU_TANH: return lt_launch<GLU, DASS_ACT_GELU_TANH>(mx, mw, mu, p, grid, st);
    case DASS_ACT_RELU: return lt_launch<GLU, DASS_ACT_RELU>(mx, mw, mu, p, grid, st);
    default: return lt_launch<GLU, DASS_ACT_NONE>(mx, mw, mu, p, grid, st);
    }
}

int device_sm_count();                                                                                       // dass_abi.cu
int *linear_status_word();                                                                                   // linear.cu
bool tc_make_map(CUtensorMap *map, const void *ptr, int64_t rows, int64_t cols, int64_t ld, int box_rows);   // calib_tc.cu
bool tc_make_map_3d(CUtensorMap *map, const void *ptr, int64_t mats, int64_t rows, int64_t cols, int64_t ld, int64_t mat_stride, int box_rows);

dass_status linear_tc_launch(const LinearArgs &a)
{
    const bool glu = a.W_up != nullptr;
    CUtensorMap mx, mw, mu;
    if (!tc_make_map(&mx, a.X, a.T, a.K, a.ldx, LT_BM) || !tc_make_map_3d(&mw, a.W, a.groups, a.N, a.K, a.ldw, a.group_stride, 128) ||
        !tc_make_map_3d(&mu, glu ? a.W_up : a.W, a.groups, a.N, a.K, a.ldw, a.group_stride, 128))
        return DASS_ERR_CUDA;
    LtParams p;
    p.offsets = a.offsets;
    p.bias = static_cast<const uint16_t *>(a.bias); p.bias_up = static_cast<const uint16_t *>(a.bias_up);
    p.residual = static_cast<const uint16_t *>(a.residual);
    p.Y = static_cast<uint16_t *>(a.Y);
    p.ldr = a.ldr; p.ldy = a.ldy; p.T = a.T;
    p.N = (int)a.N; p.groups = a.groups;
    p.cols_per_tile = glu ? LT_BN / 2 : LT_BN;
    p.col_tiles = (int)((a.N + p.cols_per_tile - 1) / p.cols_per_tile);
    p.k_blocks = (int)((a.K + LT_BK - 1) / LT_BK);
    p.y_vec = rows_vec_ok(a.Y, a.ldy, true);
    p.r_vec = a.residual && rows_vec_ok(a.residual, a.ldr, true);
    p.status = linear_status_word();
    if (!p.status) return DASS_ERR_CUDA;
    const int64_t items = ((a.T + 2 * LT_BM - 1) / (2 * LT_BM) + (a.offsets ? a.groups : 0)) * p.col_tiles;   // at most
    const int pairs = device_sm_count() / 2;
    const int grid = 2 * (int)(items < pairs ? items : pairs);
    const cudaError_t e = glu ? lt_pick<true>(a.act, mx, mw, mu, p, grid, a.st) : lt_pick<false>(a.act, mx, mw, mu, p, grid, a.st);
    return e == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

}  // namespace dass
