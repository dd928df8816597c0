// dass_linear for bf16 and many rows on the sm_100a tensor cores: Y = act(X W^T + b) [* (X W_up^T + b_up)] + R, dense or
// per expert.
//
// A persistent kernel run by CTA pairs (a cluster of 2) that drive tcgen05.mma.cta_group::2 of shape 256 x 256 x 16:
//   * M = 256 rows of X, 128 to each CTA; N = 256 accumulator columns: 256 columns of Y, or, in the GLU form, 128 of the
//     gate product (the leader CTA loads W) beside the same 128 of the up product (its peer loads W_up);
//   * two accumulators of 256 TMEM columns: the epilogue of one tile runs under the products of the next.
//   warp 0      TMA into a 6-stage, 128B-swizzled ring;  warp 1  TMEM, MMAs (leader);  warps 2..9  epilogue
// Groups: every expert's rows are cut into tiles of 256 by themselves.  A tile may begin at any row (the row coordinate
// of a TMA box is free) and reads on into the next expert's rows; those results are not stored.  The host does not know
// the offsets, so every CTA builds the prefix sums of the experts' tile counts once and finds its items in them.  Inside
// an expert the items run over 8 row tiles before they step to the next columns: the pairs at work at one time then
// share a patch of about 8 x 9 tiles through L2 (bands of 4 or 16 rows, and other cache hints than "keep" for both
// operands, are 2 to 10 % slower).
//
// Tiles of 256 columns, or of 128 where those fill the machine better (512 rows, 4096 x 4096: 21 against 30 us).  Bound by
// the tensor pipe and, run back to back, by the power it draws: 8192^3 with bias and residual takes 868 to 906 us (1267 to
// 1213 TFLOP/s; 865 without them on the card of 890, a library product 806 there), 705 us as a single burst; 16384 rows of 8 experts 4096 -> 14336 gated 3.03
// ms, 14336 -> 4096 1.60 ms.  With short contractions the epilogue bounds (16384 x 512 -> 2048: 35 us).
//
// Every wait is bounded: when one runs out the CTA raises an abort flag, counts it for dass_linear_status, lets its roles
// drain and frees its TMEM before it returns.
#include "linear_common.cuh"
#include "linear_tc.cuh"
#include "tc_common.cuh"
#include "tc_pair.cuh"

namespace dass {

constexpr int LT_BM = 128;          // rows per CTA
constexpr int LT_BK = 64;           // k per stage: one 128-byte swizzle row
constexpr int LT_EPI_WARPS = 8;     // two to a quarter of the TMEM lanes, each with half of the columns
constexpr int LT_THREADS = 64 + 32 * LT_EPI_WARPS;
constexpr int LT_BAND = 8;          // row tiles that are walked before the next columns
constexpr uint32_t LT_A_BYTES = LT_BM * LT_BK * 2;
constexpr uint32_t LT_TABLE_BYTES = (3 * LIN_MAX_GROUPS + 4) * 4;   // a group's first tile, first row and end
constexpr int LT_TURN_PITCH = 20;                                     // words from row to row of 32 bf16: 16-byte accesses of 8 rows meet no bank twice
constexpr uint32_t LT_TURN_BYTES = LT_EPI_WARPS * 32 * LT_TURN_PITCH * 4;
template <int BN> struct LtShape {  // BN: accumulator columns; each CTA of the pair loads half of them
    static constexpr uint32_t STAGE = LT_A_BYTES + BN / 2 * LT_BK * 2;
    static constexpr int STAGES = BN == 256 ? 6 : 8;
    static constexpr uint32_t BYTES = STAGES * STAGE + 1024 /* alignment slack */ + 256 /* barriers */ + LT_TABLE_BYTES + LT_TURN_BYTES;
};

struct LtParams {
    const int32_t *offsets;
    const uint16_t *bias, *bias_up, *residual;
    uint16_t *Y;
    int64_t ldr, ldy, T;
    int N, groups, col_tiles, k_blocks, cols_per_tile;
    int y_vec, r_vec;               // whole 16-byte accesses
    int *timeouts;
};

struct LtItem { int g; int row, row_end, col; };

// The idx-th item of the grid's walk; false past the last one.
__device__ __forceinline__ bool lt_item(const LtParams &p, const int *first_tile, int64_t idx, LtItem &it)
{
    const int *lo = first_tile + LIN_MAX_GROUPS + 4, *hi = lo + LIN_MAX_GROUPS;
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
    it.g = a;
    it.row = lo[a] + (band * LT_BAND + (r2 - ct * nb)) * 2 * LT_BM;
    it.row_end = hi[a];
    it.col = ct * p.cols_per_tile;
    return true;
}

// A column's bias for the lanes of a warp: lane l holds column n0 + l.
__device__ __forceinline__ float lt_bias(const uint16_t *bias, int64_t at, int n, int N)
{
    return bias && n < N ? __uint_as_float((uint32_t)DASS_LD(bias + at + n) << 16) : 0.f;
}

template <int BN, bool GLU, int ACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(LT_THREADS, 1)
linear_tc_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                 const __grid_constant__ CUtensorMap map_up, const LtParams p)
{
    constexpr int STAGES = LtShape<BN>::STAGES;
    constexpr uint32_t STAGE_BYTES = LtShape<BN>::STAGE;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;                 // swizzled tiles need 1024-byte alignment
    uint8_t *aligned = smem_raw + (base - raw);
    uint64_t *bars = reinterpret_cast<uint64_t *>(aligned + STAGES * STAGE_BYTES);
    const uint32_t bar_full = smem_u32(bars);                     // [stages], used in the leader
    const uint32_t bar_empty = bar_full + 8 * STAGES;          // [stages], per CTA
    const uint32_t bar_acc_full = bar_empty + 8 * STAGES;      // [2], per CTA
    const uint32_t bar_acc_empty = bar_acc_full + 16;             // [2], leader: the epilogue warps of both CTAs arrive
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 2 * STAGES + 4);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    int *first_tile = reinterpret_cast<int *>(reinterpret_cast<uint8_t *>(bars) + 256);

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();                      // 0 = leader
    const int64_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (threadIdx.x == 64) {                                      // the descriptors' first fetch runs beside the set-up
        tma_prefetch_map(&map_w);
        if constexpr (GLU) tma_prefetch_map(&map_up);
        tma_prefetch_map(&map_x);
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(bar_acc_full + 8 * s, 1); mbar_init(bar_acc_empty + 8 * s, 2 * LT_EPI_WARPS); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    for (int g = threadIdx.x; g < p.groups; g += LT_THREADS) {
        int64_t lo, hi;
        lin_group_rows(p.offsets, g, p.T, lo, hi);
        first_tile[g + 1] = (int)((hi - lo + 2 * LT_BM - 1) / (2 * LT_BM));
        first_tile[LIN_MAX_GROUPS + 4 + g] = (int)lo;
        first_tile[2 * LIN_MAX_GROUPS + 4 + g] = (int)hi;
    }
    if (warp == 1) {
        tmem_alloc_pair(smem_u32(tmem_slot), 2 * BN);
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

    // Both issuing warps run their loops whole and elect a lane for the instructions, which keeps the operands uniform
    // (four MMAs issued inside a one-lane branch take 225 cycles, nearly as long as they run at 128 columns).
    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer (one per CTA)
        uint32_t stage = 0, phase = 0;
        bool ok = true;
        const uint32_t leader_full = map_to_cta(bar_full, 0);
        const uint64_t pol = l2_policy_evict_last();
        const CUtensorMap *map_b = GLU && rank ? &map_up : &map_w;
        LtItem it;
        for (int64_t idx = pair; ok && lt_item(p, first_tile, idx, it); idx += pairs) {
            const int a_row = it.row + (int)rank * LT_BM;
            const int b_row = it.col + (GLU ? 0 : (int)rank * (BN / 2));
            for (int kb = 0; kb < p.k_blocks; ++kb) {
                if (!warp_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag)) { ok = false; break; }
                const uint32_t sbase = base + stage * STAGE_BYTES;
                const uint32_t fb = leader_full + 8 * stage;
                if (elect_one()) {
                    if (rank == 0) mbar_arrive_expect_tx(bar_full + 8 * stage, 2 * STAGE_BYTES);   // both CTAs' bytes
                    tma_load_2d_pair(sbase, &map_x, fb, kb * LT_BK, a_row, pol);
                    tma_load_3d_pair(sbase + LT_A_BYTES, map_b, fb, kb * LT_BK, b_row, it.g, pol);
                }
                __syncwarp();
                if (++stage == STAGES) { stage = 0; phase ^= 1u; }
            }
        }
        if (!ok && lane == 0) { *abort_flag = 1; atomicAdd(p.timeouts, 1); }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer (leader CTA only)
        if (rank == 0) {
            constexpr uint32_t idesc = idesc_bf16_f32(2 * LT_BM, BN);
            uint32_t stage = 0, phase = 0, tile = 0;
            bool ok = true;
            const int64_t items = (int64_t)first_tile[p.groups] * p.col_tiles;
            for (int64_t idx = pair; ok && idx < items; idx += pairs, ++tile) {
                const uint32_t as = tile & 1u;
                if (!warp_wait(bar_acc_empty + 8 * as, ((tile >> 1) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
                tc_fence_after();
                const uint32_t acc_addr = tmem_base + as * BN;
                for (int kb = 0; kb < p.k_blocks; ++kb) {
                    if (!warp_wait(bar_full + 8 * stage, phase, abort_flag)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t sbase = base + stage * STAGE_BYTES;
                    if (elect_one()) {
                        const uint64_t da = smem_desc_sw128(sbase);
                        const uint64_t db = smem_desc_sw128(sbase + LT_A_BYTES);
#pragma unroll
                        for (int k = 0; k < LT_BK / 16; ++k)
                            umma_bf16_pair(acc_addr, da + 2 * k, db + 2 * k, idesc, (kb > 0 || k > 0) ? 1u : 0u);   // 32 bytes per k step
                        umma_commit_pair(bar_empty + 8 * stage, (uint16_t)3);   // slot free in both CTAs
                        if (kb + 1 == p.k_blocks) umma_commit_pair(bar_acc_full + 8 * as, (uint16_t)3);   // accumulator ready in both CTAs
                    }
                    __syncwarp();
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                }
            }
            if (!ok && lane == 0) { *abort_flag = 1; atomicAdd(p.timeouts, 1); }
        }
    } else {
        // ------------------------------------------------------------ epilogue (this CTA's 128 rows)
        lin_zero_outside<true>(p.offsets, p.groups, p.T, p.N, p.Y, p.ldy, p.y_vec != 0, (int64_t)blockIdx.x * (32 * LT_EPI_WARPS) + threadIdx.x - 64,
                               (int64_t)gridDim.x * (32 * LT_EPI_WARPS));
        constexpr int COLS = GLU ? BN / 2 : BN;                  // columns of Y per tile
        const int quad = warp & 3;                               // TMEM lanes 32*quad .. 32*quad+31
        const int half = (warp - 2) >> 2;
        const uint32_t lane_addr = tmem_base + ((uint32_t)(quad * 32) << 16);
        const uint32_t leader_acc_empty = map_to_cta(bar_acc_empty, 0);
        // A TMEM lane is a row, so a thread holds 32 columns of one row.  Stored from there, a warp's access touches 32 rows
        // (1600 cycles for a 32 x 32 block, and the products wait); so a warp turns each block through shared memory and
        // moves 8 rows of 64 contiguous bytes an access, or, where rows of Y do not allow 16-byte accesses, one row of 32
        // single elements.  R comes in the same way, a block ahead of its use.
        uint32_t *turn = reinterpret_cast<uint32_t *>(first_tile) + LT_TABLE_BYTES / 4 + (warp - 2) * 32 * LT_TURN_PITCH;
        uint16_t *turn16 = reinterpret_cast<uint16_t *>(turn);
        const int vr = lane >> 2, vc = (lane & 3) * 8;           // this lane's row and column in an access of 8 rows
        uint32_t tile = 0;
        bool ok = true;
        LtItem it;
        for (int64_t idx = pair; ok && lt_item(p, first_tile, idx, it); idx += pairs, ++tile) {
            const uint32_t as = tile & 1u;
            const int64_t t0 = (int64_t)it.row + rank * LT_BM + quad * 32;                  // the warp's first row
            const int rows = it.row_end - t0 < 32 ? (int)(it.row_end - t0) : 32;             // <= 0: none
            const int64_t b_at = (int64_t)it.g * p.N;
            const int c0 = half * (COLS / 2), c1 = it.col + c0 + COLS / 2 <= p.N ? c0 + COLS / 2 : p.N - it.col;   // this warp's columns
            uint4 rv[4];
            auto fetch_residual = [&](int c) {                    // whole accesses; absent rows and columns are not touched
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = 8 * i + vr, n = it.col + c + vc;
                    if (r < rows && n + 8 <= p.N) rv[i] = DASS_LD(reinterpret_cast<const uint4 *>(p.residual + (t0 + r) * p.ldr + n));
                }
            };
            if (p.r_vec && c0 < c1) fetch_residual(c0);
            if (!warp_wait(bar_acc_full + 8 * as, (tile >> 1) & 1u, abort_flag)) { ok = false; break; }
            tc_fence_after();
            const uint32_t acc_addr = lane_addr + as * BN;
#pragma unroll 1
            for (int c = c0; c < c1; c += 32) {
                const int n0 = it.col + c;
                const bool whole = n0 + 32 <= p.N, col_in = n0 + lane < p.N;
                uint32_t w[16];
                const float bn = lt_bias(p.bias, b_at, n0 + lane, p.N);
                const float bu = GLU ? lt_bias(p.bias_up, b_at, n0 + lane, p.N) : 0.f;
                if (p.residual) {
                    if (p.r_vec && whole) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4 *>(turn16 + (8 * i + vr) * 2 * LT_TURN_PITCH + vc) = rv[i];
                        if (c + 32 < c1) fetch_residual(c + 32);
                    } else {
                        const uint16_t *res = p.residual + t0 * p.ldr + n0 + lane;
#pragma unroll 1
                        for (int r0 = 0; r0 < rows; r0 += 8, res += 8 * p.ldr) {   // 8 rows' loads in flight at once
                            uint16_t x[8];
#pragma unroll
                            for (int r = 0; r < 8; ++r) x[r] = col_in && r0 + r < rows ? DASS_LD(res + r * p.ldr) : (uint16_t)0;
#pragma unroll
                            for (int r = 0; r < 8; ++r) turn16[(r0 + r) * 2 * LT_TURN_PITCH + lane] = x[r];
                        }
                    }
                    __syncwarp();
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const uint4 x = *reinterpret_cast<const uint4 *>(turn + lane * LT_TURN_PITCH + 4 * v);
                        w[4 * v] = x.x; w[4 * v + 1] = x.y; w[4 * v + 2] = x.z; w[4 * v + 3] = x.w;
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) w[j] = 0u;
                }
#pragma unroll
                for (int q = 0; q < 2; ++q) {                     // 16 columns at a time: fewer registers
                    uint32_t a[16], u[16];
                    tmem_ld_16(acc_addr + c + 16 * q, a);
                    if constexpr (GLU) tmem_ld_16(acc_addr + BN / 2 + c + 16 * q, u);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float y[2];
                        uint32_t &wj = w[8 * q + j];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float x = __uint_as_float(a[2 * j + h]);
                            if (p.bias) x += __shfl_sync(FULL_MASK, bn, 16 * q + 2 * j + h);
                            x = lt_act<ACT>(x);
                            if constexpr (GLU) {
                                float v = __uint_as_float(u[2 * j + h]);
                                if (p.bias_up) v += __shfl_sync(FULL_MASK, bu, 16 * q + 2 * j + h);
                                x *= v;
                            }
                            y[h] = x + __uint_as_float(h ? (wj & 0xffff0000u) : (wj << 16));
                        }
                        wj = pack_bf16x2(y[0], y[1]);
                    }
                }
                __syncwarp();                                     // the last block's reads of this memory are done
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    *reinterpret_cast<uint4 *>(turn + lane * LT_TURN_PITCH + 4 * v) = make_uint4(w[4 * v], w[4 * v + 1], w[4 * v + 2], w[4 * v + 3]);
                __syncwarp();
                if (p.y_vec && whole) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = 8 * i + vr;
                        const uint4 x = *reinterpret_cast<const uint4 *>(turn16 + r * 2 * LT_TURN_PITCH + vc);
                        if (r < rows) DASS_ST(reinterpret_cast<uint4 *>(p.Y + (t0 + r) * p.ldy + n0 + vc), x);
                    }
                } else {
                    uint16_t *row = p.Y + t0 * p.ldy + n0 + lane;
#pragma unroll 4
                    for (int r = 0; r < rows; ++r, row += p.ldy)
                        if (col_in) DASS_ST(row, turn16[r * 2 * LT_TURN_PITCH + lane]);
                }
                __syncwarp();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {                                     // release the accumulator to the leader's MMA warp
                if (rank == 0) mbar_arrive(bar_acc_empty + 8 * as);
                else mbar_arrive_cluster(leader_acc_empty + 8 * as);
            }
        }
        if (!ok && lane == 0) { *abort_flag = 1; atomicAdd(p.timeouts, 1); }
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
        tmem_dealloc_pair(tmem_base, 2 * BN);
    }
}

// ------------------------------------------------------------------ host side
int device_sm_count();                                                                                       // dass_abi.cu

template <int BN, bool GLU, int ACT>
static cudaError_t lt_launch(const CUtensorMap &mx, const CUtensorMap &mw, const CUtensorMap &mu, const LtParams &p, int grid, cudaStream_t st)
{
    static DeviceMask configured{0ull};               // per device
    const cudaError_t ce = ensure_dynamic_smem(linear_tc_kernel<BN, GLU, ACT>, (int)LtShape<BN>::BYTES, configured);
    if (ce != cudaSuccess) return ce;
    linear_tc_kernel<BN, GLU, ACT><<<grid, LT_THREADS, LtShape<BN>::BYTES, st>>>(mx, mw, mu, p);
    return cudaGetLastError();
}
template <int BN, bool GLU>
static cudaError_t lt_pick(int act, const CUtensorMap &mx, const CUtensorMap &mw, const CUtensorMap &mu, const LtParams &p, int grid, cudaStream_t st)
{
    switch (act) {
    case DASS_ACT_SILU: return lt_launch<BN, GLU, DASS_ACT_SILU>(mx, mw, mu, p, grid, st);
    case DASS_ACT_GELU_TANH: return lt_launch<BN, GLU, DASS_ACT_GELU_TANH>(mx, mw, mu, p, grid, st);
    case DASS_ACT_RELU: return lt_launch<BN, GLU, DASS_ACT_RELU>(mx, mw, mu, p, grid, st);
    default: return lt_launch<BN, GLU, DASS_ACT_NONE>(mx, mw, mu, p, grid, st);
    }
}

int *linear_timeouts();                                                                                      // linear.cu
bool tc_make_map(CUtensorMap *map, const void *ptr, int64_t rows, int64_t cols, int64_t ld, int box_rows);   // calib_tc.cu

// `mats` row-major bf16 matrices [rows x cols] with pitch ld, mat_stride elements apart, as one map of three dimensions: boxes of
// 64 x box_rows elements with the 128-byte swizzle; rows past a matrix's end read as zero, not as the next matrix's.
bool tc_make_map_3d(CUtensorMap *map, const void *ptr, int64_t mats, int64_t rows, int64_t cols, int64_t ld, int64_t mat_stride, int box_rows)
{
    const EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)mats};
    const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)(mats > 1 ? mat_stride : rows * ld) * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(ptr), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// bn: 256 or 128 accumulator columns per tile
dass_status linear_tc_launch(const LinearArgs &a, int bn)
{
    const bool glu = a.W_up != nullptr;
    CUtensorMap mx, mw, mu;
    if (!tc_make_map(&mx, a.X, a.T, a.K, a.ldx, LT_BM) || !tc_make_map_3d(&mw, a.W, a.groups, a.N, a.K, a.ldw, a.group_stride, bn / 2) ||
        !tc_make_map_3d(&mu, glu ? a.W_up : a.W, a.groups, a.N, a.K, a.ldw, a.group_stride, bn / 2))
        return DASS_ERR_CUDA;
    LtParams p;
    p.offsets = a.offsets;
    p.bias = static_cast<const uint16_t *>(a.bias); p.bias_up = static_cast<const uint16_t *>(a.bias_up);
    p.residual = static_cast<const uint16_t *>(a.residual);
    p.Y = static_cast<uint16_t *>(a.Y);
    p.ldr = a.ldr; p.ldy = a.ldy; p.T = a.T;
    p.N = (int)a.N; p.groups = a.groups;
    p.cols_per_tile = glu ? bn / 2 : bn;
    p.col_tiles = (int)((a.N + p.cols_per_tile - 1) / p.cols_per_tile);
    p.k_blocks = (int)((a.K + LT_BK - 1) / LT_BK);
    p.y_vec = rows_vec_ok(a.Y, a.ldy, true);
    p.r_vec = a.residual && rows_vec_ok(a.residual, a.ldr, true);
    p.timeouts = linear_timeouts();
    if (!p.timeouts) return DASS_ERR_CUDA;
    const int64_t items = ((a.T + 2 * LT_BM - 1) / (2 * LT_BM) + (a.offsets ? a.groups : 0)) * p.col_tiles;   // at most
    const int pairs = device_sm_count() / 2;
    const int grid = 2 * (int)(items < pairs ? items : pairs);
    cudaError_t e;
    if (bn == 256) e = glu ? lt_pick<256, true>(a.act, mx, mw, mu, p, grid, a.st) : lt_pick<256, false>(a.act, mx, mw, mu, p, grid, a.st);
    else e = glu ? lt_pick<128, true>(a.act, mx, mw, mu, p, grid, a.st) : lt_pick<128, false>(a.act, mx, mw, mu, p, grid, a.st);
    return e == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

}  // namespace dass
