// dass_linear_mx4 for rows and weights in 4 bits and many rows, on the tensor cores' block-scaled 4-bit path: Y = act(X W^T
// + b) [* (X W_up^T + b_up)] + R, dense or per expert.
//
// A persistent kernel run by CTA pairs (a cluster of 2) that drive tcgen05.mma.cta_group::2.kind::mxf4 of shape 256 x BN x
// 64: e2m1 products in f32 accumulators, each block of 32 k under its scales of row and column, which the instruction reads
// from TMEM.
//   * M = 256 rows of X, 128 to each CTA; N = BN accumulator columns: BN columns of Y, or, in the GLU form, 128 of the
//     gate product (the leader CTA loads W) beside the same 128 of the up product (its peer loads W_up);
//   * a stage holds 256 k: 128 bytes of codes a row (the 128-byte swizzle) and the scale tiles, which come as the format
//     stores them and go to TMEM by tcgen05.cp, every CTA's own rows' and all columns';
//   * 256 accumulator columns leave no room for a second accumulator beside the scales, so the epilogue first takes the
//     whole accumulator into registers (128 a thread) and hands it back; arithmetic and stores then run under the next
//     tile's products.
//   warp 0      TMA;  warp 1  TMEM, scale copies and MMAs (leader);  warps 2..9  epilogue
// Groups: a scale tile covers rows 128 i .. 128 i + 127 of X wherever an expert begins, so an expert's row tiles begin at the
// multiple of 128 at or below its first row and store its own rows alone.
//
// Bound by the tensor pipe, and by the accumulator's way out: 8192^3 190 us (5.8 PFLOP/s), of a tile's 19000 cycles about 2000
// between the last product of one tile and the first of the next (181 at best; with a bias 183, a residual 192, both 216; in
// a loop of seconds, where power sets the clocks, 219 without both and 242 with); 16384 rows of 8 experts 4096 x 14336 gated
// 786 to 876 us (4.4 to 4.9 PFLOP/s; K is half as long, and an expert's first and last tiles are part empty).  The scale copies cost 3 %.
//
// Every wait is bounded, as in linear_tc.cu.
#include "linear_tc.cuh"
#include "mx4_linear.cuh"
#include "tc_common.cuh"
#include "tc_pair.cuh"

namespace dass {

constexpr int MT_BM = 128;          // rows per CTA
constexpr int MT_BK = 256;          // k per stage: one 128-byte swizzle row of codes, two scale tiles
constexpr int MT_EPI_WARPS = 8;     // two to a quarter of the TMEM lanes, each with half of the columns
constexpr int MT_THREADS = 64 + 32 * MT_EPI_WARPS;
constexpr uint32_t MT_ROW_BYTES = MT_BK / 2;
constexpr uint32_t MT_A_BYTES = MT_BM * MT_ROW_BYTES;
constexpr uint32_t MT_SCALES = 2 * MX4_TILE_BYTES;                   // 128 rows' scales of a stage
constexpr int MT_TURN_PITCH = 20;                                     // words from row to row of 32 bf16
constexpr uint32_t MT_TURN_BYTES = MT_EPI_WARPS * 32 * MT_TURN_PITCH * 4;
constexpr uint32_t MT_SF_COL = 256;                                   // TMEM columns from here on hold scales
template <int BN> struct MtShape {  // BN: accumulator columns; each CTA of the pair loads half of their codes
    static constexpr uint32_t B_BYTES = BN / 2 * MT_ROW_BYTES;
    static constexpr uint32_t STAGE = MT_A_BYTES + B_BYTES + MT_SCALES + BN / 128 * MT_SCALES;
    static constexpr int STAGES = BN == 256 ? 5 : 6;
    static constexpr int ACCS = 256 / BN;                             // accumulators
    static constexpr uint32_t SF_COLS = 8 + BN / 16;                  // TMEM columns of a stage's scales
    static constexpr uint32_t BYTES = STAGES * STAGE + 1024 /* alignment slack */ + 256 /* barriers */ + MX4_TABLE_BYTES + MT_TURN_BYTES;
    static_assert(BYTES <= 227 * 1024 && MT_SF_COL + STAGES * SF_COLS <= 512 && STAGE % 1024 == 0, "");
};

struct MtParams {
    const int32_t *offsets;
    const uint16_t *bias, *bias_up, *residual;
    uint16_t *Y;
    int64_t ldr, ldy, T;
    int N, groups, col_tiles, k_stages, cols_per_tile;
    int x_tiles, w_tiles;           // scale tiles along the rows of X, along the rows of one weight matrix
    int y_vec, r_vec;               // whole 16-byte accesses
    int *timeouts;
};

// ------------------------------------------------------------------ PTX wrappers
// 32 rows of 16 bytes to 4 TMEM columns of lanes 0 .. 31, and to the other three quarters of the lanes; in both CTAs, each
// from its own shared memory.
__device__ __forceinline__ void tmem_copy_scales_pair(uint32_t taddr, uint64_t desc)
{
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ void umma_mxf4_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "setp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
                 ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(sfa), "r"(sfb) : "memory");
}

// A column's bias for the lanes of a warp: lane l holds column n + l.
__device__ __forceinline__ float mt_bias(const uint16_t *bias, int64_t at, int n, int N)
{
    return bias && n < N ? __uint_as_float((uint32_t)DASS_LD(bias + at + n) << 16) : 0.f;
}

template <int BN, bool GLU, int ACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(MT_THREADS, 1)
mx4_tc_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_up,
              const __grid_constant__ CUtensorMap map_xs, const __grid_constant__ CUtensorMap map_ws, const __grid_constant__ CUtensorMap map_us,
              const MtParams p)
{
    using S = MtShape<BN>;
    constexpr int STAGES = S::STAGES;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;                 // swizzled tiles need 1024-byte alignment
    uint8_t *aligned = smem_raw + (base - raw);
    uint64_t *bars = reinterpret_cast<uint64_t *>(aligned + STAGES * S::STAGE);
    const uint32_t bar_full = smem_u32(bars);                     // [stages], used in the leader
    const uint32_t bar_empty = bar_full + 8 * STAGES;             // [stages], per CTA
    const uint32_t bar_acc_full = bar_empty + 8 * STAGES;         // [accumulators], per CTA
    const uint32_t bar_acc_empty = bar_acc_full + 16;             // [accumulators], leader: the epilogue warps of both CTAs arrive
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 2 * STAGES + 4);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    int *first_tile = reinterpret_cast<int *>(reinterpret_cast<uint8_t *>(bars) + 256);

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();                      // 0 = leader
    const int64_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (threadIdx.x == 64) {                                      // the descriptors' first fetch runs beside the set-up
        tma_prefetch_map(&map_w);
        tma_prefetch_map(&map_ws);
        tma_prefetch_map(&map_x);
        tma_prefetch_map(&map_xs);
        if constexpr (GLU) { tma_prefetch_map(&map_up); tma_prefetch_map(&map_us); }
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(bar_acc_full + 8 * s, 1); mbar_init(bar_acc_empty + 8 * s, 2 * MT_EPI_WARPS); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    mx4_count_tiles(first_tile, p.offsets, p.groups, p.T, MT_BM, 2 * MT_BM, MT_THREADS);
    if (warp == 1) {
        tmem_alloc_pair(smem_u32(tmem_slot), 512);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) mx4_sum_tiles(first_tile, p.groups);
    __syncthreads();
    cluster_sync_all();            // both CTAs' barriers are initialised and both TMEM allocations exist
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    // Both issuing warps run their loops whole and elect a lane for the instructions, which keeps the operands uniform.
    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer (one per CTA)
        uint32_t stage = 0, phase = 0;
        bool ok = true;
        const uint32_t leader_full = map_to_cta(bar_full, 0);
        const uint64_t pol = l2_policy_evict_last();
        const CUtensorMap *map_b = GLU && rank ? &map_up : &map_w;
        Mx4Item it;
        for (int64_t idx = pair; ok && mx4_item(first_tile, p.groups, MT_BM, 2 * MT_BM, p.col_tiles, p.cols_per_tile, idx, it); idx += pairs) {
            const int a_row = it.row + (int)rank * MT_BM;
            const int b_row = it.col + (GLU ? 0 : (int)rank * (BN / 2));
            const int a_tile = a_row / MX4_TILE_ROWS < p.x_tiles ? a_row / MX4_TILE_ROWS : p.x_tiles - 1;      // absent rows are not stored
            const int w_first = it.g * p.w_tiles, w_tile = w_first + it.col / MX4_TILE_ROWS;
            const int w_next = w_tile + 1 < w_first + p.w_tiles ? w_tile + 1 : w_tile;                           // nor absent columns
            for (int kb = 0; kb < p.k_stages; ++kb) {
                if (!warp_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag)) { ok = false; break; }
                const uint32_t sbase = base + stage * S::STAGE, scales = sbase + MT_A_BYTES + S::B_BYTES;
                const uint32_t fb = leader_full + 8 * stage;
                if (elect_one()) {
                    if (rank == 0) mbar_arrive_expect_tx(bar_full + 8 * stage, 2 * S::STAGE);   // both CTAs' bytes
                    tma_load_3d_pair(sbase, &map_x, fb, kb * (int)MT_ROW_BYTES, a_row, 0, pol);
                    tma_load_3d_pair(sbase + MT_A_BYTES, map_b, fb, kb * (int)MT_ROW_BYTES, b_row, it.g, pol);
                    tma_load_3d_pair(scales, &map_xs, fb, 0, kb * 2, a_tile, pol);
                    tma_load_3d_pair(scales + MT_SCALES, &map_ws, fb, 0, kb * 2, w_tile, pol);
                    if constexpr (GLU) tma_load_3d_pair(scales + 2 * MT_SCALES, &map_us, fb, 0, kb * 2, w_tile, pol);
                    else if constexpr (BN == 256) tma_load_3d_pair(scales + 2 * MT_SCALES, &map_ws, fb, 0, kb * 2, w_next, pol);
                }
                __syncwarp();
                if (++stage == STAGES) { stage = 0; phase ^= 1u; }
            }
        }
        if (!ok && lane == 0) { *abort_flag = 1; atomicAdd(p.timeouts, 1); }
    } else if (warp == 1) {
        // ------------------------------------------------------------ scale copies and MMAs (leader CTA only)
        if (rank == 0) {
            Mx4Ring r;
            uint32_t tile = 0;
            bool ok = true, ready = false;
            const int64_t items = (int64_t)first_tile[p.groups] * p.col_tiles;
            for (int64_t idx = pair; ok && idx < items; idx += pairs, ++tile) {
                const uint32_t as = tile % S::ACCS;
                if (!warp_wait(bar_acc_empty + 8 * as, ((tile / S::ACCS) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
                const uint32_t acc_addr = tmem_base + as * BN;
                for (int kb = 0; kb < p.k_stages; ++kb) {
                    if (!ready && !warp_wait(bar_full + 8 * r.stage, r.phase, abort_flag)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t stage = r.stage;
                    r.step(STAGES);
                    const bool next = mbar_test(bar_full + 8 * r.stage, r.phase);
                    const uint32_t sbase = base + stage * S::STAGE, scales = sbase + MT_A_BYTES + S::B_BYTES;
                    const uint32_t sfa = tmem_base + MT_SF_COL + stage * S::SF_COLS, sfb = sfa + 8;
                    if (elect_one()) {
                        // columns of a scale tile: 4; those of one k tile's BN columns side by side
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            tmem_copy_scales_pair(sfa + 4 * t, smem_desc_scales(scales + t * MX4_TILE_BYTES));
#pragma unroll
                            for (int n = 0; n < BN / 128; ++n)
                                tmem_copy_scales_pair(sfb + t * (BN / 32) + 4 * n, smem_desc_scales(scales + (1 + n) * MT_SCALES + t * MX4_TILE_BYTES));
                        }
                        const uint64_t da = smem_desc_sw128(sbase);
                        const uint64_t db = smem_desc_sw128(sbase + MT_A_BYTES);
#pragma unroll
                        for (int k = 0; k < MT_BK / 64; ++k)                      // 32 bytes of codes per k step
                            umma_mxf4_pair(acc_addr, da + 2 * k, db + 2 * k, idesc_mxf4(2 * MT_BM, BN, (k & 1) * 2), sfa + 4 * (k >> 1),
                                           sfb + (BN / 32) * (k >> 1), (kb > 0 || k > 0) ? 1u : 0u);
                        umma_commit_pair(bar_empty + 8 * stage, (uint16_t)3);   // slot free in both CTAs
                        if (kb + 1 == p.k_stages) umma_commit_pair(bar_acc_full + 8 * as, (uint16_t)3);   // accumulator ready in both CTAs
                    }
                    ready = __all_sync(FULL_MASK, next);
                }
            }
            if (!ok && lane == 0) { *abort_flag = 1; atomicAdd(p.timeouts, 1); }
        }
    } else {
        // ------------------------------------------------------------ epilogue (this CTA's 128 rows)
        lin_zero_outside<true>(p.offsets, p.groups, p.T, p.N, p.Y, p.ldy, p.y_vec != 0, (int64_t)blockIdx.x * (32 * MT_EPI_WARPS) + threadIdx.x - 64,
                               (int64_t)gridDim.x * (32 * MT_EPI_WARPS));
        constexpr int COLS = GLU ? BN / 2 : BN;                  // columns of Y per tile
        constexpr int CHUNKS = COLS / 64;                        // of 32 columns, of this warp's half
        const int quad = warp & 3;                               // TMEM lanes 32*quad .. 32*quad+31
        const int half = (warp - 2) >> 2;
        const uint32_t lane_addr = tmem_base + ((uint32_t)(quad * 32) << 16);
        const uint32_t leader_acc_empty = map_to_cta(bar_acc_empty, 0);
        // Blocks of 32 rows x 32 columns are turned through shared memory, so that an access moves runs of a row (linear_tc.cu).
        uint32_t *turn = reinterpret_cast<uint32_t *>(first_tile) + MX4_TABLE_BYTES / 4 + (warp - 2) * 32 * MT_TURN_PITCH;
        uint16_t *turn16 = reinterpret_cast<uint16_t *>(turn);
        const int vr = lane >> 2, vc = (lane & 3) * 8;           // this lane's row and column in an access of 8 rows
        uint32_t tile = 0;
        bool ok = true;
        Mx4Item it;
        for (int64_t idx = pair; ok && mx4_item(first_tile, p.groups, MT_BM, 2 * MT_BM, p.col_tiles, p.cols_per_tile, idx, it); idx += pairs, ++tile) {
            const uint32_t as = tile % S::ACCS;
            const int64_t t0 = (int64_t)it.row + rank * MT_BM + quad * 32;                  // the warp's first row
            const int r_lo = it.row_lo > t0 ? (int)(it.row_lo - t0 < 32 ? it.row_lo - t0 : 32) : 0;
            const int r_hi = it.row_hi - t0 < 32 ? (int)(it.row_hi - t0 > 0 ? it.row_hi - t0 : 0) : 32;   // rows r_lo .. r_hi - 1 are the expert's
            const int64_t b_at = (int64_t)it.g * p.N;
            if (!warp_wait(bar_acc_full + 8 * as, (tile / S::ACCS) & 1u, abort_flag)) { ok = false; break; }
            tc_fence_after();
            uint32_t acc[CHUNKS][32], up[GLU ? CHUNKS : 1][32];
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                tmem_ld_32(lane_addr + as * BN + half * (COLS / 2) + 32 * c, acc[c]);
                if constexpr (GLU) tmem_ld_32(lane_addr + as * BN + BN / 2 + half * (COLS / 2) + 32 * c, up[c]);
            }
            tmem_wait_ld();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_tmem(leader_acc_empty + 8 * as);   // release the accumulator to the leader's MMA warp
            if (r_lo >= r_hi) continue;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const int n0 = it.col + half * (COLS / 2) + 32 * c;
                if (n0 >= p.N) break;
                const bool whole = n0 + 32 <= p.N, col_in = n0 + lane < p.N;
                const float bn = mt_bias(p.bias, b_at, n0 + lane, p.N);
                const float bu = GLU ? mt_bias(p.bias_up, b_at, n0 + lane, p.N) : 0.f;
                uint32_t w[16];
                if (p.residual) {
                    if (p.r_vec && whole) {
                        uint4 rv[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int r = 8 * i + vr;
                            rv[i] = make_uint4(0u, 0u, 0u, 0u);
                            if (r >= r_lo && r < r_hi) rv[i] = DASS_LD(reinterpret_cast<const uint4 *>(p.residual + (t0 + r) * p.ldr + n0 + vc));
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4 *>(turn16 + (8 * i + vr) * 2 * MT_TURN_PITCH + vc) = rv[i];
                    } else {
                        const uint16_t *res = p.residual + t0 * p.ldr + n0 + lane;
#pragma unroll 4
                        for (int r = r_lo; r < r_hi; ++r) turn16[r * 2 * MT_TURN_PITCH + lane] = col_in ? DASS_LD(res + r * p.ldr) : (uint16_t)0;
                    }
                    __syncwarp();
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const uint4 x = *reinterpret_cast<const uint4 *>(turn + lane * MT_TURN_PITCH + 4 * v);
                        w[4 * v] = x.x; w[4 * v + 1] = x.y; w[4 * v + 2] = x.z; w[4 * v + 3] = x.w;
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) w[j] = 0u;
                }
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    float y[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float x = __uint_as_float(acc[c][2 * j + h]);
                        if (p.bias) x += __shfl_sync(FULL_MASK, bn, 2 * j + h);
                        x = lt_act<ACT>(x);
                        if constexpr (GLU) {
                            float v = __uint_as_float(up[c][2 * j + h]);
                            if (p.bias_up) v += __shfl_sync(FULL_MASK, bu, 2 * j + h);
                            x *= v;
                        }
                        y[h] = x + __uint_as_float(h ? (w[j] & 0xffff0000u) : (w[j] << 16));
                    }
                    w[j] = pack_bf16x2(y[0], y[1]);
                }
                __syncwarp();                                     // the reads of this memory are done
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    *reinterpret_cast<uint4 *>(turn + lane * MT_TURN_PITCH + 4 * v) = make_uint4(w[4 * v], w[4 * v + 1], w[4 * v + 2], w[4 * v + 3]);
                __syncwarp();
                if (p.y_vec && whole) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = 8 * i + vr;
                        const uint4 x = *reinterpret_cast<const uint4 *>(turn16 + r * 2 * MT_TURN_PITCH + vc);
                        if (r >= r_lo && r < r_hi) DASS_ST(reinterpret_cast<uint4 *>(p.Y + (t0 + r) * p.ldy + n0 + vc), x);
                    }
                } else {
                    uint16_t *row = p.Y + (t0 + r_lo) * p.ldy + n0 + lane;
#pragma unroll 4
                    for (int r = r_lo; r < r_hi; ++r, row += p.ldy)
                        if (col_in) DASS_ST(row, turn16[r * 2 * MT_TURN_PITCH + lane]);
                }
                __syncwarp();
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
        tmem_dealloc_pair(tmem_base, 512);
    }
}

// ------------------------------------------------------------------ host side
int device_sm_count();                                                                                       // dass_abi.cu
int *linear_timeouts();                                                                                      // linear.cu

struct MtMaps { CUtensorMap x, w, up, xs, ws, us; };

template <int BN, bool GLU, int ACT>
static cudaError_t mt_launch(const MtMaps &m, const MtParams &p, int grid, cudaStream_t st)
{
    static DeviceMask configured{0ull};               // per device
    const cudaError_t ce = ensure_dynamic_smem(mx4_tc_kernel<BN, GLU, ACT>, (int)MtShape<BN>::BYTES, configured);
    if (ce != cudaSuccess) return ce;
    mx4_tc_kernel<BN, GLU, ACT><<<grid, MT_THREADS, MtShape<BN>::BYTES, st>>>(m.x, m.w, m.up, m.xs, m.ws, m.us, p);
    return cudaGetLastError();
}
template <int BN, bool GLU>
static cudaError_t mt_pick(int act, const MtMaps &m, const MtParams &p, int grid, cudaStream_t st)
{
    switch (act) {
    case DASS_ACT_SILU: return mt_launch<BN, GLU, DASS_ACT_SILU>(m, p, grid, st);
    case DASS_ACT_GELU_TANH: return mt_launch<BN, GLU, DASS_ACT_GELU_TANH>(m, p, grid, st);
    case DASS_ACT_RELU: return mt_launch<BN, GLU, DASS_ACT_RELU>(m, p, grid, st);
    default: return mt_launch<BN, GLU, DASS_ACT_NONE>(m, p, grid, st);
    }
}

// bn: 256 or (without the GLU form) 128 accumulator columns per tile
dass_status mx4_tc_launch(const Mx4Args &q, int bn)
{
    const LinearArgs &a = q.a;
    const bool glu = q.up.codes != nullptr;
    const int64_t w_tiles = mx4_row_tiles(a.N);
    const Mx4Matrix &second = glu ? q.up : q.w;
    MtMaps m;
    if (!mx4_codes_map(&m.x, q.x.codes, 1, a.T, a.K, MT_BM) || !mx4_codes_map(&m.w, q.w.codes, a.groups, a.N, a.K, bn / 2) ||
        !mx4_codes_map(&m.up, second.codes, a.groups, a.N, a.K, bn / 2) || !mx4_scales_map(&m.xs, q.x.scales, mx4_row_tiles(a.T), a.K) ||
        !mx4_scales_map(&m.ws, q.w.scales, a.groups * w_tiles, a.K) || !mx4_scales_map(&m.us, second.scales, a.groups * w_tiles, a.K))
        return DASS_ERR_CUDA;
    MtParams p;
    p.offsets = a.offsets;
    p.bias = static_cast<const uint16_t *>(a.bias); p.bias_up = static_cast<const uint16_t *>(a.bias_up);
    p.residual = static_cast<const uint16_t *>(a.residual);
    p.Y = static_cast<uint16_t *>(a.Y);
    p.ldr = a.ldr; p.ldy = a.ldy; p.T = a.T;
    p.N = (int)a.N; p.groups = a.groups;
    p.cols_per_tile = glu ? bn / 2 : bn;
    p.col_tiles = (int)((a.N + p.cols_per_tile - 1) / p.cols_per_tile);
    p.k_stages = (int)((a.K + MT_BK - 1) / MT_BK);
    p.x_tiles = (int)mx4_row_tiles(a.T); p.w_tiles = (int)w_tiles;
    p.y_vec = rows_vec_ok(a.Y, a.ldy, true);
    p.r_vec = a.residual && rows_vec_ok(a.residual, a.ldr, true);
    p.timeouts = linear_timeouts();
    if (!p.timeouts) return DASS_ERR_CUDA;
    const int64_t items = ((a.T + 2 * MT_BM - 1) / (2 * MT_BM) + (a.offsets ? 2 * a.groups : 0)) * p.col_tiles;   // at most
    const int pairs = device_sm_count() / 2;
    const int grid = 2 * (int)(items < pairs ? items : pairs);
    cudaError_t e;
    if (bn == 256) e = glu ? mt_pick<256, true>(a.act, m, p, grid, a.st) : mt_pick<256, false>(a.act, m, p, grid, a.st);
    else e = mt_pick<128, false>(a.act, m, p, grid, a.st);
    return e == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

}  // namespace dass
