// dass_linear_mx4 where the time is that of reading the weights, and not so few of them that mx4_few.cu is done sooner: the
// block-scaled 4-bit products of mx4_tc.cu with the operands' sides changed, so that a tensor instruction is as long as
// there are rows, and with no arithmetic per weight at all.
//
//   * M = 128 weight rows (columns of Y), N = NT rows on the other side; a persistent kernel, one CTA to an SM, whose ring of
//     codes and scales runs on into the next tile while the last one is finished;
//   * rows in 4 bits are that other side as they are: tiles of up to 128 rows from a multiple of 128 on (a scale tile);
//   * rows in bf16 are first split into MS_PIECES 4-bit rows each (mx4_split_kernel): the nearest e2m1 value under the block's
//     own scale, then the same for what is left, and so on.  A step leaves at most a quarter of the block's largest value, so
//     12 pieces hold every value of a block of 32 to 2^-24 of the largest one in it, f32's own rounding (or to 2^-129: no
//     scale is below 2^-127).  A row is 12 columns of the accumulator, which the epilogue adds up.  The products run at four
//     times the rate of bf16 ones, and the weights, which are what there is to read, need no decoding (in registers 2
//     instructions a weight, which costs mx4_few.cu 2.3 times the bytes' time on 8 experts of 4096 x 14336).
// Bound by the weights' bytes: 8 experts of 4096 x 14336 gated, 32 bf16 rows 84 us (5.9 TB/s of weights); 64 rows in 4 bits
// through 8192 x 28672 gated 44.5 us (5.6 TB/s).  Few columns leave SMs idle: 64 rows in 4 bits through 4096 x 4096 take 9 us, 32 SMs
// at work, in bf16 18.  The split costs 3 us of latency, of which the ring's first weights hide a part (1 x 4096 x 14336 gated 15.8
// -> 13.2 us).
//   warp 0  TMA;  warp 1  TMEM, scale copies and MMAs;  warps 2..9  epilogue: a thread has one column of Y, the two warps of a
//           quarter of the TMEM lanes take its rows in turn
//
// Every wait is bounded, as in linear_tc.cu.
#include "linear_tc.cuh"
#include "mx4_linear.cuh"
#include "tc_common.cuh"

namespace dass {

constexpr int MS_PIECES = 12;        // 4-bit rows of a bf16 row
constexpr int MS_COLS = 128;         // columns of Y (weight rows) per tile: MMA M
constexpr int MS_BK = 256;           // k per stage: one 128-byte swizzle row of codes, two scale tiles
constexpr int MS_THREADS = 320;
constexpr uint32_t MS_BLOCK = 16 * 64;                              // a warp's block of Y, 16 rows of 32 columns
constexpr uint32_t MS_W_BYTES = MS_COLS * MS_BK / 2, MS_SCALES = 2 * MX4_TILE_BYTES;
constexpr uint32_t MS_SF_COL = 256;  // TMEM columns from here on hold scales
constexpr int MS_SF_SLOTS = 4;       // stages whose scales are in TMEM at a time

template <int NT, bool GLU> struct MsShape {
    static constexpr int M = GLU ? 2 : 1;
    static constexpr uint32_t X_AT = M * (MS_W_BYTES + MS_SCALES);
    static constexpr uint32_t STAGE = X_AT + NT * MS_BK / 2 + MS_SCALES;
    static constexpr int STAGES = (int)(204u * 1024u / STAGE) < 8 ? (int)(204u * 1024u / STAGE) : 8;
    static constexpr int ACCS = M * NT <= 128 ? 2 : 1;                // accumulators
    static constexpr uint32_t SF_COLS = 8 + 8 * M;                    // TMEM columns of a stage's scales
    static constexpr uint32_t BYTES = STAGES * STAGE + 1024 /* alignment slack */ + 256 /* barriers */ + MX4_TABLE_BYTES + 8 * MS_BLOCK;
    static_assert(ACCS * M * NT <= 256 && MS_SF_COL + MS_SF_SLOTS * SF_COLS <= 512 && STAGE % 1024 == 0 && BYTES <= 227 * 1024 && STAGES >= 3, "");
};

struct MsParams {
    const int32_t *offsets;
    const uint16_t *bias, *bias_up, *residual;
    uint16_t *Y;
    int64_t ldr, ldy, T;
    int N, groups, col_tiles, k_stages, w_tiles, y_vec, r_vec;
    int align, rows;                // of a row tile
    int *timeouts;
};

// ------------------------------------------------------------------ rows in bf16 as rows in 4 bits
struct SplitArgs {
    const uint16_t *X; int64_t T, K, ldx;
    uint8_t *codes, *scales;        // [tiles x 128 rows x pitch], [tiles x k tiles x 512]; row r of a tile is MS_PIECES rows from r * MS_PIECES on
    const int32_t *offsets; int groups, rows;
};

// A warp has 256 columns of one row, 8 to a lane; four lanes share a block.  grid.x columns, grid.y row tiles, grid.z rows of a tile.
__global__ void __launch_bounds__(128)
mx4_split_kernel(const SplitArgs a)
{
    grid_dependents_launch();
    const int lane = threadIdx.x & 31;
    const LinTile tile = lin_find_tile(a.offsets, a.groups, a.T, a.rows, blockIdx.y);
    if (tile.g < 0 || tile.lo + blockIdx.z >= tile.hi) return;
    const int64_t c = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 5)) * 256 + lane * 8;
    const int64_t pitch = mx4_pitch(a.K), k_tiles = mx4_k_tiles(a.K);
    const uint16_t *row = a.X + (tile.lo + blockIdx.z) * a.ldx;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (c + 8 <= a.K) {
        row_load<true, 8>(row, c, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < a.K) v[i] = __uint_as_float((uint32_t)DASS_LD(row + c + i) << 16);
    }
    uint8_t *codes = a.codes + ((int64_t)blockIdx.y * MX4_TILE_ROWS + blockIdx.z * MS_PIECES) * pitch + c / 2;
    uint8_t *scales = a.scales + ((int64_t)blockIdx.y * k_tiles + c / MX4_TILE_K) * MX4_TILE_BYTES;
    bool bad = false;
#pragma unroll 1
    for (int j = 0; j < MS_PIECES; ++j) {
        uint32_t most = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(v[i]) & 0x7fffffffu);
        most = max(most, __shfl_xor_sync(FULL_MASK, most, 1));
        most = max(most, __shfl_xor_sync(FULL_MASK, most, 2));
        // the scale that takes the largest value into (3, 6], so that none is cut: one more where its mantissa is above 1.5
        const uint32_t up_e = (most + 0x003fffffu) >> 23, e = up_e < 254u ? up_e : 254u;   // 6 x 2^125 is still a number
        bad |= most >= 0x7f800000u;                                    // NaN or infinity: the whole block is NaN, in its first piece
        const uint32_t s = bad ? (j == 0 ? 255u : 0u) : e > 2u ? e - 2u : 0u;
        const float up = __uint_as_float((254u - (bad ? 127u : s)) << 23), down = mx4_scale(bad ? 127u : s);
        uint32_t packed = 0u;
        float q[8];
        if (bad) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = v[i] * up;
        packed = mx4_encode8(q);
        mx4_decode8_f32(packed, down, q);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] -= q[i];                      // exact
        if (c < pitch * 2) DASS_ST(reinterpret_cast<uint32_t *>(codes + j * pitch), packed);
        uint32_t word = s << (8 * ((lane >> 2) & 3));
        word |= __shfl_xor_sync(FULL_MASK, word, 4);
        word |= __shfl_xor_sync(FULL_MASK, word, 8);
        const int r = blockIdx.z * MS_PIECES + j;
        if ((lane & 15) == 0 && c < k_tiles * MX4_TILE_K) DASS_ST(reinterpret_cast<uint32_t *>(scales + (r & 31) * 16 + (r >> 5) * 4), word);
    }
}

// ------------------------------------------------------------------ PTX wrappers
__device__ __forceinline__ void tmem_copy_scales(uint32_t taddr, uint64_t desc)
{
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ void umma_mxf4(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "setp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
                 ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(sfa), "r"(sfb) : "memory");
}
__device__ __forceinline__ void tmem_ld_4(uint32_t taddr, uint32_t (&r)[4])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(taddr) : "memory");
}

template <int NT, bool GLU, bool SPLIT>
__global__ void __launch_bounds__(MS_THREADS, 1)
mx4_mid_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_up,
               const __grid_constant__ CUtensorMap map_xs, const __grid_constant__ CUtensorMap map_ws, const __grid_constant__ CUtensorMap map_us,
               const MsParams p, int act)
{
    using S = MsShape<NT, GLU>;
    constexpr int M = S::M, STAGES = S::STAGES;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t *aligned = smem_raw + (base - raw);
    uint64_t *bars = reinterpret_cast<uint64_t *>(aligned + STAGES * S::STAGE);
    const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + 8 * STAGES, acc_full = bar_empty + 8 * STAGES, acc_empty = acc_full + 16;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 2 * STAGES + 4);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    int *table = reinterpret_cast<int *>(reinterpret_cast<uint8_t *>(bars) + 256);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 64) {
        tma_prefetch_map(&map_w);
        tma_prefetch_map(&map_ws);
        if constexpr (GLU) { tma_prefetch_map(&map_up); tma_prefetch_map(&map_us); }
        tma_prefetch_map(&map_x);
        tma_prefetch_map(&map_xs);
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(acc_full + 8 * s, 1); mbar_init(acc_empty + 8 * s, 8); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    mx4_count_tiles(table, p.offsets, p.groups, p.T, p.align, p.rows, MS_THREADS);
    if (warp == 1) {
        tmem_alloc(smem_u32(tmem_slot), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) mx4_sum_tiles(table, p.groups);
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    const int64_t items = (int64_t)table[p.groups] * p.col_tiles;
    Mx4Item it{};
    bool ok = true;

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer
        uint32_t stage = 0, phase = 0;
        const uint64_t pol_w = l2_policy_evict_first(), pol_x = l2_policy_evict_last();
        auto load_w = [&](uint32_t at, uint32_t full, int kb) {
            const int w_tile = it.g * p.w_tiles + it.col / MX4_TILE_ROWS;
            mbar_arrive_expect_tx(full, S::STAGE);
            tma_load_3d_hint(at, &map_w, full, kb * (MS_BK / 2), it.col, it.g, pol_w);
            tma_load_3d_hint(at + MS_W_BYTES, &map_ws, full, 0, kb * 2, w_tile, pol_w);
            if constexpr (GLU) {
                tma_load_3d_hint(at + MS_W_BYTES + MS_SCALES, &map_up, full, kb * (MS_BK / 2), it.col, it.g, pol_w);
                tma_load_3d_hint(at + 2 * MS_W_BYTES + MS_SCALES, &map_us, full, 0, kb * 2, w_tile, pol_w);
            }
        };
        // The ring's first weights are on their way before the split rows are there.
        int early = 0;
        if (SPLIT && mx4_item(table, p.groups, p.align, p.rows, p.col_tiles, MS_COLS, blockIdx.x, it)) {
            early = p.k_stages < STAGES ? p.k_stages : STAGES;
            if (elect_one())
                for (int kb = 0; kb < early; ++kb) load_w(base + kb * S::STAGE, bar_full + 8 * kb, kb);
            __syncwarp();
        }
        if (SPLIT) grid_dependency_wait();
        for (int64_t idx = blockIdx.x; ok && mx4_item(table, p.groups, p.align, p.rows, p.col_tiles, MS_COLS, idx, it); idx += gridDim.x) {
            const int x_tile = SPLIT ? it.tile : it.row / MX4_TILE_ROWS;
            for (int kb = 0; kb < p.k_stages; ++kb) {
                if (!warp_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag)) { ok = false; break; }
                const uint32_t sbase = base + stage * S::STAGE, full = bar_full + 8 * stage;
                if (elect_one()) {
                    if (early == 0) load_w(sbase, full, kb);
                    if constexpr (SPLIT) tma_load_3d_hint(sbase + S::X_AT, &map_x, full, kb * (MS_BK / 2), 0, it.tile, pol_x);
                    else tma_load_3d_hint(sbase + S::X_AT, &map_x, full, kb * (MS_BK / 2), it.row, 0, pol_x);
                    tma_load_3d_hint(sbase + S::X_AT + NT * (MS_BK / 2), &map_xs, full, 0, kb * 2, x_tile, pol_x);
                }
                __syncwarp();
                if (early > 0) --early;
                if (++stage == STAGES) { stage = 0; phase ^= 1u; }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ scale copies and MMAs
        Mx4Ring r;
        uint32_t tile = 0, slot = 0;
        bool ready = false;
        for (int64_t idx = blockIdx.x; ok && idx < items; idx += gridDim.x, ++tile) {
            const uint32_t as = tile % S::ACCS;
            if (!warp_wait(acc_empty + 8 * as, ((tile / S::ACCS) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
            const uint32_t acc = tmem_base + as * (M * NT);
            for (int kb = 0; kb < p.k_stages; ++kb) {
                if (!ready && !warp_wait(bar_full + 8 * r.stage, r.phase, abort_flag)) { ok = false; break; }
                tc_fence_after();
                const uint32_t stage = r.stage;
                r.step(STAGES);
                const bool next = mbar_test(bar_full + 8 * r.stage, r.phase);
                const uint32_t sbase = base + stage * S::STAGE;
                const uint32_t sfx = tmem_base + MS_SF_COL + slot * S::SF_COLS, sfw = sfx + 8;
                if (elect_one()) {
                    // A slot's columns are written again MS_SF_SLOTS stages later: copies and products run in the order of their issue.
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        tmem_copy_scales(sfx + 4 * t, smem_desc_scales(sbase + S::X_AT + NT * (MS_BK / 2) + t * MX4_TILE_BYTES));
#pragma unroll
                        for (int m = 0; m < M; ++m)
                            tmem_copy_scales(sfw + 8 * m + 4 * t, smem_desc_scales(sbase + m * (MS_W_BYTES + MS_SCALES) + MS_W_BYTES + t * MX4_TILE_BYTES));
                    }
                    const uint64_t db = smem_desc_sw128(sbase + S::X_AT);
#pragma unroll
                    for (int m = 0; m < M; ++m) {
                        const uint64_t da = smem_desc_sw128(sbase + m * (MS_W_BYTES + MS_SCALES));
#pragma unroll
                        for (int k = 0; k < MS_BK / 64; ++k)
                            umma_mxf4(acc + m * NT, da + 2 * k, db + 2 * k, idesc_mxf4(MS_COLS, NT, (k & 1) * 2), sfw + 8 * m + 4 * (k >> 1),
                                      sfx + 4 * (k >> 1), (kb > 0 || k > 0) ? 1u : 0u);
                    }
                    umma_commit(bar_empty + 8 * stage);
                    if (kb + 1 == p.k_stages) umma_commit(acc_full + 8 * as);
                }
                ready = __all_sync(FULL_MASK, next);
                if (++slot == MS_SF_SLOTS) slot = 0;
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue: this thread's column of Y
        constexpr int EPI = MS_THREADS - 64;
        lin_zero_outside<true>(p.offsets, p.groups, p.T, p.N, p.Y, p.ldy, p.y_vec != 0, (int64_t)blockIdx.x * EPI + threadIdx.x - 64, (int64_t)gridDim.x * EPI);
        constexpr int STEP = SPLIT ? 4 : 16;                     // rows at a time
        const int quad = warp & 3, half = (warp - 2) >> 2;
        const uint32_t lane_addr = tmem_base + ((uint32_t)(quad * 32) << 16);
        uint16_t *block = reinterpret_cast<uint16_t *>(reinterpret_cast<uint8_t *>(table) + MX4_TABLE_BYTES + (warp - 2) * MS_BLOCK);
        uint32_t tile = 0;
        for (int64_t idx = blockIdx.x; ok && mx4_item(table, p.groups, p.align, p.rows, p.col_tiles, MS_COLS, idx, it); idx += gridDim.x, ++tile) {
            const uint32_t as = tile % S::ACCS;
            const int n0 = it.col + quad * 32, left = p.N - n0;
            const int first = it.row_lo > it.row ? it.row_lo - it.row : 0;
            const int last = it.row_hi - it.row < p.rows ? it.row_hi - it.row : p.rows;      // rows first .. last - 1 of the tile are stored
            const float b = p.bias && lane < left ? __uint_as_float((uint32_t)DASS_LD(p.bias + (int64_t)it.g * p.N + n0 + lane) << 16) : 0.f;
            const float bu = GLU && p.bias_up && lane < left ? __uint_as_float((uint32_t)DASS_LD(p.bias_up + (int64_t)it.g * p.N + n0 + lane) << 16) : 0.f;
            if (!warp_wait(acc_full + 8 * as, (tile / S::ACCS) & 1u, abort_flag)) { ok = false; break; }
            tc_fence_after();
            const uint32_t acc = lane_addr + as * (M * NT);
#pragma unroll 1
            for (int r0 = (first / STEP + ((first / STEP + half) & 1)) * STEP; left > 0 && r0 < last; r0 += 2 * STEP) {
                const int lo = first > r0 ? first - r0 : 0, hi = last - r0 < STEP ? last - r0 : STEP;
                float y[M][STEP];
                if (p.residual) mx4_block_in(block, p.residual + (it.row + r0) * p.ldr + n0, p.ldr, p.r_vec, lo, hi, left);
#pragma unroll
                for (int m = 0; m < M; ++m) {
                    if constexpr (SPLIT) {
                        uint32_t v[STEP][MS_PIECES / 4][4];
#pragma unroll
                        for (int i = 0; i < STEP; ++i)
#pragma unroll
                            for (int q = 0; q < MS_PIECES / 4; ++q) {
                                const int at = (r0 + i) * MS_PIECES + 4 * q;                 // past the tile's rows: any column
                                tmem_ld_4(acc + m * NT + (at < NT ? at : 0), v[i][q]);
                            }
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < STEP; ++i) {
                            y[m][i] = 0.f;
#pragma unroll
                            for (int j = MS_PIECES - 1; j >= 0; --j) y[m][i] += __uint_as_float(v[i][j / 4][j % 4]);   // the smallest first
                        }
                    } else {
                        uint32_t v[16];
                        tmem_ld_16(acc + m * NT + r0, v);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < STEP; ++i) y[m][i] = __uint_as_float(v[i]);
                    }
                }
#pragma unroll
                for (int i = 0; i < STEP; ++i) y[0][i] += b;
                lt_act_all(y[0], act);
                if constexpr (GLU) {
#pragma unroll
                    for (int i = 0; i < STEP; ++i) y[0][i] *= y[M - 1][i] + bu;
                }
                mx4_block_set(block, 0, y[0], p.residual != nullptr);
                mx4_block_out(block, p.Y + (it.row + r0) * p.ldy + n0, p.ldy, p.y_vec, lo, hi, left);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_empty + 8 * as);
        }
    }
    if (!ok && lane == 0) { *abort_flag = 1; atomicAdd(p.timeouts, 1); }

    tc_fence_before();
    __syncthreads();
    if (*abort_flag)
        for (int i = 0; i < 20; ++i) __nanosleep(1000000);       // failure path: let what was issued land
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, 512);
    }
}

// ------------------------------------------------------------------ host side
int device_sm_count();                                                                                       // dass_abi.cu
int *linear_timeouts();                                                                                      // linear.cu

struct MsMaps { CUtensorMap x, w, up, xs, ws, us; };

template <int NT, bool GLU, bool SPLIT>
static cudaError_t ms_launch(const MsMaps &m, const MsParams &p, int act, int grid, cudaStream_t st)
{
    static DeviceMask configured{0ull};               // per device
    const cudaError_t ce = ensure_dynamic_smem(mx4_mid_kernel<NT, GLU, SPLIT>, (int)MsShape<NT, GLU>::BYTES, configured);
    if (ce != cudaSuccess) return ce;
    if (SPLIT) return launch_dependent(mx4_mid_kernel<NT, GLU, SPLIT>, dim3(grid), dim3(MS_THREADS), MsShape<NT, GLU>::BYTES, st, m.x, m.w, m.up, m.xs, m.ws, m.us, p, act);
    mx4_mid_kernel<NT, GLU, SPLIT><<<grid, MS_THREADS, MsShape<NT, GLU>::BYTES, st>>>(m.x, m.w, m.up, m.xs, m.ws, m.us, p, act);
    return cudaGetLastError();
}

// Row tiles at most, and the workspace that holds the pieces of bf16 rows.
static int64_t ms_tiles(int64_t T, int64_t groups, bool grouped, int rows)
{
    return grouped ? T / rows + (groups < T ? groups : T) : (T + rows - 1) / rows;
}
size_t mx4_mid_workspace(int64_t T, int64_t K, int64_t groups, bool grouped, int rows)
{
    return (size_t)ms_tiles(T, groups, grouped, rows) * (mx4_codes_bytes(MX4_TILE_ROWS, K) + mx4_scales_bytes(MX4_TILE_ROWS, K));
}

// rows of a tile: bf16 rows 4, 8 or 10 (48, 96 or 128 pieces), 4-bit rows 32, 64 (one group that begins at row 0) or 128
dass_status mx4_mid_launch(const Mx4Args &q, int rows, void *workspace)
{
    const LinearArgs &a = q.a;
    const bool glu = q.up.codes != nullptr, split = q.x.codes == nullptr;
    const int nt = split ? (rows == 4 ? 48 : rows == 8 ? 96 : 128) : rows;
    const int64_t w_tiles = mx4_row_tiles(a.N);
    const Mx4Matrix &second = glu ? q.up : q.w;
    const int64_t tiles = ms_tiles(a.T, a.groups, a.offsets != nullptr, rows);
    Mx4Matrix x = q.x;
    if (split) {
        x.codes = static_cast<const uint8_t *>(workspace);
        x.scales = x.codes + tiles * mx4_codes_bytes(MX4_TILE_ROWS, a.K);
    }
    MsMaps m;
    if (!mx4_codes_map(&m.x, x.codes, split ? tiles : 1, split ? MX4_TILE_ROWS : a.T, a.K, nt) || !mx4_codes_map(&m.w, q.w.codes, a.groups, a.N, a.K, MS_COLS) ||
        !mx4_codes_map(&m.up, second.codes, a.groups, a.N, a.K, MS_COLS) || !mx4_scales_map(&m.xs, x.scales, split ? tiles : mx4_row_tiles(a.T), a.K) ||
        !mx4_scales_map(&m.ws, q.w.scales, a.groups * w_tiles, a.K) || !mx4_scales_map(&m.us, second.scales, a.groups * w_tiles, a.K))
        return DASS_ERR_CUDA;
    MsParams p;
    p.offsets = a.offsets;
    p.bias = static_cast<const uint16_t *>(a.bias); p.bias_up = static_cast<const uint16_t *>(a.bias_up);
    p.residual = static_cast<const uint16_t *>(a.residual);
    p.Y = static_cast<uint16_t *>(a.Y);
    p.ldr = a.ldr; p.ldy = a.ldy; p.T = a.T;
    p.N = (int)a.N; p.groups = a.groups;
    p.col_tiles = (int)((a.N + MS_COLS - 1) / MS_COLS);
    p.k_stages = (int)((a.K + MS_BK - 1) / MS_BK);
    p.w_tiles = (int)w_tiles;
    p.y_vec = rows_vec_ok(a.Y, a.ldy, true);
    p.r_vec = a.residual && rows_vec_ok(a.residual, a.ldr, true);
    p.align = split ? 1 : MX4_TILE_ROWS;
    p.rows = rows;
    p.timeouts = linear_timeouts();
    if (!p.timeouts) return DASS_ERR_CUDA;
    if (split) {
        if (tiles > 65535) return DASS_ERR_UNSUPPORTED;
        SplitArgs s{static_cast<const uint16_t *>(a.X), a.T, a.K, a.ldx, const_cast<uint8_t *>(x.codes), const_cast<uint8_t *>(x.scales), a.offsets, a.groups, rows};
        mx4_split_kernel<<<dim3((unsigned)((a.K + 1023) / 1024), (unsigned)tiles, (unsigned)rows), 128, 0, a.st>>>(s);
        if (cudaGetLastError() != cudaSuccess) return DASS_ERR_CUDA;
    }
    const int64_t items = (split ? tiles : mx4_row_tiles(a.T) + (a.offsets ? a.groups : 0)) * p.col_tiles;       // at most
    const int sms = device_sm_count();
    const int grid = (int)(items < sms ? items : sms);
    cudaError_t e;
    if (split) {
        if (glu) e = nt == 48 ? ms_launch<48, true, true>(m, p, a.act, grid, a.st) : nt == 96 ? ms_launch<96, true, true>(m, p, a.act, grid, a.st) : ms_launch<128, true, true>(m, p, a.act, grid, a.st);
        else e = nt == 48 ? ms_launch<48, false, true>(m, p, a.act, grid, a.st) : nt == 96 ? ms_launch<96, false, true>(m, p, a.act, grid, a.st) : ms_launch<128, false, true>(m, p, a.act, grid, a.st);
    } else {
        if (glu) e = nt == 32 ? ms_launch<32, true, false>(m, p, a.act, grid, a.st) : nt == 64 ? ms_launch<64, true, false>(m, p, a.act, grid, a.st) : ms_launch<128, true, false>(m, p, a.act, grid, a.st);
        else e = nt == 32 ? ms_launch<32, false, false>(m, p, a.act, grid, a.st) : nt == 64 ? ms_launch<64, false, false>(m, p, a.act, grid, a.st) : ms_launch<128, false, false>(m, p, a.act, grid, a.st);
    }
    return e == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

}  // namespace dass
