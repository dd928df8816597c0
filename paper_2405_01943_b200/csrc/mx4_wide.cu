// dass_linear_mx4 for bf16 rows, more of them than mx4_few.cu takes: Y = act(X W^T + b) [* (X W_up^T + b_up)] + R with W in 4
// bits, on the bf16 tensor cores.
//
// The weights are decoded once per tile, straight into tensor memory: they are the left operand, M = 256 weight rows to a
// CTA pair (tcgen05.mma.cta_group::2), 128 lanes of TMEM to each CTA, and a thread that decodes a row's codes in registers
// stores them to that row's lane (tcgen05.st).  No decoded weight passes through shared memory, whose bandwidth the right
// operand needs: N = NT rows of X, half of them loaded by each CTA.
//   warp 0        TMA of X: slabs of 64 k;             warp 2  TMA of codes and scale tiles: stages of 256 k
//   warp 1        TMEM, MMAs (leader)
//   warps 4..19   decoding: a warpgroup has the 128 rows; of the four one takes a block of 32 k of every other slab or, in
//                 the GLU form, a block of one matrix of every slab
//   warps 20..27  epilogue: a TMEM lane is a column of Y, a thread has one column of half of the tile's rows
// The accumulator (NT columns, in the GLU form NT of each product) leaves TMEM room for a ring of decoded slabs and for no
// second accumulator.  So the epilogue has the residual in shared memory before the accumulator is complete, turns it into
// bf16 results there, hands it back, and stores under the next tile's products.
// A decoded slab takes 300 cycles of the integer pipe and its products 512 at NT = 256, so those bound: 8192^3 680 to 690 us (1.6
// PFLOP/s, bf16 weights in linear_tc.cu 868), 2048 x 4096 x 11008 121 us.  In the GLU form two matrices are decoded for the
// same 512 cycles, at NT = 128, and the decoding bounds: 2048 x 4096 x 14336 415 to 480 us (1.0 to
// 1.16 PFLOP/s).  A residual costs 5 us of 119 at 2048 x 4096 x 11008, a bias nothing; in a loop of seconds, where power sets
// the clocks, 146 us without both and 152 with.
// Of the steps here, in us at 2048 x 4096 x 11008: two decoding warpgroups 246; a slab announced while the next is decoded,
// without a release at cluster scope 153; epilogue in short loops 134; barriers asked for ahead of their use 131; a stage's
// codes loaded at once 121.
//
// Every wait is bounded, as in linear_tc.cu.
#include "linear_tc.cuh"
#include "mx4_linear.cuh"
#include "tc_common.cuh"
#include "tc_pair.cuh"

namespace dass {

constexpr int MW_ROWS = 128;        // weight rows of a CTA
constexpr int MW_BK = 64;           // k of a slab
constexpr int MW_STAGE_K = 256;     // k of a stage of codes
constexpr int MW_THREADS = 896;
constexpr int MW_FIRST_DECODE = 4, MW_FIRST_EPILOGUE = 20;           // warps
constexpr uint32_t MW_CODES = MW_ROWS * MW_STAGE_K / 2, MW_SCALES = 2 * MX4_TILE_BYTES;
constexpr uint32_t MW_RING_COL = 256;                                 // TMEM columns from here on hold decoded slabs

template <int NT, bool GLU> struct MwShape {
    static constexpr int M = GLU ? 2 : 1;
    static constexpr uint32_t X_BYTES = NT / 2 * MW_BK * 2;           // a CTA's half of a slab of X
    static constexpr int X_STAGES = NT == 256 ? 6 : 8;
    static constexpr uint32_t W_BYTES = M * (MW_CODES + MW_SCALES);
    static constexpr int W_STAGES = 3;
    static constexpr int A_STAGES = 8 / M;                            // of 32 TMEM columns for each matrix
    static constexpr uint32_t W_AT = X_STAGES * X_BYTES;
    static constexpr int ROWS = NT / 2;                               // rows of Y of an epilogue warp, which has 32 columns
    static constexpr uint32_t BYTES = W_AT + W_STAGES * W_BYTES + 8 * ROWS * 64 + 1024 /* alignment slack */ + 512 /* barriers */ + MX4_TABLE_BYTES;
    static_assert(M * NT <= 256 && BYTES <= 227 * 1024 && X_BYTES % 1024 == 0 && (MW_CODES + MW_SCALES) % 1024 == 0, "");
};

struct MwParams {
    const int32_t *offsets;
    const uint16_t *bias, *bias_up, *residual;
    uint16_t *Y;
    int64_t ldr, ldy, T;
    int N, groups, col_tiles, slabs, w_tiles, y_vec, r_vec;
    int *timeouts;
};

// ------------------------------------------------------------------ PTX wrappers
__device__ __forceinline__ void tmem_st_16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                   "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
                   "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// left operand in TMEM (16-bit elements, two to a column)
__device__ __forceinline__ void umma_bf16_ts_pair(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "setp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
template <int REGS> __device__ __forceinline__ void regs_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS)); }
template <int REGS> __device__ __forceinline__ void regs_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS)); }
// The launch has 896 x 72 registers; the warpgroups' shares below add up to 128 x (40 + 4 x 64 + 2 x 104) = 64512, all of them.
constexpr int MW_REGS_LAUNCH = 72, MW_REGS_ISSUE = 40, MW_REGS_DECODE = 64, MW_REGS_EPILOGUE = 104;
static_assert(128 * (MW_REGS_ISSUE + 4 * MW_REGS_DECODE + 2 * MW_REGS_EPILOGUE) <= MW_THREADS * MW_REGS_LAUNCH, "");

// 32 codes of one block (16 bytes) as 16 bf16 pairs, in order.
__device__ __forceinline__ void mw_decode32(const uint4 &v, const Mx4Factor &f, bool two, uint32_t (&out)[16])
{
    const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t w[4];
        mx4_decode8(x[i], f, two, w);
        out[4 * i] = __byte_perm(w[0], w[1], 0x5410);
        out[4 * i + 1] = __byte_perm(w[2], w[3], 0x5410);
        out[4 * i + 2] = __byte_perm(w[0], w[1], 0x7632);
        out[4 * i + 3] = __byte_perm(w[2], w[3], 0x7632);
    }
}

template <int NT, bool GLU, int ACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(MW_THREADS, 1)
mx4_wide_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_up,
                const __grid_constant__ CUtensorMap map_ws, const __grid_constant__ CUtensorMap map_us, const MwParams p)
{
    using S = MwShape<NT, GLU>;
    constexpr int M = S::M, XS = S::X_STAGES, WS = S::W_STAGES, AS = S::A_STAGES;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;                 // swizzled tiles need 1024-byte alignment
    uint8_t *aligned = smem_raw + (base - raw);
    uint64_t *bars = reinterpret_cast<uint64_t *>(aligned + S::W_AT + WS * S::W_BYTES + 8 * S::ROWS * 64);
    const uint32_t x_full = smem_u32(bars), x_empty = x_full + 8 * XS;        // full: leader; empty: per CTA
    const uint32_t w_full = x_empty + 8 * XS, w_empty = w_full + 8 * WS;      // per CTA
    const uint32_t a_full = w_empty + 8 * WS, a_empty = a_full + 8 * AS;      // full: leader, both CTAs' warps arrive; empty: per CTA
    const uint32_t acc_full = a_empty + 8 * AS, acc_empty = acc_full + 8;     // full: per CTA; empty: leader
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 2 * (XS + WS + AS) + 2);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);
    int *table = reinterpret_cast<int *>(reinterpret_cast<uint8_t *>(bars) + 512);

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();                      // 0 = leader
    const int64_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (threadIdx.x == 96) {                                      // the descriptors' first fetch runs beside the set-up
        tma_prefetch_map(&map_w);
        tma_prefetch_map(&map_ws);
        if constexpr (GLU) { tma_prefetch_map(&map_up); tma_prefetch_map(&map_us); }
        tma_prefetch_map(&map_x);
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < XS; ++s) { mbar_init(x_full + 8 * s, 1); mbar_init(x_empty + 8 * s, 1); }
        for (int s = 0; s < WS; ++s) { mbar_init(w_full + 8 * s, 1); mbar_init(w_empty + 8 * s, 16); }
        for (int s = 0; s < AS; ++s) { mbar_init(a_full + 8 * s, 2 * 8 * M); mbar_init(a_empty + 8 * s, 1); }
        mbar_init(acc_full, 1);
        mbar_init(acc_empty, 2 * 8);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    mx4_count_tiles(table, p.offsets, p.groups, p.T, 1, NT, MW_THREADS);
    if (warp == 1) {
        tmem_alloc_pair(smem_u32(tmem_slot), 512);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) mx4_sum_tiles(table, p.groups);
    __syncthreads();
    cluster_sync_all();            // both CTAs' barriers are initialised and both TMEM allocations exist
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    const int64_t items = (int64_t)table[p.groups] * p.col_tiles;
    const int w_stages = (p.slabs + 3) / 4;
    Mx4Item it;
    bool ok = true;

    if (warp < MW_FIRST_DECODE) {
        regs_dec<MW_REGS_ISSUE>();
        if (warp == 0) {
            // -------------------------------------------------------- TMA of X (one per CTA)
            uint32_t stage = 0, phase = 0;
            const uint32_t leader_full = map_to_cta(x_full, 0);
            const uint64_t pol = l2_policy_evict_last();
            for (int64_t idx = pair; ok && mx4_item(table, p.groups, 1, NT, p.col_tiles, 2 * MW_ROWS, idx, it); idx += pairs) {
                const int row = it.row + (int)rank * (NT / 2);
                for (int s = 0; s < p.slabs; ++s) {
                    if (!warp_wait(x_empty + 8 * stage, phase ^ 1u, abort_flag)) { ok = false; break; }
                    if (elect_one()) {
                        if (rank == 0) mbar_arrive_expect_tx(x_full + 8 * stage, 2 * S::X_BYTES);   // both CTAs' bytes
                        tma_load_2d_pair(base + stage * S::X_BYTES, &map_x, leader_full + 8 * stage, s * MW_BK, row, pol);
                    }
                    __syncwarp();
                    if (++stage == XS) { stage = 0; phase ^= 1u; }
                }
            }
        } else if (warp == 2) {
            // -------------------------------------------------------- TMA of codes and scales (one per CTA)
            uint32_t stage = 0, phase = 0;
            const uint64_t pol = l2_policy_evict_last();
            for (int64_t idx = pair; ok && mx4_item(table, p.groups, 1, NT, p.col_tiles, 2 * MW_ROWS, idx, it); idx += pairs) {
                const int row = it.col + (int)rank * MW_ROWS;
                const int of = row / MX4_TILE_ROWS, tile = it.g * p.w_tiles + (of < p.w_tiles ? of : p.w_tiles - 1);   // absent rows are not stored
                for (int s = 0; s < w_stages; ++s) {
                    if (!warp_wait(w_empty + 8 * stage, phase ^ 1u, abort_flag)) { ok = false; break; }
                    const uint32_t at = base + S::W_AT + stage * S::W_BYTES, full = w_full + 8 * stage;
                    if (elect_one()) {
                        mbar_arrive_expect_tx(full, S::W_BYTES);
                        tma_load_3d_hint(at, &map_w, full, s * (MW_STAGE_K / 2), row, it.g, pol);
                        tma_load_3d_hint(at + MW_CODES, &map_ws, full, 0, 2 * s, tile, pol);
                        if constexpr (GLU) {
                            tma_load_3d_hint(at + MW_CODES + MW_SCALES, &map_up, full, s * (MW_STAGE_K / 2), row, it.g, pol);
                            tma_load_3d_hint(at + 2 * MW_CODES + MW_SCALES, &map_us, full, 0, 2 * s, tile, pol);
                        }
                    }
                    __syncwarp();
                    if (++stage == WS) { stage = 0; phase ^= 1u; }
                }
            }
        } else if (warp == 1 && rank == 0) {
            // -------------------------------------------------------- MMA issuer (leader CTA only)
            constexpr uint32_t idesc = idesc_bf16_f32(2 * MW_ROWS, NT);
            Mx4Ring x, r;                                         // of X and of the decoded slabs
            uint32_t tile = 0;
            bool ready = false;
            for (int64_t idx = pair; ok && idx < items; idx += pairs, ++tile) {
                if (!warp_wait(acc_empty, (tile & 1u) ^ 1u, abort_flag)) { ok = false; break; }
                for (int s = 0; s < p.slabs; ++s) {
                    if (!ready && (!warp_wait(x_full + 8 * x.stage, x.phase, abort_flag) || !warp_wait(a_full + 8 * r.stage, r.phase, abort_flag))) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t xs = x.stage, as = r.stage;
                    x.step(XS);
                    r.step(AS);
                    const bool next_x = mbar_test(x_full + 8 * x.stage, x.phase), next_a = mbar_test(a_full + 8 * r.stage, r.phase);
                    if (elect_one()) {
                        const uint64_t db = smem_desc_sw128(base + xs * S::X_BYTES);
                        const uint32_t ring = tmem_base + MW_RING_COL + as * (32 * M);
#pragma unroll
                        for (int m = 0; m < M; ++m)
#pragma unroll
                            for (int k = 0; k < MW_BK / 16; ++k)
                                umma_bf16_ts_pair(tmem_base + m * NT, ring + 32 * m + 8 * k, db + 2 * k, idesc, (s > 0 || k > 0) ? 1u : 0u);
                        umma_commit_pair(x_empty + 8 * xs, (uint16_t)3);
                        umma_commit_pair(a_empty + 8 * as, (uint16_t)3);
                        if (s + 1 == p.slabs) umma_commit_pair(acc_full, (uint16_t)3);
                    }
                    ready = __all_sync(FULL_MASK, next_x && next_a);
                }
            }
        }
    } else if (warp < MW_FIRST_EPILOGUE) {
        // ------------------------------------------------------------ decoding: this thread's weight row
        regs_dec<MW_REGS_DECODE>();
        const int group = (warp - MW_FIRST_DECODE) >> 2;          // block of 32 k: group & 1; matrix (GLU) or parity of the slab: group >> 1
        const int block = group & 1, second = group >> 1;
        const int r = (warp & 3) * 32 + lane;
        const uint32_t lane_addr = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + MW_RING_COL;
        const uint32_t leader_full = map_to_cta(a_full, 0);
        const int chunk = r & 7;                                  // of the swizzle
        constexpr int OFF = GLU ? 1 : 2;                          // slabs from one of this warp's units to the next
        Mx4Ring wr;
        uint32_t as = 0, ap = 0;                                  // place of a stage's first slab in the ring of decoded ones
        int stored = -1;                                          // the slab whose store has not been announced: done one unit
        auto announce = [&]() {                                   // later, so that the next one is decoded meanwhile
            if (stored < 0) return;
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_tmem(leader_full + 8 * stored);
            stored = -1;
        };
        for (int64_t idx = pair; ok && idx < items; idx += pairs) {
            for (int s4 = 0; ok && s4 < w_stages; ++s4) {
                if (!warp_wait(w_full + 8 * wr.stage, wr.phase, abort_flag)) { ok = false; break; }
                const uint8_t *codes = aligned + S::W_AT + wr.stage * S::W_BYTES + (GLU ? second * (MW_CODES + MW_SCALES) : 0u);
                const uint8_t *scales = codes + MW_CODES + (r & 31) * 16 + (r >> 5) * 4;
                const uint32_t sw[2] = {*reinterpret_cast<const uint32_t *>(scales), *reinterpret_cast<const uint32_t *>(scales + MX4_TILE_BYTES)};
                const int n = p.slabs - 4 * s4 < 4 ? p.slabs - 4 * s4 : 4;                     // slabs of this stage
#pragma unroll 1
                for (int half = 0; half < (GLU ? 2 : 1); ++half) {
                    const int s0 = GLU ? 2 * half : second;       // two units, slabs s0 and s0 + OFF: 16 bytes of this row (a swizzled chunk) each
                    const uint4 c[2] = {*reinterpret_cast<const uint4 *>(codes + r * 128 + (((2 * s0 + block) ^ chunk) * 16)),
                                        *reinterpret_cast<const uint4 *>(codes + r * 128 + (((2 * (s0 + OFF) + block) ^ chunk) * 16))};
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int s = s0 + j * OFF;
                        if (s >= n) break;
                        const bool over = as + s >= AS;           // a stage's slabs may go round the ring
                        const uint32_t at = over ? as + s - AS : as + s, par = over ? ap ^ 1u : ap;
                        const bool free_now = mbar_test(a_empty + 8 * at, par ^ 1u);
                        const uint32_t e = ((GLU ? (half ? sw[1] : sw[0]) : sw[j]) >> (8 * (2 * (s & 1) + block))) & 255u;
                        const bool two = __any_sync(FULL_MASK, mx4_two(e));
                        uint32_t out[16];
                        mw_decode32(c[j], mx4_factor(e), two, out);
                        announce();
                        if (!__all_sync(FULL_MASK, free_now) && !warp_wait(a_empty + 8 * at, par ^ 1u, abort_flag)) { ok = false; break; }
                        tc_fence_after();
                        tmem_st_16(lane_addr + at * (32 * M) + (GLU ? second * 32 : 0) + block * 16, out);
                        stored = (int)at;
                    }
                    if (!ok) break;
                }
                // The stage goes back when its last codes are in TMEM: a load that has only been issued may still read the
                // memory when the next copy writes it.  The fence orders those reads before the copy's writes.
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (ok && lane == 0) mbar_arrive(w_empty + 8 * wr.stage);
                wr.step(WS);
                as += n;
                if (as >= AS) { as -= AS; ap ^= 1u; }
            }
            announce();
        }
    } else {
        // ------------------------------------------------------------ epilogue: this thread's column of Y
        regs_inc<MW_REGS_EPILOGUE>();
        constexpr int EPI = 256;                                 // threads
        lin_zero_outside<true>(p.offsets, p.groups, p.T, p.N, p.Y, p.ldy, p.y_vec != 0, (int64_t)blockIdx.x * EPI + threadIdx.x - (MW_THREADS - EPI),
                               (int64_t)gridDim.x * EPI);
        const int quad = warp & 3, half = (warp - MW_FIRST_EPILOGUE) >> 2;
        constexpr int ROWS = S::ROWS;
        const uint32_t lane_addr = tmem_base + ((uint32_t)(quad * 32) << 16) + half * ROWS;
        const uint32_t leader_acc_empty = map_to_cta(acc_empty, 0);
        uint16_t *block = reinterpret_cast<uint16_t *>(aligned + S::W_AT + WS * S::W_BYTES + (warp - MW_FIRST_EPILOGUE) * (ROWS * 64));
        uint32_t tile = 0;
        for (int64_t idx = pair; ok && mx4_item(table, p.groups, 1, NT, p.col_tiles, 2 * MW_ROWS, idx, it); idx += pairs, ++tile) {
            const int n0 = it.col + (int)rank * MW_ROWS + quad * 32, left = p.N - n0;
            const int64_t t0 = (int64_t)it.row + half * ROWS;
            const int rows = left <= 0 ? 0 : it.row_hi - t0 < ROWS ? (int)(it.row_hi - t0) : ROWS;   // <= 0: none
            const float b = p.bias && lane < left ? __uint_as_float((uint32_t)DASS_LD(p.bias + (int64_t)it.g * p.N + n0 + lane) << 16) : 0.f;
            const float bu = GLU && p.bias_up && lane < left ? __uint_as_float((uint32_t)DASS_LD(p.bias_up + (int64_t)it.g * p.N + n0 + lane) << 16) : 0.f;
            if (p.residual) mx4_block_in(block, p.residual + t0 * p.ldr + n0, p.ldr, p.r_vec, 0, rows, left);
            if (!warp_wait(acc_full, tile & 1u, abort_flag)) { ok = false; break; }
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < rows; c += 16) {
                uint32_t a[16], u[16];
                float y[16];
                tmem_ld_16(lane_addr + c, a);
                if constexpr (GLU) tmem_ld_16(lane_addr + NT + c, u);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    y[i] = lt_act<ACT>(__uint_as_float(a[i]) + b);
                    if constexpr (GLU) y[i] *= __uint_as_float(u[i]) + bu;
                }
                mx4_block_set(block, c, y, p.residual != nullptr);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_tmem(leader_acc_empty);   // release the accumulator to the leader's MMA warp
            mx4_block_out(block, p.Y + t0 * p.ldy + n0, p.ldy, p.y_vec, 0, rows, left);
        }
    }
    if (!ok && lane == 0) { *abort_flag = 1; atomicAdd(p.timeouts, 1); }

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
bool tc_make_map(CUtensorMap *map, const void *ptr, int64_t rows, int64_t cols, int64_t ld, int box_rows);   // calib_tc.cu

struct MwMaps { CUtensorMap x, w, up, ws, us; };

template <int NT, bool GLU, int ACT>
static cudaError_t mw_launch(const MwMaps &m, const MwParams &p, int grid, cudaStream_t st)
{
    static DeviceMask configured{0ull};               // per device
    const cudaError_t ce = ensure_dynamic_smem(mx4_wide_kernel<NT, GLU, ACT>, (int)MwShape<NT, GLU>::BYTES, configured);
    if (ce != cudaSuccess) return ce;
    // The warpgroups' shares are drawn on what the kernel is launched with: a build with fewer registers would wait for good.
    static std::atomic<int> registers{0};
    int have = registers.load(std::memory_order_relaxed);
    if (!have) {
        cudaFuncAttributes attr;
        const cudaError_t e = cudaFuncGetAttributes(&attr, mx4_wide_kernel<NT, GLU, ACT>);
        if (e != cudaSuccess) return e;
        registers.store(have = attr.numRegs, std::memory_order_relaxed);
    }
    if (have < MW_REGS_LAUNCH) return cudaErrorLaunchOutOfResources;
    mx4_wide_kernel<NT, GLU, ACT><<<grid, MW_THREADS, MwShape<NT, GLU>::BYTES, st>>>(m.x, m.w, m.up, m.ws, m.us, p);
    return cudaGetLastError();
}
template <int NT, bool GLU>
static cudaError_t mw_pick(int act, const MwMaps &m, const MwParams &p, int grid, cudaStream_t st)
{
    switch (act) {
    case DASS_ACT_SILU: return mw_launch<NT, GLU, DASS_ACT_SILU>(m, p, grid, st);
    case DASS_ACT_GELU_TANH: return mw_launch<NT, GLU, DASS_ACT_GELU_TANH>(m, p, grid, st);
    case DASS_ACT_RELU: return mw_launch<NT, GLU, DASS_ACT_RELU>(m, p, grid, st);
    default: return mw_launch<NT, GLU, DASS_ACT_NONE>(m, p, grid, st);
    }
}

// nt: rows of X per tile: 256 (without the GLU form), 128 or 64
dass_status mx4_wide_launch(const Mx4Args &q, int nt)
{
    const LinearArgs &a = q.a;
    const bool glu = q.up.codes != nullptr;
    const int64_t w_tiles = mx4_row_tiles(a.N);
    const Mx4Matrix &second = glu ? q.up : q.w;
    MwMaps m;
    if (!tc_make_map(&m.x, a.X, a.T, a.K, a.ldx, nt / 2) || !mx4_codes_map(&m.w, q.w.codes, a.groups, a.N, a.K, MW_ROWS) ||
        !mx4_codes_map(&m.up, second.codes, a.groups, a.N, a.K, MW_ROWS) || !mx4_scales_map(&m.ws, q.w.scales, a.groups * w_tiles, a.K) ||
        !mx4_scales_map(&m.us, second.scales, a.groups * w_tiles, a.K))
        return DASS_ERR_CUDA;
    MwParams p;
    p.offsets = a.offsets;
    p.bias = static_cast<const uint16_t *>(a.bias); p.bias_up = static_cast<const uint16_t *>(a.bias_up);
    p.residual = static_cast<const uint16_t *>(a.residual);
    p.Y = static_cast<uint16_t *>(a.Y);
    p.ldr = a.ldr; p.ldy = a.ldy; p.T = a.T;
    p.N = (int)a.N; p.groups = a.groups;
    p.col_tiles = (int)((a.N + 2 * MW_ROWS - 1) / (2 * MW_ROWS));
    p.slabs = (int)((a.K + MW_BK - 1) / MW_BK);
    p.w_tiles = (int)w_tiles;
    p.y_vec = rows_vec_ok(a.Y, a.ldy, true);
    p.r_vec = a.residual && rows_vec_ok(a.residual, a.ldr, true);
    p.timeouts = linear_timeouts();
    if (!p.timeouts) return DASS_ERR_CUDA;
    const int64_t items = ((a.T + nt - 1) / nt + (a.offsets ? a.groups : 0)) * p.col_tiles;   // at most
    const int pairs = device_sm_count() / 2;
    const int grid = 2 * (int)(items < pairs ? items : pairs);
    cudaError_t e;
    if (glu) e = nt == 128 ? mw_pick<128, true>(a.act, m, p, grid, a.st) : mw_pick<64, true>(a.act, m, p, grid, a.st);
    else e = nt == 256 ? mw_pick<256, false>(a.act, m, p, grid, a.st) : nt == 128 ? mw_pick<128, false>(a.act, m, p, grid, a.st) : mw_pick<64, false>(a.act, m, p, grid, a.st);
    return e == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

}  // namespace dass
