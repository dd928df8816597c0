// C ABI of the matrix product with 4-bit weights: validation and dispatch.  See include/dass.h.
#include "mx4_linear.cuh"

namespace dass {

dass_status mx4_few_launch(const Mx4Args &p, int eights, int sixteens, int split);     // mx4_few.cu
dass_status mx4_tc_launch(const Mx4Args &p, int columns);                              // mx4_tc.cu
dass_status mx4_mid_launch(const Mx4Args &p, int rows, void *workspace);               // mx4_mid.cu
size_t mx4_mid_workspace(int64_t T, int64_t K, int64_t groups, bool grouped, int rows);
dass_status mx4_wide_launch(const Mx4Args &p, int rows);                               // mx4_wide.cu
int device_sm_count();                                                                 // dass_abi.cu

enum Mx4Path { MX4_FEW, MX4_MID, MX4_TC, MX4_WIDE };
struct Mx4Plan { Mx4Path path; int tile, sixteens, split; };     // few: rows in eights, weight rows in sixteens, split of k; mid, wide: rows; tc: columns
struct Mx4Sizes { int64_t T, K, N, groups; bool grouped, glu, quantized; };

// Which kernel a product takes: the shortest estimate, in microseconds, of a model fitted to measurements on a B200 (rows 1 ..
// 4096, K 64 .. 14336, N 33 .. 28672, dense and per expert): on 160 such shapes, 110 of them random, the choice costs 3.5 % over
// the best kernel, tile and split on average.  Of the three worst, 1.95 and 1.72 times, two have a k below 300; 1.64 times is
// 775 uneven rows of 5 experts at k = 2488, which take tiles of 64 rows where 128 are best; 17 more are 1.2 to 1.25 or less
// (few rows at any k, where a split or a tile less would do, and gated 4-bit rows of a short k).  Every kernel has a start, then
//   mx4_few.cu    decodes every weight once per 8, 16 or 32 rows, at 5400, 4200 or 2300 (gated, bf16 rows: 1600) weights a ns;
//   mx4_mid.cu    works off stages of 256 k, one item of 128 columns (of each matrix) to an SM at a time, no faster than
//                 5.8 TB/s of weights; bf16 rows are split first, and 4, 8 or 10 of them make a tile;
//   mx4_tc.cu     the same with tiles of 256 rows and 256 (gated: 128) or 128 columns to a CTA pair;
//   mx4_wide.cu   slabs of 64 k, tiles of 64, 128 or 256 rows and 256 columns to a CTA pair.
// It goes by the rows of an average expert, since the host does not know the offsets, and has no term for uneven loads but half a
// tile a group.
static double mx4_rounds(double items, double at_a_time) { return items <= at_a_time ? 1.0 : (double)(int64_t)(items / at_a_time + 0.999); }

static Mx4Plan mx4_plan(const Mx4Sizes &z)
{
    const double sms = device_sm_count(), m = z.glu ? 2.0 : 1.0;
    const double groups = z.grouped ? (double)(z.groups < z.T ? z.groups : z.T) : 1.0;
    const double rows = (double)z.T / groups;                                          // of an average group
    const double weights = m * groups * (double)z.N * (double)z.K, bytes = weights * 0.53125 / 5.8e6;
    // row tiles of `r` rows: a group's loads are uneven, and its last tile is half full
    auto tiles = [&](double r, double extra) { const double t = z.T / r + (z.grouped ? extra * groups : 0.999); return z.grouped ? (t > groups ? t : groups) : (double)(int64_t)t; };
    Mx4Plan best{MX4_FEW, 1, 1, 1};
    double least = 1e30;
    auto take = [&](double t, const Mx4Plan &p) { if (t < least) { least = t; best = p; } };

    if (rows <= 512) {
        const double rate[3] = {5.4e3, 4.2e3, z.glu && !z.quantized ? 1.6e3 : 2.3e3};      // weights a us, in thousands
        for (int i = 0; i < 3; ++i) {
            const int nt = 1 << i, mt = nt == 1 && weights > 8e6 ? 2 : 1;
            const double blocks = groups * (double)((z.N + 16 * mt - 1) / (16 * mt));
            int split = 1;
            while (split < 8 && blocks * split * 1.3 < sms && z.K >= 1024 * split) split *= 2;
            const double passes = tiles(8.0 * nt, 0.5) / groups, waves = blocks * passes * split / (2.0 * sms);
            take(3.0 + 0.35 * nt + (waves > 1.0 ? waves - 1.0 : 0.0) * (0.6 + 0.5 * nt) + passes * weights / (rate[i] * 1e3), {MX4_FEW, nt, mt, split});
        }
    }
    const double stages = (double)((z.K + 255) / 256), slabs = (double)((z.K + 63) / 64);
    if (z.quantized) {
        for (int r = 32; r <= 128; r *= 2) {
            if (r < 128 && (z.grouped || z.T > r)) continue;
            const double items = tiles(128.0, 1.0) * (double)((z.N + 127) / 128);
            const double t = mx4_rounds(items, sms) * (stages * (z.glu ? 0.38 + 0.001 * r : 0.22 + 0.0005 * r) + 0.8 + 0.025 * (rows < r ? rows : r));
            take(4.5 + (t > bytes ? t : bytes), {MX4_MID, r, 0, 0});
        }
        for (int c = 256; c >= 128; c /= 2) {
            if (z.glu && c == 128) continue;
            const double items = tiles(256.0, 1.0) * (double)((z.N + (z.glu ? 127 : c - 1)) / (z.glu ? 128 : c));
            const double t = mx4_rounds(items, sms / 2) * (stages * (c == 256 ? 0.38 : 0.21) + 1.5);
            take((c == 256 ? 7.0 : 6.5) + (t > bytes ? t : bytes), {MX4_TC, c, 0, 0});
        }
        return best;
    }
    for (int r : {4, 8, 10}) {
        const double row_tiles = tiles((double)r, 0.5);
        if (rows > 12.0 * r || row_tiles > 8192.0) continue;
        const double items = row_tiles * (double)((z.N + 127) / 128);
        const double stage = (z.glu ? 0.36 : 0.22) + 0.0004 * 12 * r;
        const double t = mx4_rounds(items, sms) * (stages * stage + 0.5), again = bytes * (0.75 + 0.25 * row_tiles / groups);
        take(9.5 + (t > again ? t : again), {MX4_MID, r, 0, 0});
    }
    for (int r = 64; r <= 256; r *= 2) {
        if (z.glu && r == 256) continue;
        const double items = tiles((double)r, 0.5) * (double)((z.N + 255) / 256);
        const double t = mx4_rounds(items, sms / 2) * (slabs * (z.glu ? (r == 64 ? 0.40 : 0.48) : r == 256 ? 0.36 : 0.29) + 0.01 * r);
        take(6.0 + (t > bytes ? t : bytes), {MX4_WIDE, r, 0, 0});
    }
    return best;
}
static size_t mx4_workspace(const Mx4Sizes &z, const Mx4Plan &p)
{
    return p.path == MX4_MID && !z.quantized ? mx4_mid_workspace(z.T, z.K, z.groups, z.grouped, p.tile) : 0;
}
static bool mx4_too_large(int64_t T, int64_t K, int64_t N, int64_t groups)
{
    const int64_t lim = 0x7fffffffll - 512;                // 32-bit tile coordinates
    const int64_t most_rows = 1ll << 26;                   // so are sums of the counts of 64-row tiles, whatever the offsets hold
    return T > most_rows || K > lim || N > lim || groups > LIN_MAX_GROUPS;
}

}  // namespace dass

using namespace dass;

extern "C" {

dass_status dass_linear_mx4_workspace_bytes(int64_t T, int64_t K, int64_t N, int64_t groups, int has_offsets, int has_up, int x_in_4_bits, size_t *bytes)
{
    if (!bytes) return DASS_ERR_NULL;
    if (T < 0 || K < 1 || N < 1 || groups < 1 || (!has_offsets && groups != 1)) return DASS_ERR_SHAPE;
    if (mx4_too_large(T, K, N, groups)) return DASS_ERR_UNSUPPORTED;
    const Mx4Sizes z{T, K, N, groups, has_offsets != 0, has_up != 0, x_in_4_bits != 0};
    *bytes = T ? mx4_workspace(z, mx4_plan(z)) : 0;
    return DASS_OK;
}

dass_status dass_linear_mx4_plan(int64_t T, int64_t K, int64_t N, int64_t groups, int has_offsets, int has_up, int x_in_4_bits, int32_t *plan)
{
    if (!plan) return DASS_ERR_NULL;
    if (T < 1 || K < 1 || N < 1 || groups < 1 || (!has_offsets && groups != 1)) return DASS_ERR_SHAPE;
    if (mx4_too_large(T, K, N, groups)) return DASS_ERR_UNSUPPORTED;
    const Mx4Plan p = mx4_plan(Mx4Sizes{T, K, N, groups, has_offsets != 0, has_up != 0, x_in_4_bits != 0});
    const bool few = p.path == MX4_FEW;
    plan[0] = p.path;
    plan[1] = p.tile;
    plan[2] = few ? p.sixteens : 0;
    plan[3] = few ? p.split : 0;
    plan[4] = few ? mx4_few_warps(K, p.tile, p.split) : 0;
    return DASS_OK;
}

dass_status dass_linear_mx4(const void *X, int64_t ldx, const uint8_t *x_codes, const uint8_t *x_scales, int64_t T, int64_t K,
                            const uint8_t *w_codes, const uint8_t *w_scales, const uint8_t *up_codes, const uint8_t *up_scales, int64_t N,
                            const void *bias, const void *bias_up, dass_act act, const void *residual, int64_t ldr,
                            void *Y, int64_t ldy, const int32_t *offsets, int64_t groups, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    if (act != DASS_ACT_SILU && act != DASS_ACT_GELU_TANH && act != DASS_ACT_RELU && act != DASS_ACT_NONE) return DASS_ERR_DTYPE;
    if (!w_codes || !w_scales || !up_codes != !up_scales || !x_codes != !x_scales || (bias_up && !up_codes)) return DASS_ERR_NULL;
    if (T > 0 && ((!X && !x_codes) || !Y)) return DASS_ERR_NULL;
    if (X && x_codes) return DASS_ERR_UNSUPPORTED;
    if (T < 0 || K < 1 || N < 1 || (X && ldx < K) || ldy < N || (residual && ldr < N)) return DASS_ERR_SHAPE;
    if (groups < 1 || (!offsets && groups != 1)) return DASS_ERR_SHAPE;
    auto whole = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; };
    if (!whole(X) || !whole(x_codes) || !whole(x_scales) || !whole(w_codes) || !whole(w_scales) || !whole(up_codes) || !whole(up_scales) ||
        !whole(workspace) || (X && ldx % 8))
        return DASS_ERR_ALIGN;
    if (!elem_aligned(bias, true) || !elem_aligned(bias_up, true) || !elem_aligned(residual, true) || !elem_aligned(Y, true) ||
        !elem_aligned(offsets, false))
        return DASS_ERR_ALIGN;
    if (mx4_too_large(T, K, N, groups)) return DASS_ERR_UNSUPPORTED;
    if (T == 0) return DASS_OK;
    const Mx4Sizes z{T, K, N, groups, offsets != nullptr, up_codes != nullptr, x_codes != nullptr};
    const Mx4Plan plan = mx4_plan(z);
    const size_t need = mx4_workspace(z, plan);
    if (need && (!workspace || workspace_bytes < need)) return DASS_ERR_WORKSPACE;

    Mx4Args p{};
    p.a.X = X; p.a.T = T; p.a.K = K; p.a.ldx = ldx; p.a.N = N;
    p.a.bias = bias; p.a.bias_up = bias_up; p.a.residual = residual; p.a.ldr = ldr;
    p.a.Y = Y; p.a.ldy = ldy; p.a.offsets = offsets; p.a.groups = (int)groups; p.a.act = (int)act; p.a.bf16 = true;
    p.a.st = static_cast<cudaStream_t>(cuda_stream);
    p.x = {x_codes, x_scales}; p.w = {w_codes, w_scales}; p.up = {up_codes, up_scales};
    DASS_BOUNDS_SCOPE(bs);
    DASS_BOUNDS_ADD(bs, X, ((size_t)(T - 1) * ldx + K) * 2);
    DASS_BOUNDS_ADD(bs, x_codes, mx4_codes_bytes(T, K));
    DASS_BOUNDS_ADD(bs, x_scales, mx4_scales_bytes(T, K));
    DASS_BOUNDS_ADD(bs, w_codes, (size_t)groups * mx4_codes_bytes(N, K));
    DASS_BOUNDS_ADD(bs, w_scales, (size_t)groups * mx4_scales_bytes(N, K));
    DASS_BOUNDS_ADD(bs, up_codes, (size_t)groups * mx4_codes_bytes(N, K));
    DASS_BOUNDS_ADD(bs, up_scales, (size_t)groups * mx4_scales_bytes(N, K));
    DASS_BOUNDS_ADD(bs, bias, (size_t)groups * N * 2);
    DASS_BOUNDS_ADD(bs, bias_up, (size_t)groups * N * 2);
    DASS_BOUNDS_ADD(bs, residual, ((size_t)(T - 1) * ldr + N) * 2);
    DASS_BOUNDS_ADD(bs, Y, ((size_t)(T - 1) * ldy + N) * 2);
    DASS_BOUNDS_ADD(bs, offsets, (size_t)(groups + 1) * 4);
    DASS_BOUNDS_ADD(bs, workspace, need);
    DASS_BOUNDS_COMMIT(bs, p.a.st);
    switch (plan.path) {
    case MX4_FEW: return mx4_few_launch(p, plan.tile, plan.sixteens, plan.split);
    case MX4_MID: return mx4_mid_launch(p, plan.tile, workspace);
    case MX4_TC: return mx4_tc_launch(p, plan.tile);
    default: return mx4_wide_launch(p, plan.tile);
    }
}

}  // extern "C"
