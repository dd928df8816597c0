// C ABI of the matrix product with an epilogue: validation and dispatch.  See include/dass.h.
#include <atomic>

#include "linear_common.cuh"

namespace dass {

dass_status linear_f32_launch(const LinearArgs &a);        // linear_f32.cu
dass_status linear_tc_launch(const LinearArgs &a, int columns);         // linear_tc.cu
dass_status linear_few_launch(const LinearArgs &a, int eights, int split);        // linear_few.cu
dass_status linear_mid_launch(const LinearArgs &a, int rows, int split);        // linear_mid.cu
int device_sm_count();                                     // dass_abi.cu

struct LinPlan { int path, tile, split; };                 // path 1: few (rows in eights), 2: tc (columns), 3: mid (rows)


// Which kernel a bf16 product takes.
//
// linear_few.cu starts fastest (3.2 us) and slows with the rows: it takes what is small.  Between the other two the choice
// is the shorter estimate, in microseconds, of a model fitted to measurements on a B200 (rows 1 .. 8192, K 64 .. 14336, N 33
// .. 14336, dense and per expert).  On 40 random dense shapes the choice costs 3 % over the best kernel, tile and split on
// average (at worst 1.43 times), on 40 per-expert ones 5 % (1.64).  It goes by the rows of an average expert, since the host
// does not know the offsets: where one expert holds half of the rows it stays within 12 % of the best:
//   linear_tc.cu, n = 256 or 128 accumulator columns: a start, and per round of the CTA pairs the k-blocks, but no less
//   than an epilogue;
//   linear_mid.cu, nt rows a tile, split s: a start, a little for the split, and per wave of blocks the k-blocks (slower the
//   more SMs read at once) and the epilogue.
// Neither is faster than its weights, at 4.8 and 6.3 GB per ms.
static double lin_rounds_up(double x) { return (double)(int64_t)(x + 0.999999); }

LinPlan lin_plan(const LinearArgs &a)
{
    const bool glu = a.W_up != nullptr;
    const int64_t groups = lin_active_groups(a);
    const int64_t rows = a.offsets ? (a.T + a.groups - 1) / a.groups : a.T;           // of an average group
    const int64_t weights = a.N * a.K * (glu ? 2 : 1) * groups;
    const double products = (double)a.T * a.N * a.K * (glu ? 2 : 1);
    if (weights <= 8 << 20 && (products <= 32e6 || (rows <= 16 && a.T <= 64))) {
        // Weights that stay in L2 anyway are better read once per 8 rows, by more blocks (27 rows, 411 x 472: 3.9 us,
        // against 5.2 with all rows in a block).  A cluster costs more to place than a block, so k is split only where
        // most SMs would have none.
        const int64_t want = lin_rows_wanted(a), blocks = (a.N + 15) / 16 * groups;
        const int nt = want <= 8 || weights <= 2 << 20 ? 1 : want <= 16 || weights <= 4 << 20 ? 2 : 4;
        int split = 1;
        while (split < 8 && blocks * split < device_sm_count() && a.K >= 768 * split) split *= 2;
        if (blocks * (a.offsets ? 1 : (a.T + 8 * nt - 1) / (8 * nt)) <= 1024) return {1, nt, split};
    }
    const double sms = device_sm_count(), kb = (double)((a.K + 63) / 64);
    auto row_tiles = [&](int64_t r) {                                                  // about: a group's last tile is half full
        if (!a.offsets) return (double)((a.T + r - 1) / r);
        const double t = (double)a.T / r + 0.5 * groups;
        return t > groups ? t : (double)groups;
    };
    LinPlan best{2, 256, 1};
    double least = 1e30;
    for (int n = 256; n >= 128; n /= 2) {
        const double cols = (double)((a.N + (glu ? n / 2 : n) - 1) / (glu ? n / 2 : n));
        const double main = kb * (n == 256 ? 0.30 : 0.19), end = n == 256 ? 3.2 : 2.5;
        double t = lin_rounds_up(row_tiles(256) * cols / (sms / 2)) * ((main > end ? main : end) + 0.8);
        const double bytes = weights * 2.0 / 4.8e6;
        t = (n == 256 ? 7.0 : 6.5) + (t > bytes ? t : bytes);
        if (t < least) { least = t; best = {2, n, 1}; }
    }
    if (rows > 1024) return best;
    const double cols = (double)((a.N + 127) / 128);
    static const struct { int nt; double kb, end, split; } PLAIN[4] = {{16, 0.20, 1.5, 0.1}, {32, 0.20, 2.0, 0.1}, {64, 0.21, 3.1, 0.2}, {128, 0.22, 4.9, 0.3}},
                                                          GATED[4] = {{16, 0.29, 2.1, 0.5}, {32, 0.30, 2.7, 0.5}, {64, 0.31, 4.2, 0.7}, {128, 0.35, 6.7, 1.3}};
    for (int i = 0; i < 4; ++i) {
        const auto &m = glu ? GATED[i] : PLAIN[i];
        if (rows > (a.offsets ? 2 : 8) * m.nt) continue;
        // per expert the loads are uneven: tiles below twice the average leave second tiles, that read the weights again
        const double bytes = weights * 2.0 / 6.3e6 * (a.offsets && m.nt < lin_rows_wanted(a) / 2 ? 1.2 : 1.0);
        for (int s = 1; s <= 8 && (s == 1 || kb >= 4 * s); s *= 2) {
            const double blocks = row_tiles(m.nt) * cols * s, full = blocks / (s > 2 ? 0.8 * sms : sms);   // clusters do not fill every SM
            double t = (full > 1.0 ? full : 1.0) * (kb / s * (m.kb + 0.12 * (full > 1.0 ? 1.0 : full)) + m.end);
            t = 3.3 + (s == 8 ? 3 : s == 4 ? 2 : s == 2 ? 1 : 0) * m.split + (t > bytes ? t : bytes);
            if (t < least) { least = t; best = {3, m.nt, s}; }
        }
    }
    return best;
}

// Bounded waits that ran out on this device, counted and never cleared: a query that cleared it could lose what a kernel on
// another stream records meanwhile.  dass_linear_status remembers how many have been reported.
__device__ int g_linear_timeouts = 0;

// Address of the count on the current device (looked up once per device).
int *linear_timeouts()
{
    static std::atomic<int *> cached[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return nullptr;
    int *p = dev < 64 ? cached[dev].load(std::memory_order_relaxed) : nullptr;
    if (p) return p;
    void *addr = nullptr;
    if (cudaGetSymbolAddress(&addr, g_linear_timeouts) != cudaSuccess) return nullptr;
    p = static_cast<int *>(addr);
    if (dev < 64) cached[dev].store(p, std::memory_order_relaxed);
    return p;
}

}  // namespace dass

using namespace dass;

extern "C" {

dass_status dass_linear(const void *X, int64_t T, int64_t K, int64_t ldx, const void *W, const void *W_up, int64_t N, int64_t ldw,
                        int64_t group_stride, const void *bias, const void *bias_up, dass_act act, const void *residual, int64_t ldr,
                        void *Y, int64_t ldy, dass_dtype dt, const int32_t *offsets, int64_t groups, void *cuda_stream)
{
    if (dt != DASS_BF16 && dt != DASS_F32) return DASS_ERR_DTYPE;
    if (act != DASS_ACT_SILU && act != DASS_ACT_GELU_TANH && act != DASS_ACT_RELU && act != DASS_ACT_NONE) return DASS_ERR_DTYPE;
    if (!W || (T > 0 && (!X || !Y)) || (bias_up && !W_up)) return DASS_ERR_NULL;
    if (T < 0 || K < 1 || N < 1 || ldx < K || ldw < K || ldy < N || (residual && ldr < N)) return DASS_ERR_SHAPE;
    if (groups < 1 || (!offsets && groups != 1) || (groups > 1 && group_stride < (N - 1) * ldw + K)) return DASS_ERR_SHAPE;
    const bool bf16 = dt == DASS_BF16;
    const int64_t unit = bf16 ? 8 : 4;
    auto whole = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; };
    if (!whole(X) || !whole(W) || !whole(W_up) || ldx % unit || ldw % unit || (groups > 1 && group_stride % unit)) return DASS_ERR_ALIGN;
    if (!elem_aligned(bias, bf16) || !elem_aligned(bias_up, bf16) || !elem_aligned(residual, bf16) || !elem_aligned(Y, bf16) ||
        !elem_aligned(offsets, false))
        return DASS_ERR_ALIGN;
    const int64_t lim = 0x7fffffffll - 512;                // 32-bit tile coordinates
    const int64_t most_rows = 1ll << 28;                   // so are sums of tile counts, whatever the offsets hold
    if (T > most_rows || K > lim || N > lim || groups > LIN_MAX_GROUPS) return DASS_ERR_UNSUPPORTED;
    if (T == 0) return DASS_OK;

    LinearArgs a{};
    a.X = X; a.T = T; a.K = K; a.ldx = ldx;
    a.W = W; a.W_up = W_up; a.N = N; a.ldw = ldw; a.group_stride = groups > 1 ? group_stride : 0;
    a.bias = bias; a.bias_up = bias_up; a.residual = residual; a.ldr = ldr;
    a.Y = Y; a.ldy = ldy; a.offsets = offsets; a.groups = (int)groups; a.act = (int)act; a.bf16 = bf16;
    a.st = static_cast<cudaStream_t>(cuda_stream);
    DASS_BOUNDS_SCOPE(bs);
    DASS_BOUNDS_ADD(bs, X, ((size_t)(T - 1) * ldx + K) * (bf16 ? 2 : 4));
    DASS_BOUNDS_ADD(bs, W, ((size_t)(groups - 1) * a.group_stride + (size_t)(N - 1) * ldw + K) * (bf16 ? 2 : 4));
    DASS_BOUNDS_ADD(bs, W_up, ((size_t)(groups - 1) * a.group_stride + (size_t)(N - 1) * ldw + K) * (bf16 ? 2 : 4));
    DASS_BOUNDS_ADD(bs, bias, (size_t)groups * N * (bf16 ? 2 : 4));
    DASS_BOUNDS_ADD(bs, bias_up, (size_t)groups * N * (bf16 ? 2 : 4));
    DASS_BOUNDS_ADD(bs, residual, ((size_t)(T - 1) * ldr + N) * (bf16 ? 2 : 4));
    DASS_BOUNDS_ADD(bs, Y, ((size_t)(T - 1) * ldy + N) * (bf16 ? 2 : 4));
    DASS_BOUNDS_ADD(bs, offsets, (size_t)(groups + 1) * 4);
    DASS_BOUNDS_COMMIT(bs, a.st);
    if (!bf16) return linear_f32_launch(a);
    const LinPlan plan = lin_plan(a);
    return plan.path == 1 ? linear_few_launch(a, plan.tile, plan.split) : plan.path == 3 ? linear_mid_launch(a, plan.tile, plan.split) : linear_tc_launch(a, plan.tile);
}

dass_status dass_linear_status(void *cuda_stream)
{
    static std::atomic<int> reported[64];
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    int *word = linear_timeouts();
    int count = 0, dev = 0;
    if (!word || cudaGetDevice(&dev) != cudaSuccess ||
        cudaMemcpyAsync(&count, word, sizeof(int), cudaMemcpyDeviceToHost, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess)
        return DASS_ERR_CUDA;
    if (dev >= 64) return count ? DASS_ERR_TIMEOUT : DASS_OK;          // not remembered past 64 devices: reported every time
    // the remembered count only grows, whichever of several queries comes first (differences: the count may wrap)
    int before = reported[dev].load();
    while (count - before > 0 && !reported[dev].compare_exchange_weak(before, count)) {}
    return count - before > 0 ? DASS_ERR_TIMEOUT : DASS_OK;
}

}  // extern "C"
