// Token rows sorted by expert and back: the order itself (a stable counting sort of the expert ids), the copy into it,
// the weighted sum out of it, and the gradients of both.
//
// The order: flat index f = t * k + j; expert e's rows are those f with id e, ascending.  The ids are cut into one run
// per block.  Pass 1 counts each run's ids per expert.  Pass 2 needs, for its own run, what the runs before it hold of
// every expert and what all runs hold of the experts before; it counts again per warp, and then every warp walks its part
// 32 ids at a time: __match_any finds the lanes with the same expert, their order inside the warp is the rank.  Nothing
// depends on the order in which blocks or atomics run.  A short list is one run and needs no pass 1.  The sums over the
// runs are taken by every block of pass 2 itself, or, where there are many experts, once by a scan between
// the passes.
//
// The rows: a thread owns 16 bytes of a token's row and reads it once for all k copies (gather), or reads the k
// sources and sums them in f32 in j order (combine).  All of it is bound by memory: the row bytes in and out.
#include "rows_common.cuh"

namespace dass {

int device_sm_count();   // dass_abi.cu

constexpr int ER_MAX_E = 1024;
constexpr int ER_MAX_K = 32;
constexpr int64_t ER_MAX_D = 1 << 21;          // row length: accesses of a row fit a grid's y extent
// Few warps: each step of the scan over experts walks them (32 instead of 8: 4.5 instead of 2.6 us for a short list).
constexpr int ER_SORT_WARPS = 8;
constexpr int64_t ER_ONE_RUN = 4096;           // ids that one block sorts alone

// Runs of 1024 ids at least, one to an SM at most.
static int64_t er_runs(int64_t n)
{
    if (n <= ER_ONE_RUN) return 1;
    const int64_t most = device_sm_count(), want = (n + 1023) / 1024;
    return want < most ? want : most;
}
// Experts up to which every block adds up the runs itself: 32768 choices of 8 experts 5.8 us, and 7.2 with the scan; 131072
// of 128 experts 14.1 and 8.6.
constexpr int64_t ER_SUM_EXPERTS = 32;

// counts[e][run]
__global__ void __launch_bounds__(ER_SORT_WARPS * 32)
expert_count_kernel(const int32_t *__restrict__ ids, int64_t n, int64_t run_len, int E, int32_t *__restrict__ counts)
{
    extern __shared__ int32_t er_smem[];
    for (int e = threadIdx.x; e < E; e += blockDim.x) er_smem[e] = 0;
    __syncthreads();
    const int64_t f0 = blockIdx.x * run_len, f1 = f0 + run_len < n ? f0 + run_len : n;
    for (int64_t f = f0 + threadIdx.x; f < f1; f += blockDim.x) {
        const int id = DASS_LD(ids + f);
        if (id >= 0 && id < E) atomicAdd(&er_smem[id], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += blockDim.x) DASS_ST(counts + (int64_t)e * gridDim.x + blockIdx.x, er_smem[e]);
}

// One warp per expert: counts[e][0 .. runs) become what the runs before hold, totals[e] what all hold.
__global__ void __launch_bounds__(ER_SORT_WARPS * 32)
expert_scan_kernel(int32_t *__restrict__ counts, int32_t *__restrict__ totals, int runs, int E)
{
    const int lane = threadIdx.x & 31, e = blockIdx.x * ER_SORT_WARPS + (threadIdx.x >> 5);
    if (e >= E) return;
    int32_t *row = counts + (int64_t)e * runs;
    int32_t carry = 0;
    for (int r0 = 0; r0 < runs; r0 += 32) {
        const int32_t v = r0 + lane < runs ? DASS_LD(row + r0 + lane) : 0;
        int32_t inc = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t up = __shfl_up_sync(FULL_MASK, inc, o);
            inc += lane >= o ? up : 0;
        }
        if (r0 + lane < runs) DASS_ST(row + r0 + lane, carry + inc - v);
        carry += __shfl_sync(FULL_MASK, inc, 31);
    }
    if (lane == 0) DASS_ST(totals + e, carry);
}

__global__ void __launch_bounds__(ER_SORT_WARPS * 32)
expert_place_kernel(const int32_t *__restrict__ ids, int64_t n, int64_t run_len, int runs, int E, const int32_t *__restrict__ counts,
                    const int32_t *__restrict__ totals,
                    int32_t *__restrict__ offsets, int32_t *__restrict__ slot, int32_t *__restrict__ source)
{
    extern __shared__ int32_t er_smem[];
    int32_t *before = er_smem;                              // [E] rows of earlier runs, then this run's first rank
    int32_t *total = er_smem + E;                           // [E] rows of all runs, then the experts' offsets
    int32_t *mine = er_smem + 2 * E;                        // [warps][E] this run's counts by warp, then next ranks
    __shared__ int32_t warp_sum[ER_SORT_WARPS];
    constexpr int threads = ER_SORT_WARPS * 32, warps = ER_SORT_WARPS;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t f0 = blockIdx.x * run_len, f1 = f0 + run_len < n ? f0 + run_len : n;
    const int64_t part = ((f1 - f0 + warps - 1) / warps + 31) / 32 * 32;
    const int64_t w0 = f0 + warp * part, w1 = w0 + part < f1 ? w0 + part : f1;

    for (int e = threadIdx.x; e < E * warps; e += blockDim.x) mine[e] = 0;
    for (int e = threadIdx.x; e < 2 * E; e += blockDim.x) er_smem[e] = 0;
    __syncthreads();
    for (int64_t f = w0 + lane; f < w1; f += 32) {
        const int id = DASS_LD(ids + f);
        if (id >= 0 && id < E) atomicAdd(&mine[warp * E + id], 1);
    }
    if (totals) {                                           // the scan has run
        for (int e = threadIdx.x; e < E; e += threads) {
            total[e] = DASS_LD(totals + e);
            before[e] = DASS_LD(counts + (int64_t)e * runs + blockIdx.x);
        }
    } else if (runs > 1) {
        for (int e = warp; e < E; e += warps) {             // a warp per expert, lanes over the runs
            int32_t b = 0, a = 0;
            for (int r = lane; r < runs; r += 32) {
                const int32_t c = DASS_LD(counts + (int64_t)e * runs + r);
                a += c;
                b += r < (int)blockIdx.x ? c : 0;
            }
            a = __reduce_add_sync(FULL_MASK, a);
            b = __reduce_add_sync(FULL_MASK, b);
            if (lane == 0) { total[e] = a; before[e] = b; }
        }
    }
    __syncthreads();
    if (runs == 1) {
        for (int e = threadIdx.x; e < E; e += blockDim.x) {
            int32_t a = 0;
            for (int w = 0; w < warps; ++w) a += mine[w * E + e];
            total[e] = a;
        }
        __syncthreads();
    }
    // exclusive scan of total over the experts, a block's width at a time
    int32_t carry = 0;
    for (int e0 = 0; e0 < E; e0 += threads) {
        const int e = e0 + threadIdx.x;
        const int32_t v = e < E ? total[e] : 0;
        int32_t inc = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t up = __shfl_up_sync(FULL_MASK, inc, o);
            inc += lane >= o ? up : 0;
        }
        if (lane == 31) warp_sum[warp] = inc;
        __syncthreads();
        int32_t base = carry, chunk = 0;
        for (int w = 0; w < warps; ++w) {
            const int32_t s = warp_sum[w];
            base += w < warp ? s : 0;
            chunk += s;
        }
        const int32_t at = base + inc - v;
        if (e < E) {
            if (blockIdx.x == 0) DASS_ST(offsets + e, at);
            int32_t next = at + before[e];
            for (int w = 0; w < warps; ++w) {       // first rank of every warp's part
                const int32_t c = mine[w * E + e];
                mine[w * E + e] = next;
                next += c;
            }
        }
        carry += chunk;
        __syncthreads();
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) DASS_ST(offsets + E, carry);
    for (int64_t f = f0 + threadIdx.x; f < f1; f += blockDim.x)
        if (source && f >= carry) DASS_ST(source + f, -1);
    for (int64_t fb = w0; fb < w1; fb += 32) {
        const int64_t f = fb + lane;
        int id = f < w1 ? DASS_LD(ids + f) : -1;
        if (id < 0 || id >= E) id = -1;
        const unsigned peers = __match_any_sync(FULL_MASK, id);
        int32_t first = id >= 0 ? mine[warp * E + id] : 0;
        __syncwarp();
        const int rank = __popc(peers & ((1u << lane) - 1u));
        if (id >= 0 && rank == 0) mine[warp * E + id] = first + __popc(peers);
        __syncwarp();
        if (f < w1) {
            const int32_t s = id >= 0 ? first + rank : -1;
            DASS_ST(slot + f, s);
            if (source && s >= 0) DASS_ST(source + s, (int32_t)f);
        }
    }
}

// ------------------------------------------------------------------ rows
// Every kernel below cuts its rows into accesses (16 bytes, or one element where alignment does not allow them) and lays
// threads over them without a division: blockDim.x threads on a row, blockDim.y rows a block, and blocks along y for rows
// longer than a block.  Loads are held as they lie in memory until all that a thread wants are in flight.
struct ErRows {
    int64_t T, rows;                 // tokens, rows of the sorted side
    int k, step;                     // choices per token, and of them taken at once (turns alike: 6 are 3 + 3)
    int vpr;                         // accesses per row
};

constexpr int ER_THREADS = 256;
// Accesses of a row per thread: what a thread reads it reads at once, so these and BATCH, the choices it takes at once, set
// the bytes in flight.  At 16 bytes: 4 choices of 2 accesses, or 2 of 4 where there are no more than two choices (16384
// tokens, k = 2, d = 4096: the sum with residual 117 -> 89 us); 4 of 4 costs too many registers (k = 6, d = 2048: 98 ->
// 202 us).  At single elements more.
template <int VEC> constexpr int ER_GATHER_COLS = VEC == 1 ? 8 : 2;
template <int VEC, int BATCH> constexpr int ER_SUM_COLS = (VEC == 1 ? 16 : 8) / BATCH;

// Rows from *used on are zeroed, by all blocks together.
template <bool BF16, int VEC, int COLS>
__device__ __forceinline__ void er_zero_tail(const int32_t *used, int64_t rows, int vpr, void *dst, int64_t ldd, int64_t first, int64_t step, int v0)
{
    int64_t end = DASS_LD(used);
    end = end < 0 ? 0 : end;
    float zero[VEC];
#pragma unroll
    for (int c = 0; c < VEC; ++c) zero[c] = 0.f;
    for (int64_t row = end + first; row < rows; row += step)
#pragma unroll
        for (int u = 0; u < COLS; ++u)
            if (v0 + u * (int)blockDim.x < vpr) row_store<BF16, VEC>(dst, row * ldd + (int64_t)(v0 + u * blockDim.x) * VEC, zero);
}

// dst[slot[t,j]] = scale * src[t]; rows past *used are zeroed (used null: left alone)
template <bool BF16, int VEC>
__global__ void __launch_bounds__(ER_THREADS)
expert_gather_kernel(const void *__restrict__ src, int64_t lds, const int32_t *__restrict__ slot, const float *__restrict__ weight,
                     const int32_t *__restrict__ used, void *__restrict__ dst, int64_t ldd, ErRows r)
{
    constexpr int COLS = ER_GATHER_COLS<VEC>, BATCH = 4;
    const int64_t t = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const int v0 = blockIdx.y * (blockDim.x * COLS) + threadIdx.x;
    if (t < r.T && v0 < r.vpr) {
        const int32_t *to = slot + t * r.k;
        RowRaw<BF16, VEC> raw[COLS];
#pragma unroll
        for (int u = 0; u < COLS; ++u)
            if (v0 + u * (int)blockDim.x < r.vpr) raw_load<BF16, VEC, true>(raw[u], src, t * lds + (int64_t)(v0 + u * blockDim.x) * VEC);
        for (int j0 = 0; j0 < r.k; j0 += BATCH) {
            int s[BATCH];
#pragma unroll
            for (int q = 0; q < BATCH; ++q) s[q] = j0 + q < r.k ? DASS_LD(to + j0 + q) : -1;
#pragma unroll
            for (int q = 0; q < BATCH; ++q) {
                if (s[q] < 0 || s[q] >= r.rows) continue;
                const float w = weight ? DASS_LD(weight + t * r.k + j0 + q) : 1.0f;
#pragma unroll
                for (int u = 0; u < COLS; ++u) {
                    if (v0 + u * (int)blockDim.x >= r.vpr) continue;
                    float y[VEC];
                    raw_floats(raw[u], y);
                    if (weight) {
#pragma unroll
                        for (int c = 0; c < VEC; ++c) y[c] *= w;
                    }
                    row_store<BF16, VEC>(dst, s[q] * ldd + (int64_t)(v0 + u * blockDim.x) * VEC, y);
                }
            }
        }
    }
    if (used) er_zero_tail<BF16, VEC, COLS>(used, r.rows, r.vpr, dst, ldd, t, (int64_t)gridDim.x * blockDim.y, v0);
}

// out[t] = residual[t] + sum_j weight[t,j] * rows[slot[t,j]], f32, j ascending, one rounding
template <bool BF16, int VEC, int BATCH>
__global__ void __launch_bounds__(ER_THREADS)
expert_combine_kernel(const void *__restrict__ rows, int64_t ldr, const int32_t *__restrict__ slot, const float *__restrict__ weight,
                      const void *residual, int64_t ldres, void *out, int64_t ldo, ErRows r)
{
    constexpr int COLS = ER_SUM_COLS<VEC, BATCH>;
    const int64_t t = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const int v0 = blockIdx.y * (blockDim.x * COLS) + threadIdx.x;
    if (t >= r.T || v0 >= r.vpr) return;
    float acc[COLS][VEC];
    RowRaw<BF16, VEC> res[COLS];
#pragma unroll
    for (int u = 0; u < COLS; ++u) {
#pragma unroll
        for (int c = 0; c < VEC; ++c) acc[u][c] = 0.f;
        if (residual && v0 + u * (int)blockDim.x < r.vpr)
            raw_load<BF16, VEC>(res[u], residual, t * ldres + (int64_t)(v0 + u * blockDim.x) * VEC);
    }
    for (int j0 = 0; j0 < r.k; j0 += r.step) {
        int s[BATCH];
        float w[BATCH];
        RowRaw<BF16, VEC> x[BATCH][COLS];
#pragma unroll
        for (int q = 0; q < BATCH; ++q) s[q] = q < r.step && j0 + q < r.k ? DASS_LD(slot + t * r.k + j0 + q) : -1;
#pragma unroll
        for (int q = 0; q < BATCH; ++q) {
            if (s[q] >= r.rows) s[q] = -1;
            w[q] = s[q] >= 0 && weight ? DASS_LD(weight + t * r.k + j0 + q) : 1.0f;
#pragma unroll
            for (int u = 0; u < COLS; ++u)
                if (s[q] >= 0 && v0 + u * (int)blockDim.x < r.vpr)
                    raw_load<BF16, VEC, true>(x[q][u], rows, s[q] * ldr + (int64_t)(v0 + u * blockDim.x) * VEC);
        }
#pragma unroll
        for (int q = 0; q < BATCH; ++q) {
            if (s[q] < 0) continue;                               // a skipped choice adds nothing, whatever its row would hold
#pragma unroll
            for (int u = 0; u < COLS; ++u) {
                float v[VEC];
                raw_floats(x[q][u], v);
#pragma unroll
                for (int c = 0; c < VEC; ++c) acc[u][c] = fmaf(w[q], v[c], acc[u][c]);
            }
        }
    }
#pragma unroll
    for (int u = 0; u < COLS; ++u) {
        if (v0 + u * (int)blockDim.x >= r.vpr) continue;
        if (residual) {
            float v[VEC];
            raw_floats(res[u], v);
#pragma unroll
            for (int c = 0; c < VEC; ++c) acc[u][c] += v[c];
        }
        row_store<BF16, VEC>(out, t * ldo + (int64_t)(v0 + u * blockDim.x) * VEC, acc[u]);
    }
}

// Gradient of the weighted sum: drows[slot[t,j]] = weight[t,j] * dout[t] and dweight[t,j] = <dout[t], rows[slot[t,j]]>.
// blockDim.x threads per token, blockDim.y tokens a block; dout[t] is read once for BATCH choices.  Three blocks to an SM
// (held to 80 registers): 16384 tokens, k = 6, d = 2048 take 146 us, with two blocks 170.
template <bool BF16, int VEC, int BATCH>
__global__ void __launch_bounds__(ER_THREADS, VEC == 1 ? 0 : 3)
expert_combine_backward_kernel(const void *__restrict__ dout, int64_t ldo, const void *__restrict__ rows, int64_t ldr,
                               const int32_t *__restrict__ slot, const float *__restrict__ weight, const int32_t *__restrict__ used,
                               void *__restrict__ drows, int64_t lddr, float *__restrict__ dweight, ErRows r)
{
    constexpr int COLS = ER_SUM_COLS<VEC, BATCH>;
    __shared__ float part[ER_THREADS / 32][BATCH];
    const int64_t t = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const bool live = t < r.T;
    const int width = blockDim.x;
    for (int j0 = 0; j0 < r.k; j0 += r.step) {
        int s[BATCH];
        float w[BATCH], acc[BATCH];
#pragma unroll
        for (int q = 0; q < BATCH; ++q) {
            s[q] = live && q < r.step && j0 + q < r.k ? DASS_LD(slot + t * r.k + j0 + q) : -1;
            acc[q] = 0.f;
        }
#pragma unroll
        for (int q = 0; q < BATCH; ++q) {
            if (s[q] >= r.rows) s[q] = -1;
            w[q] = drows && weight && s[q] >= 0 ? DASS_LD(weight + t * r.k + j0 + q) : 1.0f;
        }
        for (int v0 = threadIdx.x; live && v0 < r.vpr; v0 += COLS * width) {
            RowRaw<BF16, VEC> g[COLS], x[BATCH][COLS];
#pragma unroll
            for (int u = 0; u < COLS; ++u) {
                const int64_t col = (int64_t)(v0 + u * width) * VEC;
                if (v0 + u * width >= r.vpr) continue;
                raw_load<BF16, VEC>(g[u], dout, t * ldo + col);
                if (dweight) {
#pragma unroll
                    for (int q = 0; q < BATCH; ++q)
                        if (s[q] >= 0) raw_load<BF16, VEC, true>(x[q][u], rows, s[q] * ldr + col);
                }
            }
#pragma unroll
            for (int u = 0; u < COLS; ++u) {
                if (v0 + u * width >= r.vpr) continue;
                float gf[VEC];
                raw_floats(g[u], gf);
#pragma unroll
                for (int q = 0; q < BATCH; ++q) {
                    if (s[q] < 0) continue;
                    float v[VEC];
                    if (dweight) {
                        raw_floats(x[q][u], v);
#pragma unroll
                        for (int c = 0; c < VEC; ++c) acc[q] = fmaf(gf[c], v[c], acc[q]);
                    }
                    if (drows) {
#pragma unroll
                        for (int c = 0; c < VEC; ++c) v[c] = w[q] * gf[c];
                        row_store<BF16, VEC>(drows, s[q] * lddr + (int64_t)(v0 + u * width) * VEC, v);
                    }
                }
            }
        }
        if (dweight) {
            const int group = width < 32 ? width : 32;               // lanes of a token within a warp
#pragma unroll
            for (int q = 0; q < BATCH; ++q)
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    const float other = __shfl_xor_sync(FULL_MASK, acc[q], o);
                    acc[q] += o < group ? other : 0.f;
                }
            if (width > 32) {                                        // a token's warps: through shared memory, in order
                const int warp = (threadIdx.y * width + threadIdx.x) >> 5, first = (threadIdx.y * width) >> 5;
                if ((threadIdx.x & 31) == 0)
#pragma unroll
                    for (int q = 0; q < BATCH; ++q) part[warp][q] = acc[q];
                __syncthreads();
#pragma unroll
                for (int q = 0; q < BATCH; ++q) {
                    acc[q] = 0.f;
                    for (int i = 0; i < width / 32; ++i) acc[q] += part[first + i][q];
                }
                __syncthreads();
            }
            if (live && threadIdx.x == 0)
#pragma unroll
                for (int q = 0; q < BATCH; ++q)
                    if (q < r.step && j0 + q < r.k) DASS_ST(dweight + t * r.k + j0 + q, acc[q]);
        }
    }
    if (drows && used)
        for (int v0 = threadIdx.x; v0 < r.vpr; v0 += COLS * width)
            er_zero_tail<BF16, VEC, COLS>(used, r.rows, r.vpr, drows, lddr, t, (int64_t)gridDim.x * blockDim.y, v0);
}

// ------------------------------------------------------------------ host side
// Threads over a row's accesses, some each, as many rows as fill the block; blocks over rows and long rows.
struct ErGrid { dim3 grid, block; };
static ErGrid er_grid(int64_t rows, const ErRows &r, int cols, int most)
{
    int x = 4;
    while (x < most && x * cols < r.vpr) x *= 2;
    const int y = ER_THREADS / x;
    return {dim3((unsigned)((rows + y - 1) / y), (unsigned)((r.vpr + x * cols - 1) / (x * cols))), dim3(x, y)};
}

static int er_sum_cols(bool vector, int64_t k)
{
    if (vector) return k <= 2 ? ER_SUM_COLS<8, 2> : ER_SUM_COLS<8, 4>;
    return k <= 2 ? ER_SUM_COLS<1, 2> : ER_SUM_COLS<1, 4>;
}

static dass_status er_check(int64_t T, int64_t k, int64_t d, int dt)
{
    if (dt != DASS_BF16 && dt != DASS_F32) return DASS_ERR_DTYPE;
    if (T < 0 || k < 1 || d < 1) return DASS_ERR_SHAPE;
    if (k > ER_MAX_K || T > ((1ll << 31) - 1) / k || d > ER_MAX_D) return DASS_ERR_UNSUPPORTED;
    return DASS_OK;
}

}  // namespace dass

using namespace dass;

extern "C" {

dass_status dass_expert_sort_workspace_bytes(int64_t T, int64_t k, int64_t E, size_t *bytes)
{
    if (!bytes) return DASS_ERR_NULL;
    if (T < 0 || k < 1 || E < 1) return DASS_ERR_SHAPE;
    if (E > ER_MAX_E || k > ER_MAX_K || T > ((1ll << 31) - 1) / k) return DASS_ERR_UNSUPPORTED;
    const int64_t runs = er_runs(T * k);
    *bytes = runs > 1 ? (size_t)(runs + 1) * (size_t)E * sizeof(int32_t) : 0;
    return DASS_OK;
}

dass_status dass_expert_sort(const int32_t *expert, int64_t T, int64_t k, int64_t E, int32_t *offsets, int32_t *slot, int32_t *source,
                             void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    if ((!expert && T > 0) || !offsets || (!slot && T > 0)) return DASS_ERR_NULL;
    size_t need = 0;
    const dass_status qs = dass_expert_sort_workspace_bytes(T, k, E, &need);
    if (qs != DASS_OK) return qs;
    if (!elem_aligned(expert, false) || !elem_aligned(offsets, false) || !elem_aligned(slot, false) || !elem_aligned(source, false))
        return DASS_ERR_ALIGN;
    if (need && (!workspace || workspace_bytes < need)) return DASS_ERR_WORKSPACE;
    if (need && (reinterpret_cast<uintptr_t>(workspace) & 15u)) return DASS_ERR_ALIGN;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const int64_t n = T * k;
    const int64_t runs = er_runs(n);
    const int64_t run_len = (n + runs - 1) / runs;
    DASS_BOUNDS_SCOPE(bs);
    DASS_BOUNDS_ADD(bs, expert, (size_t)n * 4);
    DASS_BOUNDS_ADD(bs, slot, (size_t)n * 4);
    DASS_BOUNDS_ADD(bs, source, (size_t)n * 4);
    DASS_BOUNDS_ADD(bs, offsets, (size_t)(E + 1) * 4);
    DASS_BOUNDS_ADD(bs, workspace, need);
    DASS_BOUNDS_COMMIT(bs, st);
    int32_t *counts = static_cast<int32_t *>(workspace);
    if (runs > 1) {
        expert_count_kernel<<<(unsigned)runs, ER_SORT_WARPS * 32, (size_t)E * 4, st>>>(expert, n, run_len, (int)E, counts);
        if (cudaGetLastError() != cudaSuccess) return DASS_ERR_CUDA;
    }
    int32_t *totals = runs > 1 && E > ER_SUM_EXPERTS ? counts + runs * E : nullptr;
    if (totals) {
        expert_scan_kernel<<<(unsigned)((E + ER_SORT_WARPS - 1) / ER_SORT_WARPS), ER_SORT_WARPS * 32, 0, st>>>(counts, totals, (int)runs, (int)E);
        if (cudaGetLastError() != cudaSuccess) return DASS_ERR_CUDA;
    }
    expert_place_kernel<<<(unsigned)runs, ER_SORT_WARPS * 32, (size_t)E * 4 * (2 + ER_SORT_WARPS), st>>>(expert, n, run_len, (int)runs, (int)E,
                                                                                                     counts, totals, offsets, slot, source);
    return cudaGetLastError() == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

dass_status dass_expert_gather(const void *X, int64_t T, int64_t d, int64_t ldx, dass_dtype dt, const int32_t *slot, int64_t k,
                               const float *weight, const int32_t *rows_used, void *Xs, int64_t rows, int64_t ldxs, void *cuda_stream)
{
    const dass_status cs = er_check(T, k, d, (int)dt);
    if (cs != DASS_OK) return cs;
    if (ldx < d || ldxs < d || rows < 0) return DASS_ERR_SHAPE;
    if (rows > 0 && !Xs) return DASS_ERR_NULL;
    if (T > 0 && (!X || !slot)) return DASS_ERR_NULL;
    const bool bf16 = dt == DASS_BF16;
    if (!elem_aligned(X, bf16) || !elem_aligned(Xs, bf16) || !elem_aligned(slot, false) || !elem_aligned(weight, false) ||
        !elem_aligned(rows_used, false))
        return DASS_ERR_ALIGN;
    if (rows == 0 || (T == 0 && !rows_used)) return DASS_OK;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const size_t elt = bf16 ? 2 : 4;
    const int vec = bf16 ? 8 : 4;
    const bool vector = rows_vec_ok(X, ldx, bf16) && rows_vec_ok(Xs, ldxs, bf16) && d % vec == 0;
    const ErRows r{T, rows, (int)k, (int)(k <= 2 ? k : (k + (k + 3) / 4 - 1) / ((k + 3) / 4)), (int)(vector ? d / vec : d)};
    DASS_BOUNDS_SCOPE(bs);
    if (T > 0) DASS_BOUNDS_ADD(bs, X, ((size_t)(T - 1) * ldx + d) * elt);
    DASS_BOUNDS_ADD(bs, Xs, ((size_t)(rows - 1) * ldxs + d) * elt);
    DASS_BOUNDS_ADD(bs, slot, (size_t)T * k * 4);
    DASS_BOUNDS_ADD(bs, weight, (size_t)T * k * 4);
    DASS_BOUNDS_ADD(bs, rows_used, 4);
    DASS_BOUNDS_COMMIT(bs, st);
    (void)elt;
    const ErGrid g = er_grid(T > 0 ? T : rows, r, vector ? ER_GATHER_COLS<8> : ER_GATHER_COLS<1>, ER_THREADS);
    auto launch = [&](auto kernel) { kernel<<<g.grid, g.block, 0, st>>>(X, ldx, slot, weight, rows_used, Xs, ldxs, r); };
    if (bf16 && vector) launch(expert_gather_kernel<true, 8>);
    else if (bf16) launch(expert_gather_kernel<true, 1>);
    else if (vector) launch(expert_gather_kernel<false, 4>);
    else launch(expert_gather_kernel<false, 1>);
    return cudaGetLastError() == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

dass_status dass_expert_combine(const void *Ys, int64_t rows, int64_t d, int64_t ldys, dass_dtype dt, const int32_t *slot, int64_t T,
                                int64_t k, const float *weight, const void *residual, int64_t ldr, void *Y, int64_t ldy, void *cuda_stream)
{
    const dass_status cs = er_check(T, k, d, (int)dt);
    if (cs != DASS_OK) return cs;
    if (ldys < d || ldy < d || rows < 0 || (residual && ldr < d)) return DASS_ERR_SHAPE;
    if (T > 0 && (!slot || !Y)) return DASS_ERR_NULL;
    if (T > 0 && rows > 0 && !Ys) return DASS_ERR_NULL;
    const bool bf16 = dt == DASS_BF16;
    if (!elem_aligned(Ys, bf16) || !elem_aligned(residual, bf16) || !elem_aligned(Y, bf16) || !elem_aligned(slot, false) ||
        !elem_aligned(weight, false))
        return DASS_ERR_ALIGN;
    if (T == 0) return DASS_OK;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const size_t elt = bf16 ? 2 : 4;
    const int vec = bf16 ? 8 : 4;
    const bool vector = rows_vec_ok(Ys, ldys, bf16) && rows_vec_ok(Y, ldy, bf16) && (!residual || rows_vec_ok(residual, ldr, bf16)) && d % vec == 0;
    const ErRows r{T, rows, (int)k, (int)(k <= 2 ? k : (k + (k + 3) / 4 - 1) / ((k + 3) / 4)), (int)(vector ? d / vec : d)};
    DASS_BOUNDS_SCOPE(bs);
    if (rows > 0) DASS_BOUNDS_ADD(bs, Ys, ((size_t)(rows - 1) * ldys + d) * elt);
    DASS_BOUNDS_ADD(bs, residual, ((size_t)(T - 1) * ldr + d) * elt);
    DASS_BOUNDS_ADD(bs, Y, ((size_t)(T - 1) * ldy + d) * elt);
    DASS_BOUNDS_ADD(bs, slot, (size_t)T * k * 4);
    DASS_BOUNDS_ADD(bs, weight, (size_t)T * k * 4);
    DASS_BOUNDS_COMMIT(bs, st);
    (void)elt;
    const ErGrid g = er_grid(T, r, er_sum_cols(vector, k), ER_THREADS);
    auto launch = [&](auto kernel) { kernel<<<g.grid, g.block, 0, st>>>(Ys, ldys, slot, weight, residual, ldr, Y, ldy, r); };
    if (bf16 && vector) k <= 2 ? launch(expert_combine_kernel<true, 8, 2>) : launch(expert_combine_kernel<true, 8, 4>);
    else if (bf16) k <= 2 ? launch(expert_combine_kernel<true, 1, 2>) : launch(expert_combine_kernel<true, 1, 4>);
    else if (vector) k <= 2 ? launch(expert_combine_kernel<false, 4, 2>) : launch(expert_combine_kernel<false, 4, 4>);
    else k <= 2 ? launch(expert_combine_kernel<false, 1, 2>) : launch(expert_combine_kernel<false, 1, 4>);
    return cudaGetLastError() == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

dass_status dass_expert_combine_backward(const void *dY, int64_t T, int64_t d, int64_t lddy, const void *Ys, int64_t rows, int64_t ldys,
                                         dass_dtype dt, const int32_t *slot, int64_t k, const float *weight, const int32_t *rows_used,
                                         void *dYs, int64_t lddys, float *dweight, void *cuda_stream)
{
    const dass_status cs = er_check(T, k, d, (int)dt);
    if (cs != DASS_OK) return cs;
    if (!dYs && !dweight) return DASS_ERR_NULL;
    if (lddy < d || rows < 0 || (Ys && ldys < d) || (dYs && lddys < d)) return DASS_ERR_SHAPE;
    if (T > 0 && (!dY || !slot || (dweight && !Ys && rows > 0))) return DASS_ERR_NULL;
    const bool bf16 = dt == DASS_BF16;
    if (!elem_aligned(dY, bf16) || !elem_aligned(Ys, bf16) || !elem_aligned(dYs, bf16) || !elem_aligned(slot, false) ||
        !elem_aligned(weight, false) || !elem_aligned(dweight, false) || !elem_aligned(rows_used, false))
        return DASS_ERR_ALIGN;
    if (T == 0 && !(dYs && rows_used && rows > 0)) return DASS_OK;    // without tokens dYs still has rows to be zeroed
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const size_t elt = bf16 ? 2 : 4;
    const int vec = bf16 ? 8 : 4;
    const bool vector = rows_vec_ok(dY, lddy, bf16) && (!dweight || rows_vec_ok(Ys, ldys, bf16)) && (!dYs || rows_vec_ok(dYs, lddys, bf16)) &&
                        d % vec == 0;
    const ErRows r{T, rows, (int)k, (int)(k <= 2 ? k : (k + (k + 3) / 4 - 1) / ((k + 3) / 4)), (int)(vector ? d / vec : d)};
    DASS_BOUNDS_SCOPE(bs);
    if (T > 0) DASS_BOUNDS_ADD(bs, dY, ((size_t)(T - 1) * lddy + d) * elt);
    if (rows > 0) DASS_BOUNDS_ADD(bs, Ys, ((size_t)(rows - 1) * ldys + d) * elt);
    if (rows > 0) DASS_BOUNDS_ADD(bs, dYs, ((size_t)(rows - 1) * lddys + d) * elt);
    DASS_BOUNDS_ADD(bs, slot, (size_t)T * k * 4);
    DASS_BOUNDS_ADD(bs, weight, (size_t)T * k * 4);
    DASS_BOUNDS_ADD(bs, dweight, (size_t)T * k * 4);
    DASS_BOUNDS_ADD(bs, rows_used, 4);
    DASS_BOUNDS_COMMIT(bs, st);
    (void)elt;
    // few threads a token keep its sums inside a warp; a whole block where there are few tokens
    ErGrid g = er_grid(T > 0 ? T : rows, r, er_sum_cols(vector, k), T >= (int64_t)device_sm_count() * 32 ? 64 : ER_THREADS);
    g.grid.y = 1;                                                     // a token's threads walk its whole row
    const dim3 grid = g.grid, block = g.block;
    auto launch = [&](auto kernel) { kernel<<<grid, block, 0, st>>>(dY, lddy, Ys, ldys, slot, weight, rows_used, dYs, lddys, dweight, r); };
    if (bf16 && vector) k <= 2 ? launch(expert_combine_backward_kernel<true, 8, 2>) : launch(expert_combine_backward_kernel<true, 8, 4>);
    else if (bf16) k <= 2 ? launch(expert_combine_backward_kernel<true, 1, 2>) : launch(expert_combine_backward_kernel<true, 1, 4>);
    else if (vector) k <= 2 ? launch(expert_combine_backward_kernel<false, 4, 2>) : launch(expert_combine_backward_kernel<false, 4, 4>);
    else k <= 2 ? launch(expert_combine_backward_kernel<false, 1, 2>) : launch(expert_combine_backward_kernel<false, 1, 4>);
    return cudaGetLastError() == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

}  // extern "C"
