// dass_linear for f32, in f32 FMAs.
//
// Many rows: a block owns BT rows x BN accumulator columns, a thread MT x MN of them as two halves (rows ty * MT / 2 .. and
// BT / 2 + the same; columns likewise), so that its shared-memory reads are whole accesses without conflicts.  In the GLU
// form the left half of the columns belongs to W and the right half to W_up: a thread then holds both factors of its
// outputs.  Both operands go through shared memory, transposed to k-major, BK k at a time, the next ones already in registers;
// fma.f32x2 takes two columns an instruction, which leaves issue slots for the loads.  Bound by the FMA pipes.
//
// Few rows: as linear_few.cu, a block of 8 warps owns 8 columns and up to 8 rows and the warps take k in turns of 128; a
// lane multiplies 4 k of every weight row with 4 k of every row of X.  Bound by reading the weights.
#include "linear_common.cuh"

namespace dass {


typedef unsigned long long f32pair;
__device__ __forceinline__ f32pair pair_of(float x)
{
    f32pair r;
    asm("mov.b64 %0, {%1, %1};" : "=l"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ void pair_fma(f32pair &c, f32pair a, f32pair b)
{
    asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(c) : "l"(a), "l"(b));
}
__device__ __forceinline__ void pair_split(f32pair p, float &lo, float &hi)
{
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p));
}

// 4 elements of a row from k on; those at and past K are zero (and are not touched).
__device__ __forceinline__ float4 lf_load4(const float *row, int64_t k, int64_t K)
{
    if (k + 4 <= K) return DASS_LD(reinterpret_cast<const float4 *>(row + k));
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (k < K) v.x = DASS_LD(row + k);
    if (k + 1 < K) v.y = DASS_LD(row + k + 1);
    if (k + 2 < K) v.z = DASS_LD(row + k + 2);
    return v;
}

// The value of one output: bias, activation, gating factor, residual.
__device__ __forceinline__ void lf_store(const LinearArgs &a, int g, int64_t t, int64_t n, float p, float up, bool glu)
{
    const int64_t b = (int64_t)g * a.N + n;
    if (a.bias) p += DASS_LD(static_cast<const float *>(a.bias) + b);
    p = lin_act(p, a.act);
    if (glu) p *= a.bias_up ? up + DASS_LD(static_cast<const float *>(a.bias_up) + b) : up;
    if (a.residual) p += DASS_LD(static_cast<const float *>(a.residual) + t * a.ldr + n);
    DASS_ST(static_cast<float *>(a.Y) + t * a.ldy + n, p);
}

// KG groups of threads share a tile and take turns of BK k; their sums are added at the end.
template <int BT, int BN, int MT, int MN, int BK, int KG, bool GLU>
__global__ void __launch_bounds__((BT / MT) * (BN / MN) * KG, BT == 128 && GLU ? 2 : 1)
linear_f32_tile_kernel(const __grid_constant__ LinearArgs a, int64_t n_tiles, bool y_vec)
{
    constexpr int THREADS = (BT / MT) * (BN / MN);
    constexpr int XL = BT * BK / 4 / THREADS, WL = BN * BK / 4 / THREADS;      // 4-element loads a thread and step
    static_assert(XL >= 1 && WL >= 1, "every thread loads");
    constexpr int HT = MT / 2, HN = MN / 2, OUT = GLU ? BN / 2 : BN;
    constexpr int XS = 2 * BK * (BT + 4), WS = 2 * BK * (BN + 4);                    // two buffers of each operand
    __shared__ __align__(16) float smem[KG * (XS + WS)];
    const int group = threadIdx.x / THREADS, tid = threadIdx.x % THREADS, tx = tid % (BN / MN), ty = tid / (BN / MN);
    auto &sx = *reinterpret_cast<float(*)[2][BK][BT + 4]>(smem + group * XS);
    auto &sw = *reinterpret_cast<float(*)[2][BK][BN + 4]>(smem + KG * XS + group * WS);
    lin_zero_outside<false>(a.offsets, a.groups, a.T, a.N, a.Y, a.ldy, y_vec, (int64_t)blockIdx.x * (KG * THREADS) + threadIdx.x,
                            (int64_t)gridDim.x * (KG * THREADS));
    const LinTile tile = lin_find_tile(a.offsets, a.groups, a.T, BT, blockIdx.x / n_tiles);
    if (tile.g < 0) return;
    const int64_t n0 = (blockIdx.x % n_tiles) * OUT, wbase = (int64_t)tile.g * a.group_stride;
    const float *X = static_cast<const float *>(a.X), *W = static_cast<const float *>(a.W) + wbase;
    const float *U = GLU ? static_cast<const float *>(a.W_up) + wbase : W;

    float4 rx[XL], rw[WL];
    auto fetch = [&](int64_t k0) {
#pragma unroll
        for (int i = 0; i < XL; ++i) {
            const int r = (tid + i * THREADS) / (BK / 4), c = (tid + i * THREADS) % (BK / 4) * 4;
            rx[i] = tile.lo + r < tile.hi ? lf_load4(X + (tile.lo + r) * a.ldx, k0 + c, a.K) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int i = 0; i < WL; ++i) {
            const int r = (tid + i * THREADS) / (BK / 4), c = (tid + i * THREADS) % (BK / 4) * 4;
            const int64_t n = n0 + (GLU ? r % OUT : r);
            rw[i] = n < a.N ? lf_load4((GLU && r >= OUT ? U : W) + n * a.ldw, k0 + c, a.K) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    };
    auto stash = [&](int s) {
#pragma unroll
        for (int i = 0; i < XL; ++i) {
            const int r = (tid + i * THREADS) / (BK / 4), c = (tid + i * THREADS) % (BK / 4) * 4;
            sx[s][c][r] = rx[i].x; sx[s][c + 1][r] = rx[i].y; sx[s][c + 2][r] = rx[i].z; sx[s][c + 3][r] = rx[i].w;
        }
#pragma unroll
        for (int i = 0; i < WL; ++i) {
            const int r = (tid + i * THREADS) / (BK / 4), c = (tid + i * THREADS) % (BK / 4) * 4;
            sw[s][c][r] = rw[i].x; sw[s][c + 1][r] = rw[i].y; sw[s][c + 2][r] = rw[i].z; sw[s][c + 3][r] = rw[i].w;
        }
    };
    f32pair acc[MT][MN / 2];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < MN / 2; ++j) acc[i][j] = 0ull;
    fetch(group * BK);
    stash(0);
    __syncthreads();
    int s = 0;
    for (int64_t k0 = 0; k0 < a.K; k0 += KG * BK, s ^= 1) {        // the groups of threads take turns
        const bool more = k0 + KG * BK < a.K;
        if (more) fetch(k0 + (KG + group) * BK);
#pragma unroll
        for (int k = 0; k < BK; ++k) {
            float x[MT];
            f32pair w[MN / 2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float *px = &sx[s][k][h * (BT / 2) + ty * HT], *pw = &sw[s][k][h * (BN / 2) + tx * HN];
                if constexpr (HT == 4) {
                    const float4 v = *reinterpret_cast<const float4 *>(px);
                    x[4 * h] = v.x; x[4 * h + 1] = v.y; x[4 * h + 2] = v.z; x[4 * h + 3] = v.w;
                } else {
                    const float2 v = *reinterpret_cast<const float2 *>(px);
                    x[2 * h] = v.x; x[2 * h + 1] = v.y;
                }
                if constexpr (HN == 4) {
                    const ulonglong2 v = *reinterpret_cast<const ulonglong2 *>(pw);
                    w[2 * h] = v.x; w[2 * h + 1] = v.y;
                } else {
                    w[h] = *reinterpret_cast<const f32pair *>(pw);
                }
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const f32pair xx = pair_of(x[i]);
#pragma unroll
                for (int j = 0; j < MN / 2; ++j) pair_fma(acc[i][j], xx, w[j]);
            }
        }
        if (more) stash(s ^ 1);                              // the other buffer: its readers passed the last barrier
        __syncthreads();
    }
    if constexpr (KG > 1) {                                  // the groups' sums, in order, over the operands' buffers
        float *sum = smem;
        static_assert(sizeof(smem) >= (KG - 1) * THREADS * MT * MN * 4 / 2, "two halves of the sums at a time");
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (group > 0)
#pragma unroll
                for (int i = 0; i < HT; ++i)
#pragma unroll
                    for (int j = 0; j < MN / 2; ++j)
                        *reinterpret_cast<f32pair *>(sum + 2 * ((((group - 1) * HT + i) * (MN / 2) + j) * THREADS + tid)) = acc[half * HT + i][j];
            __syncthreads();
            if (group == 0)
#pragma unroll
                for (int i = 0; i < HT; ++i)
#pragma unroll
                    for (int j = 0; j < MN / 2; ++j)
#pragma unroll
                        for (int g = 0; g < KG - 1; ++g) {
                            const f32pair v = *reinterpret_cast<const f32pair *>(sum + 2 * (((g * HT + i) * (MN / 2) + j) * THREADS + tid));
                            asm("add.rn.f32x2 %0, %0, %1;" : "+l"(acc[half * HT + i][j]) : "l"(v));
                        }
            __syncthreads();
        }
        if (group > 0) return;
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t t = tile.lo + (i / HT) * (BT / 2) + ty * HT + i % HT;
        if (t >= tile.hi) continue;
        float v[MN];
#pragma unroll
        for (int j = 0; j < MN / 2; ++j) pair_split(acc[i][j], v[2 * j], v[2 * j + 1]);
#pragma unroll
        for (int j = 0; j < (GLU ? HN : MN); ++j) {
            const int64_t n = n0 + (GLU || j < HN ? tx * HN + j : BN / 2 + tx * HN + j - HN);
            if (n < a.N) lf_store(a, tile.g, t, n, v[j], GLU ? v[HN + j] : 0.f, GLU);
        }
    }
}

constexpr int LFF_ROWS = 8, LFF_WARPS = 8, LFF_THREADS = LFF_WARPS * 32;

// COLS weight rows in all (the GLU form: COLS / 2 of W and of W_up)
template <int COLS, bool GLU>
__global__ void __launch_bounds__(LFF_THREADS)
linear_f32_few_kernel(const __grid_constant__ LinearArgs a, int64_t n_tiles, bool y_vec)
{
    constexpr int OUT = GLU ? COLS / 2 : COLS, SUMS = COLS * LFF_ROWS;
    static_assert(SUMS % 32 == 0, "the sums are spread over a warp");
    __shared__ float part[LFF_WARPS][SUMS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    lin_zero_outside<false>(a.offsets, a.groups, a.T, a.N, a.Y, a.ldy, y_vec, (int64_t)blockIdx.x * LFF_THREADS + threadIdx.x,
                            (int64_t)gridDim.x * LFF_THREADS);
    const LinTile tile = lin_find_tile(a.offsets, a.groups, a.T, LFF_ROWS, blockIdx.x / n_tiles);
    if (tile.g < 0) return;
    const int64_t n0 = (blockIdx.x % n_tiles) * OUT, wbase = (int64_t)tile.g * a.group_stride;
    const float *w[COLS], *x[LFF_ROWS];
#pragma unroll
    for (int c = 0; c < COLS; ++c) {                          // columns past the last are read as the last, rows likewise: never stored
        const int64_t n = n0 + c % OUT < a.N ? n0 + c % OUT : a.N - 1;
        w[c] = static_cast<const float *>(GLU && c >= OUT ? a.W_up : a.W) + wbase + n * a.ldw;
    }
    const int rows = (int)(tile.hi - tile.lo);
#pragma unroll
    for (int r = 0; r < LFF_ROWS; ++r) x[r] = static_cast<const float *>(a.X) + (tile.lo + (r < rows ? r : 0)) * a.ldx;
    float acc[SUMS];
#pragma unroll
    for (int i = 0; i < SUMS; ++i) acc[i] = 0.f;
    for (int64_t k = warp * 128 + lane * 4; k < a.K; k += LFF_WARPS * 128) {
        float4 wv[COLS];
#pragma unroll
        for (int c = 0; c < COLS; ++c) wv[c] = lf_load4(w[c], k, a.K);
#pragma unroll
        for (int r = 0; r < LFF_ROWS; ++r) {
            if (r >= rows) break;
            const float4 xv = lf_load4(x[r], k, a.K);
#pragma unroll
            for (int c = 0; c < COLS; ++c) {
                float &s = acc[r * COLS + c];
                s = fmaf(xv.x, wv[c].x, fmaf(xv.y, wv[c].y, fmaf(xv.z, wv[c].z, fmaf(xv.w, wv[c].w, s))));
            }
        }
    }
    // Sum over the lanes: at each step a lane keeps one half of the sums and hands the other half over.
#pragma unroll
    for (int o = 16, n = SUMS / 2; o > 0; o >>= 1, n >>= 1)
#pragma unroll
        for (int i = 0; i < SUMS / 2; ++i)
            if (i < n) {
                const float send = lane & o ? acc[i] : acc[i + n], keep = lane & o ? acc[i + n] : acc[i];
                acc[i] = keep + __shfl_xor_sync(FULL_MASK, send, o);
            }
    // lane l now holds sums SUMS / 32 * l' .. with l' the lane's bits in the order they were handed out: the highest first
    const int first = lane * (SUMS / 32);
#pragma unroll
    for (int i = 0; i < SUMS / 32; ++i) part[warp][first + i] = acc[i];
    __syncthreads();
    for (int o = threadIdx.x; o < rows * OUT; o += LFF_THREADS) {
        const int r = o / OUT, c = o % OUT;
        float p = 0.f, up = 0.f;
#pragma unroll
        for (int v = 0; v < LFF_WARPS; ++v) {
            p += part[v][r * COLS + c];
            if constexpr (GLU) up += part[v][r * COLS + OUT + c];
        }
        if (n0 + c < a.N) lf_store(a, tile.g, tile.lo + r, n0 + c, p, up, GLU);
    }
}

int device_sm_count();   // dass_abi.cu

template <int BT, int BN, int MT, int MN, int BK, int KG>
static dass_status lf_tiles(const LinearArgs &a, bool y_vec)
{
    const int out = a.W_up ? BN / 2 : BN;
    const int64_t n_tiles = (a.N + out - 1) / out, row_tiles = (a.T + BT - 1) / BT + (a.offsets ? a.groups : 0);
    if (n_tiles * row_tiles > 0x7fffffffll) return DASS_ERR_UNSUPPORTED;
    const unsigned grid = (unsigned)(n_tiles * row_tiles);
    constexpr int threads = (BT / MT) * (BN / MN) * KG;
    if (a.W_up) linear_f32_tile_kernel<BT, BN, MT, MN, BK, KG, true><<<grid, threads, 0, a.st>>>(a, n_tiles, y_vec);
    else linear_f32_tile_kernel<BT, BN, MT, MN, BK, KG, false><<<grid, threads, 0, a.st>>>(a, n_tiles, y_vec);
    return cudaGetLastError() == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

dass_status linear_f32_launch(const LinearArgs &a)
{
    const bool y_vec = rows_vec_ok(a.Y, a.ldy, false);
    const int64_t rows = a.offsets ? (a.T + a.groups - 1) / a.groups : a.T, groups = lin_active_groups(a);
    const int64_t cols = a.W_up ? 2 * a.N : a.N;
    auto tiles = [&](int64_t bt, int64_t bn) { return ((a.T + bt - 1) / bt + (a.offsets ? groups / 2 : 0)) * ((cols + bn - 1) / bn); };
    // The largest tile that still gives most SMs one (1024 rows, 4096 x 4096: 763 to 822 us with 128 x 128, 938 with 64 x 64, 1250
    // with 32 x 32; 128 rows: 422, 191, 192); few rows, while reading them again and again costs less than a tile's start
    // (4096 x 4096: 4 rows 32 against 66 us, 16 rows 86 against 63; 700 x 200 gated, 16 rows 5 against 12).
    const double products = (double)a.T * cols * a.K;
    const int path = rows <= 8 || (rows <= 16 && products <= 16e6) ? 0 : tiles(128, 128) * 10 >= 8 * device_sm_count() ? 3 : tiles(64, 64) >= device_sm_count() ? 2 : 1;
    if (path == 0) {
        const int out = a.W_up ? 4 : 8;
        const int64_t n_tiles = (a.N + out - 1) / out, row_tiles = (a.T + LFF_ROWS - 1) / LFF_ROWS + (a.offsets ? groups : 0);
        if (n_tiles * row_tiles > 0x7fffffffll) return DASS_ERR_UNSUPPORTED;
        const unsigned grid = (unsigned)(n_tiles * row_tiles);
        if (a.W_up) linear_f32_few_kernel<8, true><<<grid, LFF_THREADS, 0, a.st>>>(a, n_tiles, y_vec);
        else linear_f32_few_kernel<8, false><<<grid, LFF_THREADS, 0, a.st>>>(a, n_tiles, y_vec);
        return cudaGetLastError() == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
    }
    return path == 3 ? lf_tiles<128, 128, 8, 8, 16, 1>(a, y_vec) : path == 2 ? lf_tiles<64, 64, 4, 8, 16, 2>(a, y_vec) : lf_tiles<32, 32, 4, 4, 16, 4>(a, y_vec);
}

}  // namespace dass
