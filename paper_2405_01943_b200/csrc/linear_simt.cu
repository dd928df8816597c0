// dass_linear on the CUDA cores: a tile of 64 rows x 64 columns per block of 256 threads, 4 x 4 outputs a thread, both
// operands staged through shared memory 16 k at a time, f32 sums in ascending k.
#include "linear_common.cuh"

namespace dass {

constexpr int LS_T = 64, LS_N = 64, LS_K = 16, LS_THREADS = 256;

template <bool BF16, bool GLU>
__global__ void __launch_bounds__(LS_THREADS)
linear_simt_kernel(const LinearArgs a, int64_t n_tiles, bool y_vec)
{
    __shared__ float sx[LS_K][LS_T + 4];
    __shared__ float sw[LS_K][LS_N + 4];
    __shared__ float sv[GLU ? LS_K : 1][LS_N + 4];
    const int tid = threadIdx.x;
    lin_zero_outside<BF16>(a.offsets, a.groups, a.T, a.N, a.Y, a.ldy, y_vec, (int64_t)blockIdx.x * LS_THREADS + tid, (int64_t)gridDim.x * LS_THREADS);
    const LinTile tile = lin_find_tile(a.offsets, a.groups, a.T, LS_T, blockIdx.x / n_tiles);
    if (tile.g < 0) return;
    const int64_t n0 = (blockIdx.x % n_tiles) * LS_N;
    const int64_t wbase = (int64_t)tile.g * a.group_stride;
    const int tx = tid & 15, ty = tid >> 4;                // columns tx*4.., rows ty*4..
    float acc[4][4] = {}, acc_up[4][4] = {};
    for (int64_t k0 = 0; k0 < a.K; k0 += LS_K) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (tid >> 4) + 16 * i, c = tid & 15;
            const int64_t k = k0 + c;
            float x[1] = {0.f}, w[1] = {0.f}, v[1] = {0.f};
            if (k < a.K && tile.lo + r < tile.hi) row_load<BF16, 1>(a.X, (tile.lo + r) * a.ldx + k, x);
            if (k < a.K && n0 + r < a.N) {
                row_load<BF16, 1>(a.W, wbase + (n0 + r) * a.ldw + k, w);
                if constexpr (GLU) row_load<BF16, 1>(a.W_up, wbase + (n0 + r) * a.ldw + k, v);
            }
            sx[c][r] = x[0];
            sw[c][r] = w[0];
            if constexpr (GLU) sv[c][r] = v[0];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < LS_K; ++k) {
            float x[4], w[4], v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = sx[k][ty * 4 + i]; w[i] = sw[k][tx * 4 + i]; v[i] = GLU ? sv[k][tx * 4 + i] : 0.f; }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    acc[i][j] = fmaf(x[i], w[j], acc[i][j]);
                    if constexpr (GLU) acc_up[i][j] = fmaf(x[i], v[j], acc_up[i][j]);
                }
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t t = tile.lo + ty * 4 + i;
        if (t >= tile.hi) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t n = n0 + tx * 4 + j;
            if (n >= a.N) continue;
            float b[1] = {0.f}, bu[1] = {0.f}, r[1] = {0.f};
            if (a.bias) row_load<BF16, 1>(a.bias, tile.g * a.N + n, b);
            if (GLU && a.bias_up) row_load<BF16, 1>(a.bias_up, tile.g * a.N + n, bu);
            if (a.residual) row_load<BF16, 1>(a.residual, t * a.ldr + n, r);
            float y[1] = {lin_act(acc[i][j] + b[0], a.act)};
            if constexpr (GLU) y[0] *= acc_up[i][j] + bu[0];
            y[0] += r[0];
            row_store<BF16, 1>(a.Y, t * a.ldy + n, y);
        }
    }
}

dass_status linear_simt_launch(const LinearArgs &a)
{
    const int64_t n_tiles = (a.N + LS_N - 1) / LS_N;
    const int64_t row_tiles = (a.T + LS_T - 1) / LS_T + (a.offsets ? a.groups : 0);
    if (n_tiles * row_tiles > 0x7fffffffll) return DASS_ERR_UNSUPPORTED;
    const unsigned grid = (unsigned)(n_tiles * row_tiles);
    const bool y_vec = rows_vec_ok(a.Y, a.ldy, a.bf16);
    if (a.bf16) {
        if (a.W_up) linear_simt_kernel<true, true><<<grid, LS_THREADS, 0, a.st>>>(a, n_tiles, y_vec);
        else linear_simt_kernel<true, false><<<grid, LS_THREADS, 0, a.st>>>(a, n_tiles, y_vec);
    } else {
        if (a.W_up) linear_simt_kernel<false, true><<<grid, LS_THREADS, 0, a.st>>>(a, n_tiles, y_vec);
        else linear_simt_kernel<false, false><<<grid, LS_THREADS, 0, a.st>>>(a, n_tiles, y_vec);
    }
    return cudaGetLastError() == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

}  // namespace dass
