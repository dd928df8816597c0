// What the kernels of dass_linear share: the arguments, the walk over groups of rows, the epilogue's arithmetic.
// Internal header.
#pragma once

#include "rows_common.cuh"

namespace dass {

constexpr int LIN_MAX_GROUPS = 1024;

struct LinearArgs {
    const void *X; int64_t T, K, ldx;
    const void *W, *W_up; int64_t N, ldw, group_stride;    // group g's matrix starts at W + g * group_stride
    const void *bias, *bias_up;                            // [groups x N], nullable
    const void *residual; int64_t ldr;                     // [T x N], nullable
    void *Y; int64_t ldy;
    const int32_t *offsets; int groups;                    // offsets null: one group of all T rows
    int act;
    bool bf16;
    cudaStream_t st;
};

// What the host can say about the groups, whose sizes only the device knows: how many have rows at most, and how many
// rows a tile should hold so that a group's weights are read once -- twice the average and a little, since a router does
// not spread its tokens evenly.
inline int64_t lin_active_groups(const LinearArgs &a) { return a.offsets ? (a.groups < a.T ? a.groups : a.T) : 1; }
inline int64_t lin_rows_wanted(const LinearArgs &a)
{
    const int64_t twice = a.offsets ? 2 * ((a.T + a.groups - 1) / a.groups) + 6 : a.T;
    return twice < a.T ? twice : a.T;
}

// Whether 8 bf16 columns of Y, of the residual and of a group's row of either bias are one aligned 16-byte access each.
// Row g of a bias [groups x N] begins g * N elements in: past the first group N decides, whichever bias is there.
inline bool lin_wide_ok(const LinearArgs &a)
{
    auto whole = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; };
    return rows_vec_ok(a.Y, a.ldy, true) && (!a.residual || rows_vec_ok(a.residual, a.ldr, true)) && whole(a.bias) && whole(a.bias_up) &&
           ((!a.bias && !a.bias_up) || a.groups == 1 || a.N % 8 == 0);
}

// Rows [lo, hi) of group g, whatever the offsets hold: never outside [0, T).
__device__ __forceinline__ void lin_group_rows(const int32_t *offsets, int g, int64_t T, int64_t &lo, int64_t &hi)
{
    if (!offsets) { lo = 0; hi = T; return; }
    const int64_t a = DASS_LD(offsets + g), b = DASS_LD(offsets + g + 1);
    lo = a < 0 ? 0 : (a > T ? T : a);
    hi = b < lo ? lo : (b > T ? T : b);
}

struct LinTile { int g; int64_t lo, hi; };                 // group, rows of the tile; g < 0: there is no such tile

// The index-th tile of `rows` rows when every group is cut into tiles by itself, groups in order.  Called by a whole warp.
__device__ __forceinline__ LinTile lin_find_tile(const int32_t *offsets, int groups, int64_t T, int rows, int64_t index)
{
    const int lane = threadIdx.x & 31;
    LinTile r{-1, 0, 0};
    for (int g0 = 0; g0 < groups; g0 += 32) {
        int64_t lo = 0, hi = 0;
        if (g0 + lane < groups) lin_group_rows(offsets, g0 + lane, T, lo, hi);
        const int tiles = (int)((hi - lo + rows - 1) / rows);
        int inc = tiles;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(FULL_MASK, inc, o);
            inc += lane >= o ? up : 0;
        }
        const unsigned past = __ballot_sync(FULL_MASK, index < inc);
        if (past) {
            const int src = __ffs(past) - 1;
            const int64_t at = lo + (index - (inc - tiles)) * rows;
            r.g = g0 + src;
            r.lo = __shfl_sync(FULL_MASK, at, src);
            r.hi = __shfl_sync(FULL_MASK, at + rows < hi ? at + rows : hi, src);
            return r;
        }
        index -= __shfl_sync(FULL_MASK, inc, 31);
    }
    return r;
}

// max(x, 0) that keeps NaN, as the other activations do (fmaxf gives the number where one side is NaN).
__device__ __forceinline__ float lin_relu(float x)
{
    float y;
    asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(y) : "f"(x));
    return y;
}

// The activation in f32, from accurate functions.
__device__ __forceinline__ float lin_act(float x, int act)
{
    switch (act) {
    case DASS_ACT_SILU: return x / (1.0f + expf(-x));
    case DASS_ACT_GELU_TANH: return 0.5f * x * (1.0f + tanhf(0.7978845608028654f * (x + 0.044715f * x * x * x)));
    case DASS_ACT_RELU: return lin_relu(x);
    default: return x;
    }
}

// Rows of no group are zero.  Strided over all threads of the grid.
template <bool BF16>
__device__ __forceinline__ void lin_zero_outside(const int32_t *offsets, int groups, int64_t T, int64_t N, void *Y, int64_t ldy, bool vec,
                                                 int64_t thread, int64_t threads)
{
    if (!offsets) return;
    int64_t first, last, ignore;
    lin_group_rows(offsets, 0, T, first, ignore);
    lin_group_rows(offsets, groups - 1, T, ignore, last);
    const int64_t outside = first + (T - last);
    const int64_t wide = vec ? N / ROW_VEC<BF16> : 0;              // whole accesses of a row, then single elements
    const int64_t per = wide + (N - wide * ROW_VEC<BF16>);
    for (int64_t i = thread; i < outside * per; i += threads) {
        const int64_t r = i / per, c = i - r * per;
        const int64_t at = (r < first ? r : last + r - first) * ldy;
        if (c < wide) {
            float zero[ROW_VEC<BF16>] = {};
            row_store<BF16, ROW_VEC<BF16>>(Y, at + c * ROW_VEC<BF16>, zero);
        } else {
            const float zero[1] = {0.f};
            row_store<BF16, 1>(Y, at + wide * ROW_VEC<BF16> + (c - wide), zero);
        }
    }
}

}  // namespace dass
