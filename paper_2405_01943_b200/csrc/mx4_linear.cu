// C ABI of the matrix product with 4-bit weights: validation and dispatch.  See include/dass.h.
#include "mx4_linear.cuh"

namespace dass {

dass_status mx4_few_launch(const Mx4Args &p, int eights, int sixteens, int split);     // mx4_few.cu
dass_status mx4_tc_launch(const Mx4Args &p, int columns);                              // mx4_tc.cu
dass_status mx4_wide_launch(const Mx4Args &p, int rows);                               // mx4_wide.cu
int device_sm_count();                                                                 // dass_abi.cu

}  // namespace dass

using namespace dass;

extern "C" {

dass_status dass_linear_mx4(const void *X, int64_t ldx, const uint8_t *x_codes, const uint8_t *x_scales, int64_t T, int64_t K,
                            const uint8_t *w_codes, const uint8_t *w_scales, const uint8_t *up_codes, const uint8_t *up_scales, int64_t N,
                            const void *bias, const void *bias_up, dass_act act, const void *residual, int64_t ldr,
                            void *Y, int64_t ldy, const int32_t *offsets, int64_t groups, void *cuda_stream)
{
    if (act != DASS_ACT_SILU && act != DASS_ACT_GELU_TANH && act != DASS_ACT_RELU && act != DASS_ACT_NONE) return DASS_ERR_DTYPE;
    if (!w_codes || !w_scales || !up_codes != !up_scales || !x_codes != !x_scales || (bias_up && !up_codes)) return DASS_ERR_NULL;
    if (T > 0 && ((!X && !x_codes) || !Y)) return DASS_ERR_NULL;
    if (X && x_codes) return DASS_ERR_UNSUPPORTED;
    if (T < 0 || K < 1 || N < 1 || (X && ldx < K) || ldy < N || (residual && ldr < N)) return DASS_ERR_SHAPE;
    if (groups < 1 || (!offsets && groups != 1)) return DASS_ERR_SHAPE;
    auto whole = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; };
    if (!whole(X) || !whole(x_codes) || !whole(x_scales) || !whole(w_codes) || !whole(w_scales) || !whole(up_codes) || !whole(up_scales) ||
        (X && ldx % 8))
        return DASS_ERR_ALIGN;
    if (!elem_aligned(bias, true) || !elem_aligned(bias_up, true) || !elem_aligned(residual, true) || !elem_aligned(Y, true) ||
        !elem_aligned(offsets, false))
        return DASS_ERR_ALIGN;
    const int64_t lim = 0x7fffffffll - 512;                // 32-bit tile coordinates
    const int64_t most_rows = 1ll << 28;                   // so are sums of tile counts, whatever the offsets hold
    if (T > most_rows || K > lim || N > lim || groups > LIN_MAX_GROUPS) return DASS_ERR_UNSUPPORTED;
    if (T == 0) return DASS_OK;

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
    DASS_BOUNDS_COMMIT(bs, p.a.st);
    if (x_codes && T > 32) return mx4_tc_launch(p, 256);
    if (!x_codes && T > 64) return mx4_wide_launch(p, up_codes ? 128 : 256);
    const int64_t want = lin_rows_wanted(p.a), blocks = (N + 31) / 32 * lin_active_groups(p.a);
    const int nt = want <= 8 ? 1 : want <= 16 ? 2 : 4;
    int split = 1;
    while (split < 8 && blocks * split < device_sm_count() && K >= 1024 * split) split *= 2;
    return mx4_few_launch(p, nt, nt == 1 ? 2 : 1, split);
}

}  // extern "C"
