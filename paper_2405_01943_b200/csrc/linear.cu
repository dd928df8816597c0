// C ABI of the matrix product with an epilogue: validation and dispatch.  See include/dass.h.
#include <atomic>

#include "linear_common.cuh"

namespace dass {

dass_status linear_simt_launch(const LinearArgs &a);       // linear_simt.cu
dass_status linear_tc_launch(const LinearArgs &a);         // linear_tc.cu

__device__ int g_linear_status = 0;      // DASS_OK or DASS_ERR_TIMEOUT; read and cleared through dass_linear_status

// Address of the record on the current device (looked up once per device).
int *linear_status_word()
{
    static std::atomic<int *> cached[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return nullptr;
    int *p = dev < 64 ? cached[dev].load(std::memory_order_relaxed) : nullptr;
    if (p) return p;
    void *addr = nullptr;
    if (cudaGetSymbolAddress(&addr, g_linear_status) != cudaSuccess) return nullptr;
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
    return bf16 ? linear_tc_launch(a) : linear_simt_launch(a);
}

dass_status dass_linear_status(void *cuda_stream)
{
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    int *word = linear_status_word();
    int host = 0;
    if (!word || cudaMemcpyAsync(&host, word, sizeof(int), cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaMemsetAsync(word, 0, sizeof(int), st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess)
        return DASS_ERR_CUDA;
    return host == 0 ? DASS_OK : DASS_ERR_TIMEOUT;
}

}  // extern "C"
