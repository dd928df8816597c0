// Quantisation of rows or weights to microscaled 4-bit values, and back.
//
// A block of 32 consecutive values of a row shares the scale 2^(s - 127), s = max(0, floor(log2 max|x|) - 2 + 127): the
// exponent that puts the largest value into e2m1's top binade [4, 8).  With a the bits of max|x| that is
// max(0, (a >> 23) - 2), no logarithm needed.  x 2^(127 - s) is exact up to values that round to zero anyway; one
// conversion rounds it to the nearest code, ties to even, beyond 6 to 6.
//
// Four lanes share a block, 8 values (16 bytes of bf16) to a lane, so a warp reads 256 consecutive values of a row, and of
// four rows at a time.  Scales go to tiles of 128 rows x 4 blocks (the order in which the tensor cores take them); the
// four scales of a row in a tile are one word, put together by two shuffles.
//
// Bound by the memory.
#include "mx4_common.cuh"
#include "rows_common.cuh"

namespace dass {

constexpr int MQ_THREADS = 128;
constexpr int MQ_ROWS = 4;           // rows of a warp
constexpr int MQ_COLS = 256;         // columns of a warp

// Two floats to two codes each, four pairs: v[0] in the lowest bits.
__device__ __forceinline__ uint32_t mx4_encode8(const float (&v)[8])
{
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}

// 8 values of a row from column c on; absent ones are zero.
template <bool BF16, bool VECTOR>
__device__ __forceinline__ void mq_load8(const void *X, int64_t row, int64_t c, int64_t K, float (&v)[8])
{
    if (VECTOR && c + 8 <= K) {
        if constexpr (BF16) {
            row_load<true, 8>(X, row + c, v);
        } else {
            float a[4], b[4];
            row_load<false, 4>(X, row + c, a);
            row_load<false, 4>(X, row + c + 4, b);
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float x[1] = {0.f};
        if (c + i < K) row_load<BF16, 1>(X, row + c + i, x);
        v[i] = x[0];
    }
}

template <bool BF16, bool VECTOR>
__global__ void __launch_bounds__(MQ_THREADS)
mx4_quantize_kernel(const void *__restrict__ X, int64_t rows, int64_t K, int64_t ldx, int64_t group_stride,
                    uint8_t *__restrict__ codes, uint8_t *__restrict__ scales, int col_chunks, int64_t row_chunks, int64_t chunks)
{
    const int64_t chunk = (int64_t)blockIdx.x * (MQ_THREADS / 32) + (threadIdx.x >> 5);
    if (chunk >= chunks) return;
    const int lane = threadIdx.x & 31;
    const int64_t across = chunk / col_chunks;
    const int64_t g = across / row_chunks, r0 = (across - g * row_chunks) * MQ_ROWS;
    const int64_t c = (chunk - across * col_chunks) * MQ_COLS + lane * 8;
    const int64_t pitch = mx4_pitch(K), k_tiles = mx4_k_tiles(K);
    uint8_t *const gcodes = codes + g * rows * pitch;
    uint8_t *const gscales = scales + g * mx4_row_tiles(rows) * k_tiles * MX4_TILE_BYTES;
    float v[MQ_ROWS][8];
#pragma unroll
    for (int i = 0; i < MQ_ROWS; ++i) {
        if (r0 + i < rows) {
            mq_load8<BF16, VECTOR>(X, g * group_stride + (r0 + i) * ldx, c, K, v[i]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < MQ_ROWS; ++i) {
        const int64_t r = r0 + i;
        uint32_t most = 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(v[i][j]) & 0x7fffffffu);
        most = max(most, __shfl_xor_sync(FULL_MASK, most, 1));
        most = max(most, __shfl_xor_sync(FULL_MASK, most, 2));
        const uint32_t e = most >> 23;
        const uint32_t s = e == 255u ? 255u : e > 2u ? e - 2u : 0u;
        const float up = s == 255u ? 0.f : __uint_as_float((254u - s) << 23);
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = s == 255u ? 0.f : v[i][j] * up;
        const uint32_t packed = mx4_encode8(y);
        if (r < rows && c < pitch * 2) DASS_ST(reinterpret_cast<uint32_t *>(gcodes + r * pitch + c / 2), packed);
        uint32_t word = s << (8 * ((lane >> 2) & 3));
        word |= __shfl_xor_sync(FULL_MASK, word, 4);
        word |= __shfl_xor_sync(FULL_MASK, word, 8);
        if ((lane & 15) == 0 && c < k_tiles * MX4_TILE_K)
            DASS_ST(reinterpret_cast<uint32_t *>(gscales + mx4_scale_word(r, c / MX4_TILE_K, k_tiles)), word);
    }
}

template <bool BF16, bool VECTOR>
__global__ void __launch_bounds__(MQ_THREADS)
mx4_dequantize_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, int64_t rows, int64_t K,
                      void *__restrict__ Y, int64_t ldy, int64_t group_stride, int col_chunks, int64_t row_chunks, int64_t chunks)
{
    const int64_t chunk = (int64_t)blockIdx.x * (MQ_THREADS / 32) + (threadIdx.x >> 5);
    if (chunk >= chunks) return;
    const int lane = threadIdx.x & 31;
    const int64_t across = chunk / col_chunks;
    const int64_t g = across / row_chunks, r0 = (across - g * row_chunks) * MQ_ROWS;
    const int64_t c = (chunk - across * col_chunks) * MQ_COLS + lane * 8;
    const int64_t pitch = mx4_pitch(K), k_tiles = mx4_k_tiles(K);
    const uint8_t *const gcodes = codes + g * rows * pitch;
    const uint8_t *const gscales = scales + g * mx4_row_tiles(rows) * k_tiles * MX4_TILE_BYTES;
    if (c >= K) return;
    uint32_t x[MQ_ROWS], s[MQ_ROWS];
#pragma unroll
    for (int i = 0; i < MQ_ROWS; ++i) {
        const int64_t r = r0 + i;
        x[i] = r < rows ? DASS_LD_CS(reinterpret_cast<const uint32_t *>(gcodes + r * pitch + c / 2)) : 0u;
        s[i] = r < rows ? DASS_LD(gscales + mx4_scale_word(r, c / MX4_TILE_K, k_tiles) + ((c / MX4_BLOCK) & 3)) : 0u;
    }
#pragma unroll
    for (int i = 0; i < MQ_ROWS; ++i) {
        const int64_t r = r0 + i, at = g * group_stride + r * ldy + c;
        if (r >= rows) break;
        float v[8];
        mx4_decode8_f32(x[i], mx4_scale(s[i]), v);
        if (VECTOR && c + 8 <= K) {
            if constexpr (BF16) {
                row_store<true, 8>(Y, at, v);
            } else {
                const float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
                row_store<false, 4>(Y, at, a);
                row_store<false, 4>(Y, at + 4, b);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float one[1] = {v[j]};
                if (c + j < K) row_store<BF16, 1>(Y, at + j, one);
            }
        }
    }
}

static dass_status mq_check(int64_t groups, int64_t rows, int64_t K, int64_t ld, int64_t group_stride, int dt)
{
    if (dt != DASS_BF16 && dt != DASS_F32) return DASS_ERR_DTYPE;
    if (groups < 1 || rows < 0 || K < 1 || ld < K || (groups > 1 && rows > 0 && group_stride < (rows - 1) * ld + K)) return DASS_ERR_SHAPE;
    const int64_t lim = 0x7fffffffll - 512;
    if (rows > lim || K > lim || groups > lim) return DASS_ERR_UNSUPPORTED;
    return DASS_OK;
}

struct MqGrid { int col_chunks; int64_t row_chunks, chunks; unsigned blocks; };
// False where there are more warps than a grid holds.
static bool mq_grid(int64_t groups, int64_t padded_rows, int64_t K, MqGrid &q)
{
    q.col_chunks = (int)((K + MQ_COLS - 1) / MQ_COLS);
    q.row_chunks = (padded_rows + MQ_ROWS - 1) / MQ_ROWS;
    if (q.row_chunks > (int64_t)0x7fffffff * (MQ_THREADS / 32) / q.col_chunks / groups) return false;
    q.chunks = groups * q.row_chunks * q.col_chunks;
    q.blocks = (unsigned)((q.chunks + MQ_THREADS / 32 - 1) / (MQ_THREADS / 32));
    return true;
}

}  // namespace dass

using namespace dass;

extern "C" {

dass_status dass_mx4_bytes(int64_t rows, int64_t K, size_t *codes, size_t *scales)
{
    if (!codes && !scales) return DASS_ERR_NULL;
    if (rows < 0 || K < 1) return DASS_ERR_SHAPE;
    const int64_t lim = 0x7fffffffll - 512;
    if (rows > lim || K > lim) return DASS_ERR_UNSUPPORTED;
    if (codes) *codes = (size_t)mx4_codes_bytes(rows, K);
    if (scales) *scales = (size_t)mx4_scales_bytes(rows, K);
    return DASS_OK;
}

dass_status dass_mx4_quantize(const void *X, int64_t groups, int64_t rows, int64_t K, int64_t ldx, int64_t group_stride, dass_dtype dt,
                              uint8_t *codes, uint8_t *scales, void *cuda_stream)
{
    if (rows > 0 && (!X || !codes || !scales)) return DASS_ERR_NULL;
    const dass_status cs = mq_check(groups, rows, K, ldx, group_stride, (int)dt);
    if (cs != DASS_OK) return cs;
    const bool bf16 = dt == DASS_BF16;
    if (!elem_aligned(X, bf16) || (reinterpret_cast<uintptr_t>(codes) & 15u) || (reinterpret_cast<uintptr_t>(scales) & 15u)) return DASS_ERR_ALIGN;
    if (rows == 0) return DASS_OK;
    MqGrid q;
    if (!mq_grid(groups, mx4_row_tiles(rows) * MX4_TILE_ROWS, K, q)) return DASS_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const int64_t stride = groups > 1 ? group_stride : 0;
    DASS_BOUNDS_SCOPE(bs);
    DASS_BOUNDS_ADD(bs, X, ((size_t)(groups - 1) * stride + (size_t)(rows - 1) * ldx + K) * (bf16 ? 2 : 4));
    DASS_BOUNDS_ADD(bs, codes, (size_t)groups * mx4_codes_bytes(rows, K));
    DASS_BOUNDS_ADD(bs, scales, (size_t)groups * mx4_scales_bytes(rows, K));
    DASS_BOUNDS_COMMIT(bs, st);
    const bool vec = rows_vec_ok(X, ldx, bf16) && (groups == 1 || stride % (bf16 ? 8 : 4) == 0);
    auto go = [&](auto kernel) { kernel<<<q.blocks, MQ_THREADS, 0, st>>>(X, rows, K, ldx, stride, codes, scales, q.col_chunks, q.row_chunks, q.chunks); };
    if (bf16) vec ? go(mx4_quantize_kernel<true, true>) : go(mx4_quantize_kernel<true, false>);
    else vec ? go(mx4_quantize_kernel<false, true>) : go(mx4_quantize_kernel<false, false>);
    return cudaGetLastError() == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

dass_status dass_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t groups, int64_t rows, int64_t K,
                                void *Y, int64_t ldy, int64_t group_stride, dass_dtype dt, void *cuda_stream)
{
    if (rows > 0 && (!Y || !codes || !scales)) return DASS_ERR_NULL;
    const dass_status cs = mq_check(groups, rows, K, ldy, group_stride, (int)dt);
    if (cs != DASS_OK) return cs;
    const bool bf16 = dt == DASS_BF16;
    if (!elem_aligned(Y, bf16) || (reinterpret_cast<uintptr_t>(codes) & 15u) || (reinterpret_cast<uintptr_t>(scales) & 15u)) return DASS_ERR_ALIGN;
    if (rows == 0) return DASS_OK;
    MqGrid q;
    if (!mq_grid(groups, rows, K, q)) return DASS_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const int64_t stride = groups > 1 ? group_stride : 0;
    DASS_BOUNDS_SCOPE(bs);
    DASS_BOUNDS_ADD(bs, Y, ((size_t)(groups - 1) * stride + (size_t)(rows - 1) * ldy + K) * (bf16 ? 2 : 4));
    DASS_BOUNDS_ADD(bs, codes, (size_t)groups * mx4_codes_bytes(rows, K));
    DASS_BOUNDS_ADD(bs, scales, (size_t)groups * mx4_scales_bytes(rows, K));
    DASS_BOUNDS_COMMIT(bs, st);
    const bool vec = rows_vec_ok(Y, ldy, bf16) && (groups == 1 || stride % (bf16 ? 8 : 4) == 0);
    auto go = [&](auto kernel) { kernel<<<q.blocks, MQ_THREADS, 0, st>>>(codes, scales, rows, K, Y, ldy, stride, q.col_chunks, q.row_chunks, q.chunks); };
    if (bf16) vec ? go(mx4_dequantize_kernel<true, true>) : go(mx4_dequantize_kernel<true, false>);
    else vec ? go(mx4_dequantize_kernel<false, true>) : go(mx4_dequantize_kernel<false, false>);
    return cudaGetLastError() == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

}  // extern "C"
