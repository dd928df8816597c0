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

constexpr int MQ_WARPS = 4;
constexpr int MQ_THREADS = MQ_WARPS * 32;
constexpr int MQ_ROWS = 4;           // rows of a warp
constexpr int MQ_COLS = 256;         // columns of a warp

// A block's warps lie side by side along the columns, or, where a row is shorter, over each other: `across` (1, 2 or 4) of
// them side by side.  grid.x columns, grid.y rows, grid.z matrices; the last two wrap around.
struct MqGrid { int across; int64_t row_groups, groups; };

// 8 values of a lane as they lie in memory: 16-byte pieces where rows allow them; else single elements, 32 consecutive ones to
// an access of the warp, that change lanes through shared memory (mq_turn).
template <bool BF16, bool VECTOR> struct MqRaw { RowRaw<BF16, VECTOR ? ROW_VEC<BF16> : 1> piece[VECTOR ? 8 / ROW_VEC<BF16> : 8]; };

template <bool BF16, bool VECTOR>
__device__ __forceinline__ void mq_load(MqRaw<BF16, VECTOR> &r, const void *X, int64_t row, int64_t c0, int lane, int64_t K)
{
    constexpr int W = VECTOR ? ROW_VEC<BF16> : 1;
#pragma unroll
    for (int i = 0; i < 8 / W; ++i) {
        const int64_t c = VECTOR ? c0 + lane * 8 + i * W : c0 + i * 32 + lane;
        if (c + W <= K) {
            raw_load<BF16, W, true>(r.piece[i], X, row + c);
        } else if constexpr (W == 1) {
            r.piece[i].w = 0;
        } else {                                                       // a row that ends inside the piece
            uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int j = 0; j < W; ++j) {
                if (c + j >= K) continue;
                if constexpr (BF16) w[j / 2] |= (uint32_t)DASS_LD(static_cast<const uint16_t *>(X) + row + c + j) << (16 * (j & 1));
                else w[j] = DASS_LD(static_cast<const uint32_t *>(X) + row + c + j);
            }
            r.piece[i].w = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}
// The lane's 8 consecutive values.
template <bool BF16, bool VECTOR>
__device__ __forceinline__ void mq_floats(const MqRaw<BF16, VECTOR> &r, float *turn, int lane, float (&v)[8])
{
    constexpr int W = VECTOR ? ROW_VEC<BF16> : 1;
    if constexpr (VECTOR) {
#pragma unroll
        for (int i = 0; i < 8 / W; ++i) {
            float x[W];
            raw_floats<BF16, W>(r.piece[i], x);
#pragma unroll
            for (int j = 0; j < W; ++j) v[i * W + j] = x[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float x[1];
            raw_floats<BF16, 1>(r.piece[i], x);
            turn[i * 32 + lane] = x[0];
        }
        __syncwarp();
        const float4 a = *reinterpret_cast<const float4 *>(turn + lane * 8), b = *reinterpret_cast<const float4 *>(turn + lane * 8 + 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        __syncwarp();
    }
}

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// The scale of a block from its largest value's exponent field: 255 where it holds a NaN or an infinity.
__device__ __forceinline__ uint32_t mq_scale(uint32_t e) { return e == 255u ? 255u : e > 2u ? e - 2u : 0u; }

template <bool BF16, bool VECTOR>
__global__ void __launch_bounds__(MQ_THREADS)
mx4_quantize_kernel(const void *__restrict__ X, int64_t rows, int64_t K, int64_t ldx, int64_t group_stride,
                    uint8_t *__restrict__ codes, uint8_t *__restrict__ scales, const MqGrid q)
{
    __shared__ float turn[VECTOR ? 1 : MQ_WARPS][VECTOR ? 4 : MQ_COLS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c0 = ((int64_t)blockIdx.x * q.across + (warp & (q.across - 1))) * MQ_COLS, c = c0 + lane * 8;
    const int64_t pitch = mx4_pitch(K), k_tiles = mx4_k_tiles(K);
    const int64_t first = (int64_t)blockIdx.y * (MQ_WARPS / q.across) + warp / q.across;
    for (int64_t g = blockIdx.z; g < q.groups; g += gridDim.z)
        for (int64_t rg = first; rg < q.row_groups; rg += (int64_t)gridDim.y * (MQ_WARPS / q.across)) {
            const int64_t r0 = rg * MQ_ROWS;
            uint8_t *const gcodes = codes + (g * rows + r0) * pitch + c / 2;
            uint8_t *const gscales = scales + g * mx4_row_tiles(rows) * k_tiles * MX4_TILE_BYTES + mx4_scale_word(r0, c / MX4_TILE_K, k_tiles);
            MqRaw<BF16, VECTOR> raw[MQ_ROWS];
#pragma unroll
            for (int i = 0; i < MQ_ROWS; ++i)
                mq_load<BF16, VECTOR>(raw[i], X, g * group_stride + (r0 + i) * ldx, c0, lane, r0 + i < rows ? K : 0);
#pragma unroll
            for (int i = 0; i < MQ_ROWS; ++i) {
                uint32_t s;
                float y[8];
                if constexpr (BF16 && VECTOR) {
                    // two values to a word: maximum and product by a power of two of both halves at once
                    const uint32_t w[4] = {raw[i].piece[0].w.x, raw[i].piece[0].w.y, raw[i].piece[0].w.z, raw[i].piece[0].w.w};
                    uint32_t most = max_u16x2(max_u16x2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), max_u16x2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
                    most = max_u16x2(most, __shfl_xor_sync(FULL_MASK, most, 1));
                    most = max_u16x2(most, __shfl_xor_sync(FULL_MASK, most, 2));
                    const uint32_t e = max(most >> 23, (most >> 7) & 255u);
                    s = mq_scale(e);
                    const uint32_t up = e == 255u ? 0u : (254u - s) * 0x00800080u;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t p = mul_bf16x2(w[j], up);
                        y[2 * j] = __uint_as_float(p << 16);
                        y[2 * j + 1] = __uint_as_float(p & 0xffff0000u);
                    }
                } else {
                    float v[8];
                    mq_floats<BF16, VECTOR>(raw[i], turn[VECTOR ? 0 : warp], lane, v);
                    uint32_t most = 0u;
#pragma unroll
                    for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(v[j]) & 0x7fffffffu);
                    most = max(most, __shfl_xor_sync(FULL_MASK, most, 1));
                    most = max(most, __shfl_xor_sync(FULL_MASK, most, 2));
                    s = mq_scale(most >> 23);
                    const float up = __uint_as_float((254u - s) << 23);
#pragma unroll
                    for (int j = 0; j < 8; ++j) y[j] = v[j] * up;
                }
                const uint32_t packed = s == 255u ? 0u : mx4_encode8(y);
                if (r0 + i < rows && c < pitch * 2) DASS_ST_CS(reinterpret_cast<uint32_t *>(gcodes + i * pitch), packed);
                uint32_t word = s << (8 * ((lane >> 2) & 3));
                word |= __shfl_xor_sync(FULL_MASK, word, 4);
                word |= __shfl_xor_sync(FULL_MASK, word, 8);
                if ((lane & 15) == 0 && c < k_tiles * MX4_TILE_K) DASS_ST(reinterpret_cast<uint32_t *>(gscales + i * 16), word);   // the four rows' slots are neighbours
            }
        }
}

template <bool BF16, bool VECTOR>
__global__ void __launch_bounds__(MQ_THREADS)
mx4_dequantize_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, int64_t rows, int64_t K,
                      void *__restrict__ Y, int64_t ldy, int64_t group_stride, const MqGrid q)
{
    __shared__ float turn[VECTOR ? 1 : MQ_WARPS][VECTOR ? 4 : MQ_COLS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c0 = ((int64_t)blockIdx.x * q.across + (warp & (q.across - 1))) * MQ_COLS, c = c0 + lane * 8;
    const int64_t pitch = mx4_pitch(K), k_tiles = mx4_k_tiles(K);
    const int64_t first = (int64_t)blockIdx.y * (MQ_WARPS / q.across) + warp / q.across;
    for (int64_t g = blockIdx.z; g < q.groups; g += gridDim.z)
        for (int64_t rg = first; rg < q.row_groups; rg += (int64_t)gridDim.y * (MQ_WARPS / q.across)) {
            const int64_t r0 = rg * MQ_ROWS;
            const uint8_t *const gcodes = codes + (g * rows + r0) * pitch + c / 2;
            const uint8_t *const gscales = scales + g * mx4_row_tiles(rows) * k_tiles * MX4_TILE_BYTES + mx4_scale_word(r0, c / MX4_TILE_K, k_tiles) +
                                           ((c / MX4_BLOCK) & 3);
            uint32_t x[MQ_ROWS], s[MQ_ROWS];
#pragma unroll
            for (int i = 0; i < MQ_ROWS; ++i) {
                const bool in = r0 + i < rows && c < K;
                x[i] = in ? DASS_LD_CS(reinterpret_cast<const uint32_t *>(gcodes + i * pitch)) : 0u;
                s[i] = in ? DASS_LD(gscales + i * 16) : 0u;
            }
#pragma unroll
            for (int i = 0; i < MQ_ROWS; ++i) {
                if (r0 + i >= rows) break;
                const int64_t at = g * group_stride + (r0 + i) * ldy;
                // every value is a bf16 number, or past the range of f32 as well
                uint32_t w[4];
                mx4_decode8(x[i], mx4_factor(s[i]), mx4_two(s[i]), w);
                const uint32_t pairs[4] = {__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410), __byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632)};
                float v[8];
#pragma unroll
                for (int j = 0; j < 4; ++j) { v[2 * j] = __uint_as_float(pairs[j] << 16); v[2 * j + 1] = __uint_as_float(pairs[j] & 0xffff0000u); }
                if constexpr (VECTOR) {
                    if (c + 8 <= K) {
                        if constexpr (BF16) {
                            DASS_ST_CS(reinterpret_cast<uint4 *>(static_cast<uint16_t *>(Y) + at + c), make_uint4(pairs[0], pairs[1], pairs[2], pairs[3]));
                        } else {
                            const float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
                            row_store<false, 4>(Y, at + c, a);
                            row_store<false, 4>(Y, at + c + 4, b);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const float one[1] = {v[j]};
                            if (c + j < K) row_store<BF16, 1>(Y, at + c + j, one);
                        }
                    }
                } else {
                    float *const mine = turn[warp];
                    *reinterpret_cast<float4 *>(mine + lane * 8) = make_float4(v[0], v[1], v[2], v[3]);
                    *reinterpret_cast<float4 *>(mine + lane * 8 + 4) = make_float4(v[4], v[5], v[6], v[7]);
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float one[1] = {mine[j * 32 + lane]};
                        if (c0 + j * 32 + lane < K) row_store<BF16, 1>(Y, at + c0 + j * 32 + lane, one);
                    }
                    __syncwarp();
                }
            }
        }
}

static dass_status mq_check(int64_t groups, int64_t rows, int64_t K, int64_t ld, int64_t group_stride, int dt)
{
    if (dt != DASS_BF16 && dt != DASS_F32) return DASS_ERR_DTYPE;
    if (groups < 1 || rows < 0 || K < 1 || ld < K || (groups > 1 && rows > 0 && group_stride < (rows - 1) * ld + K)) return DASS_ERR_SHAPE;
    const int64_t lim = 0x7fffffffll - 512;
    if (rows > lim || K > lim || groups > lim || rows > (1ll << 48) / K / groups) return DASS_ERR_UNSUPPORTED;   // more than any memory holds
    return DASS_OK;
}

static dim3 mq_grid(int64_t groups, int64_t padded_rows, int64_t K, MqGrid &q)
{
    const int64_t chunks = (K + MQ_COLS - 1) / MQ_COLS;
    q.across = chunks >= 4 ? 4 : chunks >= 2 ? 2 : 1;
    q.row_groups = (padded_rows + MQ_ROWS - 1) / MQ_ROWS;
    q.groups = groups;
    const int64_t y = (q.row_groups + MQ_WARPS / q.across - 1) / (MQ_WARPS / q.across);
    return dim3((unsigned)((chunks + q.across - 1) / q.across), (unsigned)(y < 65535 ? y : 65535), (unsigned)(groups < 65535 ? groups : 65535));
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
    const dim3 grid = mq_grid(groups, mx4_row_tiles(rows) * MX4_TILE_ROWS, K, q);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const int64_t stride = groups > 1 ? group_stride : 0;
    DASS_BOUNDS_SCOPE(bs);
    DASS_BOUNDS_ADD(bs, X, ((size_t)(groups - 1) * stride + (size_t)(rows - 1) * ldx + K) * (bf16 ? 2 : 4));
    DASS_BOUNDS_ADD(bs, codes, (size_t)groups * mx4_codes_bytes(rows, K));
    DASS_BOUNDS_ADD(bs, scales, (size_t)groups * mx4_scales_bytes(rows, K));
    DASS_BOUNDS_COMMIT(bs, st);
    const bool vec = rows_vec_ok(X, ldx, bf16) && (groups == 1 || stride % (bf16 ? 8 : 4) == 0);
    auto go = [&](auto kernel) { kernel<<<grid, MQ_THREADS, 0, st>>>(X, rows, K, ldx, stride, codes, scales, q); };
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
    const dim3 grid = mq_grid(groups, rows, K, q);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const int64_t stride = groups > 1 ? group_stride : 0;
    DASS_BOUNDS_SCOPE(bs);
    DASS_BOUNDS_ADD(bs, Y, ((size_t)(groups - 1) * stride + (size_t)(rows - 1) * ldy + K) * (bf16 ? 2 : 4));
    DASS_BOUNDS_ADD(bs, codes, (size_t)groups * mx4_codes_bytes(rows, K));
    DASS_BOUNDS_ADD(bs, scales, (size_t)groups * mx4_scales_bytes(rows, K));
    DASS_BOUNDS_COMMIT(bs, st);
    const bool vec = rows_vec_ok(Y, ldy, bf16) && (groups == 1 || stride % (bf16 ? 8 : 4) == 0);
    auto go = [&](auto kernel) { kernel<<<grid, MQ_THREADS, 0, st>>>(codes, scales, rows, K, Y, ldy, stride, q); };
    if (bf16) vec ? go(mx4_dequantize_kernel<true, true>) : go(mx4_dequantize_kernel<true, false>);
    else vec ? go(mx4_dequantize_kernel<false, true>) : go(mx4_dequantize_kernel<false, false>);
    return cudaGetLastError() == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

}  // extern "C"
