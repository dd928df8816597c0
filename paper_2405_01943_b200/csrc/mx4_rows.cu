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
// Bound by the memory: a 28672 x 8192 matrix in bf16 101 us (5.88 TB/s of 6.57), back 98 us (6.09).  With 64-bit divisions for a
// warp's place it took 276 us, with bounds tested at every access 141, with six blocks to an SM instead of eight 111, with the
// decoding of single floats 142 back.  Rows that are not 16-byte aligned change lanes through shared memory: 3001 x 1001 f32
// 5.1 us, 4.4 back (element by element 8.4 and 19.0).
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

// MQ_ROWS rows of 8 values a lane.  INSIDE: all rows and columns exist and are read 16 bytes at a time.
template <bool BF16, bool VECTOR, bool INSIDE>
__device__ __forceinline__ void mq_encode(const char *src, int64_t row_bytes, int64_t c0, int64_t rows, int64_t K, int lane, float *turn,
                                          uint8_t *codes, int64_t pitch, uint8_t *scales, int64_t scale_cols)
{
    constexpr int ES = BF16 ? 2 : 4;
    const int64_t c = c0 + lane * 8;
    MqRaw<BF16, VECTOR> raw[MQ_ROWS];
#pragma unroll
    for (int i = 0; i < MQ_ROWS; ++i) {
        const char *row = src + i * row_bytes;
        if constexpr (INSIDE) {
            constexpr int W = ROW_VEC<BF16>;
#pragma unroll
            for (int j = 0; j < 8 / W; ++j) raw[i].piece[j].w = DASS_LD_CS(reinterpret_cast<const uint4 *>(row + (lane * 8 + j * W) * ES));
        } else {
            mq_load<BF16, VECTOR>(raw[i], row - c0 * ES, 0, c0, lane, i < rows ? K : 0);
        }
    }
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
            s = mq_scale(max(most >> 23, (most >> 7) & 255u));
            const uint32_t up = s == 255u ? 0u : (254u - s) * 0x00800080u;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t p = mul_bf16x2(w[j], up);
                y[2 * j] = __uint_as_float(p << 16);
                y[2 * j + 1] = __uint_as_float(p & 0xffff0000u);
            }
        } else {
            float v[8];
            mq_floats<BF16, VECTOR>(raw[i], turn, lane, v);
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
        if (INSIDE || (i < rows && c < pitch * 2)) DASS_ST_CS(reinterpret_cast<uint32_t *>(codes + i * pitch), packed);
        uint32_t word = s << (8 * ((lane >> 2) & 3));
        word |= __shfl_xor_sync(FULL_MASK, word, 4);
        word |= __shfl_xor_sync(FULL_MASK, word, 8);
        if ((lane & 15) == 0 && (INSIDE || c < scale_cols)) DASS_ST(reinterpret_cast<uint32_t *>(scales + i * 16), word);   // the four rows' slots are neighbours
    }
}

template <bool BF16, bool VECTOR>
__global__ void __launch_bounds__(MQ_THREADS, VECTOR ? 8 : 4)
mx4_quantize_kernel(const void *__restrict__ X, int64_t rows, int64_t K, int64_t ldx, int64_t group_stride,
                    uint8_t *__restrict__ codes, uint8_t *__restrict__ scales, const MqGrid q)
{
    constexpr int ES = BF16 ? 2 : 4;
    __shared__ __align__(16) float turn[VECTOR ? 1 : MQ_WARPS][VECTOR ? 4 : MQ_COLS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float *const mine = turn[VECTOR ? 0 : warp];
    const int64_t c0 = ((int64_t)blockIdx.x * q.across + (warp & (q.across - 1))) * MQ_COLS, c = c0 + lane * 8;
    const int64_t pitch = mx4_pitch(K), k_tiles = mx4_k_tiles(K);
    const int64_t first = (int64_t)blockIdx.y * (MQ_WARPS / q.across) + warp / q.across, step = (int64_t)gridDim.y * (MQ_WARPS / q.across);
    for (int64_t g = blockIdx.z; g < q.groups; g += gridDim.z) {
        const char *src = static_cast<const char *>(X) + (g * group_stride + first * MQ_ROWS * ldx + c0) * ES;
        uint8_t *dst = codes + (g * rows + first * MQ_ROWS) * pitch + c / 2;
        uint8_t *const gscales = scales + (g * mx4_row_tiles(rows) * k_tiles + c / MX4_TILE_K) * MX4_TILE_BYTES;
        for (int64_t rg = first; rg < q.row_groups; rg += step, src += step * MQ_ROWS * ldx * ES, dst += step * MQ_ROWS * pitch) {
            uint8_t *const word = gscales + mx4_scale_word(rg * MQ_ROWS, 0, k_tiles);
            if (VECTOR && c0 + MQ_COLS <= K && rg * MQ_ROWS + MQ_ROWS <= rows)
                mq_encode<BF16, VECTOR, VECTOR>(src, ldx * ES, c0, MQ_ROWS, K, lane, mine, dst, pitch, word, k_tiles * MX4_TILE_K);
            else
                mq_encode<BF16, VECTOR, false>(src, ldx * ES, c0, rows - rg * MQ_ROWS, K, lane, mine, dst, pitch, word, k_tiles * MX4_TILE_K);
        }
    }
}

// The four rows again, decoded.  INSIDE as above, for Y.
template <bool BF16, bool VECTOR, bool INSIDE>
__device__ __forceinline__ void mq_decode(const uint8_t *codes, int64_t pitch, const uint8_t *scales, int64_t c0, int64_t rows, int64_t K, int lane,
                                          float *turn, char *dst, int64_t row_bytes)
{
    constexpr int ES = BF16 ? 2 : 4;
    const int64_t c = c0 + lane * 8;
    uint32_t x[MQ_ROWS], s[MQ_ROWS];
#pragma unroll
    for (int i = 0; i < MQ_ROWS; ++i) {
        const bool in = INSIDE || (i < rows && c < K);
        x[i] = in ? DASS_LD_CS(reinterpret_cast<const uint32_t *>(codes + i * pitch)) : 0u;
        s[i] = in ? DASS_LD(scales + i * 16) : 0u;
    }
#pragma unroll
    for (int i = 0; i < MQ_ROWS; ++i) {
        if (!INSIDE && i >= rows) break;
        char *const row = dst + i * row_bytes;                         // column c0
        // every value is a bf16 number, or past the range of f32 as well
        uint32_t w[4];
        mx4_decode8(x[i], mx4_factor(s[i]), mx4_two(s[i]), w);
        const uint32_t pairs[4] = {__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410), __byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632)};
        uint4 *const at = reinterpret_cast<uint4 *>(row + lane * 8 * ES);
        if constexpr (VECTOR && BF16) {
            if (INSIDE || c + 8 <= K) {
                DASS_ST_CS(at, make_uint4(pairs[0], pairs[1], pairs[2], pairs[3]));
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < K) DASS_ST(reinterpret_cast<uint16_t *>(at) + j, (uint16_t)(pairs[j / 2] >> (16 * (j & 1))));
            }
        } else {
            uint32_t v[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) { v[2 * j] = pairs[j] << 16; v[2 * j + 1] = pairs[j] & 0xffff0000u; }
            if constexpr (VECTOR) {
                if constexpr (INSIDE) {
                    // a lane's 32 bytes in two accesses would be half a sector each: neighbours swap, and write a sector together
                    uint32_t mine[4], theirs[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        mine[j] = lane & 1 ? v[4 + j] : v[j];
                        theirs[j] = __shfl_xor_sync(FULL_MASK, lane & 1 ? v[j] : v[4 + j], 1);
                    }
                    uint4 *const pair = reinterpret_cast<uint4 *>(row + (lane & ~1) * 8 * ES) + (lane & 1);
                    DASS_ST_CS(pair, lane & 1 ? make_uint4(theirs[0], theirs[1], theirs[2], theirs[3]) : make_uint4(mine[0], mine[1], mine[2], mine[3]));
                    DASS_ST_CS(pair + 2, lane & 1 ? make_uint4(mine[0], mine[1], mine[2], mine[3]) : make_uint4(theirs[0], theirs[1], theirs[2], theirs[3]));
                } else if (c + 8 <= K) {
                    DASS_ST(at, make_uint4(v[0], v[1], v[2], v[3]));
                    DASS_ST(at + 1, make_uint4(v[4], v[5], v[6], v[7]));
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (c + j < K) DASS_ST(reinterpret_cast<uint32_t *>(at) + j, v[j]);
                }
            } else {
                *reinterpret_cast<uint4 *>(turn + lane * 8) = make_uint4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<uint4 *>(turn + lane * 8 + 4) = make_uint4(v[4], v[5], v[6], v[7]);
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t one = __float_as_uint(turn[j * 32 + lane]);
                    if (c0 + j * 32 + lane >= K) continue;
                    if constexpr (BF16) DASS_ST(reinterpret_cast<uint16_t *>(row) + j * 32 + lane, (uint16_t)(one >> 16));
                    else DASS_ST(reinterpret_cast<uint32_t *>(row) + j * 32 + lane, one);
                }
                __syncwarp();
            }
        }
    }
}

template <bool BF16, bool VECTOR>
__global__ void __launch_bounds__(MQ_THREADS, 8)
mx4_dequantize_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, int64_t rows, int64_t K,
                      void *__restrict__ Y, int64_t ldy, int64_t group_stride, const MqGrid q)
{
    constexpr int ES = BF16 ? 2 : 4;
    __shared__ __align__(16) float turn[VECTOR ? 1 : MQ_WARPS][VECTOR ? 4 : MQ_COLS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float *const mine = turn[VECTOR ? 0 : warp];
    const int64_t c0 = ((int64_t)blockIdx.x * q.across + (warp & (q.across - 1))) * MQ_COLS, c = c0 + lane * 8;
    const int64_t pitch = mx4_pitch(K), k_tiles = mx4_k_tiles(K);
    const int64_t first = (int64_t)blockIdx.y * (MQ_WARPS / q.across) + warp / q.across, step = (int64_t)gridDim.y * (MQ_WARPS / q.across);
    for (int64_t g = blockIdx.z; g < q.groups; g += gridDim.z) {
        char *dst = static_cast<char *>(Y) + (g * group_stride + first * MQ_ROWS * ldy + c0) * ES;
        const uint8_t *src = codes + (g * rows + first * MQ_ROWS) * pitch + c / 2;
        const uint8_t *const gscales = scales + (g * mx4_row_tiles(rows) * k_tiles + c / MX4_TILE_K) * MX4_TILE_BYTES + ((c / MX4_BLOCK) & 3);
        for (int64_t rg = first; rg < q.row_groups; rg += step, src += step * MQ_ROWS * pitch, dst += step * MQ_ROWS * ldy * ES) {
            const uint8_t *const byte = gscales + mx4_scale_word(rg * MQ_ROWS, 0, k_tiles);
            if (VECTOR && c0 + MQ_COLS <= K && rg * MQ_ROWS + MQ_ROWS <= rows)
                mq_decode<BF16, VECTOR, VECTOR>(src, pitch, byte, c0, MQ_ROWS, K, lane, mine, dst, ldy * ES);
            else
                mq_decode<BF16, VECTOR, false>(src, pitch, byte, c0, rows - rg * MQ_ROWS, K, lane, mine, dst, ldy * ES);
        }
    }
}

int device_sm_count();   // dass_abi.cu

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
    const int64_t x = (chunks + q.across - 1) / q.across, z = groups < 65535 ? groups : 65535;
    int64_t y = (q.row_groups + MQ_WARPS / q.across - 1) / (MQ_WARPS / q.across);
    const int64_t turns = x * y * z / (32 * (int64_t)device_sm_count());   // a block's set-up is spread over up to 8 groups of rows
    y = (y + (turns < 1 ? 1 : turns < 8 ? turns : 8) - 1) / (turns < 1 ? 1 : turns < 8 ? turns : 8);
    return dim3((unsigned)x, (unsigned)(y < 65535 ? y : 65535), (unsigned)z);
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
