// dass_linear_mx4 for few rows (a decode step): every weight is read once, 4.25 bits of it, and meets at most 32 rows of X,
// given in bf16 or in 4 bits.
//
// A block of 8 or 16 warps owns MT * 16 weight rows (columns of Y); the warps take k in turns of 128.  A lane loads 16 bytes of
// codes of a weight row, which are the 32 k of one scale, and decodes them in registers to bf16 fragments of mma.m16n8k16.
// A dot product may take its k in any order as long as both sides agree: a word of 8 codes gives pairs (p, p + 4), since
// those are 16 bits apart, and the rows of X are paired the same way (one byte permutation a word; rows in 4 bits come out
// of the same decoding).  A cluster of SPLIT blocks shares the columns and splits k further where there are few columns;
// sums over the warps and the cluster's blocks are taken in a fixed order.
//
// 32 weight rows a block (MT = 2) halve the traffic of X from L2, which in bf16 has four times the bytes of a weight's.
//
// Bound by the decoding, 17 instructions for 8 codes in a thread: 5400 weights a ns (8 experts of 4096 x 14336 gated, 32 rows:
// 174 us where the bytes take 76 and mx4_mid.cu 84), and for small products by the launch and the latency of a few turns:
// 1 x 4096 x 4096 6.8 us (the bytes: 1.4), 1 x 1000 x 689 3.5 us.
#include "linear_tc.cuh"
#include "mx4_linear.cuh"
#include "tc_pair.cuh"

namespace dass {

constexpr int MF_STEP = 128;         // k of a warp's turn: a scale tile

__device__ __forceinline__ void mma_bf16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 8 elements of a bf16 row from k on; elements at and past K read as zero (and are not touched).
__device__ __forceinline__ uint4 mf_load8(const uint16_t *row, int64_t k, int64_t K)
{
    if (k + 8 <= K) return DASS_LD_G(reinterpret_cast<const uint4 *>(row + k));
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (k + i < K) w[i >> 1] |= (uint32_t)DASS_LD(row + k + i) << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// NT: rows of X in eights; MT: weight rows in sixteens; XQ: X in 4 bits; WARPS of a block.  Grid: SPLIT x column tiles x row tiles, clusters
// of SPLIT along x.
template <int NT, int MT, bool GLU, bool XQ, int WARPS>
__global__ void __launch_bounds__(WARPS * 32)
mx4_few_kernel(const Mx4Args p, int col_tiles, int split)
{
    constexpr int M = GLU ? 2 : 1, THREADS = WARPS * 32;
    constexpr int COLS = MT * 16;
    constexpr int SUMS = M * COLS * NT * 8;
    __shared__ float part[WARPS][SUMS];
    __shared__ float sum[SUMS];
    const LinearArgs &a = p.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, q = lane & 3;
    const int64_t block = blockIdx.x / split;
    const int rank = blockIdx.x - (int)block * split;
    lin_zero_outside<true>(a.offsets, a.groups, a.T, a.N, a.Y, a.ldy, false, (int64_t)blockIdx.x * THREADS + threadIdx.x,
                           (int64_t)gridDim.x * THREADS);
    const LinTile tile = lin_find_tile(a.offsets, a.groups, a.T, NT * 8, block / col_tiles);
    if (tile.g < 0) return;                                  // the whole cluster
    const int64_t n0 = (block % col_tiles) * COLS;
    const int64_t pitch = mx4_pitch(a.K), k_tiles = mx4_k_tiles(a.K);

    const uint8_t *w[M][MT][2], *ws[M][MT][2];               // this lane's rows of codes and of scales
#pragma unroll
    for (int m = 0; m < M; ++m) {
        const Mx4Matrix mat = mx4_group(m ? p.up : p.w, tile.g, a.N, a.K);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {                    // rows past the last column are read as the last: never stored
                const int64_t at = n0 + 16 * i + 8 * h + g, n = at < a.N ? at : a.N - 1;
                w[m][i][h] = mat.codes + n * pitch + q * 16;
                ws[m][i][h] = mat.scales + mx4_scale_word(n, 0, k_tiles) + q;
            }
    }
    const uint16_t *x[NT];
    const uint8_t *xc[NT], *xs[NT];
    bool has[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int64_t t = tile.lo + i * 8 + g;
        has[i] = t < tile.hi;
        if constexpr (XQ) {
            xc[i] = p.x.codes + t * pitch + q * 16;
            xs[i] = p.x.scales + mx4_scale_word(t, 0, k_tiles) + q;
        } else {
            x[i] = static_cast<const uint16_t *>(a.X) + t * a.ldx + q * 32;
        }
    }
    float acc[M][MT][NT][4];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int j = 0; j < MT; ++j)
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[m][j][i][c] = 0.f;

    for (int64_t kt = rank * WARPS + warp; kt < k_tiles; kt += split * WARPS) {
        const int64_t k0 = kt * MF_STEP;
        const bool inside = k0 + q * 32 < a.K;                // this lane's block of 32
        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
        uint4 wv[M][MT][2];
        uint32_t sv[M][MT][2];
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int j = 0; j < MT; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    wv[m][j][h] = inside ? DASS_LD_CS(reinterpret_cast<const uint4 *>(w[m][j][h] + kt * 64)) : zero;
                    sv[m][j][h] = inside ? DASS_LD_CS(ws[m][j][h] + kt * MX4_TILE_BYTES) : 0u;
                }
        uint4 xv[NT][XQ ? 1 : 4];
        uint32_t xsv[NT];
        bool two = false;                                    // some scale above 2: see mx4_factor
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            xsv[i] = 0u;
            if constexpr (XQ) {
                xv[i][0] = has[i] && inside ? DASS_LD_G(reinterpret_cast<const uint4 *>(xc[i] + kt * 64)) : zero;
                xsv[i] = has[i] && inside ? DASS_LD_G(xs[i] + kt * MX4_TILE_BYTES) : 0u;
                two |= mx4_two(xsv[i]);
            } else {
#pragma unroll
                for (int s = 0; s < 4; ++s) xv[i][s] = has[i] ? mf_load8(x[i], k0 + s * 8, a.K - q * 32) : zero;
            }
        }
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int j = 0; j < MT; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) two |= mx4_two(sv[m][j][h]);
        two = __any_sync(FULL_MASK, two);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            uint32_t b[NT][4];
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                if constexpr (XQ) {
                    const uint32_t c = s == 0 ? xv[i][0].x : s == 1 ? xv[i][0].y : s == 2 ? xv[i][0].z : xv[i][0].w;
                    mx4_decode8(c, mx4_factor(xsv[i]), two, b[i]);
                } else {
                    const uint4 v = xv[i][s];
                    b[i][0] = __byte_perm(v.x, v.z, 0x5410);
                    b[i][1] = __byte_perm(v.x, v.z, 0x7632);
                    b[i][2] = __byte_perm(v.y, v.w, 0x5410);
                    b[i][3] = __byte_perm(v.y, v.w, 0x7632);
                }
            }
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int j = 0; j < MT; ++j) {
                    uint32_t lo[4], hi[4];
                    const uint4 v0 = wv[m][j][0], v1 = wv[m][j][1];
                    mx4_decode8(s == 0 ? v0.x : s == 1 ? v0.y : s == 2 ? v0.z : v0.w, mx4_factor(sv[m][j][0]), two, lo);
                    mx4_decode8(s == 0 ? v1.x : s == 1 ? v1.y : s == 2 ? v1.z : v1.w, mx4_factor(sv[m][j][1]), two, hi);
#pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        mma_bf16_16816(acc[m][j][i], lo[0], hi[0], lo[1], hi[1], b[i][0], b[i][1]);
                        mma_bf16_16816(acc[m][j][i], lo[2], hi[2], lo[3], hi[3], b[i][2], b[i][3]);
                    }
                }
        }
    }
    // sum over the warps, then over the cluster's blocks
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int j = 0; j < MT; ++j)
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    part[warp][(m * NT * 8 + i * 8 + 2 * q + (c & 1)) * COLS + 16 * j + g + 8 * (c >> 1)] = acc[m][j][i][c];
    __syncthreads();
    for (int o = threadIdx.x; o < SUMS; o += THREADS) {
        float s = part[0][o];
#pragma unroll
        for (int v = 1; v < WARPS; ++v) s += part[v][o];
        sum[o] = s;
    }
    __syncwarp();                                            // the cluster barrier wants whole warps
    if (split > 1) cluster_sync_all(); else __syncthreads();
    const int rows = (int)(tile.hi - tile.lo);
    const uint32_t sum_addr = smem_u32(sum);
    for (int o = threadIdx.x + rank * THREADS; o < rows * COLS; o += split * THREADS) {
        const int64_t t = tile.lo + o / COLS, n = n0 + o % COLS;
        if (n >= a.N) continue;
        float s[M];
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int at = m * NT * 8 * COLS + o;
            if (split > 1) {
                s[m] = 0.f;
                for (int r = 0; r < split; ++r) s[m] += ld_cluster(map_to_cta(sum_addr + at * 4, r));
            } else {
                s[m] = sum[at];
            }
        }
        float b[1] = {0.f};
        if (a.bias) { row_load<true, 1>(a.bias, (int64_t)tile.g * a.N + n, b); s[0] += b[0]; }
        float y[1] = {s[0]};
        lt_act_all(y, a.act);
        if constexpr (GLU) {
            if (a.bias_up) { row_load<true, 1>(a.bias_up, (int64_t)tile.g * a.N + n, b); s[1] += b[0]; }
            y[0] *= s[1];
        }
        if (a.residual) { row_load<true, 1>(a.residual, t * a.ldr + n, b); y[0] += b[0]; }
        row_store<true, 1>(a.Y, t * a.ldy + n, y);
    }
    __syncwarp();
    if (split > 1) cluster_sync_all();                       // the others may still read this block's sums
}

template <int NT, int MT, bool GLU, bool XQ, int WARPS>
static cudaError_t mf_launch(const Mx4Args &p, int64_t row_tiles, int split)
{
    const int col_tiles = (int)((p.a.N + MT * 16 - 1) / (MT * 16));
    if (row_tiles * col_tiles * split > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(row_tiles * col_tiles * split));
    cfg.blockDim = dim3(WARPS * 32);
    cfg.stream = p.a.st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, mx4_few_kernel<NT, MT, GLU, XQ, WARPS>, p, col_tiles, split);
}
template <int MT, bool GLU, bool XQ>
static cudaError_t mf_one(const Mx4Args &p, int64_t row_tiles, int split)
{
    if (mx4_few_warps(p.a.K, 1, split) == 16) return mf_launch<1, MT, GLU, XQ, 16>(p, row_tiles, split);
    return mf_launch<1, MT, GLU, XQ, 8>(p, row_tiles, split);
}
template <bool GLU, bool XQ>
static cudaError_t mf_pick(const Mx4Args &p, int64_t row_tiles, int nt, int mt, int split)
{
    if (nt == 1) return mt == 2 ? mf_one<2, GLU, XQ>(p, row_tiles, split) : mf_one<1, GLU, XQ>(p, row_tiles, split);
    if (nt == 2) return mf_launch<2, 1, GLU, XQ, 8>(p, row_tiles, split);
    return mf_launch<4, 1, GLU, XQ, 8>(p, row_tiles, split);
}

// nt: rows of X in eights (1, 2 or 4); mt: weight rows in sixteens (2 only with nt 1); split: blocks that share the contraction
dass_status mx4_few_launch(const Mx4Args &p, int nt, int mt, int split)
{
    const int64_t row_tiles = p.a.offsets ? p.a.T / (8 * nt) + lin_active_groups(p.a) : (p.a.T + 8 * nt - 1) / (8 * nt);
    const bool glu = p.up.codes != nullptr, xq = p.x.codes != nullptr;
    cudaError_t e;
    if (glu) e = xq ? mf_pick<true, true>(p, row_tiles, nt, mt, split) : mf_pick<true, false>(p, row_tiles, nt, mt, split);
    else e = xq ? mf_pick<false, true>(p, row_tiles, nt, mt, split) : mf_pick<false, false>(p, row_tiles, nt, mt, split);
    return e == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

}  // namespace dass
