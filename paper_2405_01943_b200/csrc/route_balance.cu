// The router's balance loss, the experts' loads, and the gradient.
//
// With n tokens that have a choice, c_e choices of expert e, p_t the softmax of token t's unmasked logits:
//     P_e = 1/n sum_t p_te,   f_e = c_e / (n k),   loss = E sum_e f_e P_e,   dloss/dl_te = E/n p_te (f_e - sum_i f_i p_ti).
//
// A token's row is held by a group of L lanes in 16-byte pieces that are dealt out in turn, so a lane has the same columns
// of every token it meets: the column sums stay in its registers over all of its tokens, and nothing but the row's
// maximum and sum crosses lanes.  At the end the groups of a block add up, then the 8 blocks of a cluster, which
// writes one row of partial sums, and a second kernel adds the rows, all in a fixed order.  Small calls are one cluster and
// one launch.  Choices are counted in shared memory; integer sums do not depend on their order.  Sums of probabilities are in
// f32: a mean over 65536 tokens is off by 1.3e-7 of itself at most; added up in 64 bits, f32 probabilities leave 0.6e-7.
//
// Bound by latency: 65536 x 128 f32, k = 8 18.8 us for the loss (its bytes: 5.4), of which the second kernel takes 3.7, and 14.0
// for the gradient (10.5): four rounds of loads, softmax and sums a warp.  Loads taken one by one 52, a row's loads together
// and a round ahead 31, whole rows without column checks and two blocks to an SM 19.6; 8 columns a lane instead of 16, for
// more warps, 20.3; faster exponentials 18.0 (not taken: 2 to 3 times the error).  4096 x 8 4.4 us, one cluster (a second
// kernel over 128 rows at a time 12.6).
#include "linear_tc.cuh"

namespace dass {

constexpr int RB_THREADS = 512;            // of the loss
constexpr int RB_BACK_THREADS = 256;       // of the gradient
constexpr int RB_MAX_E = 1024;
constexpr int RB_MAX_K = 32;
constexpr int RB_BLOCKS = 296;             // at most: two to each of 148 SMs
constexpr int RB_CLUSTER = 8;              // blocks whose sums make one row

// -inf and NaN are masked (fmaxf drops a NaN); +inf counts as the largest finite value.
__device__ __forceinline__ float rb_logit(float x) { return fminf(fmaxf(x, -INFINITY), 3.402823466e38f); }

template <int L> __device__ __forceinline__ float rb_max(float v)
{
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(FULL_MASK, v, o));
    return v;
}
template <int L> __device__ __forceinline__ float rb_sum(float v)
{
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(FULL_MASK, v, o);
    return v;
}

// The column of a lane's element i * W + c.
template <int L, int W> __device__ __forceinline__ int rb_col(int gl, int i) { return (i * L + gl) * W; }

// FULL: the row has exactly the group's V L columns.  Else columns past E are absent.
// A row as it lies in memory, all of its loads in flight before the first is used; absent columns hold bits that
// rb_floats does not look at.
template <bool BF16, int W, int V> struct RbRow { RowRaw<BF16, W> piece[V / W]; RowRaw<BF16, 1> tail[W > 1 ? W : 1]; };

template <bool BF16, int W, int V, int L, bool FULL>
__device__ __forceinline__ void rb_load(RbRow<BF16, W, V> &r, const void *logits, int64_t row, int gl, int E)
{
#pragma unroll
    for (int i = 0; i < V / W; ++i) {
        const int e = rb_col<L, W>(gl, i);
        if (FULL || e + W <= E) raw_load<BF16, W>(r.piece[i], logits, row + e);
        else if (W > 1 && e < E) {                                     // the one ragged piece of the row
#pragma unroll
            for (int c = 0; c < W; ++c)
                if (e + c < E) raw_load<BF16, 1>(r.tail[W > 1 ? c : 0], logits, row + e + c);
        }
    }
}
// The row's masked logits; absent columns are -inf.
template <bool BF16, int W, int V, int L, bool FULL>
__device__ __forceinline__ void rb_floats(const RbRow<BF16, W, V> &r, int gl, int E, float (&x)[V])
{
#pragma unroll
    for (int i = 0; i < V / W; ++i) {
        const int e = rb_col<L, W>(gl, i);
        float v[W];
        raw_floats<BF16, W>(r.piece[i], v);
        if (!FULL && W > 1 && e < E && e + W > E) {
#pragma unroll
            for (int c = 0; c < W; ++c) {
                float one[1];
                raw_floats<BF16, 1>(r.tail[W > 1 ? c : 0], one);
                v[c] = one[0];
            }
        }
#pragma unroll
        for (int c = 0; c < W; ++c) x[i * W + c] = FULL || e + c < E ? rb_logit(v[c]) : -INFINITY;
    }
}

// x becomes exp(x - max), and the result is 1 / sum (0 for a row without unmasked logits).
template <int V, int L>
__device__ __forceinline__ float rb_softmax(float (&x)[V])
{
    float top = x[0];
#pragma unroll
    for (int i = 1; i < V; ++i) top = fmaxf(top, x[i]);
    top = rb_max<L>(top);
    top = top > -INFINITY ? top : 0.f;                               // nothing unmasked: every exponential is 0
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        x[i] = expf(x[i] - top);
        sum += x[i];
    }
    sum = rb_sum<L>(sum);
    return sum > 0.f ? 1.0f / sum : 0.f;
}

// A lane's choices of a token: j = gl, gl + L, ...
template <int L> constexpr int RB_IDS = L >= 8 ? RB_MAX_K / L : 4;     // held in registers; the others (of few lanes' tokens) are read when they are looked at
template <int L>
__device__ __forceinline__ void rb_load_ids(int (&id)[RB_IDS<L>], const int32_t *expert, int64_t t, int k, int gl, bool live)
{
#pragma unroll
    for (int i = 0; i < RB_IDS<L>; ++i) {
        id[i] = -1;
        if (i * L < k && live && gl + i * L < k) id[i] = DASS_LD(expert + t * k + gl + i * L);
    }
}
// Whether the token has a choice inside [0, E), for all lanes of its group; COUNT: the choices are counted too.
template <int L, bool COUNT>
__device__ __forceinline__ bool rb_chosen(const int (&id)[RB_IDS<L>], const int32_t *expert, int64_t t, int k, int E, int gl, bool live, int *count)
{
    bool any = false;
    auto look = [&](int e) {
        if (e >= 0 && e < E) {
            any = true;
            if (COUNT) atomicAdd(count + e, 1);
        }
    };
#pragma unroll
    for (int i = 0; i < RB_IDS<L>; ++i)
        if (i * L < k) look(id[i]);
    if (live)
        for (int j = gl + RB_IDS<L> * L; j < k; j += L) look(DASS_LD(expert + t * k + j));
    const unsigned group = (L == 32 ? FULL_MASK : ((1u << (L & 31)) - 1u)) << (threadIdx.x & 31 & ~(L - 1));
    return (__ballot_sync(FULL_MASK, any) & group) != 0u;
}

// loss, share and the last count from sums and counts; called by a whole block with both complete in shared memory.
__device__ __forceinline__ void rb_finish(const float *sum, const int *count, int E, int k, float *loss, int32_t *counts, float *share)
{
    __shared__ float parts[32];
    const int n = count[E];
    const float inverse = n > 0 ? 1.0f / (float)n : 0.f;
    float dot = 0.f;
    for (int e = threadIdx.x; e < E; e += blockDim.x) {
        const float P = sum[e] * inverse;
        DASS_ST(share + e, P);
        DASS_ST(counts + e, (int32_t)count[e]);
        dot += P * ((float)count[e] * inverse);
    }
    if (threadIdx.x == 0) DASS_ST(counts + E, (int32_t)n);
    dot = rb_sum<32>(dot);
    if ((threadIdx.x & 31) == 0) parts[threadIdx.x >> 5] = dot;
    __syncthreads();
    if (threadIdx.x == 0) {
        float total = 0.f;
        for (int w = 0; w < (int)blockDim.x / 32; ++w) total += parts[w];
        DASS_ST(loss, total * ((float)E / (float)k));
    }
}

// One row of partial sums and counts per cluster of blocks (partial null: the only cluster, whose first block finishes).
template <bool BF16, int W, int V, int L, bool FULL>
__global__ void __launch_bounds__(RB_THREADS, V <= 16 ? 2 : 1)
route_balance_kernel(const void *__restrict__ logits, int64_t T, int E, int64_t ld, int k, const int32_t *__restrict__ expert,
                     float *__restrict__ partial, int32_t *__restrict__ partial_counts, float *loss, int32_t *counts, float *share, int cluster)
{
    constexpr int TOKENS = RB_THREADS / L, WARPS = RB_THREADS / 32;
    extern __shared__ float rb_smem[];
    float *sums = rb_smem;                                          // [WARPS x E], then the block's in the first row
    int *count = reinterpret_cast<int *>(rb_smem + WARPS * E);      // [E + 1], then the cluster's
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gl = threadIdx.x & (L - 1);
    if (partial) grid_dependents_launch();                           // the second kernel may take its place and wait there
    for (int e = threadIdx.x; e <= E; e += RB_THREADS) count[e] = 0;
    __syncthreads();
    float acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.f;
    int seen = 0;
    const int rounds = (int)((T + TOKENS - 1) / TOKENS);            // every lane takes part in every round of its warp
    for (int r = blockIdx.x; r < rounds; r += gridDim.x) {
        const int64_t t = (int64_t)r * TOKENS + threadIdx.x / L;
        const bool live = t < T;
        RbRow<BF16, W, V> row;
        int id[RB_IDS<L>];
        float x[V];
        rb_load<BF16, W, V, L, FULL>(row, logits, (live ? t : 0) * ld, gl, E);
        rb_load_ids<L>(id, expert, t, k, gl, live);
        rb_floats<BF16, W, V, L, FULL>(row, gl, E, x);
        const bool in = rb_chosen<L, true>(id, expert, t, k, E, gl, live, count);
        const float inv = rb_softmax<V, L>(x) * (in ? 1.f : 0.f);   // a row past the last has no choice
        seen += in && gl == 0;
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = fmaf(x[i], inv, acc[i]);
    }
    // over the groups of a warp, then over the warps, then over the cluster's blocks, in order
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int o = L; o < 32; o <<= 1) acc[i] += __shfl_xor_sync(FULL_MASK, acc[i], o);
    }
    if (lane < L) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = rb_col<L, W>(gl, i / W) + i % W;
            if (e < E) sums[warp * E + e] = acc[i];
        }
    }
    if (seen) atomicAdd(count + E, seen);
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += RB_THREADS) {
        float s = sums[e];
#pragma unroll
        for (int w = 1; w < WARPS; ++w) s += sums[w * E + e];
        sums[e] = s;
    }
    __syncwarp();                                                    // the cluster barrier wants whole warps
    if (cluster > 1) cluster_sync_all(); else __syncthreads();
    const int rank = (int)(blockIdx.x % cluster);
    const int64_t out = blockIdx.x / cluster;
    const uint32_t sums_addr = smem_u32(sums), count_addr = smem_u32(count);
    // the cluster's blocks share the columns of its row, or the first block has them all
    const int from = partial ? threadIdx.x + rank * RB_THREADS : rank == 0 ? threadIdx.x : 2 * E + 1, by = partial ? cluster * RB_THREADS : RB_THREADS;
    for (int e = from; cluster > 1 && e < 2 * E + 1; e += by) {
        if (e < E) {
            float v[RB_CLUSTER], s = 0.f;                            // all loads in flight, then their sum in order
#pragma unroll
            for (int r = 0; r < RB_CLUSTER; ++r) v[r] = r < cluster ? ld_cluster(map_to_cta(sums_addr + 4 * e, r)) : 0.f;
#pragma unroll
            for (int r = 0; r < RB_CLUSTER; ++r) s += v[r];
            if (partial) DASS_ST(partial + out * E + e, s);
            else sums[E + e] = s;                                    // the second warp's place: a block has several
        } else {
            int v[RB_CLUSTER], c = 0;
#pragma unroll
            for (int r = 0; r < RB_CLUSTER; ++r) v[r] = r < cluster ? __float_as_int(ld_cluster(map_to_cta(count_addr + 4 * (e - E), r))) : 0;
#pragma unroll
            for (int r = 0; r < RB_CLUSTER; ++r) c += v[r];
            if (partial) DASS_ST(partial_counts + out * (E + 1) + e - E, (int32_t)c);
            else count[E + 1 + e - E] = c;                           // past the block's own
        }
    }
    __syncwarp();
    if (cluster > 1) cluster_sync_all();                             // the others may still read this block's sums
    if (!partial && rank == 0) {
        if (cluster > 1) rb_finish(sums + E, count + E + 1, E, k, loss, counts, share);
        else rb_finish(sums, count, E, k, loss, counts, share);
    }
}

// Rows that the second kernel reads at a time, each by E of its 1024 threads.
__host__ __device__ __forceinline__ int rb_deep(int E, int rows) { return 1024 / E < rows ? 1024 / E : rows; }

// The rows of partial sums added up.
__global__ void __launch_bounds__(1024)
route_balance_finish_kernel(const float *__restrict__ partial, const int32_t *__restrict__ partial_counts, int rows, int E, int k,
                            float *loss, int32_t *counts, float *share)
{
    extern __shared__ float rb_smem[];
    grid_dependency_wait();                                          // the partial sums
    const int lanes = E, deep = rb_deep(E, rows);
    float *sums = rb_smem;                                           // [deep x E]
    int *count = reinterpret_cast<int *>(rb_smem + deep * E);        // [deep x (E + 1)]
    const int d = threadIdx.x / lanes, e = threadIdx.x - d * lanes;
    if (d < deep) {
        float s = 0.f;
        int c = 0, n = 0;
#pragma unroll 8
        for (int r = d; r < rows; r += deep) {
            s += DASS_LD(partial + (int64_t)r * E + e);
            c += DASS_LD(partial_counts + (int64_t)r * (E + 1) + e);
            if (e == 0) n += DASS_LD(partial_counts + (int64_t)r * (E + 1) + E);
        }
        sums[d * E + e] = s;
        count[d * (E + 1) + e] = c;
        if (e == 0) count[d * (E + 1) + E] = n;
    }
    __syncthreads();
    if (threadIdx.x < lanes) {
        for (int i = 1; i < deep; ++i) { sums[e] += sums[i * E + e]; count[e] += count[i * (E + 1) + e]; }
    }
    if (threadIdx.x == 0)
        for (int i = 1; i < deep; ++i) count[E] += count[i * (E + 1) + E];
    __syncthreads();
    rb_finish(sums, count, E, k, loss, counts, share);
}

// dlogits = add + dloss * E/n p (f - sum f p); 0 + add for tokens without a choice.
template <bool BF16, int W, int V, int L, bool FULL>
__global__ void __launch_bounds__(RB_BACK_THREADS, V <= 16 ? 4 : 2)
route_balance_backward_kernel(const void *__restrict__ logits, int64_t T, int E, int64_t ld, int k, const int32_t *__restrict__ expert,
                              const int32_t *__restrict__ counts, const float *__restrict__ dloss, const void *add, int64_t lda,
                              void *dlogits, int64_t ldd)
{
    constexpr int TOKENS = RB_BACK_THREADS / L;
    const int gl = threadIdx.x & (L - 1);
    const int n = DASS_LD(counts + E);
    const float inverse = n > 0 ? 1.0f / (float)n : 0.f;
    const float factor = (dloss ? DASS_LD(dloss) : 1.0f) * (float)E * inverse;
    float f[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = rb_col<L, W>(gl, i / W) + i % W;
        f[i] = e < E ? (float)DASS_LD(counts + e) * inverse / (float)k : 0.f;
    }
    const int rounds = (int)((T + TOKENS - 1) / TOKENS);
    for (int r = blockIdx.x; r < rounds; r += gridDim.x) {
        const int64_t t = (int64_t)r * TOKENS + threadIdx.x / L;
        const bool live = t < T;
        RbRow<BF16, W, V> row;
        int id[RB_IDS<L>];
        float x[V];
        rb_load<BF16, W, V, L, FULL>(row, logits, (live ? t : 0) * ld, gl, E);
        rb_load_ids<L>(id, expert, t, k, gl, live);
        rb_floats<BF16, W, V, L, FULL>(row, gl, E, x);
        const bool in = rb_chosen<L, false>(id, expert, t, k, E, gl, live, nullptr);
        const float inv = rb_softmax<V, L>(x);
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) dot = fmaf(x[i], f[i], dot);
        dot = rb_sum<L>(dot) * inv;
        if (!live) continue;
        const float g = in ? factor * inv : 0.f;
#pragma unroll
        for (int i = 0; i < V / W; ++i) {
            const int e = rb_col<L, W>(gl, i);
            float y[W];
#pragma unroll
            for (int c = 0; c < W; ++c) y[c] = in ? g * x[i * W + c] * (f[i * W + c] - dot) : 0.f;
            if (FULL || e + W <= E) {
                if (add) {
                    float a[W];
                    row_load<BF16, W>(add, t * lda + e, a);
#pragma unroll
                    for (int c = 0; c < W; ++c) y[c] += a[c];
                }
                row_store<BF16, W>(dlogits, t * ldd + e, y);
            } else {
#pragma unroll
                for (int c = 0; c < W; ++c) {
                    if (e + c >= E) continue;
                    float a[1] = {0.f};
                    if (add) row_load<BF16, 1>(add, t * lda + e + c, a);
                    const float one[1] = {y[c] + a[0]};
                    row_store<BF16, 1>(dlogits, t * ldd + e + c, one);
                }
            }
        }
    }
}

struct BalanceArgs {
    const void *logits; int64_t T; int E; int64_t ld; int k; const int32_t *expert;
    float *partial; int32_t *partial_counts; float *loss; int32_t *counts; float *share;              // forward
    const int32_t *load; const float *dloss; const void *add; int64_t lda; void *dlogits; int64_t ldd;   // backward (dlogits not null)
    bool vector; int blocks, cluster; cudaStream_t st;
};

int device_sm_count();   // dass_abi.cu

// Blocks that share T tokens.  Up to three rounds each of one cluster's blocks are done sooner than a second kernel; else
// enough to fill the SMs, in clusters whose blocks add up, which leaves the second kernel few rows.
static int rb_blocks(int64_t T, int64_t E)
{
    const int64_t lanes = E <= 8 ? 1 : E <= 16 ? 2 : E <= 32 ? 4 : E <= 128 ? 8 : E <= 256 ? 16 : 32;
    const int64_t rounds = (T * lanes + RB_THREADS - 1) / RB_THREADS;
    if (rounds <= 3 * RB_CLUSTER) return rounds >= 8 ? 8 : rounds >= 4 ? 4 : rounds >= 2 ? 2 : 1;
    return (int)((rounds < RB_BLOCKS ? rounds : RB_BLOCKS) / RB_CLUSTER * RB_CLUSTER);
}
static int rb_cluster(int blocks) { return blocks < RB_CLUSTER ? blocks : RB_CLUSTER; }

template <bool BF16, int W, int V, int L, bool FULL>
static cudaError_t rb_go(const BalanceArgs &a)
{
    if (a.dlogits) {
        constexpr int TOKENS = RB_BACK_THREADS / L;
        const int64_t rounds = (a.T + TOKENS - 1) / TOKENS, most = 8 * (int64_t)device_sm_count();
        route_balance_backward_kernel<BF16, W, V, L, FULL><<<(unsigned)(rounds < most ? rounds : most), RB_BACK_THREADS, 0, a.st>>>(
            a.logits, a.T, a.E, a.ld, a.k, a.expert, a.load, a.dloss, a.add, a.lda, a.dlogits, a.ldd);
        return cudaGetLastError();
    }
    const size_t smem = ((size_t)(RB_THREADS / 32) * a.E + 2 * (a.E + 1)) * 4;   // at most 72 KB
    if (smem > 47 * 1024) {                                                      // E above 668; rb_finish's static 128 bytes count too
        static DeviceMask configured{0ull};                                      // per device
        const cudaError_t e = ensure_dynamic_smem(route_balance_kernel<BF16, W, V, L, FULL>, 72 * 1024 + 8, configured);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.blocks);
    cfg.blockDim = dim3(RB_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = a.st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)a.cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, route_balance_kernel<BF16, W, V, L, FULL>, a.logits, a.T, a.E, a.ld, a.k, a.expert, a.partial, a.partial_counts,
                              a.loss, a.counts, a.share, a.cluster);
}
template <bool BF16, int W, int V, int L>
static cudaError_t rb_launch(const BalanceArgs &a)
{
    return a.E == V * L ? rb_go<BF16, W, V, L, true>(a) : rb_go<BF16, W, V, L, false>(a);
}
template <bool BF16, bool VECTOR>
static cudaError_t rb_pick(const BalanceArgs &a)
{
    constexpr int W = VECTOR ? ROW_VEC<BF16> : 1;
    if (a.E <= 8) return rb_launch<BF16, W, 8, 1>(a);
    if (a.E <= 16) return rb_launch<BF16, W, 8, 2>(a);
    if (a.E <= 32) return rb_launch<BF16, W, 8, 4>(a);
    if (a.E <= 64) return rb_launch<BF16, W, 8, 8>(a);
    if (a.E <= 128) return rb_launch<BF16, W, 16, 8>(a);
    if (a.E <= 256) return rb_launch<BF16, W, 16, 16>(a);
    if (a.E <= 512) return rb_launch<BF16, W, 16, 32>(a);
    return rb_launch<BF16, W, 32, 32>(a);
}
static cudaError_t rb_dispatch(const BalanceArgs &a, bool bf16)
{
    if (bf16) return a.vector ? rb_pick<true, true>(a) : rb_pick<true, false>(a);
    return a.vector ? rb_pick<false, true>(a) : rb_pick<false, false>(a);
}

static dass_status rb_check(int64_t T, int64_t E, int64_t ld, int dt, int64_t k)
{
    if (dt != DASS_BF16 && dt != DASS_F32) return DASS_ERR_DTYPE;
    if (T < 0 || E < 1 || ld < E || k < 1) return DASS_ERR_SHAPE;
    if (E > RB_MAX_E || k > RB_MAX_K || T > ((1ll << 31) - 1) / k) return DASS_ERR_UNSUPPORTED;   // counts are 32 bits
    return DASS_OK;
}
static size_t rb_workspace(int64_t T, int64_t E)
{
    const int blocks = rb_blocks(T, E);
    return blocks > RB_CLUSTER ? (size_t)(blocks / RB_CLUSTER) * (2 * E + 1) * 4 : 0;
}

}  // namespace dass

using namespace dass;

extern "C" {

dass_status dass_route_balance_workspace_bytes(int64_t T, int64_t E, size_t *bytes)
{
    if (!bytes) return DASS_ERR_NULL;
    if (T < 0 || E < 1) return DASS_ERR_SHAPE;
    if (E > RB_MAX_E || T > (1ll << 31) - 1) return DASS_ERR_UNSUPPORTED;
    *bytes = rb_workspace(T, E);
    return DASS_OK;
}

dass_status dass_route_balance(const void *logits, int64_t T, int64_t E, int64_t ld, dass_dtype dt, const int32_t *expert, int64_t k,
                               float *loss, int32_t *counts, float *share, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    if (!loss || !counts || !share || (T > 0 && (!logits || !expert))) return DASS_ERR_NULL;
    const dass_status cs = rb_check(T, E, ld, (int)dt, k);
    if (cs != DASS_OK) return cs;
    const bool bf16 = dt == DASS_BF16;
    if (!elem_aligned(logits, bf16) || !elem_aligned(expert, false) || !elem_aligned(loss, false) || !elem_aligned(counts, false) ||
        !elem_aligned(share, false) || (reinterpret_cast<uintptr_t>(workspace) & 15u))
        return DASS_ERR_ALIGN;
    const size_t need = rb_workspace(T, E);
    if (need && (!workspace || workspace_bytes < need)) return DASS_ERR_WORKSPACE;
    BalanceArgs a{};
    a.logits = logits; a.T = T; a.E = (int)E; a.ld = ld; a.k = (int)k; a.expert = expert;
    a.loss = loss; a.counts = counts; a.share = share;
    a.blocks = rb_blocks(T, E);
    a.cluster = rb_cluster(a.blocks);
    const int partial_rows = a.blocks / a.cluster;
    a.vector = rows_vec_ok(logits, ld, bf16);
    a.st = static_cast<cudaStream_t>(cuda_stream);
    if (a.blocks > RB_CLUSTER) {
        a.partial = static_cast<float *>(workspace);
        a.partial_counts = reinterpret_cast<int32_t *>(a.partial + (int64_t)partial_rows * E);
    }
    DASS_BOUNDS_SCOPE(bs);
    if (T > 0) {
        DASS_BOUNDS_ADD(bs, logits, ((size_t)(T - 1) * ld + E) * (bf16 ? 2 : 4));
        DASS_BOUNDS_ADD(bs, expert, (size_t)T * k * 4);
    }
    DASS_BOUNDS_ADD(bs, loss, 4);
    DASS_BOUNDS_ADD(bs, counts, (size_t)(E + 1) * 4);
    DASS_BOUNDS_ADD(bs, share, (size_t)E * 4);
    DASS_BOUNDS_ADD(bs, workspace, need);
    DASS_BOUNDS_COMMIT(bs, a.st);
    if (rb_dispatch(a, bf16) != cudaSuccess) return DASS_ERR_CUDA;
    if (a.blocks > RB_CLUSTER) {
        const int deep = rb_deep((int)E, partial_rows);
        if (launch_dependent(route_balance_finish_kernel, dim3(1), dim3(1024), (size_t)deep * (2 * E + 1) * 4, a.st, (const float *)a.partial,
                             (const int32_t *)a.partial_counts, partial_rows, (int)E, (int)k, loss, counts, share) != cudaSuccess)
            return DASS_ERR_CUDA;
    }
    return DASS_OK;
}

dass_status dass_route_balance_backward(const void *logits, int64_t T, int64_t E, int64_t ld, dass_dtype dt, const int32_t *expert, int64_t k,
                                        const int32_t *counts, const float *dloss, const void *add, int64_t lda,
                                        void *dlogits, int64_t ldd, void *cuda_stream)
{
    if (!counts || (T > 0 && (!logits || !expert || !dlogits))) return DASS_ERR_NULL;
    const dass_status cs = rb_check(T, E, ld, (int)dt, k);
    if (cs != DASS_OK) return cs;
    if (ldd < E || (add && lda < E)) return DASS_ERR_SHAPE;
    const bool bf16 = dt == DASS_BF16;
    if (!elem_aligned(logits, bf16) || !elem_aligned(dlogits, bf16) || !elem_aligned(add, bf16) || !elem_aligned(expert, false) ||
        !elem_aligned(counts, false) || !elem_aligned(dloss, false))
        return DASS_ERR_ALIGN;
    if (T == 0) return DASS_OK;
    BalanceArgs a{};
    a.logits = logits; a.T = T; a.E = (int)E; a.ld = ld; a.k = (int)k; a.expert = expert;
    a.load = counts; a.dloss = dloss; a.add = add; a.lda = lda; a.dlogits = dlogits; a.ldd = ldd;
    a.vector = rows_vec_ok(logits, ld, bf16) && rows_vec_ok(dlogits, ldd, bf16) && (!add || rows_vec_ok(add, lda, bf16));
    a.st = static_cast<cudaStream_t>(cuda_stream);
    DASS_BOUNDS_SCOPE(bs);
    DASS_BOUNDS_ADD(bs, logits, ((size_t)(T - 1) * ld + E) * (bf16 ? 2 : 4));
    DASS_BOUNDS_ADD(bs, expert, (size_t)T * k * 4);
    DASS_BOUNDS_ADD(bs, counts, (size_t)(E + 1) * 4);
    DASS_BOUNDS_ADD(bs, dloss, 4);
    DASS_BOUNDS_ADD(bs, add, ((size_t)(T - 1) * lda + E) * (bf16 ? 2 : 4));
    DASS_BOUNDS_ADD(bs, dlogits, ((size_t)(T - 1) * ldd + E) * (bf16 ? 2 : 4));
    DASS_BOUNDS_COMMIT(bs, a.st);
    return rb_dispatch(a, bf16) == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

}  // extern "C"
