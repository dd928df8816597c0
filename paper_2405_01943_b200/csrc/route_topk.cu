// The router's selection: the k experts with the highest logits of every token, their softmax weights, and the gradient.
//
// A token's row is held in registers by a group of L lanes (a power of two), V consecutive logits to a lane, so a warp
// works on 32 / L tokens.  A logit becomes an unsigned key of the same order (masked: 0).  Its last log2(V L) bits give
// way to the index, lower indices above higher ones: keys are then unique.  Up to 8 of up to 256 experts: every lane sorts
// its 8 keys and log2 L merges of two lists leave the group's 8 largest in order.  Else each of k rounds is a maximum over
// the group and a compare that removes it.  For bf16 nothing is lost, the bits are empty.  For f32 two chosen logits, or a
// chosen one and one left out, that agree in all but those bits leave the order open: such a warp (one in about a hundred
// on random logits of 128 experts) repeats its tokens with whole keys, each round finding the lowest lane and element that
// hold the maximum.  Sums are in f32 and in a fixed order.
//
// Bound: with many tokens the selection by integer instructions (65536 x 128, k = 8: f32 28.7 us, bf16 23.5, where the bytes
// would take 5.8 and 3.2; rounds instead of sorted lists 31.5 and 28), the gradient by the latency of the choices' ids, then
// their logits (f32 15.9, bf16 12.0 over the chosen, 23.8 and 22.5 over all); with few the launch.
#include "rows_common.cuh"

namespace dass {

constexpr int RT_THREADS = 128;
constexpr int RT_MAX_E = 1024;
constexpr int RT_MAX_K = 32;

// Order-preserving key of a logit: 0 for a masked one (-inf, NaN); -0 and +0 are one value, +inf is the largest finite one.
__device__ __forceinline__ uint32_t rt_key(float x)
{
    if (!(x > -INFINITY)) return 0u;
    const uint32_t u = __float_as_uint(fminf(x, 3.402823466e38f) + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
// The logit a key stands for.
__device__ __forceinline__ float rt_value(uint32_t key)
{
    return __uint_as_float((key & 0x80000000u) ? (key ^ 0x80000000u) : ~key);
}

template <int L> __device__ __forceinline__ uint32_t group_max(uint32_t v)
{
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(FULL_MASK, v, o));
    return v;
}
template <int L> __device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(FULL_MASK, v, o);
    return v;
}

// V consecutive logits from element e0 of a row of E, as keys (absent ones are masked).
template <bool BF16, bool VECTOR, int V>
__device__ __forceinline__ void rt_load(const void *logits, int64_t row, int e0, int E, uint32_t (&key)[V])
{
    constexpr int W = VECTOR ? ROW_VEC<BF16> : 1;
#pragma unroll
    for (int i = 0; i < V; i += W) {
        if (e0 + i + W <= E) {
            float x[W];
            row_load<BF16, W>(logits, row + e0 + i, x);
#pragma unroll
            for (int c = 0; c < W; ++c) key[i + c] = rt_key(x[c]);
        } else {
#pragma unroll
            for (int c = 0; c < W; ++c) {
                float x[1] = {0.f};
                if (e0 + i + c < E) row_load<BF16, 1>(logits, row + e0 + i + c, x);
                key[i + c] = e0 + i + c < E ? rt_key(x[0]) : 0u;
            }
        }
    }
}

__device__ __forceinline__ void order_pair(uint32_t &a, uint32_t &b)
{
    const uint32_t hi = max(a, b);
    b = min(a, b);
    a = hi;
}
// 8 keys in descending order (an odd-even merge network of 19 comparators)
__device__ __forceinline__ void sort8(uint32_t (&k)[8])
{
#pragma unroll
    for (int i = 0; i < 8; i += 2) order_pair(k[i], k[i + 1]);
#pragma unroll
    for (int i = 0; i < 8; i += 4) { order_pair(k[i], k[i + 2]); order_pair(k[i + 1], k[i + 3]); order_pair(k[i + 1], k[i + 2]); }
#pragma unroll
    for (int i = 0; i < 4; ++i) order_pair(k[i], k[i + 4]);
    order_pair(k[2], k[4]); order_pair(k[3], k[5]);
    order_pair(k[1], k[2]); order_pair(k[3], k[4]); order_pair(k[5], k[6]);
}
// The 8 largest of the group's keys, descending, in every lane: the 8 largest of two descending lists are the larger of
// each key and its counterpart from the other end, a bitonic list that three strides order.
template <int L> __device__ __forceinline__ void merge8(uint32_t (&k)[8])
{
#pragma unroll
    for (int o = 1; o < L; o <<= 1) {
        uint32_t other[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) other[i] = __shfl_xor_sync(FULL_MASK, k[7 - i], o);
#pragma unroll
        for (int i = 0; i < 8; ++i) k[i] = max(k[i], other[i]);
#pragma unroll
        for (int s = 4; s > 0; s >>= 1)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (!(i & s)) order_pair(k[i], k[i + s]);
    }
}

template <bool BF16, bool VECTOR, int V, int L>
__global__ void __launch_bounds__(RT_THREADS)
route_topk_kernel(const void *__restrict__ logits, int64_t T, int E, int64_t ld, int k, bool over_all,
                  int32_t *__restrict__ expert, float *__restrict__ weight)
{
    extern __shared__ uint32_t rt_smem[];
    constexpr int TOKENS = RT_THREADS / L;
    const int lane = threadIdx.x & 31;
    const int gl = lane & (L - 1);                                  // lane within the token's group
    const int64_t t = (int64_t)blockIdx.x * TOKENS + threadIdx.x / L;
    const bool live = t < T;
    int32_t *s_id = reinterpret_cast<int32_t *>(rt_smem) + (threadIdx.x / L) * k;
    uint32_t *s_key = rt_smem + TOKENS * k + (threadIdx.x / L) * k;

    constexpr uint32_t LOW = V * L - 1;                             // the bits that hold V * L - 1 - index
    uint32_t key[V];
    auto load_keys = [&]() { rt_load<BF16, VECTOR, V>(logits, (live ? t : 0) * ld, gl * V, live ? E : 0, key); };
    load_keys();
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = key[i] ? (key[i] & ~LOW) | (LOW - (gl * V + i)) : 0u;
    uint32_t best = 0u, last = 0u;
    bool open = false;
    if (V == 8 && k <= 8) {
        uint32_t top8[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) top8[i] = key[i % V];
        sort8(top8);
        merge8<L>(top8);
        uint32_t edge = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i < k) edge = top8[i];
            if (i < k && gl == 0) s_key[i] = top8[i];
            if (i > 0) open |= i < k && top8[i] && ((top8[i] ^ top8[i > 0 ? i - 1 : 0]) & ~LOW) == 0u;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) open |= edge && key[i] < edge && ((key[i] ^ edge) & ~LOW) == 0u;
        open &= !BF16;
    } else {
        for (int j = 0; j <= k; ++j) {
            best = 0u;
#pragma unroll
            for (int i = 0; i < V; ++i) { key[i] = key[i] == last ? 0u : key[i]; best = max(best, key[i]); }
            const uint32_t m = group_max<L>(best);
            open |= !BF16 && m && ((last ^ m) & ~LOW) == 0u;
            if (j < k && gl == 0) s_key[j] = m;
            last = m;
        }
    }
    const bool fast = !__any_sync(FULL_MASK, open);
    if (!fast) {
        load_keys();
        best = 0u;
#pragma unroll
        for (int i = 0; i < V; ++i) best = max(best, key[i]);
        const unsigned group_bits = (L == 32 ? FULL_MASK : ((1u << (L & 31)) - 1u)) << (lane & ~(L - 1));
        for (int j = 0; j < k; ++j) {
            const uint32_t m = group_max<L>(best);
            const unsigned holders = __ballot_sync(FULL_MASK, best == m) & group_bits;
            if (lane == __ffs(holders) - 1) {
                int at = 0;
#pragma unroll
                for (int i = V - 1; i >= 0; --i) at = key[i] == m ? i : at;
                s_id[j] = m ? gl * V + at : -1;
                s_key[j] = m;
                best = 0u;
#pragma unroll
                for (int i = 0; i < V; ++i) { key[i] = i == at ? 0u : key[i]; best = max(best, key[i]); }
            }
        }
    }
    __syncwarp();
    for (int j = gl; live && fast && j < k; j += L) {               // the exact logits of the indices found
        const uint32_t m = s_key[j];
        const int id = m ? (int)(LOW - (m & LOW)) : -1;
        float x[1] = {0.f};
        if (m) row_load<BF16, 1>(logits, t * ld + id, x);
        s_id[j] = id;
        s_key[j] = m ? rt_key(x[0]) : 0u;
    }
    __syncwarp();
    const float top = rt_value(s_key[0]);
    float all = 0.f, chosen = 0.f;
    if (over_all) {
        rt_load<BF16, VECTOR, V>(logits, (live ? t : 0) * ld, gl * V, live ? E : 0, key);
#pragma unroll
        for (int i = 0; i < V; ++i) all += key[i] ? expf(rt_value(key[i]) - top) : 0.f;
    }
    if (!over_all)
        for (int j = gl; j < k; j += L) chosen += s_key[j] ? expf(rt_value(s_key[j]) - top) : 0.f;
    const float total = group_sum<L>(over_all ? all : chosen);
    if (!live) return;
    for (int j = gl; j < k; j += L) {
        const uint32_t m = s_key[j];
        DASS_ST(expert + t * k + j, s_id[j]);
        DASS_ST(weight + t * k + j, m ? expf(rt_value(m) - top) / total : 0.f);
    }
}

// dlogits.  With p the softmax (over the chosen, or over all unmasked) and s = sum_j w_j dw_j over the chosen:
// dl_e = p_e ([e chosen] dw_e - s), 0 for what p leaves out.  The row is written as it is for experts that were not
// chosen, then (after a warp barrier, which orders the two) the chosen elements over it.
template <bool BF16, bool VECTOR, int V, int L>
__global__ void __launch_bounds__(RT_THREADS)
route_topk_backward_kernel(const void *__restrict__ logits, int64_t T, int E, int64_t ld, int k, bool over_all,
                           const int32_t *__restrict__ expert, const float *__restrict__ dweight,
                           void *__restrict__ dlogits, int64_t ldd)
{
    constexpr int TOKENS = RT_THREADS / L;
    constexpr int W = VECTOR ? ROW_VEC<BF16> : 1;
    const int gl = threadIdx.x & (L - 1);
    const int64_t t = (int64_t)blockIdx.x * TOKENS + threadIdx.x / L;
    const bool live = t < T;
    uint32_t key[V];
    uint32_t m = 0u;
    if (over_all) {
        rt_load<BF16, VECTOR, V>(logits, (live ? t : 0) * ld, gl * V, live ? E : 0, key);
#pragma unroll
        for (int i = 0; i < V; ++i) m = max(m, key[i]);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = 0u;
    }
    constexpr int J = L >= 4 ? 32 / L : 8;                           // choices of a lane: k <= min(32, V L)
    int id[J];
    uint32_t ck[J];
    float dw[J], ce[J];
#pragma unroll
    for (int q = 0; q < J; ++q) {
        const int j = gl + q * L;
        id[q] = live && j < k ? DASS_LD(expert + t * k + j) : -1;
        dw[q] = live && j < k ? DASS_LD(dweight + t * k + j) : 0.f;
    }
#pragma unroll
    for (int q = 0; q < J; ++q) {
        float x[1] = {0.f};
        const bool in = id[q] >= 0 && id[q] < E;
        if (in) row_load<BF16, 1>(logits, t * ld + id[q], x);
        ck[q] = in ? rt_key(x[0]) : 0u;
        m = max(m, ck[q]);
    }
    const float top = rt_value(group_max<L>(m));
    float sum = 0.f, dot = 0.f;
    if (over_all) {
#pragma unroll
        for (int i = 0; i < V; ++i) sum += key[i] ? expf(rt_value(key[i]) - top) : 0.f;
    }
#pragma unroll
    for (int q = 0; q < J; ++q) {
        ce[q] = ck[q] ? expf(rt_value(ck[q]) - top) : 0.f;
        if (!over_all) sum += ce[q];
        if (ck[q]) dot += ce[q] * dw[q];
    }
    sum = group_sum<L>(sum);
    dot = group_sum<L>(dot);
    const float share = sum > 0.f ? 1.0f / sum : 0.f;
    const float s = dot * share;
    if (live) {
#pragma unroll
        for (int i = 0; i < V; i += W) {
            const int e = gl * V + i;
            float g[W];
#pragma unroll
            for (int c = 0; c < W; ++c) g[c] = key[i + c] ? -s * (expf(rt_value(key[i + c]) - top) * share) : 0.f;
            if (e + W <= E) row_store<BF16, W>(dlogits, t * ldd + e, g);
            else {
#pragma unroll
                for (int c = 0; c < W; ++c) {
                    const float one[1] = {g[c]};
                    if (e + c < E) row_store<BF16, 1>(dlogits, t * ldd + e + c, one);
                }
            }
        }
    }
    __syncwarp();
#pragma unroll
    for (int q = 0; q < J; ++q) {
        if (!ck[q]) continue;
        const float g[1] = {ce[q] * share * (dw[q] - s)};
        row_store<BF16, 1>(dlogits, t * ldd + id[q], g);
    }
}

struct RouteArgs {
    const void *logits; int64_t T; int E; int64_t ld; int k; bool over_all;
    int32_t *expert; float *weight;                                  // forward
    const int32_t *chosen; const float *dweight; void *dlogits; int64_t ldd;   // backward (dlogits not null)
    bool vector; cudaStream_t st;
};

template <bool BF16, bool VECTOR, int V, int L>
static cudaError_t rt_launch(const RouteArgs &a)
{
    constexpr int TOKENS = RT_THREADS / L;
    const unsigned grid = (unsigned)((a.T + TOKENS - 1) / TOKENS);
    if (a.dlogits)
        route_topk_backward_kernel<BF16, VECTOR, V, L><<<grid, RT_THREADS, 0, a.st>>>(a.logits, a.T, a.E, a.ld, a.k, a.over_all,
                                                                                      a.chosen, a.dweight, a.dlogits, a.ldd);
    else
        route_topk_kernel<BF16, VECTOR, V, L><<<grid, RT_THREADS, (size_t)TOKENS * a.k * 8, a.st>>>(a.logits, a.T, a.E, a.ld, a.k,
                                                                                                    a.over_all, a.expert, a.weight);
    return cudaGetLastError();
}
template <bool BF16, bool VECTOR>
static cudaError_t rt_pick(const RouteArgs &a)
{
    if (a.E <= 8) return rt_launch<BF16, VECTOR, 8, 1>(a);
    if (a.E <= 16) return rt_launch<BF16, VECTOR, 8, 2>(a);
    if (a.E <= 32) return rt_launch<BF16, VECTOR, 8, 4>(a);
    if (a.E <= 64) return rt_launch<BF16, VECTOR, 8, 8>(a);
    if (a.E <= 128) return rt_launch<BF16, VECTOR, 8, 16>(a);
    if (a.E <= 256) return rt_launch<BF16, VECTOR, 8, 32>(a);
    if (a.E <= 512) return rt_launch<BF16, VECTOR, 16, 32>(a);
    return rt_launch<BF16, VECTOR, 32, 32>(a);
}
static cudaError_t rt_dispatch(const RouteArgs &a, bool bf16)
{
    if (bf16) return a.vector ? rt_pick<true, true>(a) : rt_pick<true, false>(a);
    return a.vector ? rt_pick<false, true>(a) : rt_pick<false, false>(a);
}

static dass_status rt_check(int64_t T, int64_t E, int64_t ld, int dt, int k, int norm)
{
    if (dt != DASS_BF16 && dt != DASS_F32) return DASS_ERR_DTYPE;
    if (norm != DASS_ROUTE_CHOSEN && norm != DASS_ROUTE_ALL) return DASS_ERR_DTYPE;
    if (T < 0 || E < 1 || ld < E || k < 1 || k > E) return DASS_ERR_SHAPE;
    if (E > RT_MAX_E || k > RT_MAX_K || T > (1ll << 31) - 1) return DASS_ERR_UNSUPPORTED;
    return DASS_OK;
}

}  // namespace dass

using namespace dass;

extern "C" {

dass_status dass_route_topk(const void *logits, int64_t T, int64_t E, int64_t ld, dass_dtype dt, int k, dass_route_norm norm,
                            int32_t *expert, float *weight, void *cuda_stream)
{
    if (T > 0 && (!logits || !expert || !weight)) return DASS_ERR_NULL;
    const dass_status cs = rt_check(T, E, ld, (int)dt, k, (int)norm);
    if (cs != DASS_OK) return cs;
    const bool bf16 = dt == DASS_BF16;
    if (!elem_aligned(logits, bf16) || !elem_aligned(expert, false) || !elem_aligned(weight, false)) return DASS_ERR_ALIGN;
    if (T == 0) return DASS_OK;
    RouteArgs a{};
    a.logits = logits; a.T = T; a.E = (int)E; a.ld = ld; a.k = k; a.over_all = norm == DASS_ROUTE_ALL;
    a.expert = expert; a.weight = weight;
    a.vector = rows_vec_ok(logits, ld, bf16);
    a.st = static_cast<cudaStream_t>(cuda_stream);
    DASS_BOUNDS_SCOPE(bs);
    DASS_BOUNDS_ADD(bs, logits, ((size_t)(T - 1) * ld + E) * (bf16 ? 2 : 4));
    DASS_BOUNDS_ADD(bs, expert, (size_t)T * k * 4);
    DASS_BOUNDS_ADD(bs, weight, (size_t)T * k * 4);
    DASS_BOUNDS_COMMIT(bs, a.st);
    return rt_dispatch(a, bf16) == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

dass_status dass_route_topk_backward(const void *logits, int64_t T, int64_t E, int64_t ld, dass_dtype dt, int k, dass_route_norm norm,
                                     const int32_t *expert, const float *dweight, void *dlogits, int64_t ldd, void *cuda_stream)
{
    if (T > 0 && (!logits || !expert || !dweight || !dlogits)) return DASS_ERR_NULL;
    const dass_status cs = rt_check(T, E, ld, (int)dt, k, (int)norm);
    if (cs != DASS_OK) return cs;
    if (ldd < E) return DASS_ERR_SHAPE;
    const bool bf16 = dt == DASS_BF16;
    if (!elem_aligned(logits, bf16) || !elem_aligned(dlogits, bf16) || !elem_aligned(expert, false) || !elem_aligned(dweight, false))
        return DASS_ERR_ALIGN;
    if (T == 0) return DASS_OK;
    RouteArgs a{};
    a.logits = logits; a.T = T; a.E = (int)E; a.ld = ld; a.k = k; a.over_all = norm == DASS_ROUTE_ALL;
    a.chosen = expert; a.dweight = dweight; a.dlogits = dlogits; a.ldd = ldd;
    a.vector = rows_vec_ok(logits, ld, bf16) && rows_vec_ok(dlogits, ldd, bf16);
    a.st = static_cast<cudaStream_t>(cuda_stream);
    DASS_BOUNDS_SCOPE(bs);
    DASS_BOUNDS_ADD(bs, logits, ((size_t)(T - 1) * ld + E) * (bf16 ? 2 : 4));
    DASS_BOUNDS_ADD(bs, expert, (size_t)T * k * 4);
    DASS_BOUNDS_ADD(bs, dweight, (size_t)T * k * 4);
    DASS_BOUNDS_ADD(bs, dlogits, ((size_t)(T - 1) * ldd + E) * (bf16 ? 2 : 4));
    DASS_BOUNDS_COMMIT(bs, a.st);
    return rt_dispatch(a, bf16) == cudaSuccess ? DASS_OK : DASS_ERR_CUDA;
}

}  // extern "C"
