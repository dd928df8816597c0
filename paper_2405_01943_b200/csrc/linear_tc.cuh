// What the tensor-core kernels of dass_linear share.  Internal header.
#pragma once

#include "linear_common.cuh"
#include "tc_common.cuh"
#include "tc_pair.cuh"

namespace dass {

// ------------------------------------------------------------------ PTX wrappers
__device__ __forceinline__ void tma_load_3d_hint(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y, int z, uint64_t policy)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4, %5}], [%2], %6;"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "r"(z), "l"(policy) : "memory");
}
// True in one lane of a converged warp.  Around tcgen05 and TMA instructions this, unlike `lane == 0`, lets the compiler
// keep their operands in uniform registers.
__device__ __forceinline__ bool elect_one()
{
    uint32_t is;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
    return is != 0;
}
// A bounded wait of a whole warp with one answer for all its lanes: where the wait runs out for some of them only, none
// goes on into an instruction that expects the others.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag)
{
    return __all_sync(FULL_MASK, mbar_wait(bar, parity, abort_flag));
}
__device__ __forceinline__ void tma_prefetch_map(const CUtensorMap *map)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}
// loads from another CTA's shared memory (addresses from map_to_cta)
__device__ __forceinline__ float ld_cluster(uint32_t addr)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap *map, uint32_t bar_cluster_addr,
                                                 int x, int y, int z, uint64_t policy)
{
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
                 " [%0], [%1, {%3, %4, %5}], [%2], %6;"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar_cluster_addr), "r"(x), "r"(y), "r"(z), "l"(policy)
                 : "memory");
}

// ------------------------------------------------------------------ the epilogue's arithmetic

__device__ __forceinline__ float rcp_approx(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float ex2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The activation before a rounding to bf16 (8 bits): an exponential and a reciprocal of the special-function unit, a few
// units of f32's last place off, are exact enough by 2^10 and keep the epilogue at two such instructions per element.
// x / (1 + e^-x) holds at the ends too: e^-x = inf gives a reciprocal of 0.  Both instructions flush subnormals, so that
// results below 1e-36 in size (SiLU of x < -87.3) come out as zero.
template <int ACT>
__device__ __forceinline__ float lt_act(float x)
{
    constexpr float LOG2E = 1.4426950408889634f;
    if constexpr (ACT == DASS_ACT_SILU) return x * rcp_approx(1.0f + ex2_approx(-LOG2E * x));
    else if constexpr (ACT == DASS_ACT_GELU_TANH)           // 0.5 (1 + tanh z) = sigmoid(2 z), z = sqrt(2 / pi) (x + 0.044715 x^3)
        return x * rcp_approx(1.0f + ex2_approx(-1.5957691216057308f * LOG2E * x * fmaf(0.044715f * x, x, 1.0f)));
    else if constexpr (ACT == DASS_ACT_RELU) return lin_relu(x);
    else return x;
}
template <int ACT, int V> __device__ __forceinline__ void lt_act_each(float (&x)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = lt_act<ACT>(x[i]);
}
template <int V> __device__ __forceinline__ void lt_act_all(float (&x)[V], int act)
{
    switch (act) {
    case DASS_ACT_SILU: lt_act_each<DASS_ACT_SILU>(x); break;
    case DASS_ACT_GELU_TANH: lt_act_each<DASS_ACT_GELU_TANH>(x); break;
    case DASS_ACT_RELU: lt_act_each<DASS_ACT_RELU>(x); break;
    default: break;
    }
}

}  // namespace dass
