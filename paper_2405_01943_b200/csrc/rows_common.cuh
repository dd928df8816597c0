// Row access shared by the router, expert-row and linear kernels: VEC consecutive elements of a bf16 or f32 row as
// floats.  VEC elements fill one 16-byte access where pointers and pitches allow it; VEC = 1 is the form for any
// alignment.  Internal header.
#pragma once

#include "dass_device.cuh"

namespace dass {

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));     // first source -> upper half
    return r;
}

// Elements of one 16-byte access.
template <bool BF16> constexpr int ROW_VEC = BF16 ? 8 : 4;

template <bool BF16, int VEC>
__device__ __forceinline__ void row_load(const void *base, int64_t off, float (&v)[VEC])
{
    if constexpr (VEC == 1) {
        if constexpr (BF16) v[0] = __uint_as_float((uint32_t)DASS_LD(static_cast<const uint16_t *>(base) + off) << 16);
        else v[0] = DASS_LD(static_cast<const float *>(base) + off);
    } else if constexpr (BF16) {
        const uint4 w = DASS_LD(reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(base) + off));
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(x[i] << 16); v[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u); }
    } else {
        const float4 w = DASS_LD(reinterpret_cast<const float4 *>(static_cast<const float *>(base) + off));
        v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
    }
}

template <bool BF16, int VEC>
__device__ __forceinline__ void row_store(void *base, int64_t off, const float (&v)[VEC])
{
    if constexpr (VEC == 1) {
        if constexpr (BF16) DASS_ST(static_cast<uint16_t *>(base) + off, (uint16_t)(pack_bf16x2(v[0], 0.f) & 0xffffu));
        else DASS_ST(static_cast<float *>(base) + off, v[0]);
    } else if constexpr (BF16) {
        DASS_ST(reinterpret_cast<uint4 *>(static_cast<uint16_t *>(base) + off),
                make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])));
    } else {
        DASS_ST(reinterpret_cast<float4 *>(static_cast<float *>(base) + off), make_float4(v[0], v[1], v[2], v[3]));
    }
}

// One access of a row as it lies in memory, for kernels that hold many in flight before they use the first.
template <bool BF16, int VEC> struct RowRaw { uint4 w; };
template <> struct RowRaw<true, 1> { uint16_t w; };
template <> struct RowRaw<false, 1> { float w; };

template <bool BF16, int VEC, bool ONCE = false>
__device__ __forceinline__ void raw_load(RowRaw<BF16, VEC> &r, const void *base, int64_t off)
{
    using W = decltype(r.w);
    const W *p = reinterpret_cast<const W *>(static_cast<const char *>(base) + off * (BF16 ? 2 : 4));
    if constexpr (ONCE) r.w = DASS_LD_CS(p); else r.w = DASS_LD(p);
}
template <bool BF16, int VEC>
__device__ __forceinline__ void raw_floats(const RowRaw<BF16, VEC> &r, float (&v)[VEC])
{
    if constexpr (VEC == 1) {
        if constexpr (BF16) v[0] = __uint_as_float((uint32_t)r.w << 16); else v[0] = r.w;
    } else {
        const uint32_t x[4] = {r.w.x, r.w.y, r.w.z, r.w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (BF16) { v[2 * i] = __uint_as_float(x[i] << 16); v[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u); }
            else v[i] = __uint_as_float(x[i]);
        }
    }
}

// Whether rows that start at `p` and are `ld` elements apart can be read 16 bytes at a time.
inline bool rows_vec_ok(const void *p, int64_t ld, bool bf16)
{
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld % (bf16 ? 8 : 4) == 0;
}
inline bool elem_aligned(const void *p, bool bf16) { return (reinterpret_cast<uintptr_t>(p) & (bf16 ? 1u : 3u)) == 0; }

}  // namespace dass
