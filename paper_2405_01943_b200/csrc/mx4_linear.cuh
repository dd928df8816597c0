// What the kernels of dass_linear_mx4 share: the arguments.  Internal header.
#pragma once

#include "linear_common.cuh"
#include "mx4_common.cuh"

namespace dass {

struct Mx4Matrix { const uint8_t *codes, *scales; };       // null codes: absent

struct Mx4Args {
    LinearArgs a;              // X null where x holds the rows; W, W_up and their strides unused; bf16
    Mx4Matrix x, w, up;        // rows [T x K]; weights [groups x N x K]
};

// Codes and scales of group g's matrix.
__host__ __device__ __forceinline__ Mx4Matrix mx4_group(const Mx4Matrix &m, int64_t g, int64_t N, int64_t K)
{
    return {m.codes + g * N * mx4_pitch(K), m.scales + g * ((N + MX4_TILE_ROWS - 1) / MX4_TILE_ROWS) * mx4_k_tiles(K) * MX4_TILE_BYTES};
}

}  // namespace dass
