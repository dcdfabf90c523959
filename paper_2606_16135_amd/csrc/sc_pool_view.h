// Device-side addressing of a pool's blocks (rope.hip, decode_attn.hip).
#pragma once

#include "sc_internal.h"

namespace sc {

// t / block_size for 0 <= t < 2^31.
__device__ __forceinline__ int block_of(const PoolView &p, int t) {
  return (int)(((uint64_t)(uint32_t)t * p.block_magic) >> (31 + p.block_shift));
}

// The layer's slice of block `id` (its K half), or nullptr for an id outside
// the pool or beyond the HBM blocks it lends.
__device__ __forceinline__ char *block_layer(const PoolView &p, int32_t id) {
  if (id < 0 || id >= p.n_ids) return nullptr;
  const int tier = id < p.first[0] ? 0 : id < p.first[1] ? 1 : 2;
  if (tier == 0 && id >= p.lent) return nullptr;
  const int64_t local = id - (tier == 0 ? 0 : p.first[tier - 1]);
  return p.tier[tier] + local * p.block_bytes + p.layer_off;
}

}  // namespace sc
